// The router in front of grouped products: host side of route.hip.
#pragma once
#include "common.hpp"

namespace brg {

constexpr int64_t kMostExperts = 1024, kMostChosen = 16;

struct RouteCall {
    int dtype;                          // BRGEMM_DTYPE_* of the logits
    int64_t M;
    int experts, chosen;                // E, and how many of them a row takes
    const void *logits;
    int64_t ld;
    const uint8_t *valid;               // a byte a row, or nullptr: 0 marks padding
    int level;                          // 1: a row's gates add up to 1
    int64_t *ids;                       // M x chosen
    float *gates;
    int64_t *offsets;                   // E + 1
    int64_t *rows, *place;              // M * chosen
    float *balance;                     // loss, rows counted, mean probability of every expert
    const float *dgates, *dloss;        // gradients (dgates, dloss: or nullptr)
    void *dlogits;
    int64_t ldd;
    void *workspace;
    size_t workspace_bytes;
    hipStream_t stream;
};

size_t route_workspace(int64_t M, int64_t experts);
hipError_t launch_route(const RouteCall &c);
hipError_t launch_route_grad(const RouteCall &c);

}  // namespace brg
