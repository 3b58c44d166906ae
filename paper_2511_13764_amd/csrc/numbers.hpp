// Numbers of the types that the router and the packer of 4-bit images read and write, in fp32 and back.
#pragma once
#include "../../include/brgemm.h"
#include "common.hpp"

namespace brg {

namespace {

template <int DT> struct Num;
template <> struct Num<BRGEMM_DTYPE_F32> {
    typedef float type;
    static __device__ float wide(float v) { return v; }
    static __device__ float narrow(float v) { return v; }
};
template <> struct Num<BRGEMM_DTYPE_BF16> {
    typedef uint16_t type;
    static __device__ float wide(uint16_t v) { return bf16_to_f32(v); }
    static __device__ uint16_t narrow(float v) { return f32_to_bf16_rne(v); }
};
template <> struct Num<BRGEMM_DTYPE_F16> {
    typedef uint16_t type;
    static __device__ float wide(uint16_t v) { return f16_to_f32(v); }
    static __device__ uint16_t narrow(float v) { return f32_to_f16_rne(v); }
};

}  // namespace

}  // namespace brg
