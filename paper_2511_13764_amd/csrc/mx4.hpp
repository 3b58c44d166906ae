// 4-bit operands that share a power of two in blocks of 32 (E2M1 elements, E8M0 powers): what host and kernels agree on.
//
// An image of R x K numbers, Kp = K rounded up to a multiple of 256:
//   codes    R rows of Kp / 2 bytes, element 2 i of a row in the low half of byte i, zeros past K;
//   powers   behind them Kp / 256 planes of R x 8 bytes: 2^(byte - 127), 255 not a number, of the 8 blocks of those 256 columns in
//            the order 0 4 1 5 2 6 3 7.
// Why so: the 16 x 16 x 128 matrix instruction takes 32 codes a lane (row l % 16, block l / 16), so 256 columns are two 16-byte reads a lane, blocks
// l / 16 and 4 + l / 16 of a row of 128 bytes, the same reads as for the 16-bit types, and their two powers are neighbours in the lane's 16
// bits.  16 rows' powers of 256 columns are one line of 128 bytes, from whatever row a group starts at.
// K is padded because a reduction then has whole blocks only: 256 zeros cost less than a tail in every kernel.
#pragma once
#include "grouped.hpp"

namespace brg {

constexpr int MX_K = 256;               // columns of a block of the image
constexpr int MX_ROW = 128;             // bytes of it in a row

// The other operand: an image too, or 16-bit rows.
enum Mx4Left { LEFT_MX4, LEFT_BF16, LEFT_F16 };

__host__ __device__ inline int64_t mx4_blocks(int64_t K) { return (K + MX_K - 1) / MX_K; }
__host__ __device__ inline int64_t mx4_bytes(int64_t rows, int64_t K) { return rows * mx4_blocks(K) * (MX_ROW + 8); }
// What an image's address, and the step from one to the next, is a multiple of: 16, or 8 where the size is none of 16 (rows and blocks
// both odd), so that images of any size can stand one behind the other.  No kernel takes codes to be aligned to more than 8 bytes.
inline int64_t mx4_alignment(int64_t rows, int64_t K) { return mx4_bytes(rows, K) % 16 ? 8 : 16; }

struct Mx4Args {
    int64_t M, N, K;
    int blocks;                         // of 256 columns
    const char *A;                      // codes or 16-bit rows
    int64_t lda;                        // bytes
    const char *a_powers;               // LEFT_MX4
    int64_t a_plane;                    // bytes from one 256 columns' powers to the next's
    const char *B;
    int64_t ldb;
    const char *b_powers;
    int64_t b_plane;
    int64_t stride_b;                   // bytes from one group's image to the next's
    Epilogue epi;
    int tiles_m, tiles_n;
    Walk walk;
    int split, per;                     // of the reduction, over blockIdx.y: blocks of a slice, sums to `partial`
    float *partial;
};

struct Mx4Call {
    Mx4Args a;
    Mx4Left left;
    bool grouped;
    GroupArgs g;
    hipStream_t stream;
    void *workspace;
    size_t workspace_bytes;
};

// Point a product at the rows and weights of its group.
__device__ __forceinline__ void select_piece(Mx4Args &p, const GroupArgs &g, const GroupTile &t)
{
    p.M = t.rows;
    p.A += t.first * p.lda;
    p.a_powers += (int64_t)t.first * 8;
    p.B += t.weights * p.stride_b;
    p.b_powers += t.weights * p.stride_b;
    select_piece(p.epi, g, t);
}

typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef int32_t mx4_codes __attribute__((ext_vector_type(4), aligned(8)));      // 32 codes of an image

// 2^(byte - 127) in fp32.
__device__ __forceinline__ float mx4_power(uint32_t byte)
{
    const uint32_t bits = byte == 0 ? 0x00400000u : byte << 23;
    return __uint_as_float(byte == 255 ? 0x7fc00000u : bits);
}

// D = A x B + C of v_mfma_scale_f32_16x16x128_f8f6f4 on 4-bit operands; powers: byte OP of each lane's register.
// Sums of products that share their powers are exact, others are cut off 20 bits and more below the largest product.
template <int OP_A, int OP_B>
__device__ __forceinline__ f32x4 mfma_mx4(i32x4 a, i32x4 b, f32x4 c, int powers_a, int powers_b)
{
    const i32x4 z = {0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(__builtin_shufflevector(a, z, 0, 1, 2, 3, 4, 5, 6, 7),
                                                            __builtin_shufflevector(b, z, 0, 1, 2, 3, 4, 5, 6, 7), c, 4, 4,
                                                            OP_A, powers_a, OP_B, powers_b);
}

// Eight codes widened to what the 16-bit matrix instruction takes: exact in bf16 for powers up to 2^125 (the packer's most; 4 x 2^126 becomes an
// infinity), in binary16 for 2^-23 .. 2^13.
__device__ __forceinline__ bf16x8 widen_bf16(uint32_t codes, float power)
{
    typedef __attribute__((ext_vector_type(2))) __bf16 h2;
    const h2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, power, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, power, 1);
    const h2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, power, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, power, 3);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
__device__ __forceinline__ f16x8 widen_f16(uint32_t codes, float power)
{
    typedef __attribute__((ext_vector_type(2))) _Float16 h2;
    const h2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, power, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, power, 1);
    const h2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, power, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, power, 3);
    return f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
constexpr uint32_t MX_F16_LEAST = 127 - 23, MX_F16_MOST = 127 + 13;

// Eight binary16 values as the sum of two bf16 each, exactly: 8 of the 11 bits, then the other 3.
__device__ __forceinline__ void split_f16(f16x8 x, bf16x8 &high, bf16x8 &low)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float v = (float)x[i];
        const __bf16 h = (__bf16)v;
        high[i] = h;
        low[i] = __builtin_isfinite(v) ? (__bf16)(v - (float)h) : (__bf16)0.0f;
    }
}

// load16_to_lds_saddr with 4 bytes a lane.
__device__ __forceinline__ void load4_to_lds_saddr(const char *base, uint32_t lane_off, uint32_t lds_addr)
{
    const uint64_t b = (uint64_t)base;
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)b);
    const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(b >> 32));
    const uint64_t ub = ((uint64_t)hi << 32) | lo;
    const uint32_t la = __builtin_amdgcn_readfirstlane(lds_addr);
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2"
                 :
                 : "s"(la), "v"(lane_off), "s"(ub)
                 : "m0");
}

// Launch a kernel of BM x BN tiles.  NARROW: find_mixed_tile<true> looks for them, and a group's last row of tiles may be two workgroups a tile.
template <int BM, int BN, bool NARROW = false>
inline hipError_t mx4_launch(void (*kern)(Mx4Args, GroupArgs), const Mx4Call &c, int threads, size_t lds)
{
    Mx4Args a = c.a;
    GroupArgs g = c.g;
    a.tiles_n = (int)((a.N + BN - 1) / BN);
    a.tiles_m = (int)((a.M + BM - 1) / BM);
    int64_t rows = a.tiles_m;
    if (c.grouped)
        rows = g.max_tiles = (int)most_row_tiles(a.M, g.groups, BM);
    if (NARROW && c.grouped)
        rows += rows < g.groups ? rows : g.groups;
    a.walk = make_walk(c.grouped ? 1 : a.tiles_m, a.tiles_n, 1, 1, 1, (int64_t)kWalkRows * a.tiles_n);
    a.per = (a.blocks + a.split - 1) / a.split;
    if (lds > 65536) {
        static thread_local const void *configured[32] = {nullptr};
        const hipError_t e = raise_lds((const void *)kern, lds, configured);
        if (e != hipSuccess)
            return e;
    }
    hipLaunchKernelGGL(kern, dim3((unsigned)(rows * a.tiles_n), (unsigned)a.split), dim3((unsigned)threads), lds, c.stream, a, g);
    return hipGetLastError();
}

// mx4_direct.hip: tiles whose operands go from memory to registers.
hipError_t mx4_direct(const Mx4Call &c);
// mx4_pingpong.hip: 256 x 256 tiles of two images.
hipError_t mx4_pingpong(const Mx4Call &c);
// mx4_stream.hip: tiles of 128 x 128, 64 x 128 and 64 x 64, of 16-bit rows 32 x 64 and 16 x 64, too (the same rows).
hipError_t mx4_stream(const Mx4Call &c, int bm, int bn);
// mx4_half.hip: 256 x 256 tiles of 16-bit rows (16-byte aligned, and readable, with zeros, up to a multiple of 64 columns).
hipError_t mx4_half(const Mx4Call &c);
// mx4_pack.hip
struct Mx4Pack {
    int dtype;                          // BRGEMM_DTYPE_* of the numbers
    int trans;
    int64_t rows, K;
    const void *X;                      // read by the packer, written by the other
    int64_t ldx, x_rows;
    const int64_t *source;
    char *image;
    hipStream_t stream;
};
hipError_t launch_pack_mx4(const Mx4Pack &p);
hipError_t launch_unpack_mx4(const Mx4Pack &p);
// Rows of K 16-bit values, `lda` bytes apart at any alignment, to rows of `pitch` bytes (a multiple of 16), zeros behind K.
hipError_t launch_mx4_rows(const char *A, int64_t lda, int64_t M, int64_t K, char *out, int64_t pitch, hipStream_t stream);
// mx4.hip.  The kernel a call takes, as the variant whose tile it has: V_GENERIC (mx4_direct), V_BF16_PP256 (mx4_pingpong, mx4_half), V_BF16_STREAM128
// (128 x 128), V_BF16_STREAM64 (64 x 128), V_BF16_STREAM32 (32 x 64, 16 x 64) and with form GEN_64 (64 x 64; mx4_stream).
int plan_mx4(const Mx4Call &c, int forced_variant, int forced_split, int forced_form, Plan *out);
hipError_t launch_mx4(const Mx4Call &c, const Plan &plan);
// Whether a call's rows go through a copy, and that copy, after which the call reads it.
bool mx4_copies(const Mx4Call &c);
hipError_t mx4_copy(Mx4Call &c);

}  // namespace brg
