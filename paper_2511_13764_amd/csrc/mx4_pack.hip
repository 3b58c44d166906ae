// Numbers to 4-bit images (mx4.hpp) and back.  For a block of 32 with largest magnitude m: power e = floor(log2 m) - 2, at least -127, and
// every x becomes the nearest of 0 .5 1 1.5 2 3 4 6 to |x| / 2^e, of two the one whose last bit is clear, 6 where x / 2^e is larger (it is
// below 8).  Blocks of zeros have power -127; infinities and NaN make a block not a number (power byte 255).
#include "../../include/brgemm.h"
#include "mx4.hpp"
#include "numbers.hpp"

namespace brg {

namespace {

__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// Power byte of a block whose largest magnitude has these bits.
__device__ __forceinline__ uint32_t power_byte(uint32_t largest)
{
    const uint32_t e = largest >> 23;
    return e == 255 ? 255 : e > 2 ? e - 2 : 0;
}

// Eight numbers as codes.
__device__ __forceinline__ uint32_t codes_of(const float (&x)[8], uint32_t power)
{
    const float s = mx4_power(power);
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[0], x[1], s, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], s, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4], x[5], s, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6], x[7], s, 3);
    return power == 255 ? 0 : c;
}

// Place of block b (of 8) among the powers of its 256 columns.
__device__ __forceinline__ int power_place(int b) { return 2 * (b & 3) + (b >> 2); }

template <class T> struct Eight;
template <> struct Eight<float> { typedef float type __attribute__((ext_vector_type(4), aligned(4))); };
template <> struct Eight<uint16_t> { typedef uint16_t type __attribute__((ext_vector_type(8), aligned(2))); };

// Eight numbers of a row of `left` that remain (any alignment), zeros behind them.
template <int DT>
__device__ __forceinline__ void load8(const typename Num<DT>::type *x, int64_t left, float (&out)[8])
{
    typedef typename Num<DT>::type T;
    typedef typename Eight<T>::type V;
    constexpr int n = sizeof(V) / sizeof(T);
    if (left >= 8) {
#pragma unroll
        for (int i = 0; i < 8; i += n) {
            const V v = *(const V *)(x + i);
#pragma unroll
            for (int j = 0; j < n; ++j)
                out[i + j] = Num<DT>::wide(v[j]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            out[i] = i < left ? Num<DT>::wide(x[i]) : 0.0f;
    }
}

// Blocks of 256 columns are numbered row by row; half a wave takes one, eight numbers a lane, or of 16-bit numbers two neighbours at once (4096 x 11008
// bf16 out of memory and to it: packing 25.3 us with one and 24.5 with two, 27.4 with four, back 29.4, 26.9 and 25.4; fp32 packing 37.3 and
// 37.9, back 43.5 and 53.9).  (A whole wave for 512 columns: 60000 x 256 16.5 us, so 10.1.)
struct Blocks {
    int64_t rows, K;
    int blocks;                                 // of a row
    Fastdiv by_blocks;                          // or {0, 0}: there are more than 31 bits hold
    __device__ __forceinline__ int64_t total() const { return rows * blocks; }
    __device__ __forceinline__ void find(int64_t i, int64_t &r, int &kb) const
    {
        r = by_blocks.mul ? div_by((int)i, by_blocks) : i / blocks;
        kb = (int)(i - r * blocks);
    }
};

template <int DT, int AT_ONCE>
__global__ void __launch_bounds__(256)
pack_rows_kernel(Blocks at, const typename Num<DT>::type *X, int64_t ldx, int64_t x_rows, const int64_t *source, char *codes, char *powers)
{
    const int lane = threadIdx.x & 31, half = (int)blockIdx.x * 8 + (threadIdx.x >> 5);
    const int64_t step = (int64_t)gridDim.x * 8 * AT_ONCE, total = at.total();
    for (int64_t i0 = (int64_t)half * AT_ONCE; __builtin_amdgcn_ballot_w64(i0 < total) != 0; i0 += step) {
        int64_t r[AT_ONCE];
        int kb[AT_ONCE];
        bool is[AT_ONCE];
        float x[AT_ONCE][8];
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) {
            is[j] = i0 + j < total;
            at.find(is[j] ? i0 + j : total - 1, r[j], kb[j]);
            const int64_t from = source ? source[r[j]] : r[j], k = (int64_t)kb[j] * MX_K + lane * 8;
#pragma unroll
            for (int v = 0; v < 8; ++v)
                x[j][v] = 0.0f;
            if (from >= 0 && from < x_rows && k < at.K)
                load8<DT>(X + from * ldx + k, at.K - k, x[j]);
        }
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) {
            uint32_t m = 0;
#pragma unroll
            for (int v = 0; v < 8; ++v)
                m = m > magnitude(x[j][v]) ? m : magnitude(x[j][v]);
            uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xb1, 0xf, 0xf, true);     // lanes 1 0 3 2
            m = m > o ? m : o;
            o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4e, 0xf, 0xf, true);              // lanes 2 3 0 1
            m = m > o ? m : o;
            const uint32_t power = power_byte(m);
            if (is[j]) {
                *(uint32_t *)(codes + (r[j] * at.blocks + kb[j]) * MX_ROW + lane * 4) = codes_of(x[j], power);
                if ((lane & 3) == 0)
                    powers[((int64_t)kb[j] * at.rows + r[j]) * 8 + power_place(lane >> 2)] = (char)power;
            }
        }
    }
}

// Columns become rows (X is K x rows): 64 of them and 256 k a workgroup, a wave for each block of 32.  A load is 64 numbers of 32 bits, a
// lane having a column, or of 16 bits two rows of 64, a lane having two columns and every other k (4096 x 11008 bf16 one row a load: 43 us).  The codes go through LDS so that rows
// are written in whole lines.
template <int DT>
__global__ void __launch_bounds__(512)
pack_columns_kernel(int64_t rows, int64_t K, const typename Num<DT>::type *X, int64_t ldx, char *codes, char *powers, int64_t tiles)
{
    typedef typename Num<DT>::type T;
    constexpr int C = 4 / sizeof(T);            // columns of a lane
    typedef T Run __attribute__((ext_vector_type(C), aligned(sizeof(T))));
    constexpr int PITCH = MX_ROW + 16;
    __shared__ __attribute__((aligned(16))) char stage[64 * PITCH];
    const int lane = threadIdx.x & 63, b = threadIdx.x >> 6;
    const int column = lane % (64 / C) * C, part = lane / (64 / C);         // k0 + 32 / C part and on
    const int64_t blocks = mx4_blocks(K), strips = (rows + 63) / 64;
    for (int64_t t = blockIdx.x; t < tiles; t += gridDim.x) {
        const int64_t kb = t / strips, r0 = (t - kb * strips) * 64, r = r0 + column, k0 = kb * MX_K + b * 32 + part * (32 / C);
        float x[C][4 / C][8];
        uint32_t m[C] = {};
#pragma unroll
        for (int i = 0; i < 32 / C; ++i) {
            const T *from = X + (k0 + i) * ldx + r;
            Run v = {};
            if (k0 + i < K) {
                if (r + C <= rows)
                    v = *(const Run *)from;
                else if (r < rows)
                    v[0] = from[0];
            }
#pragma unroll
            for (int c = 0; c < C; ++c) {
                x[c][i / 8][i % 8] = Num<DT>::wide(v[c]);
                const uint32_t a = magnitude(x[c][i / 8][i % 8]);
                m[c] = m[c] > a ? m[c] : a;
            }
        }
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if constexpr (C == 2) {
                const auto both = __builtin_amdgcn_permlane32_swap(m[c], m[c], false, false);
                m[c] = both[0] > both[1] ? both[0] : both[1];
            }
            const uint32_t power = power_byte(m[c]);
#pragma unroll
            for (int i = 0; i < 4 / C; i += 2)
                *(u32x2 *)(stage + (column + c) * PITCH + b * 16 + part * (16 / C) + i * 4) = u32x2{codes_of(x[c][i], power), codes_of(x[c][i + 1], power)};
            if (part == 0 && r + c < rows)
                powers[(kb * rows + r + c) * 8 + power_place(b)] = (char)power;
        }
        __syncthreads();
        const int row = threadIdx.x >> 3, chunk = threadIdx.x & 7;
        if (r0 + row < rows)
            *(mx4_codes *)(codes + (r0 + row) * blocks * MX_ROW + kb * MX_ROW + chunk * 16) = *(const i32x4 *)(stage + row * PITCH + chunk * 16);
        __syncthreads();
    }
}

// Back, the same way.
template <int DT, int AT_ONCE>
__global__ void __launch_bounds__(256)
unpack_kernel(Blocks at, const char *codes, const char *powers, typename Num<DT>::type *out, int64_t ldo)
{
    typedef typename Num<DT>::type T;
    typedef typename Eight<T>::type V;
    constexpr int n = sizeof(V) / sizeof(T);
    const int lane = threadIdx.x & 31, half = (int)blockIdx.x * 8 + (threadIdx.x >> 5);
    const int64_t step = (int64_t)gridDim.x * 8 * AT_ONCE, total = at.total();
    for (int64_t i0 = (int64_t)half * AT_ONCE; i0 < total; i0 += step) {
        int64_t r[AT_ONCE];
        int kb[AT_ONCE];
        uint32_t c[AT_ONCE];
        uint8_t power[AT_ONCE];
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) {
            at.find(i0 + j < total ? i0 + j : total - 1, r[j], kb[j]);
            c[j] = *(const uint32_t *)(codes + (r[j] * at.blocks + kb[j]) * MX_ROW + lane * 4);
            power[j] = (uint8_t)powers[((int64_t)kb[j] * at.rows + r[j]) * 8 + power_place(lane >> 2)];
        }
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) {
            const int64_t k = (int64_t)kb[j] * MX_K + lane * 8, left = i0 + j < total ? at.K - k : 0;
            const float s = mx4_power(power[j]);
            typedef __attribute__((ext_vector_type(2))) float f2;
            const f2 p0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[j], s, 0), p1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[j], s, 1);
            const f2 p2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[j], s, 2), p3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[j], s, 3);
            const float v[8] = {p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
            T *to = out + r[j] * ldo + k;
            if (left >= 8) {
#pragma unroll
                for (int i = 0; i < 8; i += n) {
                    V o;
#pragma unroll
                    for (int e = 0; e < n; ++e)
                        o[e] = Num<DT>::narrow(v[i + e]);
                    *(V *)(to + i) = o;
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i < left)
                        to[i] = Num<DT>::narrow(v[i]);
            }
        }
    }
}

__global__ void __launch_bounds__(256)
rows_kernel(const char *A, int64_t lda, int64_t M, int64_t K, char *out, int64_t pitch)
{
    const int64_t chunks = pitch / 16, total = M * chunks;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t m = i / chunks, k = (i - m * chunks) * 8;
        const uint16_t *x = (const uint16_t *)(A + m * lda) + k;
        s16x8 v = {0, 0, 0, 0, 0, 0, 0, 0};
        if (k + 8 <= K) {
            v = *(const s16x8_any2 *)x;
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (k + j < K)
                    v[j] = (short)x[j];
        }
        *(s16x8 *)(out + m * pitch + k * 2) = v;
    }
}

// Workgroups of a grid whose kernels walk on by themselves.
unsigned grid_of(int64_t groups) { return (unsigned)(groups < 65536 ? groups : 65536); }

Blocks blocks_of(const Mx4Pack &p)
{
    const int64_t blocks = mx4_blocks(p.K);
    return Blocks{p.rows, p.K, (int)blocks, p.rows * blocks < (int64_t)1 << 31 ? fastdiv(blocks) : Fastdiv{0, 0}};
}
// Blocks at once, and workgroups of eight half waves for that.  (Few blocks one by one: 16 x 4096 2.4 us, two at once 3.0.)
template <int DT> constexpr int kAtOnce = 4 / sizeof(typename Num<DT>::type);
template <int DT>
int at_once(const Blocks &at) { return at.rows * at.blocks >= 16384 ? kAtOnce<DT> : 1; }
unsigned half_waves(const Blocks &at, int n) { return grid_of((at.rows * at.blocks + 8 * n - 1) / (8 * n)); }

template <int DT>
hipError_t pack(const Mx4Pack &p)
{
    typedef typename Num<DT>::type T;
    const int64_t blocks = mx4_blocks(p.K);
    char *powers = p.image + p.rows * blocks * MX_ROW;
    if (p.trans) {
        const int64_t tiles = (p.rows + 63) / 64 * blocks;
        hipLaunchKernelGGL(pack_columns_kernel<DT>, dim3(grid_of(tiles)), dim3(512), 0, p.stream, p.rows, p.K, (const T *)p.X, p.ldx,
                           p.image, powers, tiles);
    } else {
        const Blocks at = blocks_of(p);
        const int n = at_once<DT>(at);
        hipLaunchKernelGGL((n > 1 ? pack_rows_kernel<DT, kAtOnce<DT>> : pack_rows_kernel<DT, 1>), dim3(half_waves(at, n)), dim3(256), 0, p.stream, at, (const T *)p.X, p.ldx, p.x_rows, p.source, p.image, powers);
    }
    return hipGetLastError();
}

template <int DT>
hipError_t unpack(const Mx4Pack &p)
{
    const Blocks at = blocks_of(p);
    const int n = at_once<DT>(at);
    hipLaunchKernelGGL((n > 1 ? unpack_kernel<DT, kAtOnce<DT>> : unpack_kernel<DT, 1>), dim3(half_waves(at, n)), dim3(256), 0, p.stream, at, p.image, p.image + p.rows * at.blocks * MX_ROW,
                       (typename Num<DT>::type *)p.X, p.ldx);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_mx4_rows(const char *A, int64_t lda, int64_t M, int64_t K, char *out, int64_t pitch, hipStream_t stream)
{
    hipLaunchKernelGGL(rows_kernel, dim3(grid_of((M * (pitch / 16) + 255) / 256)), dim3(256), 0, stream, A, lda, M, K, out, pitch);
    return hipGetLastError();
}

hipError_t launch_pack_mx4(const Mx4Pack &p)
{
    return p.dtype == BRGEMM_DTYPE_F32 ? pack<BRGEMM_DTYPE_F32>(p) : p.dtype == BRGEMM_DTYPE_BF16 ? pack<BRGEMM_DTYPE_BF16>(p)
                                                                                              : pack<BRGEMM_DTYPE_F16>(p);
}

hipError_t launch_unpack_mx4(const Mx4Pack &p)
{
    return p.dtype == BRGEMM_DTYPE_F32 ? unpack<BRGEMM_DTYPE_F32>(p) : p.dtype == BRGEMM_DTYPE_BF16 ? unpack<BRGEMM_DTYPE_BF16>(p)
                                                                                                : unpack<BRGEMM_DTYPE_F16>(p);
}

}  // namespace brg
