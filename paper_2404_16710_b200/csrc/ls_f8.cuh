// The 8-bit number format of a layer's products, and the kernels around them: conversion of rows and weights and
// back, RMSNorm and SwiGLU that leave their result in it.  (LayerSkip computes in 16 bits; what bounds its prompt pass
// are the projections, which the tensor cores do at twice the rate on 8-bit operands, and its decode loop their bytes.)
//
// A block of values x shares a scale s = 2^(e - 127), kept as the byte e; a value stands for c * s, c an e4m3 code
// (sign, 4 exponent and 3 mantissa bits: at most 448, no infinities).  Blocks are 128 columns of one row
// (activations) or 128 rows x 128 columns (weights).
//   s = the smallest power of two with max |x| <= 448 s, held in 2^-117 .. 2^119;  c = x / s rounded to nearest even.
// Why a power of two and not max |x| / 448: the codes' relative precision does not depend on s, x / s is exact, so that
// codes are decided exactly in fp32, and c * s has 4 significant bits: it IS a bf16 number (the lowest, 2^-9 * 2^-117, is
// 2^-126), so that expanding loses nothing.  The price: codes reach down to 2^-17 of the largest value instead of 2^-18.
// Ends: a block of zeros has s = 2^-117; beyond 448 * 2^119 = 1.75 * 2^127 codes saturate; a block with a NaN or an
// infinity gets e = 255, codes 0, and stands for NaN.
//
// Codes are rows of K bytes, K a multiple of 16; scale bytes are rows of 4 * ceil(K / 512), one 32-bit word for 512
// columns, the bytes behind the last block zero.
#pragma once
#include "ls_common.cuh"

namespace ls {

constexpr int kF8Block = 128;

__host__ __device__ constexpr int64_t f8_scale_width(int64_t K) { return (K + 511) / 512 * 4; }

// scale byte of a block whose largest |x| has the fp32 bits a: 448 is 1.75 * 2^8, and mantissas above 1.75 carry
__device__ __forceinline__ uint32_t f8_scale_byte(uint32_t a)
{
    const int e = (int)((a + 0x1fffffu) >> 23) - 8;
    return a >= 0x7f800000u ? 255u : (uint32_t)min(max(e, 10), 246);
}
// 1 / s as a float; 0 for a NaN block, whose codes are all 0 (f8_codes4)
__device__ __forceinline__ float f8_inverse(uint32_t e) { return __uint_as_float(e == 255u ? 0u : (254u - e) << 23); }
// s as a float: 2^-127 is below the normal numbers, 255 is NaN
__device__ __forceinline__ float f8_scale(uint32_t e)
{
    return __uint_as_float(e == 255u ? 0x7fc00000u : e == 0u ? 0x00400000u : e << 23);
}
// codes of four values, the first in the lowest byte
__device__ __forceinline__ uint32_t f8_codes4(float a, float b, float c, float d, float r)
{
    uint32_t w;
    asm("{\n\t.reg .b16 lo, hi;\n\t"
        "cvt.rn.satfinite.e4m3x2.f32 lo, %2, %1;\n\t"
        "cvt.rn.satfinite.e4m3x2.f32 hi, %4, %3;\n\t"
        "mov.b32 %0, {lo, hi};\n\t}"
        : "=r"(w)
        : "f"(a * r), "f"(b * r), "f"(c * r), "f"(d * r));
    return r == 0.f ? 0u : w;  // inf * 0 is NaN
}
// values of two codes (the first in the low byte) times s, as bf16: exact
__device__ __forceinline__ uint32_t f8_values2(uint32_t codes, float s)
{
    uint32_t h;
    asm("{\n\t.reg .b16 c;\n\tcvt.u16.u32 c, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, c;\n\t}" : "=r"(h) : "r"(codes));
    float lo, hi;
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}" : "=f"(lo), "=f"(hi) : "r"(h));
    return pack_bf16(lo * s, hi * s);
}

// 16 bytes of a row as floats: four of fp32, eight of bf16.  Coherent loads past L1 (the operation ahead may have
// written them, and under programmatic dependent launch been running when this kernel started).
template <typename T>
struct F8In;
template <>
struct F8In<float> {
    static constexpr int V = 4;
    static __device__ __forceinline__ void load(const float* p, float (&v)[4])
    {
        const float4 f = __ldcg(reinterpret_cast<const float4*>(p));
        v[0] = f.x, v[1] = f.y, v[2] = f.z, v[3] = f.w;
    }
    static __device__ __forceinline__ void store(float* p, const float (&v)[4])
    {
        *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    }
    static __device__ __forceinline__ float kept(float v) { return v; }
};
template <>
struct F8In<uint16_t> {  // bf16
    static constexpr int V = 8;
    static __device__ __forceinline__ void load(const uint16_t* p, float (&v)[8])
    {
        const uint4 u = __ldcg(reinterpret_cast<const uint4*>(p));
        v[0] = bf16lo(u.x), v[1] = bf16hi(u.x), v[2] = bf16lo(u.y), v[3] = bf16hi(u.y);
        v[4] = bf16lo(u.z), v[5] = bf16hi(u.z), v[6] = bf16lo(u.w), v[7] = bf16hi(u.w);
    }
    static __device__ __forceinline__ void store(uint16_t* p, const float (&v)[8])
    {
        *reinterpret_cast<uint4*>(p) =
            make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
    }
    static __device__ __forceinline__ float kept(float v) { return bf16f(f2bf(v)); }  // the value that store() leaves
};

template <int V>
__device__ __forceinline__ uint32_t f8_absmax(const float (&v)[V])  // bits, not values: NaN counts as largest
{
    uint32_t a = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) a = max(a, __float_as_uint(v[i]) & 0x7fffffffu);
    return a;
}
// largest over the 128 / V lanes that hold a block
template <int V>
__device__ __forceinline__ uint32_t f8_block_max(uint32_t a)
{
    if (V == 4) return __reduce_max_sync(0xffffffffu, a);
#pragma unroll
    for (int o = 64 / V; o > 0; o >>= 1) a = max(a, __shfl_xor_sync(0xffffffffu, a, o));
    return a;
}
template <int V>
__device__ __forceinline__ void f8_store_codes(unsigned char* p, const float (&v)[V], float r)
{
    uint32_t w[V / 4];
#pragma unroll
    for (int i = 0; i < V / 4; ++i) w[i] = f8_codes4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3], r);
    if (V == 4) *reinterpret_cast<uint32_t*>(p) = w[0];
    else *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[V / 4 - 1]);
}
// A warp's 32 V columns of a row, from column k0 (a multiple of 128; lane l holds columns k0 + V l ..): codes and scale
// bytes, and zeros behind the row's last block.  Lanes beyond K hold zeros.
template <int V>
__device__ __forceinline__ void f8_store_row_part(const float (&v)[V], int k0, int K, int width, unsigned char* codes,
                                                  unsigned char* scales)
{
    const int lane = threadIdx.x & 31, k = k0 + V * lane;
    const uint32_t e = f8_scale_byte(f8_block_max<V>(f8_absmax<V>(v)));
    if (k < K) f8_store_codes<V>(codes + k, v, f8_inverse(e));
    if (k % kF8Block == 0 && k / kF8Block < width) scales[k / kF8Block] = k < K ? (unsigned char)e : 0;
}

// ------------------------------------------------------------------ rows and weights -> 8 bits, and back
// Rows: a warp takes 512 columns of a row, one word of scales.  grid.x * 8 warps cover the parts of all rows.
template <typename T>
__global__ void __launch_bounds__(256) quantize_f8_rows_kernel(const T* __restrict__ x, int64_t ldx, int K, int parts, long long items,
                                                               unsigned char* __restrict__ codes, unsigned char* __restrict__ scales)
{
    constexpr int V = F8In<T>::V, STEP = 32 * V, N = 512 / STEP;
    pdl_launch_dependents();
    pdl_wait();
    const long long it = (long long)blockIdx.x * 8 + threadIdx.x / 32;
    if (it >= items) return;  // whole warps
    const long long m = it / parts;
    const int k0 = (int)(it - m * parts) * 512, lane = threadIdx.x & 31, width = 4 * parts;
    float v[N][V];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int k = k0 + i * STEP + V * lane;
#pragma unroll
        for (int j = 0; j < V; ++j) v[i][j] = 0.f;
        if (k < K) F8In<T>::load(x + m * ldx + k, v[i]);  // K is a multiple of 16: the octet is in or out
    }
#pragma unroll
    for (int i = 0; i < N; ++i) f8_store_row_part<V>(v[i], k0 + i * STEP, K, width, codes + m * K, scales + m * width);
}

// Weights: a CTA takes a block of 128 x 128.  grid (blocks of a row of them, rows of blocks).
template <typename T>
__global__ void __launch_bounds__(256) quantize_f8_weights_kernel(const T* __restrict__ x, int64_t ldx, int M, int K,
                                                                  unsigned char* __restrict__ codes, unsigned char* __restrict__ scales)
{
    constexpr int V = F8In<T>::V, LANES = kF8Block / V, ROWS = 256 / LANES, N = kF8Block / ROWS;  // ROWS rows a step
    __shared__ uint32_t wmax[8];
    pdl_wait();
    const int tid = threadIdx.x, k = blockIdx.x * kF8Block + V * (tid % LANES);
    const long long m0 = (long long)blockIdx.y * kF8Block + tid / LANES;
    float v[N][V];
    uint32_t a = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
#pragma unroll
        for (int j = 0; j < V; ++j) v[i][j] = 0.f;
        if (k < K && m0 + i * ROWS < M) F8In<T>::load(x + (m0 + i * ROWS) * ldx + k, v[i]);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) a = max(a, f8_absmax<V>(v[i]));
    a = __reduce_max_sync(0xffffffffu, a);
    if ((tid & 31) == 0) wmax[tid >> 5] = a;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 8; ++w) a = max(a, wmax[w]);
    const uint32_t e = f8_scale_byte(a);
    const float r = f8_inverse(e);
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (k < K && m0 + i * ROWS < M) f8_store_codes<V>(codes + (m0 + i * ROWS) * K + k, v[i], r);
    const int width = (int)f8_scale_width(K);
    unsigned char* row = scales + (long long)blockIdx.y * width;
    if (tid == 0) row[blockIdx.x] = (unsigned char)e;
    if (blockIdx.x + 1 == gridDim.x && tid > 0 && (int)blockIdx.x + tid < width) row[blockIdx.x + tid] = 0;  // at most 3
}

// Codes and scales -> bf16 [M, K].  A warp takes 512 columns of a row; `shift`: log2 of a block's rows.
__global__ void __launch_bounds__(256) expand_f8_kernel(const unsigned char* __restrict__ codes, const unsigned char* __restrict__ scales,
                                                        int K, int parts, long long items, int shift, int signal, uint16_t* __restrict__ out)
{
    if (signal) pdl_launch_dependents();
    pdl_wait();
    const long long it = (long long)blockIdx.x * 8 + threadIdx.x / 32;
    if (it >= items) return;
    const long long m = it / parts;
    const int k = (int)(it - m * parts) * 512 + 16 * (threadIdx.x & 31);
    if (k >= K) return;
    const float s = f8_scale(__ldcg(scales + (m >> shift) * (4ll * parts) + k / kF8Block));
    const uint4 c = __ldcg(reinterpret_cast<const uint4*>(codes + m * K + k));
    uint4 lo, hi;
    lo.x = f8_values2(c.x, s), lo.y = f8_values2(c.x >> 16, s), lo.z = f8_values2(c.y, s), lo.w = f8_values2(c.y >> 16, s);
    hi.x = f8_values2(c.z, s), hi.y = f8_values2(c.z >> 16, s), hi.z = f8_values2(c.w, s), hi.w = f8_values2(c.w >> 16, s);
    uint4* dst = reinterpret_cast<uint4*>(out + m * K + k);
    dst[0] = lo;
    dst[1] = hi;
}

// ------------------------------------------------------------------ RMSNorm with the residual's addition, into 8 bits
// x' = x + d rounded to x's type, y = x' / sqrt(mean x'^2 + eps) * gain, sums in fp32.  A CTA takes a row; with NV > 0 a
// thread keeps its NV pieces of it in registers, else (rows too long for that) x' is read again, from x_out where it was
// written.  d and x_out may be null, x_out may be x.
template <typename T, typename TD, int NV>
__global__ void __launch_bounds__(NV == 8 ? 512 : 1024)
rmsnorm_f8_kernel(const T* x, int64_t ldx, const TD* d, int64_t ldd, T* x_out, int64_t ldo, const uint16_t* __restrict__ gain, int D,
                  float eps, unsigned char* __restrict__ codes, unsigned char* __restrict__ scales)
{
    constexpr int V = F8In<T>::V, KEEP = NV > 0 ? NV : 1;
    __shared__ float part[32];
    pdl_launch_dependents();
    pdl_wait();
    const int tid = threadIdx.x, T0 = blockDim.x;
    const long long m = blockIdx.x;
    x += m * ldx;
    if (d) d += m * ldd;
    if (x_out) x_out += m * ldo;
    const int width = (int)f8_scale_width(D), cover = width * kF8Block;  // columns with a scale byte
    auto fetch = [&](int k, float (&v)[V]) {
        F8In<T>::load(x + k, v);
        if (d) {
            float a[V];
            if constexpr (F8In<TD>::V == V) {
                F8In<TD>::load(d + k, a);
            } else if constexpr (V == 8) {  // fp32 d for bf16 x
                float lo[4], hi[4];
                F8In<float>::load(d + k, lo);
                F8In<float>::load(d + k + 4, hi);
#pragma unroll
                for (int j = 0; j < 4; ++j) a[j] = lo[j], a[4 + j] = hi[j];
            } else {
                const uint2 u = __ldcg(reinterpret_cast<const uint2*>(d + k));
                a[0] = bf16lo(u.x), a[1] = bf16hi(u.x), a[2] = bf16lo(u.y), a[3] = bf16hi(u.y);
            }
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = F8In<T>::kept(v[j] + a[j]);
        }
    };
    float v[KEEP][V], ss = 0.f;
    auto square = [&](const float (&u)[V]) {
        float s = 0.f;
#pragma unroll
        for (int j = 0; j < V; ++j) s = fmaf(u[j], u[j], s);
        ss += s;
    };
    if (NV > 0) {
#pragma unroll
        for (int i = 0; i < KEEP; ++i) {
            const int k = (i * T0 + tid) * V;
#pragma unroll
            for (int j = 0; j < V; ++j) v[i][j] = 0.f;
            if (k < D) fetch(k, v[i]);
        }
#pragma unroll
        for (int i = 0; i < KEEP; ++i) {
            const int k = (i * T0 + tid) * V;
            if (x_out && k < D) F8In<T>::store(x_out + k, v[i]);
            square(v[i]);
        }
    } else {
        for (int k = tid * V; k < D; k += T0 * V) {
            fetch(k, v[0]);
            if (x_out) F8In<T>::store(x_out + k, v[0]);
            square(v[0]);
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    if ((tid & 31) == 0) part[tid >> 5] = ss;
    __syncthreads();
    ss = (tid & 31) < T0 / 32 ? part[tid & 31] : 0.f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    const float r = 1.0f / sqrtf(ss / (float)D + eps);
    auto finish = [&](int k, float (&u)[V]) {  // whole warps
        if (k < D) {
            float g[V];
            if constexpr (V == 8) {
                F8In<uint16_t>::load(gain + k, g);
            } else {
                const uint2 w = __ldcg(reinterpret_cast<const uint2*>(gain + k));
                g[0] = bf16lo(w.x), g[1] = bf16hi(w.x), g[2] = bf16lo(w.y), g[3] = bf16hi(w.y);
            }
#pragma unroll
            for (int j = 0; j < V; ++j) u[j] = u[j] * r * g[j];
        }
        f8_store_row_part<V>(u, k - V * (tid & 31), D, width, codes + m * D, scales + m * width);
    };
    if (NV > 0) {
#pragma unroll
        for (int i = 0; i < KEEP; ++i)
            if ((i * T0 + (tid & ~31)) * V < cover) finish((i * T0 + tid) * V, v[i]);
    } else {
        for (int k = tid * V; k - V * (tid & 31) < cover; k += T0 * V) {
#pragma unroll
            for (int j = 0; j < V; ++j) v[0][j] = 0.f;
            if (k < D) {
                if (x_out) F8In<T>::load(x_out + k, v[0]);  // this thread wrote it
                else fetch(k, v[0]);
            }
            finish(k, v[0]);
        }
    }
}

// ------------------------------------------------------------------ SwiGLU into 8 bits
// y = gate / (1 + exp(-gate)) * up.  A warp takes 512 features of a row.
template <typename T>
__global__ void __launch_bounds__(256) swiglu_f8_kernel(const T* __restrict__ gate, const T* __restrict__ up, int64_t ld, int F, int parts,
                                                        long long items, unsigned char* __restrict__ codes,
                                                        unsigned char* __restrict__ scales)
{
    constexpr int V = F8In<T>::V, STEP = 32 * V, N = 512 / STEP;
    pdl_launch_dependents();
    pdl_wait();
    const long long it = (long long)blockIdx.x * 8 + threadIdx.x / 32;
    if (it >= items) return;
    const long long m = it / parts;
    const int k0 = (int)(it - m * parts) * 512, lane = threadIdx.x & 31, width = 4 * parts;
    float g[N][V], u[N][V];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int k = k0 + i * STEP + V * lane;
#pragma unroll
        for (int j = 0; j < V; ++j) g[i][j] = u[i][j] = 0.f;
        if (k < F) {
            F8In<T>::load(gate + m * ld + k, g[i]);
            F8In<T>::load(up + m * ld + k, u[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
#pragma unroll
        for (int j = 0; j < V; ++j) g[i][j] = g[i][j] / (1.0f + expf(-g[i][j])) * u[i][j];
        f8_store_row_part<V>(g[i], k0 + i * STEP, F, width, codes + m * F, scales + m * width);
    }
}

}  // namespace ls
