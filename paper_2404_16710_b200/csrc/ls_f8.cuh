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

// 32 bytes of a row: eight values of fp32, sixteen of bf16.  One access where `wide` says that rows begin at 32-byte boundaries,
// else two.  Coherent loads that L1 does not keep (the operation ahead may have written the data, and under programmatic
// dependent launch been running when this kernel started).
struct F8Raw {
    uint32_t w[8];
};
template <bool LAST = false>  // LAST: nobody reads it again, L2 may drop it first
__device__ __forceinline__ F8Raw f8_ld32(const void* p, bool wide)
{
    F8Raw r;
    if (LAST && wide) {
        asm volatile("ld.global.L1::no_allocate.L2::evict_first.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                     : "=r"(r.w[0]), "=r"(r.w[1]), "=r"(r.w[2]), "=r"(r.w[3]), "=r"(r.w[4]), "=r"(r.w[5]), "=r"(r.w[6]), "=r"(r.w[7])
                     : "l"(p)
                     : "memory");
    } else if (wide) {
        asm volatile("ld.global.L1::no_allocate.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                     : "=r"(r.w[0]), "=r"(r.w[1]), "=r"(r.w[2]), "=r"(r.w[3]), "=r"(r.w[4]), "=r"(r.w[5]), "=r"(r.w[6]), "=r"(r.w[7])
                     : "l"(p)
                     : "memory");
    } else {
        const uint4 a = __ldcg(reinterpret_cast<const uint4*>(p)), b = __ldcg(reinterpret_cast<const uint4*>(p) + 1);
        r.w[0] = a.x, r.w[1] = a.y, r.w[2] = a.z, r.w[3] = a.w, r.w[4] = b.x, r.w[5] = b.y, r.w[6] = b.z, r.w[7] = b.w;
    }
    return r;
}
__device__ __forceinline__ void f8_st32(void* p, const uint32_t (&w)[8], bool wide)
{
    if (wide) {
        asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                     ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                     : "memory");
    } else {
        reinterpret_cast<uint4*>(p)[0] = make_uint4(w[0], w[1], w[2], w[3]);
        reinterpret_cast<uint4*>(p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
    }
}
template <typename T>
struct F8In;
template <>
struct F8In<float> {
    static constexpr int V = 8;
    static __device__ __forceinline__ void unpack(const F8Raw& r, float (&v)[8])
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r.w[i]);
    }
    static __device__ __forceinline__ void store(float* p, const float (&v)[8], bool wide)
    {
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(v[i]);
        f8_st32(p, w, wide);
    }
    static __device__ __forceinline__ float kept(float v) { return v; }
    static __device__ __forceinline__ float load(const float* p) { return __ldcg(p); }
};
template <>
struct F8In<uint16_t> {  // bf16
    static constexpr int V = 16;
    static __device__ __forceinline__ void unpack(const F8Raw& r, float (&v)[16])
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[2 * i] = bf16lo(r.w[i]), v[2 * i + 1] = bf16hi(r.w[i]);
    }
    static __device__ __forceinline__ void store(uint16_t* p, const float (&v)[16], bool wide)
    {
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
        f8_st32(p, w, wide);
    }
    static __device__ __forceinline__ float kept(float v) { return bf16f(f2bf(v)); }  // the value that store() leaves
    static __device__ __forceinline__ float load(const uint16_t* p) { return bf16f(__ldcg(p)); }
};

__device__ __forceinline__ float max_nan(float a, float b)  // a NaN wins
{
    float m;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(a), "f"(b));
    return m;
}
template <int V>
__device__ __forceinline__ uint32_t f8_absmax(const float (&v)[V])  // bits of the largest |v|; a NaN's are larger than any number's
{
    float a[V / 2];
#pragma unroll
    for (int i = 0; i < V / 2; ++i) a[i] = max_nan(fabsf(v[2 * i]), fabsf(v[2 * i + 1]));
#pragma unroll
    for (int n = V / 4; n > 0; n /= 2)
#pragma unroll
        for (int i = 0; i < n; ++i) a[i] = max_nan(a[i], a[i + n]);
    return __float_as_uint(a[0]) & 0x7fffffffu;
}
template <int V>
__device__ __forceinline__ void f8_store_codes(unsigned char* p, const float (&v)[V], float r)
{
    uint32_t w[V / 4];
#pragma unroll
    for (int i = 0; i < V / 4; ++i) w[i] = f8_codes4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3], r);
    if constexpr (V == 8) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    else *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
// largest over the 128 / V lanes that hold a block
template <int V>
__device__ __forceinline__ uint32_t f8_block_max(uint32_t a)
{
#pragma unroll
    for (int o = 64 / V; o > 0; o >>= 1) a = max(a, __shfl_xor_sync(0xffffffffu, a, o));
    return a;
}
// A double as a float, rounded to odd: where it is inexact the last bit is set, so that a later rounding to fewer bits, and a
// comparison with a number of fewer bits, decide as the double would.
__device__ __forceinline__ float f8_odd(double y)
{
    const float n = (float)y, f = __double2float_rz(y);
    return (double)n == y || isinf(n) ? n : __uint_as_float(__float_as_uint(f) | 1u);
}
// Values computed in fp32, off by up to W 2^-24 of theirs, are rounded to 4 bits here.  What lies so near a border between two
// codes (one value in 2^20 / 2 W) or two scales is computed again, by fix(k) for column k: in 64 bits, rounded to odd, so
// that codes and scales are those of the exact values (of 18 million, fp32 alone gave 10 the neighbouring code).  Borders
// have 0x80000 in the 20 bits behind the code's three; of t (1 + W 2^-24), with t near one, they are up to 2 W + 1 above
// that.  Codes below 2^-6 s (8 of the 127, a fixed distance apart) keep the fp32 value's rounding.
__device__ __forceinline__ uint32_t f8_above_border(float t) { return (__float_as_uint(t) ^ 0x80000u) & 0xfffffu; }
struct F8AsIs {};  // with W = 0: the values are what they are
// The two rare ways are calls, whose registers and instructions the others do not carry: the columns of a lane that `todo`
// names, and a warp's whole part where the scale is in doubt.
// fix() loads from L2: a line that an operation of the chain left in L1 may be older than the data (f8_ld32 leaves none).
template <typename Fix>
__device__ __noinline__ void f8_fix_codes(Fix fix, int k, uint32_t todo, float r, unsigned char* codes)
{
    for (; todo; todo &= todo - 1) {
        const int j = __ffs(todo) - 1;
        codes[k + j] = (unsigned char)f8_codes4(fix(k + j), 0.f, 0.f, 0.f, r);
    }
}
template <int V, typename Fix>
__device__ __noinline__ void f8_fix_part(Fix fix, int k, int K, int width, unsigned char* codes, unsigned char* scales)
{
    uint32_t a = 0;
#pragma unroll 1
    for (int j = 0; j < V; ++j)
        if (k < K) a = max(a, __float_as_uint(fix(k + j)) & 0x7fffffffu);
    const uint32_t e = f8_scale_byte(f8_block_max<V>(a));
    if (k < K) f8_fix_codes(fix, k, (1u << V) - 1, f8_inverse(e), codes);
    if (k % kF8Block == 0 && k / kF8Block < width) scales[k / kF8Block] = k < K ? (unsigned char)e : 0;
}
// A warp's 32 V columns of a row, from column k0 (a multiple of 128; lane l holds columns k0 + V l ..): codes and scale
// bytes, and zeros behind the row's last block.  Lanes beyond K hold zeros.
template <int V, int W, typename Fix>
__device__ __forceinline__ void f8_store_row_part(const float (&v)[V], int k0, int K, int width, unsigned char* codes,
                                                  unsigned char* scales, Fix fix)
{
    const int k = k0 + V * (threadIdx.x & 31);
    const uint32_t a = f8_block_max<V>(f8_absmax<V>(v));
    if constexpr (W > 0) {
        if (__any_sync(0xffffffffu, (a & 0x7fffffu) - (0x600000u - W) <= 2u * W)) {  // 448 = 1.75 2^8
            f8_fix_part<V>(fix, k, K, width, codes, scales);
            return;
        }
    }
    const uint32_t e = f8_scale_byte(a);
    const float r = f8_inverse(e);
    if (k < K) f8_store_codes<V>(codes + k, v, r);
    if (k % kF8Block == 0 && k / kF8Block < width) scales[k / kF8Block] = k < K ? (unsigned char)e : 0;
    if constexpr (W > 0) {
        const float q = r * (1.f + W * 0x1p-24f);
        uint32_t near = 0xfffffu;
#pragma unroll
        for (int j = 0; j < V; j += 2) near = __vimin3_u32(near, f8_above_border(v[j] * q), f8_above_border(v[j + 1] * q));
        if (near <= 2 * W + 1) {
            uint32_t todo = 0;
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (f8_above_border(v[j] * q) <= 2 * W + 1) todo |= 1u << j;
            f8_fix_codes(fix, k, todo, r, codes);
        }
    }
}

// ------------------------------------------------------------------ rows and weights -> 8 bits, and back
// Rows: a warp takes 1024 columns of a row.  grid.x * 8 warps cover the parts of all rows.  (1030 x 4096 bf16: 5.6 us, launch 2.2 of them.)
constexpr int kF8RowPart = 1024;
template <typename T>
__global__ void __launch_bounds__(256) quantize_f8_rows_kernel(const T* __restrict__ x, int64_t ldx, int K, int parts, long long items, int wide,
                                                               unsigned char* __restrict__ codes, unsigned char* __restrict__ scales)
{
    constexpr int V = F8In<T>::V, STEP = 32 * V, N = kF8RowPart / STEP;
    pdl_launch_dependents();
    pdl_wait();
    const long long it = (long long)blockIdx.x * 8 + threadIdx.x / 32;
    if (it >= items) return;  // whole warps
    const long long m = it / parts;
    const int k0 = (int)(it - m * parts) * kF8RowPart, lane = threadIdx.x & 31, width = (int)f8_scale_width(K);
    F8Raw raw[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int k = k0 + i * STEP + V * lane;
        raw[i] = F8Raw{};
        if (k < K) raw[i] = f8_ld32<true>(x + m * ldx + k, wide);  // K is a multiple of 16: all of the piece is in or out
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        float v[V];
        F8In<T>::unpack(raw[i], v);
        if (k0 + i * STEP < width * kF8Block) f8_store_row_part<V, 0>(v, k0 + i * STEP, K, width, codes + m * K, scales + m * width, F8AsIs{});
    }
}

// Weights: a CTA takes a block of 128 x 128.  grid (blocks of a row of them, rows of blocks).  Bound by the loads of a CTA's only
// block: pieces stay as they were loaded, so that more CTAs fit an SM (11008 x 4096 bf16: 27 us, 5.0 TB/s; as floats, and
// 16 bytes at a time, 60).
template <typename T>
__global__ void __launch_bounds__(256, F8In<T>::V == 16 ? 3 : 2)
quantize_f8_weights_kernel(const T* __restrict__ x, int64_t ldx, int M, int K, int wide, unsigned char* __restrict__ codes,
                           unsigned char* __restrict__ scales)
{
    constexpr int V = F8In<T>::V, LANES = kF8Block / V, ROWS = 256 / LANES, N = kF8Block / ROWS;  // ROWS rows a step
    __shared__ uint32_t wmax[8];
    pdl_wait();
    const int tid = threadIdx.x, k = blockIdx.x * kF8Block + V * (tid % LANES);
    const long long m0 = (long long)blockIdx.y * kF8Block + tid / LANES;
    F8Raw raw[N];
    uint32_t a = 0;
    const T* src = x + m0 * ldx + k;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        raw[i] = F8Raw{};
        if (k < K && m0 + i * ROWS < M) raw[i] = f8_ld32<true>(src, wide);
        src += ROWS * ldx;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        float v[V];
        F8In<T>::unpack(raw[i], v);
        a = max(a, f8_absmax<V>(v));
    }
    a = __reduce_max_sync(0xffffffffu, a);
    if ((tid & 31) == 0) wmax[tid >> 5] = a;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 8; ++w) a = max(a, wmax[w]);
    const uint32_t e = f8_scale_byte(a);
    const float r = f8_inverse(e);
    unsigned char* dst = codes + m0 * K + k;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        float v[V];
        F8In<T>::unpack(raw[i], v);
        if (k < K && m0 + i * ROWS < M) f8_store_codes<V>(dst, v, r);
        dst += (int64_t)ROWS * K;
    }
    const int width = (int)f8_scale_width(K);
    unsigned char* row = scales + (long long)blockIdx.y * width;
    if (tid == 0) row[blockIdx.x] = (unsigned char)e;
    if (blockIdx.x + 1 == gridDim.x && tid > 0 && (int)blockIdx.x + tid < width) row[blockIdx.x + tid] = 0;  // at most 3
}

// Codes and scales -> bf16 [M, K].  A warp takes 2048 columns of a row, a lane 16 neighbouring ones at a time: 32 bytes of
// output (4096 x 11008: 22.8 us, 5.9 TB/s; 16 bytes of codes a warp's lane at a time, stored in two halves, 39).  `shift`: log2 of a
// block's rows.
constexpr int kF8ExpandPart = 2048;
__global__ void __launch_bounds__(256) expand_f8_kernel(const unsigned char* __restrict__ codes, const unsigned char* __restrict__ scales,
                                                        int K, int parts, long long items, int shift, int signal, int wide,
                                                        uint16_t* __restrict__ out)
{
    constexpr int N = kF8ExpandPart / 512;
    if (signal) pdl_launch_dependents();
    pdl_wait();
    const long long it = (long long)blockIdx.x * 8 + threadIdx.x / 32;
    if (it >= items) return;
    const long long m = it / parts;
    const int k0 = (int)(it - m * parts) * kF8ExpandPart + 16 * (threadIdx.x & 31);
    const unsigned char *row = scales + (m >> shift) * f8_scale_width(K), *src = codes + m * K + k0;
    uint4 c[N];
    uint32_t e[N];
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (k0 + 512 * i < K) {
            c[i] = __ldcg(reinterpret_cast<const uint4*>(src + 512 * i));
            e[i] = __ldcg(row + (k0 + 512 * i) / kF8Block);
        }
    uint16_t* dst = out + m * K + k0;
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (k0 + 512 * i < K) {
            const float s = f8_scale(e[i]);
            const uint32_t u[4] = {c[i].x, c[i].y, c[i].z, c[i].w};
            uint32_t w[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) w[2 * j] = f8_values2(u[j], s), w[2 * j + 1] = f8_values2(u[j] >> 16, s);
            f8_st32(dst + 512 * i, w, wide);
        }
}

// ------------------------------------------------------------------ RMSNorm with the residual's addition, into 8 bits
// x' = x + d rounded to x's type, y = x' / sqrt(mean x'^2 + eps) * gain.  Squares are added in 64 bits (exact products, so that the sum's
// error is nothing beside a rounding to fp32, and no row's squares overflow or vanish); the rest is fp32, off by 4.5 2^-24: the mean's rounding,
// halved by the root, and those of root, reciprocal and two products.  Where the mean is not a normal number of fp32, x' is
// multiplied by p, a power of two, and the mean by p^2.  A CTA
// takes a row; with NV > 0 a thread keeps its NV pieces of it in registers, else (rows too long for that) x' is read again,
// from x_out where it was written.  d and x_out may be null, x_out may be x or d.  Bound by memory and, since the borders
// are checked, by registers: 4096 x 4096, fp32 x and bf16 d 37.1 us, 5.0 TB/s (36.8 with squares in
// fp32; without the check 31.5; that with 16-byte accesses 41); one row 2.8 us, a launch.
__device__ __forceinline__ float f8_norm_exact(float x, float g, double mean) { return f8_odd((double)x * (1.0 / sqrt(mean)) * (double)g); }
template <typename T, typename TD, int NV>
__global__ void __launch_bounds__(NV >= 4 ? 512 : 1024)
rmsnorm_f8_kernel(const T* x, int64_t ldx, const TD* d, int64_t ldd, T* x_out, int64_t ldo, const uint16_t* gain, int D, double inv_D, float eps, int wide,
                  unsigned char* __restrict__ codes, unsigned char* __restrict__ scales)
{
    constexpr int V = F8In<T>::V, KEEP = NV > 0 ? NV : 1;
    __shared__ double part[32];
    pdl_launch_dependents();
    pdl_wait();
    const int tid = threadIdx.x, T0 = blockDim.x;
    const long long m = blockIdx.x;
    x += m * ldx;
    if (d) d += m * ldd;
    if (x_out) x_out += m * ldo;
    const int width = (int)f8_scale_width(D), cover = width * kF8Block;  // columns with a scale byte
    auto fetch = [&](int k, float (&v)[V]) {
        F8In<T>::unpack(f8_ld32(x + k, wide), v);
        if (d) {
            float a[V];
            if constexpr (F8In<TD>::V == V) {
                F8In<TD>::unpack(f8_ld32(d + k, wide), a);
            } else if constexpr (V == 16) {  // fp32 d for bf16 x
                float lo[8], hi[8];
                F8In<float>::unpack(f8_ld32(d + k, wide), lo);
                F8In<float>::unpack(f8_ld32(d + k + 8, wide), hi);
#pragma unroll
                for (int j = 0; j < 8; ++j) a[j] = lo[j], a[8 + j] = hi[j];
            } else {
                const uint4 u = __ldcg(reinterpret_cast<const uint4*>(d + k));
                a[0] = bf16lo(u.x), a[1] = bf16hi(u.x), a[2] = bf16lo(u.y), a[3] = bf16hi(u.y);
                a[4] = bf16lo(u.z), a[5] = bf16hi(u.z), a[6] = bf16lo(u.w), a[7] = bf16hi(u.w);
            }
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = F8In<T>::kept(v[j] + a[j]);
        }
    };
    float v[KEEP][V];
    double ss = 0, ss1 = 0;  // two chains
    auto square = [&](const float (&u)[V]) {
#pragma unroll
        for (int j = 0; j < V; j += 2) {
            ss = fma((double)u[j], (double)u[j], ss);
            ss1 = fma((double)u[j + 1], (double)u[j + 1], ss1);
        }
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
            if (x_out && k < D) F8In<T>::store(x_out + k, v[i], wide);
            square(v[i]);
        }
    } else {
        for (int k = tid * V; k < D; k += T0 * V) {
            fetch(k, v[0]);
            if (x_out) F8In<T>::store(x_out + k, v[0], wide);
            square(v[0]);
        }
    }
    ss += ss1;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    if ((tid & 31) == 0) part[tid >> 5] = ss;
    __syncthreads();
    ss = (tid & 31) < T0 / 32 ? part[tid & 31] : 0.0;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    const double mean = ss * inv_D + (double)eps;
    const float p = mean > 0x1p127 ? 0x1p-65f : mean < 0x1p-126 ? 0x1p100f : 1.f;
    const float r = 1.0f / sqrtf((float)(mean * p * p));
    auto exact = [=](int k) {
        float u = F8In<T>::load(x_out ? x_out + k : x + k);
        if (!x_out && d) u = F8In<T>::kept(u + F8In<TD>::load(d + k));
        return f8_norm_exact(u, bf16f(gain[k]), mean);
    };
    auto finish = [&](int k, float (&u)[V]) {  // whole warps
        if (p != 1.f)
#pragma unroll
            for (int j = 0; j < V; ++j) u[j] *= p;
        if (k < D) {
#pragma unroll
            for (int j = 0; j < V; j += 8) {
                const uint4 g = ld_reuse16(gain + k + j);
                const uint32_t w[4] = {g.x, g.y, g.z, g.w};
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    u[j + 2 * q] = u[j + 2 * q] * r * bf16lo(w[q]);
                    u[j + 2 * q + 1] = u[j + 2 * q + 1] * r * bf16hi(w[q]);
                }
            }
        }
        f8_store_row_part<V, 6>(u, k - V * (tid & 31), D, width, codes + m * D, scales + m * width, exact);
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
                if (x_out) F8In<T>::unpack(f8_ld32(x_out + k, wide), v[0]);  // this thread wrote it
                else fetch(k, v[0]);
            }
            finish(k, v[0]);
        }
    }
}

// ------------------------------------------------------------------ SwiGLU into 8 bits
// y = gate / (1 + exp(-gate)) * up.  exp(-g) = 2^t (1 + d ln 2), t = -g log2 e rounded down, d what it was rounded by (the product's
// error, which the fma gives exactly, and that of log2 e), so that the exponential is off by little more than ex2.approx,
// 2^-22 of its value; in all y is off by 10 2^-24 of its value.  (With expf and a division the kernel issued 2.75 instructions a cycle and took
// 86 us, 4096 x 11008 bf16.)  From t = 126 on (gates below -87.3) the
// reciprocal is not a normal number and counts as 0.
// d is held to 0 .. 1, which costs nothing: of far gates t overflows, or is rounded by more than it may be.  As t is rounded down, d is
// negative only for positive gates, by log2 e's part: with exp(-g) beside 1 that is less than 2^-27 of y.
// The reciprocal is multiplied by up first: that cannot overflow, and the bits it loses below the normal numbers are below the
// codes'; half of a subnormal gate would lose bits that count.
__device__ __forceinline__ float f8_silu_times(float g, float u)
{
    const float c = -1.44269502e+00f, c_lo = -1.92596299e-08f, ln2 = 0.693147182f;  // -log2 e in two parts
    const float t = __fmul_rd(g, c), d = __saturatef(fmaf(g, c_lo, fmaf(g, c, -t)));  // of a NaN: 0
    float e, r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(fminf(t, 127.f)));
    e = fmaf(e, d * ln2, e);
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + e));
    return g * (r * u);
}
__device__ __forceinline__ float f8_silu_exact(float g, float u)
{
    const double q = 1.0 + exp(-(double)g);
    return f8_odd((q > 0x1p126 ? (double)g * 0.0 : (double)g / q) * (double)u);
}
// A warp takes 32 V features of a row at a time, and loads its next piece before it works on this one: the check of the borders
// leaves 32 warps an SM, whose loads alone would not cover the memory's latency (4096 x 11008 bf16: 51 us without, 46.4 with (46.8 since
// far gates are right); unrolled twice 50).  4.8 TB/s; without the check 39, 5.8.
template <typename T>
__global__ void __launch_bounds__(256, 4) swiglu_f8_kernel(const T* __restrict__ gate, const T* __restrict__ up, int64_t ld, int M, int F,
                                                           int parts, int dm, int dp, int wide, unsigned char* __restrict__ codes,
                                                           unsigned char* __restrict__ scales)
{
    constexpr int V = F8In<T>::V, STEP = 32 * V;
    pdl_launch_dependents();
    pdl_wait();
    const int it = blockIdx.x * 8 + threadIdx.x / 32, lane = threadIdx.x & 31, width = parts * STEP / kF8Block;
    uint32_t m = it / parts;  // m1 may pass 2^31
    int p = it - (int)m * parts;
    F8Raw g, u;
    auto load = [&](uint32_t m, int p, F8Raw& g, F8Raw& u) {
        const int k = p * STEP + V * lane;
        g = u = F8Raw{};
        if (m < (uint32_t)M && k < F) {
            g = f8_ld32<true>(gate + m * ld + k, wide);
            u = f8_ld32<true>(up + m * ld + k, wide);
        }
    };
    load(m, p, g, u);
#pragma unroll 1
    while (m < (uint32_t)M) {
        F8Raw g1, u1;
        uint32_t m1 = m + dm;
        int p1 = p + dp;
        if (p1 >= parts) ++m1, p1 -= parts;
        load(m1, p1, g1, u1);
        float a[V], b[V];
        F8In<T>::unpack(g, a);
        F8In<T>::unpack(u, b);
#pragma unroll
        for (int j = 0; j < V; ++j) a[j] = f8_silu_times(a[j], b[j]);
        const T *gm = gate + m * ld, *um = up + m * ld;
        auto exact = [=](int k) { return f8_silu_exact(F8In<T>::load(gm + k), F8In<T>::load(um + k)); };
        f8_store_row_part<V, 12>(a, p * STEP, F, width, codes + (int64_t)m * F, scales + (int64_t)m * width, exact);
        m = m1, p = p1, g = g1, u = u1;
    }
}

}  // namespace ls
