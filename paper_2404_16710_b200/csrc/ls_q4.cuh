// The 4-bit number format that the packed weights and the 4-bit KV cache share, and the kernels that only
// convert: weights and cache rows to 4 bits and back.  (LayerSkip keeps weights and cache in 16 bits; what
// bounds its decode loop is the bytes of both, which this format cuts by 3.5.)
//
// A group of values x shares a scale s; a value stands for c * s with an integer code c in -7..7:
//   a = max |x|,  s = a / 7 rounded UP to 5 significant bits,  c = rint(x / s), ties to even.
// s is kept as bf16.  A code has 3 significant bits, so c * s has at most 8: it IS a bf16 number, and the
// bf16 operators (the prompt pass) see on expanded data exactly the values the 4-bit operators use.  The
// price is a step up to 6 % wider (3 % on average) than a / 7.  Codes decide exactly in fp32: x has 8
// significant bits and a border (k + 1/2) s at most 9, so x / s either is k + 1/2 or differs from it by at least
// 2^-17 of its value, 2^-18 or more.
// Ends of the range: s = 0 (all codes 0) if a = 0; s >= 2^-126, so that c * s never is a subnormal number;
// s <= 1.125 * 2^125, so that 7 s is finite.  A group with a NaN or an infinity gets a NaN scale and stands
// for NaN.  A nibble holds c + 8.
//
// Rows of 128 values (64 for a cache of head dim 64) are stored in the order in which mma.sync m16n8k16
// wants its A operand: lane 4 g + t of a warp owns row g and needs, per group of 32 columns, 8 of them.
// The 16-byte piece t of a row holds columns 32 j + 8 t .. + 7 for j = 0..3, one 32-bit word each, so a
// lane reads all its codes with one 16-byte access and a warp's accesses are contiguous.  Inside a word
// column e of the eight sits at nibble e / 2 + 4 (e % 2): (word >> 4 i) & 0x000f000f leaves columns 2 i and
// 2 i + 1 in the two halves of a register.
#pragma once
#include "ls_common.cuh"

namespace ls {

constexpr int kQ4Rows = 16;                  // rows of a block of weights, tokens of a tile of the cache
constexpr int kQ4Cols = 128;                 // columns of a block of weights
constexpr int kQ4CodeBytes = kQ4Rows * kQ4Cols / 2;
enum : int { DEV_BAD_PAGE = 4 };             // a page-table entry outside the pool (beside DevStatus)

// bytes of a block of 16 rows x 128 columns of weights: codes, then scales [16][128 / group]
__host__ __device__ constexpr int w4_block_bytes(int ng) { return kQ4CodeBytes + kQ4Rows * ng * 2; }
// bytes of a tile of 16 tokens of one KV head: K codes, K scales [16][hd / 32], V codes, V scales [hd / 32][16]
__host__ __device__ constexpr int kv4_tile_bytes(int hd) { return kQ4Rows * (hd + hd / 8); }

// scale of a group whose largest |x| has the bf16 bits amax (sign bit clear)
__device__ __forceinline__ float q4_scale(uint32_t amax)
{
    // a / 7 from below: a has 8 significant bits, so a / 7 either has 5 or is farther than 2^-11 of its value
    // from every number that does, and a product short of it by less than 2^-19 rounds up to the same one
    const float q = __uint_as_float(amax << 16) * 0.14285700f;
    // up to the next multiple of 2^19 ulps: 4 of the 23 mantissa bits stay
    float s = __uint_as_float((__float_as_uint(q) + 0x7ffffu) & ~0x7ffffu);
    s = fminf(fmaxf(s, 0x1p-126f), 1.125f * 0x1p125f);
    if (amax == 0) s = 0.f;
    return amax >= 0x7f80u ? __uint_as_float(0x7fff0000u) : s;  // an infinity or a NaN in the group
}
// 1 / s to within an ulp; 0 for s = 0 or NaN: every code is then 0
__device__ __forceinline__ float q4_rcp(float s)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(s));
    return s > 0.f ? r : 0.f;
}
// A float whose bits are kQ4Base + u, u = c + 8, for the bf16 value v; r = q4_rcp(s).  v r + 24 is rounded to a multiple
// of 2^-19: the product is off by at most 7.1 * 2^-23 < 2^-20, so what lies on a border (k + 1/2) comes out on
// it, and what does not lies at least 2^-18 off and stays off.  Adding 3 * 2^22 then rounds to an integer, borders
// to the even one, and leaves 24 + c in the low bits.
constexpr uint32_t kQ4Base = 0x4b400000u + 16u;
__device__ __forceinline__ uint32_t q4_code_bits(float v, float r)
{
    return __float_as_uint(__fadd_rn(__fmaf_rn(v, r, 24.f), 12582912.f));
}

__device__ __forceinline__ uint32_t absmax_bf16x2(uint32_t m, uint32_t w)  // bits, not values: NaN counts as largest
{
    return max(m, max(w & 0x7fffu, (w >> 16) & 0x7fffu));
}
__device__ __forceinline__ uint32_t absmax8(const uint4& v)
{
    return absmax_bf16x2(absmax_bf16x2(absmax_bf16x2(absmax_bf16x2(0, v.x), v.y), v.z), v.w);
}
// Codes of 8 values as a word, value e at nibble e / 2 + 4 (e % 2) (ROW) or e: the sum of the codes' bits in their places,
// less what kQ4Base adds to each.  Under a NaN scale all codes are 0.
template <bool ROW>
__device__ __forceinline__ uint32_t q4_word8(const uint4& v, float s, float r)
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    uint32_t word = 0u - kQ4Base * 0x11111111u;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int pos = ROW ? e / 2 + 4 * (e % 2) : e;
        word += q4_code_bits(e & 1 ? bf16hi(w[e / 2]) : bf16lo(w[e / 2]), r) << (4 * pos);
    }
    return s == s ? word : 0x88888888u;
}
__device__ __forceinline__ uint32_t q4_word(const uint4& v, float s, float r) { return q4_word8<true>(v, s, r); }         // a row's
__device__ __forceinline__ uint32_t q4_word_plain(const uint4& v, float s, float r) { return q4_word8<false>(v, s, r); }  // lowest first (V)

// Floats are made of nibbles by or-ing them into the mantissa of a power of two and subtracting it, a published method
// (for 4-bit weights e.g. Kim et al. 2022, arXiv 2211.10017); the constants follow from the formats.
// codes i and i + 4 of a word as two bf16 numbers c (exact): 0x4300 | u is 128 + u
__device__ __forceinline__ uint32_t q4_bf16x2(uint32_t w, int i)
{
    uint32_t r;
    asm("lop3.b32 %0, %1, 0x000f000f, 0x43004300, 0xea;" : "=r"(r) : "r"(w >> (4 * i)));
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(r), "r"(0x43084308u));  // - 136
    return r;
}
// codes of nibbles 0 (i = 0) or 1 (i = 1) of the two halves of w as f16 numbers c (exact), which has bits enough for both
__device__ __forceinline__ uint32_t q4_f16x2(uint32_t w, int i)
{
    uint32_t r;
    if (i == 0) {
        asm("lop3.b32 %0, %1, 0x000f000f, 0x64006400, 0xea;" : "=r"(r) : "r"(w));
        asm("add.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(r), "r"(0xe408e408u));  // 1024 + u - 1032
    } else {
        asm("lop3.b32 %0, %1, 0x00f000f0, 0x64006400, 0xea;" : "=r"(r) : "r"(w));
        asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(r), "r"(0x2c002c00u), "r"(0xd480d480u));  // (1024 + 16 u) / 16 - 72
    }
    return r;
}
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// the 8 values a row word stands for, in column order; s2: the scale in both halves
__device__ __forceinline__ uint4 q4_values(uint32_t w, uint32_t s2)
{
    return make_uint4(mul_bf16x2(q4_bf16x2(w, 0), s2), mul_bf16x2(q4_bf16x2(w, 1), s2),
                      mul_bf16x2(q4_bf16x2(w, 2), s2), mul_bf16x2(q4_bf16x2(w, 3), s2));
}

// D (fp32, 16x8) = A (f16, 16x16) * B (f16, 16x8) + C
__device__ __forceinline__ void mma_f16_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                              uint32_t b0, uint32_t b1, float c0, float c1, float c2, float c3)
{
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
        "{%10,%11,%12,%13};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c0), "f"(c1), "f"(c2), "f"(c3));
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// Coherent loads of data that the kernel before this one may have written, under programmatic dependent launch after this one's
// CTAs had started (ld_reuse16 says why): positions and page tables, and what is read once, from L2.
__device__ __forceinline__ int ld_now(const int32_t* p)
{
    int v;
    asm volatile("ld.global.b32 %0, [%1];" : "=r"(v) : "l"(p));
    return v;
}
template <typename T>
__device__ __forceinline__ T ld_once(const void* p)
{
    return __ldcg(reinterpret_cast<const T*>(p));
}

// ------------------------------------------------------------------ weights: bf16 -> blocks, blocks -> bf16
// Both are bound by memory: 11008 x 4096, packed and expanded again: 39 us (0.80 of the measured copy rate), 4096 x 4096: 19.4
// (0.60), in four launches: fence_kernel follows either and takes 0.8 us.  A code costs about 5 instructions; with a
// division, floor and comparison each (16, two of them on the quarter-rate conversion pipe) the latter took 8 us more.
// One warp per block of 16 rows x 128 columns: lane 4 g + t holds rows g and g + 8, columns 32 j + 8 t .. + 7.
// NG groups of 128 / NG columns per block.  grid.x * warps covers the blocks of all rows, row blocks slowest.
template <int NG>
__global__ void __launch_bounds__(256) quantize_w4_kernel(const uint16_t* __restrict__ w, int N, int K, int kblocks,
                                                          long long blocks, unsigned char* __restrict__ packed)
{
    pdl_wait();
    const long long blk = (long long)blockIdx.x * (blockDim.x / 32) + threadIdx.x / 32;
    if (blk >= blocks) return;  // whole warps
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const long long n0 = blk / kblocks * kQ4Rows;
    const int k0 = (int)(blk % kblocks) * kQ4Cols;
    unsigned char* dst = packed + blk * w4_block_bytes(NG);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const long long n = n0 + g + 8 * half;
        uint4 v[4];
        uint32_t am[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int k = k0 + 32 * j + 8 * t;
            v[j] = make_uint4(0, 0, 0, 0);
            if (n < N && k < K) v[j] = ld_once<uint4>(w + n * K + k);  // K is a multiple of 8: the octet is in or out
            am[j] = absmax8(v[j]);
        }
        if (NG <= 2) am[0] = am[1] = max(am[0], am[1]), am[2] = am[3] = max(am[2], am[3]);
        if (NG == 1) am[0] = am[1] = am[2] = am[3] = max(am[0], am[2]);
        uint32_t words[4], sc[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            am[j] = max(am[j], __shfl_xor_sync(0xffffffffu, am[j], 1));
            am[j] = max(am[j], __shfl_xor_sync(0xffffffffu, am[j], 2));
            const float s = q4_scale(am[j]), r = q4_rcp(s);
            sc[j] = __float_as_uint(s) >> 16;
            words[j] = q4_word(v[j], s, r);
        }
        *reinterpret_cast<uint4*>(dst + half * (kQ4CodeBytes / 2) + lane * 16) =
            make_uint4(words[0], words[1], words[2], words[3]);
        if (t == 0) {
            unsigned char* sd = dst + kQ4CodeBytes + (g + 8 * half) * NG * 2;
            if (NG == 4) *reinterpret_cast<uint2*>(sd) = make_uint2(sc[0] | sc[1] << 16, sc[2] | sc[3] << 16);
            if (NG == 2) *reinterpret_cast<uint32_t*>(sd) = sc[0] | sc[2] << 16;
            if (NG == 1) *reinterpret_cast<uint16_t*>(sd) = (uint16_t)sc[0];
        }
    }
}

// Does nothing.  Launched without the attribute behind what writes weights: it starts when they are written and visible,
// and the next operation's early reads of weights start after it.
__global__ void fence_kernel() {}

// scales of one row of a block in both halves of a register each, group by group
template <int NG>
__device__ __forceinline__ void q4_row_scales(const unsigned char* sd, uint32_t (&s2)[NG])
{
    if (NG == 4) {
        const uint2 v = ld_once<uint2>(sd);
        s2[0] = __byte_perm(v.x, 0, 0x1010), s2[1 % NG] = __byte_perm(v.x, 0, 0x3232);
        s2[2 % NG] = __byte_perm(v.y, 0, 0x1010), s2[3 % NG] = __byte_perm(v.y, 0, 0x3232);
    } else if (NG == 2) {
        const uint32_t v = ld_once<uint32_t>(sd);
        s2[0] = __byte_perm(v, 0, 0x1010), s2[1 % NG] = __byte_perm(v, 0, 0x3232);
    } else {
        const uint32_t v = ld_once<uint16_t>(sd);
        s2[0] = __byte_perm(v, 0, 0x1010);
    }
}

template <int NG>
__global__ void __launch_bounds__(256) expand_w4_kernel(const unsigned char* __restrict__ packed, int N, int K,
                                                        int kblocks, long long blocks, uint16_t* __restrict__ out)
{
    pdl_wait();
    const long long blk = (long long)blockIdx.x * (blockDim.x / 32) + threadIdx.x / 32;
    if (blk >= blocks) return;
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const long long n0 = blk / kblocks * kQ4Rows;
    const int k0 = (int)(blk % kblocks) * kQ4Cols;
    const unsigned char* src = packed + blk * w4_block_bytes(NG);
    uint4 c[2];
    uint32_t s2[2][NG];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        c[half] = ld_once<uint4>(src + half * (kQ4CodeBytes / 2) + lane * 16);
        q4_row_scales<NG>(src + kQ4CodeBytes + (g + 8 * half) * NG * 2, s2[half]);
    }
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const long long n = n0 + g + 8 * half;
        const uint32_t words[4] = {c[half].x, c[half].y, c[half].z, c[half].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int k = k0 + 32 * j + 8 * t;
            if (n < N && k < K) *reinterpret_cast<uint4*>(out + n * K + k) = q4_values(words[j], s2[half][j * NG / 4]);
        }
    }
}

// ------------------------------------------------------------------ cache: bf16 rows -> tiles, tiles -> bf16 pages
// Where position p of sequence b lives: the tile's first byte, or null (with a status) if the position or
// the page-table entry is out of range.
struct Kv4Cache {
    const int32_t* table;  // [n_seq][table_stride]
    int table_stride, page_shift, max_seq, n_pages, Hkv;
};
template <int HD>
__device__ __forceinline__ long long kv4_tile_offset(const Kv4Cache& c, int page, int p, int head)
{
    const int tiles = 1 << (c.page_shift - 4);  // tiles of a page and head
    return (((long long)page * c.Hkv + head) * tiles + ((p >> 4) & (tiles - 1))) * kv4_tile_bytes(HD);
}
__device__ __forceinline__ int kv4_entry(const Kv4Cache& c, int b, int p)
{
    return ld_now(c.table + (long long)b * c.table_stride + (p >> c.page_shift));
}
__device__ __forceinline__ int kv4_page(const Kv4Cache& c, int page, int32_t* status)
{
    if ((unsigned)page < (unsigned)c.n_pages) return page;
    if (status) *status = DEV_BAD_PAGE;
    return -1;
}
// position of row m of a sequence whose row 0 is at pos0: -1 (nothing to do) below 0, -1 and a status beyond the cache
__device__ __forceinline__ int kv4_position(int pos0, int m, int max_seq, int32_t* status)
{
    const long long p = (long long)pos0 + m;
    if (p < 0) return -1;
    if (p < max_seq) return (int)p;
    if (status) *status = DEV_POS_OVERFLOW;
    return -1;
}
// byte offset inside a tile of the V piece of channels (hd / 8) g .. of token i
template <int HD>
__device__ __forceinline__ int kv4_v_piece(int i, int g)
{
    return 9 * HD + ((((i >> 3) * 8 + g) * 4 + ((i >> 1) & 3)) * 2 + (i & 1)) * (HD / 16);
}

// A warp takes 8 rows of one head; lane 4 g + t row g: of K the columns 32 j + 8 t, of V the pieces t and
// t + 4.  grid (ceil(M / (8 warps)), Hkv, n_seq).  4096 rows of 8 heads, appended and expanded: 14.4 us in two launches
// (0.41 of the measured copy rate): one wave of CTAs, each behind the chain position, page, data; one row of 32 heads: 2.5 us.
template <int HD>
__global__ void __launch_bounds__(256) append_kv4_kernel(const uint16_t* __restrict__ k, const uint16_t* __restrict__ v,
                                                         long long seq_stride, long long row_stride, long long head_stride,
                                                         int M, const int32_t* __restrict__ pos0, const Kv4Cache cache,
                                                         unsigned char* __restrict__ pages, int32_t* status)
{
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3, head = blockIdx.y, b = blockIdx.z;
    const int m = (blockIdx.x * (blockDim.x / 32) + threadIdx.x / 32) * 8 + g;
    constexpr int G = HD / 32, O = HD / 64;  // groups of a row, octets of a V piece
    // the first loads are all on their way before the first is used
    const int start = ld_now(pos0 + b);
    const long long at = b * seq_stride + (long long)m * row_stride + head * head_stride;
    uint4 xk[G], xv[2][O];
#pragma unroll
    for (int j = 0; j < G; ++j) xk[j] = m < M ? ld_once<uint4>(k + at + 32 * j + 8 * t) : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int o = 0; o < O; ++o)
            xv[h][o] = m < M ? ld_once<uint4>(v + at + (t + 4 * h) * (HD / 8) + 8 * o) : make_uint4(0, 0, 0, 0);
    const int p = m < M ? kv4_position(start, m, cache.max_seq, status) : -1;
    const int page = p >= 0 ? kv4_page(cache, kv4_entry(cache, b, p), status) : -1;  // -1: the row is left out, its lanes stay for the shuffles
    unsigned char* tile = pages + (page >= 0 ? kv4_tile_offset<HD>(cache, page, p, head) : 0);
    const int i = p & 15;
    {
        uint32_t words[G], sc[G];
#pragma unroll
        for (int j = 0; j < G; ++j) {
            uint32_t am = absmax8(xk[j]);
            am = max(am, __shfl_xor_sync(0xffffffffu, am, 1));
            am = max(am, __shfl_xor_sync(0xffffffffu, am, 2));
            const float s = q4_scale(am), r = q4_rcp(s);
            sc[j] = __float_as_uint(s) >> 16;
            words[j] = q4_word(xk[j], s, r);
        }
        if (page >= 0) {
            unsigned char* cd = tile + i * (HD / 2) + t * (HD / 8);
            unsigned char* sd = tile + 8 * HD + i * (HD / 16);
            if (HD == 128) {
                *reinterpret_cast<uint4*>(cd) = make_uint4(words[0], words[1], words[2 % G], words[3 % G]);
                if (t == 0) *reinterpret_cast<uint2*>(sd) = make_uint2(sc[0] | sc[1] << 16, sc[2 % G] | sc[3 % G] << 16);
            } else {
                *reinterpret_cast<uint2*>(cd) = make_uint2(words[0], words[1]);
                if (t == 0) *reinterpret_cast<uint32_t*>(sd) = sc[0] | sc[1] << 16;
            }
        }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int piece = t + 4 * h;  // of HD / 8 channels: two pieces to a group (HD = 128) or four
        uint32_t am = absmax8(xv[h][0]);
        if (O == 2) am = max(am, absmax8(xv[h][O - 1]));
        am = max(am, __shfl_xor_sync(0xffffffffu, am, 1));
        if (HD == 64) am = max(am, __shfl_xor_sync(0xffffffffu, am, 2));
        const float s = q4_scale(am), r = q4_rcp(s);
        if (page < 0) continue;
        unsigned char* cd = tile + kv4_v_piece<HD>(i, piece);
        const uint32_t w0 = q4_word_plain(xv[h][0], s, r);
        if (O == 2)
            *reinterpret_cast<uint2*>(cd) = make_uint2(w0, q4_word_plain(xv[h][O - 1], s, r));
        else
            *reinterpret_cast<uint32_t*>(cd) = w0;
        const int grp = piece * (HD / 8) / 32;
        if (piece * (HD / 8) % 32 == 0)
            *reinterpret_cast<uint16_t*>(tile + 17 * HD + (grp * 16 + i) * 2) = (uint16_t)(__float_as_uint(s) >> 16);
    }
}

// The same lanes the other way round, to pages [page][Hkv][page_size][hd] of a bf16 cache with a table of its own.
template <int HD>
__global__ void __launch_bounds__(256) expand_kv4_kernel(const unsigned char* __restrict__ pages, int M,
                                                         const int32_t* __restrict__ pos0, const Kv4Cache cache,
                                                         const Kv4Cache dst, uint16_t* __restrict__ kp,
                                                         uint16_t* __restrict__ vp, int32_t* status)
{
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3, head = blockIdx.y, b = blockIdx.z;
    const int m = (blockIdx.x * (blockDim.x / 32) + threadIdx.x / 32) * 8 + g;
    if (m >= M) return;
    const int p = kv4_position(ld_now(pos0 + b), m, cache.max_seq, status);
    if (p < 0) return;
    const int entry = kv4_entry(cache, b, p), to_entry = kv4_entry(dst, b, p);
    const int page = kv4_page(cache, entry, status), to = kv4_page(dst, to_entry, status);
    if (page < 0 || to < 0) return;
    const unsigned char* tile = pages + kv4_tile_offset<HD>(cache, page, p, head);
    const int slot = p & ((1 << cache.page_shift) - 1), i = p & 15;
    const long long at = ((((long long)to * cache.Hkv + head) << cache.page_shift) + slot) * HD;
    constexpr int G = HD / 32;
    uint32_t s2[G], words[G];
    q4_row_scales<G>(tile + 8 * HD + i * (HD / 16), s2);
    const unsigned char* cd = tile + i * (HD / 2) + t * (HD / 8);
    if (HD == 128) {
        const uint4 c = ld_once<uint4>(cd);
        words[0] = c.x, words[1] = c.y, words[2 % G] = c.z, words[3 % G] = c.w;
    } else {
        const uint2 c = ld_once<uint2>(cd);
        words[0] = c.x, words[1] = c.y;
    }
    uint32_t sv[2], wv[2][HD / 64];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int piece = t + 4 * h;
        sv[h] = ld_once<uint16_t>(tile + 17 * HD + (piece * (HD / 8) / 32 * 16 + i) * 2);
#pragma unroll
        for (int o = 0; o < HD / 64; ++o) wv[h][o] = ld_once<uint32_t>(tile + kv4_v_piece<HD>(i, piece) + 4 * o);
    }
#pragma unroll
    for (int j = 0; j < G; ++j) *reinterpret_cast<uint4*>(kp + at + 32 * j + 8 * t) = q4_values(words[j], s2[j]);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t s = __byte_perm(sv[h], 0, 0x1010);
#pragma unroll
        for (int o = 0; o < HD / 64; ++o) {
            // lowest nibble first -> the row order of q4_values: even columns to nibbles 0..3, odd to 4..7
            uint32_t e = 0;
#pragma unroll
            for (int n = 0; n < 4; ++n) e |= ((wv[h][o] >> (8 * n)) & 0xfu) << (4 * n) | ((wv[h][o] >> (8 * n + 4)) & 0xfu) << (4 * n + 16);
            *reinterpret_cast<uint4*>(vp + at + (t + 4 * h) * (HD / 8) + 8 * o) = q4_values(e, s);
        }
    }
}

}  // namespace ls
