// Attention over a KV cache held in 4 bits (format and tile layout: ls_q4.cuh): the draft and verify passes
// of LayerSkip Sec. 4.3.3 for one or several sequences, up to 16 rows each.
//
//   o[m] = sum_i p_i v_i / sum_i p_i,  p_i = exp(q[m] . k_i / sqrt(hd)) for the positions i <= pos0 + m
//
// Tokens are the 16-row operand of mma.sync in both products, queries (row, head of the KV group) the
// 8-column one: S^T = K Q^T and O^T = V^T P^T.  At 4 bits a value the kernel is bound by the instructions
// that turn nibbles into operands, so both products run in f16, whose formats make those few:
// * K: a nibble u = c + 8 or-ed to 1024 is 1024 + u (bits 0..3) or 1024 + 16 u (bits 4..7), and one instruction makes
//   c of it: 9 instructions for 8 codes, 11 in bf16, which has too few bits for the second kind.  (The bare nibble is
//   an f16 denormal, u 2^-24, that the tensor cores multiply without any conversion -- but they align products by
//   exponent fields, and sums of denormals came out with an error of 2^-20 instead of 2^-24.)  Queries are scaled by
//   powers of two of their own so that the largest component is in [2^14, 2^15): what f16 then cannot hold is 2^-39 of it.
// * V: a nibble moved to bits 4..7 or-ed to 1024 is 1024 + 16 u, and one multiply-add makes c s of it:
//   (1024 + 16 u) (s / 16) - 72 s.  A scale has 5 significant bits, so every step is exact, for scales down to 2^-23
//   of the largest one that the warp has met in the channel group (a lane's channels are of one group, and the power of
//   two it divides by is its own); what is smaller still is off by less than 2^-21 of that one.
// * p is rounded to f16's 11 bits (2^-12 of it), well below the rounding of a bf16 result.  2^7 p stands in f16: p is at most
//   2^8 and the largest so far 1 or more, so that weights keep those bits down to 2^-21 and are off by 2^-32 below, which
//   thousands of positions beside one that outweighs them by 2^25 need.  Scores, maxima, sums and O are fp32.
// Some 360 instructions go into a tile of 16 tokens of one KV head (2304 bytes) and up to 8 queries, all else included, 85
// more for each further 8; two CTAs of 8 warps an SM issue 2.4 of them a cycle.  131072 tokens, 8 KV heads: 42.4 us (0.54 of
// the measured copy rate; first form 130); 1030 tokens, 32 heads: 6.9 us, of which the launch is 1.4, the first loads and
// the queries 2, a chunk 1.4, joining the warps and CTAs 2.  With 25 to 32 queries of head size 128 a thread has 255 registers and
// spills 23 more (64 queries over 131072 tokens: 196 us).
#pragma once
#include "ls_attention.cuh"
#include "ls_w4.cuh"

namespace ls {

constexpr int kKv4Chunk = 32;   // positions a warp takes at a time: two tiles
constexpr int kKv4Warps = 8;
// How far beyond a V scale the unit goes that it raises: units are then raised rarely after a warp's first chunk (4103
// positions, 7 rows: 0.3 us of 11 less than with 0)
constexpr int kKv4Headroom = 1;
constexpr int kKv4WeightBits = 7;  // softmax weights are held times 2^7

__device__ __forceinline__ uint32_t movmatrix_trans(uint32_t a)
{
    uint32_t d;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
    return d;
}
__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// 2^e, 0 below the denormals
__device__ __forceinline__ float exp2_int(int e)
{
    if (e >= -126) return __uint_as_float((uint32_t)(min(e, 127) + 127) << 23);
    return e >= -149 ? __uint_as_float(1u << (e + 149)) : 0.f;
}
__device__ __forceinline__ void st_cluster_f4(uint32_t addr, float4 v)
{
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}
__device__ __forceinline__ uint32_t map_cluster(uint32_t addr, int rank)
{
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t fma_f16x2(uint32_t a, uint32_t b, uint32_t c)
{
    uint32_t r;
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
    return r;
}
// c s of nibble i of the two halves of w, as f16: s16 = s / 16, s72 = -72 s
__device__ __forceinline__ uint32_t q4_scaled_f16x2(uint32_t w, int i, uint32_t s16, uint32_t s72)
{
    uint32_t r;
    asm("lop3.b32 %0, %1, 0x00f000f0, 0x64006400, 0xea;" : "=r"(r) : "r"(i == 0 ? w << 4 : w >> (4 * i - 4)));
    return fma_f16x2(r, s16, s72);
}

// shared memory of a CTA: rings (later each warp's O in its own), queries and their factors, the
// warps' statistics, and what the CTAs of the cluster send one another
constexpr int kKv4MaxCluster = 8;
template <int HD, int NT>
struct Kv4Smem {
    static constexpr int W = kKv4Warps;
    // chunks of a warp's ring: no more than its O needs (16384 positions, 16 queries a head: 15.6 us with 2, 16.9 with 4)
    static constexpr int kStages = NT <= 2 ? 2 : NT;
    static constexpr int kTile = kv4_tile_bytes(HD);
    static constexpr int kWarpRing = kStages * 2 * kTile;
    static constexpr int kItems = NT * HD / 16 * 32;           // float4 pieces of O: [NT][HD / 16][lane]
    static constexpr int kRing = W * kWarpRing;
    static constexpr int kQ = NT * HD / 32 * 32 * 16;          // [NT][group][lane] 16 bytes
    static constexpr int kInbox = (kItems + kKv4MaxCluster) * 16;  // [CTA][a share of the pieces]
    static constexpr int kFactor = NT * 8 * 4;                 // 2^e [query]
    static constexpr int kStat = W * NT * 8 * 8 + W * HD / 32 * NT * 8 * 4;  // (max, sum) of the warps, units of their O
    static constexpr int kInStat = kKv4MaxCluster * NT * 8 * 8;  // (max, sum) of the CTAs
    static constexpr int kBytes = kRing + kQ + kInbox + kFactor + kStat + kInStat;
    static_assert(kItems / (NT * 32) * 512 * NT <= kWarpRing, "a warp's O fits its ring");
};

// where the results of split s of (sequence b, block row y of the grid) stand in the scratch memory
__device__ __forceinline__ long long kv4_partial(int b, int rows, int y, int splits, int s)
{
    return ((long long)b * rows + y) * splits + s;
}
// log2(e) / sqrt(hd), over the 2^14 that queries are scaled to
__device__ __forceinline__ float kv4_unit(int hd) { return 0x1p-14f * 1.4426950408889634f / sqrtf((float)hd); }

// grid (S times the splits, or a part of them, Hkv * query tiles, n_seq) in clusters of S CTAs.  The warps of a (sequence, KV head) take
// the 32-position chunks of the cache in turn by absolute position, each through a cp.async ring of its own and
// with a running (max, sum, O) of its own.  At the end every thread adds up, in warp order, the pieces of O it is
// given and sends them to the CTA of the cluster that finishes them, through distributed shared memory: one
// CTA barrier, one cluster barrier.  With one split that is the result; a GPC has room for few large clusters
// (148 SMs: 33 of 4 CTAs, 15 of 8, 7 of 16 where one fills an SM), so that few heads over a long cache take several splits,
// which a second kernel joins.  A row's result depends on its position and on the grid, not on M or the other
// rows: what other rows add to the tokens a CTA looks at has weight 0, and all factors that are shared are powers
// of two that lose nothing (where they would, a row has its own: `work`).
template <int HD, int NT>
__global__ void __launch_bounds__(kKv4Warps * 32, NT == 1 ? 2 : 1)
attention_kv4_kernel(const uint16_t* __restrict__ q, int M, int G, const int32_t* __restrict__ pos0_dev,
                     const Kv4Cache cache, const unsigned char* __restrict__ pages, int S, int n_splits, uint32_t div_S,
                     uint32_t div_G, uint32_t div_Hkv, uint16_t* __restrict__ out, float* __restrict__ scratch, int32_t* status)
{
    using SM = Kv4Smem<HD, NT>;
    constexpr int W = kKv4Warps;
    constexpr int NJ = HD / 32;   // groups of a row
    constexpr int CT = HD / 16;   // 16-channel tiles of O^T
    constexpr int TB = SM::kTile, D = SM::kStages;
    extern __shared__ __align__(128) unsigned char kv4_smem[];
    unsigned char* at = kv4_smem + SM::kRing;
    uint4* sQ = reinterpret_cast<uint4*>(at);
    float4* sIn = reinterpret_cast<float4*>(at += SM::kQ);
    float* sF = reinterpret_cast<float*>(at += SM::kInbox);
    float2* sStat = reinterpret_cast<float2*>(at += SM::kFactor);   // [W][NT * 8]
    float* sUnit = reinterpret_cast<float*>(sStat + W * NT * 8);     // [W][channel group][NT * 8]
    float2* sInStat = reinterpret_cast<float2*>(at += SM::kStat);   // [CTA][NT * 8]
    pdl_wait();
    const int splits = NT == 1 ? fastdiv(gridDim.x, S, div_S) : n_splits;
    const int first_split = fastdiv(blockIdx.x, S, div_S), rank = blockIdx.x - first_split * S, b = blockIdx.z;
    if (S > 1) cluster_arrive_relaxed();  // this CTA is there
    const int tile_y = fastdiv(blockIdx.y, cache.Hkv, div_Hkv), head = blockIdx.y - tile_y * cache.Hkv, q0 = tile_y * (NT * 8);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int Q = M * G, Hq = cache.Hkv * G;

    // The first accesses to memory, all before the first use of any (volatile: the compiler moves plain loads down to
    // their use, one latency after the other): this thread's piece of a query, the page-table entries of its warp's first
    // chunk, the position.
    constexpr int PER = NJ * 4, PIECES = (NT * 8 * PER + W * 32 - 1) / (W * 32);  // threads that make a query's operand; a thread's share
    uint4 piece[PIECES];
#pragma unroll
    for (int k = 0; k < PIECES; ++k) {
        const int i = threadIdx.x + k * W * 32, qi = q0 + i / PER, row = fastdiv(qi, G, div_G);
        piece[k] = make_uint4(0, 0, 0, 0);
        if (i < NT * 8 * PER && qi < Q)
            piece[k] = ld_reuse16(q + (((long long)b * M + row) * Hq + head * G + qi - row * G) * HD + 8 * (i % PER));
    }
    // page-table entries of this warp's next chunk (a chunk lies in one page, unless pages are of 16), read before
    // anything says whether it is needed: the positions below max_seq have entries
    const int step = (NT == 1 ? gridDim.x : splits * S) * W * kKv4Chunk;
    int split = first_split, base0 = (blockIdx.x * W + warp) * kKv4Chunk;
    const int32_t* table = cache.table + (long long)b * cache.table_stride;
    int next_page[2];
    auto look_up = [&](int base) {
        next_page[0] = next_page[1] = 0;
        if (base < cache.max_seq) next_page[0] = ld_now(table + (base >> cache.page_shift));
        if (cache.page_shift == 4 && base + 16 < cache.max_seq) next_page[1] = ld_now(table + ((base + 16) >> 4));
    };
    look_up(base0);
    const int pos0 = ld_now(pos0_dev + b);

    // last position that this lane's two queries of each 8 see, and over the CTA's queries that see any the last and the
    // first of those
    int lim[NT][2], top = -1, low = 0x7fffffff;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int qi = q0 + nt * 8 + 2 * t + e;
            lim[nt][e] = qi < Q ? kv4_position(pos0, fastdiv(qi, G, div_G), cache.max_seq, status) : -1;
            top = max(top, lim[nt][e]);
            if (lim[nt][e] >= 0) low = min(low, lim[nt][e]);
        }
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    low = min(low, __shfl_xor_sync(0xffffffffu, low, 1));
    low = min(low, __shfl_xor_sync(0xffffffffu, low, 2));

    // the ring: chunks of this warp, D - 1 ahead of their use.  ok_bits: which tiles of the chunks in flight exist
    const uint32_t ring = smem_u32(kv4_smem) + warp * D * 2 * TB;
    int in_base = base0, in_stage = 0, in_count = 0;
    uint32_t ok_bits = 0;
    const unsigned char* mine = pages + ((long long)head << (cache.page_shift - 4)) * TB + lane * 16;
    const uint32_t page_bytes = (uint32_t)(cache.Hkv << (cache.page_shift - 4)) * TB, tile_mask = (1u << (cache.page_shift - 4)) - 1;
    auto fetch = [&]() {
        if (in_base <= top) {
            const uint32_t dst = ring + in_stage * 2 * TB + lane * 16;
            auto source = [&](int p, int page) {
                return mine + (unsigned long long)page_bytes * (uint32_t)page + ((uint32_t)(p >> 4) & tile_mask) * TB;
            };
            if (in_base + 16 <= top && cache.page_shift > 4 && (unsigned)next_page[0] < (unsigned)cache.n_pages) {
                const unsigned char* src = source(in_base, next_page[0]);  // two tiles in a row
#pragma unroll
                for (int i = 0; i < 2 * TB / 512; ++i) cp_async16_cg(dst + 512 * i, src + 512 * i, 16);
                if (2 * TB % 512 && lane < 2 * TB % 512 / 16) cp_async16_cg(dst + 2 * TB / 512 * 512, src + 2 * TB / 512 * 512, 16);
                ok_bits |= 3u << (2 * in_count);
            } else {
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int p = in_base + 16 * u;
                    if (p > top) continue;
                    const int page = cache.page_shift > 4 ? next_page[0] : next_page[u];
                    if ((unsigned)page >= (unsigned)cache.n_pages) {
                        if (status) *status = DEV_BAD_PAGE;
                        continue;
                    }
                    ok_bits |= 1u << (2 * in_count + u);
                    const unsigned char* src = source(p, page);
#pragma unroll
                    for (int i = 0; i < TB / 512; ++i) cp_async16_cg(dst + u * TB + 512 * i, src + 512 * i, 16);
                    if (lane < TB % 512 / 16) cp_async16_cg(dst + u * TB + TB / 512 * 512, src + TB / 512 * 512, 16);
                }
            }
            in_base += step;
            ++in_count;
            if (++in_stage == D) in_stage = 0;
            look_up(in_base);
        }
        cp_async_commit();
    };
#pragma unroll
    for (int i = 0; i < D - 1; ++i) fetch();

    // Queries as B operands: lane 4 g + t of group j holds channels 32 j + 8 t .. + 7 of query g.
#pragma unroll
    for (int k = 0; k < PIECES; ++k) {
        const int i = threadIdx.x + k * W * 32, qq = i / PER, j = i % PER / 4, tt = i % 4;
        if (i >= NT * 8 * PER) break;  // whole warps
        const uint32_t x[4] = {piece[k].x, piece[k].y, piece[k].z, piece[k].w};
        uint32_t am = 0;  // the largest finite component
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const uint32_t lo = x[v] & 0x7fffu, hi = x[v] >> 16 & 0x7fffu;
            am = max(am, max(lo < 0x7f80u ? lo : 0u, hi < 0x7f80u ? hi : 0u));
        }
#pragma unroll
        for (int o = 1; o < PER; o *= 2) am = max(am, __shfl_xor_sync(0xffffffffu, am, o));
        const int e = max((int)(am >> 7), 15) - 127;  // |q| < 2^(e + 1)
        const float up = exp2_int(14 - e);
        float y[8];
#pragma unroll
        for (int v = 0; v < 8; ++v) y[v] = (v & 1 ? bf16hi(x[v / 2]) : bf16lo(x[v / 2])) * up;
        sQ[((qq / 8) * NJ + j) * 32 + (qq % 8) * 4 + tt] =
            make_uint4(pack_f16(y[0], y[1]), pack_f16(y[2], y[3]), pack_f16(y[4], y[5]), pack_f16(y[6], y[7]));
        if (i % PER == 0) sF[qq] = exp2_int(e);
    }
    __syncthreads();
    float fa[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) fa[nt][e] = sF[nt * 8 + 2 * t + e];
    // score * log2(e) = sum_g s_g c_g * 2^e * fb
    const float fb = kv4_unit(HD);

    for (;;) {  // one split after the other, where there are fewer clusters than splits
        float o[NT][CT][4] = {}, mx[NT][2], sum[NT][2] = {};
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) mx[nt][0] = mx[nt][1] = -INFINITY;
        float top_m[NT][2];
        // O is kept in units of 2^(vexp - 135), and of 2^-7 for the weights; vexp: no less than the exponent field of any V
        // scale so far of this lane's channel group, at least 17
        int vexp = 17;
        float vscale = exp2_int(135 - vexp);  // scales become less than 2^9, the largest [2^7, 2^8) when it raises vexp

        // The products of a chunk, for all queries or (ROW) for those of one row, whose lim is `only`.  True, and nothing done, if
        // the rows have to be gone through one by one: if later rows' own tokens, which only a warp's last chunk can hold, would
        // take V's unit so far up that the products of rows which do not see them lose bits.
        int base = base0;
        uint32_t ok, chunk;  // tiles of the chunk that exist; where it is
        auto work = [&](auto row, int only) __attribute__((always_inline)) -> bool {
            constexpr bool ROW = decltype(row)::value;
            const bool whole = ok == 3u && base + kKv4Chunk - 1 <= low;  // every query sees every token

            float s[NT][2][4];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const uint32_t tile = chunk + u * TB;
                uint32_t wl[NJ], wh[NJ];
                if (HD == 128) {
                    const uint4 x = lds16(tile + lane * 16), y = lds16(tile + 512 + lane * 16);
                    wl[0] = x.x, wl[1] = x.y, wl[2 % NJ] = x.z, wl[3 % NJ] = x.w;
                    wh[0] = y.x, wh[1] = y.y, wh[2 % NJ] = y.z, wh[3 % NJ] = y.w;
                } else {
                    const uint2 x = lds8(tile + lane * 8), y = lds8(tile + 256 + lane * 8);
                    wl[0] = x.x, wl[1] = x.y;
                    wh[0] = y.x, wh[1] = y.y;
                }
                float s_lo[NJ], s_hi[NJ];
                const uint32_t sd = tile + 8 * HD + g * (HD / 16);
                if (HD == 128) {
                    const uint2 x = lds8(sd), y = lds8(sd + 8 * (HD / 16));
                    s_lo[0] = bf16lo(x.x), s_lo[1] = bf16hi(x.x), s_lo[2 % NJ] = bf16lo(x.y), s_lo[3 % NJ] = bf16hi(x.y);
                    s_hi[0] = bf16lo(y.x), s_hi[1] = bf16hi(y.x), s_hi[2 % NJ] = bf16lo(y.y), s_hi[3 % NJ] = bf16hi(y.y);
                } else {
                    const uint32_t x = lds4(sd), y = lds4(sd + 8 * (HD / 16));
                    s_lo[0] = bf16lo(x), s_lo[1] = bf16hi(x);
                    s_hi[0] = bf16lo(y), s_hi[1] = bf16hi(y);
                }
#pragma unroll
                for (int j = 0; j < NJ; ++j) {
                    uint32_t a[8];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        a[2 * i] = q4_f16x2(wl[j] >> (8 * (i / 2)), i % 2);
                        a[2 * i + 1] = q4_f16x2(wh[j] >> (8 * (i / 2)), i % 2);
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        const uint4 bq = sQ[(nt * NJ + j) * 32 + lane];
                        float c[4];
                        mma_f16_16816(c, a[0], a[1], a[2], a[3], bq.x, bq.y, 0.f, 0.f, 0.f, 0.f);
                        mma_f16_16816(c, a[4], a[5], a[6], a[7], bq.z, bq.w, c[0], c[1], c[2], c[3]);
                        if (j == 0) {
                            s[nt][u][0] = s_lo[j] * c[0], s[nt][u][1] = s_lo[j] * c[1];
                            s[nt][u][2] = s_hi[j] * c[2], s[nt][u][3] = s_hi[j] * c[3];
                        } else {
                            s[nt][u][0] = fmaf(s_lo[j], c[0], s[nt][u][0]);
                            s[nt][u][1] = fmaf(s_lo[j], c[1], s[nt][u][1]);
                            s[nt][u][2] = fmaf(s_hi[j], c[2], s[nt][u][2]);
                            s[nt][u][3] = fmaf(s_hi[j], c[3], s[nt][u][3]);
                        }
                    }
                }
            }
            // V scales of this lane's group, tokens 2 t, 2 t + 1 and 8 more of each tile
            uint32_t sc[2][2];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int r = 0; r < 2; ++r)
                    sc[u][r] = lds4(chunk + u * TB + 17 * HD + g * (HD / 8) / 32 * 32 + r * 16 + t * 4);
            if (!whole) {
                // a score that its query does not see is -inf, the V scale of a token that none sees 0, whatever
                // bits the tile holds there
                const int to = ROW ? only : top;
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const bool here = ok >> u & 1u;
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int l = lim[nt][e & 1];
                            if (!here || (ROW && l != only) || base + 16 * u + g + 8 * (e >> 1) > l) s[nt][u][e] = -INFINITY;
                        }
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const int p = base + 16 * u + 8 * r + 2 * t;
                        if (!here || p > to) sc[u][r] &= 0xffff0000u;
                        if (!here || p + 1 > to) sc[u][r] &= 0x0000ffffu;
                    }
                }
            }
            // Running softmax, in units of 1 / fb.  A query's reference moves up only when its maximum has outgrown it by
            // 2^8, so that O is rarely rescaled: p <= 2^8 then, and some p so far has been 1 or more.
            bool grown = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
#pragma unroll
                    for (int u = 0; u < 2; ++u) s[nt][u][e] *= fa[nt][e], s[nt][u][e + 2] *= fa[nt][e];
                    float m = fmaxf(fmaxf(s[nt][0][e], s[nt][0][e + 2]), fmaxf(s[nt][1][e], s[nt][1][e + 2]));
                    m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 4));
                    m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
                    top_m[nt][e] = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16));
                    grown |= top_m[nt][e] * fb > fmaf(mx[nt][e], fb, 8.f);
                }
            // V scales beyond what O's unit allows for, or not finite (of values that are not)
            const uint32_t m2 = __vmaxu2(__vmaxu2(sc[0][0], sc[0][1]), __vmaxu2(sc[1][0], sc[1][1]));
            grown |= max(m2 & 0xffffu, m2 >> 16) >> 7 > (uint32_t)vexp;
            bool odd = false;
            float poison[NT][2] = {};
            if (__any_sync(0xffffffffu, grown)) {
                auto largest = [](const uint32_t (&v)[2][2]) {  // scale of this lane's channel group: 32 / NJ lanes side by side
                    uint32_t x = __vmaxu2(__vmaxu2(v[0][0], v[0][1]), __vmaxu2(v[1][0], v[1][1]));
#pragma unroll
                    for (int d = 1; d < 32 / NJ; d *= 2) x = __vmaxu2(x, __shfl_xor_sync(0xffffffffu, x, d));
                    return max(x & 0xffffu, x >> 16);
                };
                uint32_t vmax = largest(sc);
                odd = __any_sync(0xffffffffu, vmax >= 0x7f80u);
                if (odd) [[unlikely]] {  // 0 in the product, and NaN for the queries that see them
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        for (int i = 0; i < 16; ++i) {
                            const uint32_t x = lds4(chunk + u * TB + 17 * HD + g * (HD / 8) / 32 * 32 + (i & ~1) * 2) >> (16 * (i & 1));
                            if ((x & 0x7f80u) != 0x7f80u || !(ok >> u & 1u)) continue;
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                                for (int e = 0; e < 2; ++e)
                                    if (base + 16 * u + i <= lim[nt][e]) poison[nt][e] = __uint_as_float(0x7fffffffu);
                        }
#pragma unroll
                        for (int r = 0; r < 2; ++r) {
                            if ((sc[u][r] & 0x7f80u) == 0x7f80u) sc[u][r] &= 0xffff0000u;
                            if ((sc[u][r] & 0x7f800000u) == 0x7f800000u) sc[u][r] &= 0x0000ffffu;
                        }
                    }
                    __syncwarp();
                    vmax = largest(sc);
                }
                const int vnew = (int)(vmax >> 7) > vexp ? (int)(vmax >> 7) + kKv4Headroom : vexp;
                if (!ROW && low < top && base + kKv4Chunk - 1 > low) {
                    // Rows differ in what they see of this chunk.  A unit taken up by tokens that the first does not see changes
                    // nothing for it, being a power of two, while all products stay normal f16 numbers (scales down to 2^-22 of
                    // the largest) and what is in O stays normal (bits below 2^-149 of the unit are not looked after).
                    uint32_t seen[2][2], least = 0xffffffffu;  // scales of what the first row sees; the smallest but 0, less 1
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t x = sc[i / 2][i % 2];
                        const int p = base + 16 * (i / 2) + 8 * (i % 2) + 2 * t;
                        seen[i / 2][i % 2] = p < low ? x : p == low ? x & 0xffffu : 0u;
                        least = __vminu2(least, __vsub2(x, 0x00010001u));
                    }
                    const bool raised = (int)(vmax >> 7) > max(vexp, (int)(largest(seen) >> 7));
                    const int by = vnew - (int)(min(least & 0xffffu, least >> 16) >> 7);
                    if (__any_sync(0xffffffffu, raised && (by > 22 || (base > base0 && vnew - vexp > 22)))) return true;
                }
                const float shrink = exp2_int(vexp - vnew);
                vexp = vnew;
                vscale = exp2_int(135 - vexp);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float alpha = 1.f;
                        if (top_m[nt][e] * fb > fmaf(mx[nt][e], fb, 8.f)) {
                            alpha = exp2_fast((mx[nt][e] - top_m[nt][e]) * fb);
                            mx[nt][e] = top_m[nt][e];
                        }
                        sum[nt][e] *= alpha;
                        if (!ROW || lim[nt][e] == only) alpha *= shrink;
#pragma unroll
                        for (int i = 0; i < CT; ++i) o[nt][i][e] *= alpha, o[nt][i][e + 2] *= alpha;
                    }
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    // 2^7 p; nothing seen so far: every score is -inf
                    const float off = mx[nt][e] == -INFINITY ? 0.f : fmaf(-mx[nt][e], fb, kKv4WeightBits);
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        s[nt][u][e] = exp2_fast(fmaf(s[nt][u][e], fb, off));
                        s[nt][u][e + 2] = exp2_fast(fmaf(s[nt][u][e + 2], fb, off));
                        sum[nt][e] += s[nt][u][e] + s[nt][u][e + 2];
                    }
                }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                constexpr int CW = HD / 64;  // code words of a lane's piece: channels (HD / 8) g ..
                uint32_t p[NT][2], s16[2], s72[2], w[2][2][CW];  // w: [tokens 2 t, 2 t + 1 | 8 more][token][word]
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int r = 0; r < 2; ++r) p[nt][r] = movmatrix_trans(pack_f16(s[nt][u][2 * r], s[nt][u][2 * r + 1]));
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const uint32_t vs = pack_f16(bf16lo(sc[u][r]) * vscale, bf16hi(sc[u][r]) * vscale);
                    s16[r] = mul_f16x2(vs, 0x2c002c00u), s72[r] = mul_f16x2(vs, 0xd480d480u);  // 1 / 16, -72
                    const uint32_t vc = chunk + u * TB + 9 * HD + r * (4 * HD) + lane * (HD / 8);
                    if (HD == 128) {
                        const uint4 x = lds16(vc);
                        w[r][0][0] = x.x, w[r][0][CW - 1] = x.y, w[r][1][0] = x.z, w[r][1][CW - 1] = x.w;
                    } else {
                        const uint2 x = lds8(vc);
                        w[r][0][0] = x.x, w[r][1][0] = x.y;
                    }
                }
#pragma unroll
                for (int i = 0; i < CT; ++i) {  // channels (HD / 8) g + 2 i and + 1: nibbles 2 i, 2 i + 1 of the piece
                    uint32_t a[4];
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const uint32_t two = __byte_perm(w[r][0][i / 4], w[r][1][i / 4], i % 4 < 2 ? 0x5410 : 0x7632);
                        a[2 * r] = q4_scaled_f16x2(two, 2 * (i % 2), s16[r], s72[r]);
                        a[2 * r + 1] = q4_scaled_f16x2(two, 2 * (i % 2) + 1, s16[r], s72[r]);
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
                        mma_f16_16816(o[nt][i], a[0], a[1], a[2], a[3], p[nt][0], p[nt][1], o[nt][i][0], o[nt][i][1], o[nt][i][2],
                                      o[nt][i][3]);
                }
            }
            if (odd) [[unlikely]] {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < CT; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[nt][i][e] += poison[nt][e & 1];
            }
            return false;
        };
        int stage = 0;
        bool apart = false;
        for (; base <= top; base += step) {
            fetch();
            cp_async_wait<D - 1>();
            __syncwarp();
            ok = ok_bits & 3u;
            ok_bits >>= 2;
            --in_count;
            chunk = ring + stage * 2 * TB;
            if (++stage == D) stage = 0;
            if ((apart = work(std::false_type(), -1))) break;
            __syncwarp();  // every lane has read the chunk before the ring comes round to it
        }
        // where O's units go: of the 32 / NJ lanes of a channel group the first four have two queries of each 8 each
        float* units = sUnit + (warp * NJ + lane / (32 / NJ)) * NT * 8 + 2 * t;
        auto unit = [&]() { return exp2_int(vexp - 135 - kKv4WeightBits); };  // no less than 2^-125
        if (apart) {
            const int before = vexp;
            for (int only = low; only <= top; ++only) {
                work(std::true_type(), only);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        if (lim[nt][e] == only && lane % (32 / NJ) < 4) units[nt * 8 + e] = unit();
                vexp = before, vscale = exp2_int(135 - vexp);
                __syncwarp();
            }
        } else if (lane % (32 / NJ) < 4) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) *reinterpret_cast<float2*>(units + nt * 8) = make_float2(unit(), unit());
        }

        // The next operation may come in from here on: earlier, its CTAs would take the free SMs two at a time (a layer of 4096
        // channels over 16000 positions: 68 us, 66.5).
        pdl_launch_dependents();
        // ---- the warps' results, each where its ring was
        cp_async_wait<0>();
        __syncwarp();
        float4* mineO = reinterpret_cast<float4*>(kv4_smem + warp * SM::kWarpRing);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int i = 0; i < CT; ++i)
                mineO[(nt * CT + i) * 32 + lane] = make_float4(o[nt][i][0], o[nt][i][1], o[nt][i][2], o[nt][i][3]);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                sum[nt][e] += __shfl_xor_sync(0xffffffffu, sum[nt][e], 4);
                sum[nt][e] += __shfl_xor_sync(0xffffffffu, sum[nt][e], 8);
                sum[nt][e] += __shfl_xor_sync(0xffffffffu, sum[nt][e], 16);
                if (g == 0)
                    sStat[warp * NT * 8 + nt * 8 + 2 * t + e] = make_float2(mx[nt][e], sum[nt][e] * exp2_int(-kKv4WeightBits));
            }
        }
        __syncwarp();  // the cluster's barriers want whole warps
        if (S > 1) cluster_wait();  // the others are there
        __syncthreads();
        // ---- the CTA's, sent to the CTA that finishes them: piece x holds two queries x two channels
        const int share = fastdiv(SM::kItems + S - 1, S, div_S);  // pieces a CTA finishes; the last one may have fewer
        for (int x = threadIdx.x; x < SM::kItems; x += W * 32) {
            const int c = x / (CT * 32) * 8 + 2 * (x & 3);  // its first query
            if (q0 + c >= Q) continue;
            float m0 = -INFINITY, m1 = -INFINITY;
#pragma unroll
            for (int w = 0; w < W; ++w) m0 = fmaxf(m0, sStat[w * NT * 8 + c].x), m1 = fmaxf(m1, sStat[w * NT * 8 + c + 1].x);
            float4 r = make_float4(0.f, 0.f, 0.f, 0.f);
            float l0 = 0.f, l1 = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const float4 v = *reinterpret_cast<const float4*>(kv4_smem + w * SM::kWarpRing + x * 16);
                const float2 s0 = sStat[w * NT * 8 + c], s1 = sStat[w * NT * 8 + c + 1];
                const float f0 = m0 == -INFINITY ? 0.f : exp2_fast((s0.x - m0) * fb);
                const float f1 = m1 == -INFINITY ? 0.f : exp2_fast((s1.x - m1) * fb);
                const float2 unit = *reinterpret_cast<const float2*>(sUnit + (w * NJ + (x & 31) / (32 / NJ)) * NT * 8 + c);
                l0 = fmaf(f0, s0.y, l0), l1 = fmaf(f1, s1.y, l1);
                r.x = fmaf(f0 * unit.x, v.x, r.x), r.z = fmaf(f0 * unit.x, v.z, r.z);
                r.y = fmaf(f1 * unit.y, v.y, r.y), r.w = fmaf(f1 * unit.y, v.w, r.w);
            }
            int to = 0;  // x / share
            for (int edge = share; edge <= x; edge += share) ++to;
            st_cluster_f4(map_cluster(smem_u32(sIn) + (rank * share + x - to * share) * 16, to), r);
            if ((x / 4) % (CT * 8) == 0)  // one of the pieces with these queries: their statistics, to all
                for (int d = 0; d < S; ++d) {
                    const uint32_t a = map_cluster(smem_u32(sInStat) + (rank * NT * 8 + c) * 8, d);
                    st_cluster_f2(a, m0, l0);
                    st_cluster_f2(a + 8, m1, l1);
                }
        }
        __syncwarp();
        if (S > 1)
            cluster_sync_all();  // after it nobody touches another CTA's memory
        else
            __syncthreads();
        for (int y = threadIdx.x; y < 2 * share; y += W * 32) {  // one query and two channels a thread
            const int x = rank * share + y / 2, e = y & 1, l = x & 31, c = x / (CT * 32) * 8 + 2 * (l & 3) + e, qi = q0 + c;
            if (x >= SM::kItems || qi >= Q) continue;
            float m = -INFINITY, sum_l = 0.f, v0 = 0.f, v1 = 0.f;
            for (int r = 0; r < S; ++r) m = fmaxf(m, sInStat[r * NT * 8 + c].x);
#pragma unroll 4
            for (int r = 0; r < S; ++r) {
                const float2 st = sInStat[r * NT * 8 + c];
                const float f = m == -INFINITY ? 0.f : exp2_fast((st.x - m) * fb);
                const float* v = reinterpret_cast<const float*>(sIn + r * share + y / 2);
                sum_l = fmaf(f, st.y, sum_l), v0 = fmaf(f, v[e], v0), v1 = fmaf(f, v[e + 2], v1);
            }
            const int row = fastdiv(qi, G, div_G), ch = (l >> 2) * (HD / 8) + 2 * (x / 32 % CT);
            if (splits > 1) {  // to be finished by combine_kv4_kernel
                float* to = scratch + (kv4_partial(b, gridDim.y, blockIdx.y, splits, split) * (NT * 8) + c) * (HD + 2);
                *reinterpret_cast<float2*>(to + ch) = make_float2(v0, v1);
                if (ch == 0) *reinterpret_cast<float2*>(to + HD) = make_float2(m, sum_l);
                continue;
            }
            const bool none = (long long)pos0 + row < 0 || (long long)pos0 + row >= cache.max_seq;
            const float inv = 1.f / sum_l;
            const uint32_t v = none ? 0u : pack_bf16(v0 * inv, v1 * inv);
            *reinterpret_cast<uint32_t*>(out + (((long long)b * M + row) * Hq + head * G + qi - row * G) * HD + ch) = v;
        }
        if (NT == 1) break;
        const int ahead = fastdiv(gridDim.x, S, div_S);
        if ((split += ahead) >= splits) break;
        __syncwarp();
        if (S > 1) cluster_arrive();  // what the others sent here has been read
        in_base = base0 += ahead * S * W * kKv4Chunk, in_stage = in_count = 0, ok_bits = 0;
        look_up(base0);
#pragma unroll
        for (int i = 0; i < D - 1; ++i) fetch();
    }
}

// Joins the splits.  grid (M, Hq, n_seq), block 2 HD: a thread has two channels of a row and every fourth split.  NT, rows
// (gridDim.y), splits: of the attention kernel's launch.
constexpr int kKv4MaxSplits = 64;
template <int HD>
__global__ void __launch_bounds__(2 * HD)
combine_kv4_kernel(const float* __restrict__ scratch, int G, const int32_t* __restrict__ pos0_dev, int max_seq, int NT, int Hkv,
                   int rows, int splits, uint16_t* __restrict__ out)
{
    __shared__ float2 stat[kKv4MaxSplits];  // (max, sum) of a split, later (weight, weight * sum)
    __shared__ float2 part[3][HD / 2];
    pdl_launch_dependents();
    pdl_wait();
    const int m = blockIdx.x, hq = blockIdx.y, b = blockIdx.z, lane = threadIdx.x % (HD / 2), quarter = threadIdx.x / (HD / 2);
    const int qi = m * G + hq % G, y = qi / (NT * 8) * Hkv + hq / G, c = qi % (NT * 8);
    const float* from = scratch + (kv4_partial(b, rows, y, splits, 0) * (NT * 8) + c) * (HD + 2);
    const long long stride = (long long)NT * 8 * (HD + 2), p = (long long)ld_now(pos0_dev + b) + m;
    const float fb = kv4_unit(HD);
    const bool mine = threadIdx.x < splits;
    const float2 st = mine ? ld_once<float2>(from + threadIdx.x * stride + HD) : make_float2(0.f, 0.f);
    if (mine) stat[threadIdx.x] = st;
    __syncthreads();
    float top = -INFINITY;
    for (int s = 0; s < splits; ++s) top = fmaxf(top, stat[s].x);
    __syncthreads();
    if (mine) {
        const float f = top == -INFINITY ? 0.f : exp2_fast((st.x - top) * fb);
        stat[threadIdx.x] = make_float2(f, f * st.y);
    }
    __syncthreads();
    float x0 = 0.f, x1 = 0.f;
#pragma unroll 4
    for (int s = quarter; s < splits; s += 4) {
        const float2 v = ld_once<float2>(from + s * stride + 2 * lane);
        x0 = fmaf(stat[s].x, v.x, x0), x1 = fmaf(stat[s].x, v.y, x1);
    }
    if (quarter) part[quarter - 1][lane] = make_float2(x0, x1);
    __syncthreads();
    if (quarter) return;
    float l = 0.f;
    for (int s = 0; s < splits; ++s) l += stat[s].y;
#pragma unroll
    for (int i = 0; i < 3; ++i) x0 += part[i][lane].x, x1 += part[i][lane].y;
    const float inv = 1.f / l;
    const uint32_t r = p < 0 || p >= max_seq ? 0u : pack_bf16(x0 * inv, x1 * inv);
    *reinterpret_cast<uint32_t*>(out + (((long long)b * gridDim.x + m) * gridDim.y + hq) * HD + 2 * lane) = r;
}

}  // namespace ls
