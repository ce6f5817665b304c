// Attention over a KV cache held in 4 bits (format and tile layout: ls_q4.cuh): the draft and verify passes
// of LayerSkip Sec. 4.3.3 for one or several sequences, up to 16 rows each.
//
//   o[m] = sum_i p_i v_i / sum_i p_i,  p_i = exp(q[m] . k_i / sqrt(hd)) for the positions i <= pos0 + m
//
// Tokens are the 16-row operand of mma.sync in both products, queries (row, head of the KV group) the
// 8-column one: S^T = K Q^T with K's codes as A; O^T = V^T P^T with V^T's values as A -- a tile stores V so
// that a lane finds two neighbouring tokens of a channel in the same nibble of two words, so the
// transposition costs one byte permutation.
#pragma once
#include "ls_w4.cuh"

namespace ls {

constexpr int kKv4Warps = 8;
constexpr int kKv4Threads = kKv4Warps * 32;
constexpr int kKv4Chunk = 32;  // positions a warp takes at a time: two tiles

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
__device__ __forceinline__ float ld_cluster_f32(uint32_t addr)
{
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t map_cluster(uint32_t addr, int rank)
{
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}

// shared memory, in floats: the halves of the warps' outputs while they are added up, then the CTA's (O, m, l)
template <int HD, int NT>
__host__ __device__ constexpr int kv4_o_floats() { return (kKv4Warps / 2) * NT * 8 * HD; }
template <int HD, int NT>
constexpr size_t kv4_smem_bytes()
{
    return sizeof(float) * (kv4_o_floats<HD, NT>() + (kKv4Warps + 2) * NT * 8) + NT * 8 * HD * 2;
}

// grid (S, Hkv * query tiles, n_seq) in clusters of S CTAs.  The warps of a cluster take the 32-position
// chunks of the cache in turn by absolute position, each with a running (max, sum, O) of its own; the warps'
// results are added up in a fixed order, then the CTAs' through distributed shared memory.  A row's result
// depends on its position and on S, not on M or the other rows.
template <int HD, int NT>
__global__ void __launch_bounds__(kKv4Threads)
attention_kv4_kernel(const uint16_t* __restrict__ q, int M, int G, const int32_t* __restrict__ pos0_dev,
                     const Kv4Cache cache, const unsigned char* __restrict__ pages, uint16_t* __restrict__ out,
                     int32_t* status)
{
    constexpr int NJ = HD / 32;   // groups of a row
    constexpr int CT = HD / 16;   // 16-channel tiles of O^T
    extern __shared__ __align__(16) float kv4_smem[];
    float* sO = kv4_smem;                                       // [4][NT * 8][HD]
    float* sM = kv4_smem + kv4_o_floats<HD, NT>();              // [warps][NT * 8], then the CTA's max and sum
    float* sML = sM + kKv4Warps * NT * 8;                 // [2][NT * 8]
    uint4* sQ = reinterpret_cast<uint4*>(sML + 2 * NT * 8);  // [NT][NJ][32 lanes]
    pdl_launch_dependents();
    pdl_wait();
    const int S = gridDim.x, rank = blockIdx.x, b = blockIdx.z;
    const int head = blockIdx.y % cache.Hkv, q0 = blockIdx.y / cache.Hkv * (NT * 8);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int Q = M * G, Hq = cache.Hkv * G, pos0 = pos0_dev[b];

    for (int i = threadIdx.x; i < NT * NJ * 32; i += kKv4Threads) {
        const int l = i % 32, j = i / 32 % NJ, qi = q0 + i / 32 / NJ * 8 + (l >> 2);
        uint4 v = make_uint4(0, 0, 0, 0);
        if (qi < Q)
            v = *reinterpret_cast<const uint4*>(q + (((long long)b * M + qi / G) * Hq + head * G + qi % G) * HD + 32 * j +
                                                8 * (l & 3));
        sQ[i] = v;
    }
    // last visible position of this lane's two queries of each tile, and of all queries of the CTA
    int lim[NT][2], top = -1;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int qi = q0 + nt * 8 + 2 * t + e;
            lim[nt][e] = qi < Q ? kv4_position(pos0, qi / G, cache.max_seq, status) : -1;
            top = max(top, lim[nt][e]);
        }
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    __syncthreads();

    float o[NT][CT][4] = {}, mx[NT][2], sum[NT][2] = {};
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) mx[nt][0] = mx[nt][1] = -INFINITY;
    const float scale = 1.4426950408889634f / sqrtf((float)HD);

    for (int base = (rank * kKv4Warps + warp) * kKv4Chunk; base <= top; base += S * kKv4Warps * kKv4Chunk) {
        const unsigned char* tile[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int p = base + 16 * u, page = p <= top ? kv4_page(cache, b, p, status) : -1;
            tile[u] = page >= 0 ? pages + kv4_tile_offset<HD>(cache, page, p, head) : nullptr;
        }
        float s[NT][2][4];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            uint32_t wl[4] = {}, wh[4] = {}, s_lo[NJ] = {}, s_hi[NJ] = {};
            if (tile[u]) {
                if (HD == 128) {
                    const uint4 x = ld_stream16(tile[u] + lane * 16), y = ld_stream16(tile[u] + 512 + lane * 16);
                    wl[0] = x.x, wl[1] = x.y, wl[2] = x.z, wl[3] = x.w;
                    wh[0] = y.x, wh[1] = y.y, wh[2] = y.z, wh[3] = y.w;
                } else {
                    const uint2 x = *reinterpret_cast<const uint2*>(tile[u] + lane * 8);
                    const uint2 y = *reinterpret_cast<const uint2*>(tile[u] + 256 + lane * 8);
                    wl[0] = x.x, wl[1] = x.y;
                    wh[0] = y.x, wh[1] = y.y;
                }
                q4_row_scales<NJ>(tile[u] + 8 * HD + g * (HD / 16), s_lo);
                q4_row_scales<NJ>(tile[u] + 8 * HD + (g + 8) * (HD / 16), s_hi);
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) s[nt][u][0] = s[nt][u][1] = s[nt][u][2] = s[nt][u][3] = 0.f;
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                uint32_t a[8];
#pragma unroll
                for (int i = 0; i < 4; ++i) a[2 * i] = q4_bf16x2(wl[j], i), a[2 * i + 1] = q4_bf16x2(wh[j], i);
                const float s0 = bf16lo(s_lo[j]), s1 = bf16lo(s_hi[j]);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const uint4 bq = sQ[(nt * NJ + j) * 32 + lane];
                    float c[4];
                    mma_bf16_16816_new(c, a[0], a[1], a[2], a[3], bq.x, bq.y);
                    mma_bf16_16816(c, a[4], a[5], a[6], a[7], bq.z, bq.w);
                    s[nt][u][0] = fmaf(s0, c[0], s[nt][u][0]);
                    s[nt][u][1] = fmaf(s0, c[1], s[nt][u][1]);
                    s[nt][u][2] = fmaf(s1, c[2], s[nt][u][2]);
                    s[nt][u][3] = fmaf(s1, c[3], s[nt][u][3]);
                }
            }
        }
        // running softmax; a score that its query does not see is -inf whatever the tile holds there
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int p = base + 16 * u + g + 8 * (e >> 1);
                    s[nt][u][e] = tile[u] && p <= lim[nt][e & 1] ? s[nt][u][e] * scale : -INFINITY;
                }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float m = fmaxf(fmaxf(s[nt][0][e], s[nt][0][e + 2]), fmaxf(s[nt][1][e], s[nt][1][e + 2]));
                m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 4));
                m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
                m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16));
                m = fmaxf(m, mx[nt][e]);
                const float ref = m == -INFINITY ? 0.f : m;  // nothing seen so far
                const float alpha = exp2_fast(mx[nt][e] - ref);
                mx[nt][e] = m;
                float add = 0.f;
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    s[nt][u][e] = exp2_fast(s[nt][u][e] - ref);
                    s[nt][u][e + 2] = exp2_fast(s[nt][u][e + 2] - ref);
                    add += s[nt][u][e] + s[nt][u][e + 2];
                }
                sum[nt][e] = sum[nt][e] * alpha + add;
#pragma unroll
                for (int i = 0; i < CT; ++i) o[nt][i][e] *= alpha, o[nt][i][e + 2] *= alpha;
            }
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            if (!tile[u]) continue;  // the whole warp
            // p as the sum of two bf16 numbers (16 bits): rounding it to one would cost as much as the
            // rounding of the result
            uint32_t ph[NT][2], pl[NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const float x = s[nt][u][2 * r], y = s[nt][u][2 * r + 1];
                    const uint32_t hi = pack_bf16(x, y);
                    ph[nt][r] = movmatrix_trans(hi);
                    pl[nt][r] = movmatrix_trans(pack_bf16(x - bf16lo(hi), y - bf16hi(hi)));
                }
            constexpr int W = HD / 64;  // code words of a lane's piece: channels (HD / 8) g ..
            const unsigned char* vc = tile[u] + 9 * HD + lane * (HD / 8);
            const unsigned char* vs = tile[u] + 17 * HD + g * (HD / 8) / 32 * 32 + t * 4;
            uint32_t w[2][2][W], sc[2];  // [tokens 2 t, 2 t + 1 | 2 t + 8, 2 t + 9][token][word]
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                if (HD == 128) {
                    const uint4 x = ld_stream16(vc + r * 512);
                    w[r][0][0] = x.x, w[r][0][W - 1] = x.y, w[r][1][0] = x.z, w[r][1][W - 1] = x.w;
                } else {
                    const uint2 x = *reinterpret_cast<const uint2*>(vc + r * 256);
                    w[r][0][0] = x.x, w[r][1][0] = x.y;
                }
                sc[r] = *reinterpret_cast<const uint32_t*>(vs + r * 16);
            }
            // Scales that are not finite: those of slots behind the last token (whatever bits are there),
            // and of values that are not finite themselves.  0 in the product for both; the latter make
            // NaN of what the queries that see them sum up.
            bool odd = false;
#pragma unroll
            for (int r = 0; r < 2; ++r)
                odd |= (sc[r] & 0x7f80u) == 0x7f80u || (sc[r] & 0x7f800000u) == 0x7f800000u;
            float poison[NT][2] = {};
            const bool any_odd = __any_sync(0xffffffffu, odd);
            if (any_odd) {
                const uint16_t* gs = reinterpret_cast<const uint16_t*>(tile[u] + 17 * HD + g * (HD / 8) / 32 * 32);
                for (int i = 0; i < 16; ++i) {
                    if ((gs[i] & 0x7f80u) != 0x7f80u) continue;
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 2; ++e)
                            if (base + 16 * u + i <= lim[nt][e]) poison[nt][e] = __uint_as_float(0x7fffffffu);
                }
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    if ((sc[r] & 0x7f80u) == 0x7f80u) sc[r] &= 0xffff0000u;
                    if ((sc[r] & 0x7f800000u) == 0x7f800000u) sc[r] &= 0xffffu;
                }
            }
#pragma unroll
            for (int i = 0; i < CT; ++i) {  // channels (HD / 8) g + 2 i and + 1: nibbles 2 i, 2 i + 1 of the piece
                uint32_t a[4];
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const uint32_t two = __byte_perm(w[r][0][i / 4], w[r][1][i / 4], i % 4 < 2 ? 0x5410 : 0x7632);
                    a[2 * r] = mul_bf16x2(q4_bf16x2(two, 2 * (i % 2)), sc[r]);
                    a[2 * r + 1] = mul_bf16x2(q4_bf16x2(two, 2 * (i % 2) + 1), sc[r]);
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    mma_bf16_16816(o[nt][i], a[0], a[1], a[2], a[3], ph[nt][0], ph[nt][1]);
                    mma_bf16_16816(o[nt][i], a[0], a[1], a[2], a[3], pl[nt][0], pl[nt][1]);
                }
            }
            if (any_odd) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < CT; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[nt][i][e] += poison[nt][e & 1];
            }
        }
    }

    // ---- the warps of the CTA: common maximum, then halves added in a fixed order
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            sum[nt][e] += __shfl_xor_sync(0xffffffffu, sum[nt][e], 4);
            sum[nt][e] += __shfl_xor_sync(0xffffffffu, sum[nt][e], 8);
            sum[nt][e] += __shfl_xor_sync(0xffffffffu, sum[nt][e], 16);
            if (g == 0) sM[warp * NT * 8 + nt * 8 + 2 * t + e] = mx[nt][e];
        }
    __syncthreads();
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int c = nt * 8 + 2 * t + e;
            float m = -INFINITY;
#pragma unroll
            for (int w = 0; w < kKv4Warps; ++w) m = fmaxf(m, sM[w * NT * 8 + c]);
            const float f = m == -INFINITY ? 0.f : exp2_fast(mx[nt][e] - m);
            sum[nt][e] *= f;
#pragma unroll
            for (int i = 0; i < CT; ++i) o[nt][i][e] *= f, o[nt][i][e + 2] *= f;
            if (warp == 0 && g == 0) sML[c] = m;
        }
    __syncthreads();
    for (int half = kKv4Warps / 2; half >= 1; half /= 2) {
        if (warp >= half && warp < 2 * half) {
            float* dst = sO + (warp - half) * NT * 8 * HD;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float* d = dst + (nt * 8 + 2 * t + e) * HD + g * (HD / 8);
#pragma unroll
                    for (int i = 0; i < CT; ++i)
                        *reinterpret_cast<float2*>(d + 2 * i) = make_float2(o[nt][i][e], o[nt][i][e + 2]);
                    if (g == 0) sM[(warp - half) * NT * 8 + nt * 8 + 2 * t + e] = sum[nt][e];
                }
        }
        __syncthreads();
        if (warp < half) {
            const float* src = sO + warp * NT * 8 * HD;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float* d = src + (nt * 8 + 2 * t + e) * HD + g * (HD / 8);
#pragma unroll
                    for (int i = 0; i < CT; ++i) {
                        const float2 v = *reinterpret_cast<const float2*>(d + 2 * i);
                        o[nt][i][e] += v.x, o[nt][i][e + 2] += v.y;
                    }
                    sum[nt][e] += sM[warp * NT * 8 + nt * 8 + 2 * t + e];
                }
        }
        __syncthreads();
    }
    if (warp == 0) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int c = nt * 8 + 2 * t + e;
#pragma unroll
                for (int i = 0; i < CT; ++i)
                    *reinterpret_cast<float2*>(sO + c * HD + g * (HD / 8) + 2 * i) =
                        make_float2(o[nt][i][e], o[nt][i][e + 2]);
                if (g == 0) sML[NT * 8 + c] = sum[nt][e];
            }
    }
    // ---- the CTAs of the cluster: CTA r finishes every S-th pair of output elements
    if (S > 1)
        cluster_sync_all();
    else
        __syncthreads();
    const uint32_t aO = (uint32_t)__cvta_generic_to_shared(sO), aML = (uint32_t)__cvta_generic_to_shared(sML);
    for (int i = rank * kKv4Threads + threadIdx.x; i < NT * 8 * HD / 2; i += S * kKv4Threads) {
        const int c = i / (HD / 2), ch = 2 * (i % (HD / 2)), qi = q0 + c;
        if (qi >= Q) continue;
        float m = -INFINITY;
        for (int r = 0; r < S; ++r) m = fmaxf(m, ld_cluster_f32(map_cluster(aML + 4 * c, r)));
        float l = 0.f, x = 0.f, y = 0.f;
        for (int r = 0; r < S; ++r) {
            const float mr = ld_cluster_f32(map_cluster(aML + 4 * c, r));
            const float f = m == -INFINITY ? 0.f : exp2_fast(mr - m);
            l = fmaf(f, ld_cluster_f32(map_cluster(aML + 4 * (NT * 8 + c), r)), l);
            x = fmaf(f, ld_cluster_f32(map_cluster(aO + 4 * (c * HD + ch), r)), x);
            y = fmaf(f, ld_cluster_f32(map_cluster(aO + 4 * (c * HD + ch + 1), r)), y);
        }
        const int m_row = qi / G;
        const bool none = (long long)pos0 + m_row < 0 || (long long)pos0 + m_row >= cache.max_seq;
        const uint32_t v = none ? 0u : pack_bf16(x / l, y / l);
        *reinterpret_cast<uint32_t*>(out + (((long long)b * M + m_row) * Hq + head * G + qi % G) * HD + ch) = v;
    }
    if (S > 1) cluster_sync_all();  // no CTA leaves while another still reads its results
}

}  // namespace ls
