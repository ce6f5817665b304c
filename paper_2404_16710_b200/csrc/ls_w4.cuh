// Linear layer of the decode loop on 4-bit weights: out[m, n] (+)= sum_k c[n, k] s[n, k / group] h[m, k] for
// M <= 16 rows (LayerSkip Sec. 4.3: a draft pass has one row, a verify pass num_draft + 1).  Format and
// block layout: ls_q4.cuh.
#pragma once
#include <type_traits>

#include "ls_prefill.cuh"
#include "ls_q4.cuh"

namespace ls {

__device__ __forceinline__ uint2 lds8(uint32_t addr)
{
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(addr));
    return v;
}
__device__ __forceinline__ uint32_t lds4(uint32_t addr)
{
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(addr));
    return v;
}
// D = A * B: the first product of a sum
__device__ __forceinline__ void mma_bf16_16816_new(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                                   uint32_t b0, uint32_t b1)
{
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
        "{%10,%10,%10,%10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
constexpr int kW4SmemMax = 227 * 1024;

// shared memory: the warps' sums of a tile, then D blocks a warp, then (HS) the rows of h, each padded by 64 bytes
// (two rows' 64-byte pieces then fall on different banks)
template <int NT, int W>
__host__ __device__ constexpr int w4_part_bytes() { return W * 32 * NT * 16; }
template <int NG, int W>
__host__ __device__ constexpr int w4_ring_bytes(int D) { return W * D * w4_block_bytes(NG); }
__host__ __device__ constexpr int w4_h_stride(int kblocks) { return kblocks * kQ4Cols * 2 + 64; }

// what a lane reads of a block: the codes of rows g and g + 8 (its 16-byte pieces) and the rows' scales
template <int NG>
struct W4Regs {
    uint4 lo, hi;
    uint32_t s_lo[(NG + 1) / 2], s_hi[(NG + 1) / 2];
    __device__ __forceinline__ void load(uint32_t blk, int lane)  // of a block in shared memory
    {
        lo = lds16(blk + lane * 16);
        hi = lds16(blk + kQ4CodeBytes / 2 + lane * 16);
        const uint32_t sd = blk + kQ4CodeBytes + (lane >> 2) * NG * 2;
        if (NG == 4) {
            const uint2 x = lds8(sd), y = lds8(sd + 8 * NG * 2);
            s_lo[0] = x.x, s_lo[(NG + 1) / 2 - 1] = x.y, s_hi[0] = y.x, s_hi[(NG + 1) / 2 - 1] = y.y;
        } else if (NG == 2) {
            s_lo[0] = lds4(sd), s_hi[0] = lds4(sd + 8 * NG * 2);
        } else {
            uint16_t x, y;
            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(x) : "r"(sd));
            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(y) : "r"(sd + 8 * NG * 2));
            s_lo[0] = x, s_hi[0] = y;
        }
    }
    __device__ __forceinline__ static float scale(const uint32_t (&s)[(NG + 1) / 2], int i)
    {
        return i & 1 ? bf16hi(s[i / 2]) : bf16lo(s[i / 2]);
    }
};

// acc (rows g, g + 8 x columns 2 t, 2 t + 1) += the block's values times the NT * 8 rows of h in b
template <int NG, int NT>
__device__ __forceinline__ void w4_block_mma(const W4Regs<NG>& w, const uint4 (&b)[NT][4], float (&acc)[NT][4])
{
    const uint32_t wl[4] = {w.lo.x, w.lo.y, w.lo.z, w.lo.w}, wh[4] = {w.hi.x, w.hi.y, w.hi.z, w.hi.w};
    float c[NT][4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        uint32_t a[8];
#pragma unroll
        for (int p = 0; p < 4; ++p) a[2 * p] = q4_bf16x2(wl[j], p), a[2 * p + 1] = q4_bf16x2(wh[j], p);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            if (j % (4 / NG) == 0)
                mma_bf16_16816_new(c[nt], a[0], a[1], a[2], a[3], b[nt][j].x, b[nt][j].y);
            else
                mma_bf16_16816(c[nt], a[0], a[1], a[2], a[3], b[nt][j].x, b[nt][j].y);
            mma_bf16_16816(c[nt], a[4], a[5], a[6], a[7], b[nt][j].z, b[nt][j].w);
            if ((j + 1) % (4 / NG) == 0) {
                const float s0 = W4Regs<NG>::scale(w.s_lo, j * NG / 4), s1 = W4Regs<NG>::scale(w.s_hi, j * NG / 4);
                acc[nt][0] = fmaf(s0, c[nt][0], acc[nt][0]);
                acc[nt][1] = fmaf(s0, c[nt][1], acc[nt][1]);
                acc[nt][2] = fmaf(s1, c[nt][2], acc[nt][2]);
                acc[nt][3] = fmaf(s1, c[nt][3], acc[nt][3]);
            }
        }
    }
}

// One CTA per SM; its W warps form teams of 2^lks, and a team takes every (teams of the grid)-th group of TG tiles of
// 16 rows (TG = 2 halves what is read of h in shared memory, which bounds the kernel for 16 rows of h).  Of a tile's
// blocks each warp of the team has a fixed share, consecutive along K, and keeps the next blocks of its sequence (which
// runs on across tiles) in flight in a ring of its own, of D blocks; the team meets once per tile, to add its sums up.  HS: h
// is copied to shared memory once (columns beyond K as zeros); otherwise, for h larger than that, it comes through L1.
// The codes are the A operand of mma.sync, the rows of h the B operand; a group's products are summed in fp32 by
// the tensor cores and multiplied by the group's scale (a lane holds rows g and g + 8 of a tile) when they join
// the running sum.  Turning codes into operands bounds the kernel: 11 instructions for 8 codes, 7 of them on the
// half-rate integer pipe, which is 50 % busy on average and collides with the products of the other warps.  With the
// conversion left out the loads alone take 43 us for 128256 x 4096 (the copy rate), 4.0 us for 4096 x 4096; with it, one
// row of h: 56 us (0.77 of the measured copy rate) and 5.5 us (0.24: 2 us are the launch).  What HS = false costs, groups of
// 64: 4096 x 11008, 7 rows 10.0 us, 8 rows (h no longer fits) 11.1, 9 12.7, 16 13.2; 8192 x 8192, 9 rows 14.4, 10 (no longer)
// 17.0, 16 17.6; 4096 x 14336, 5 rows 11.0, 6 12.7.  Tried and not kept: bulk
// copies with h from L1 (143 us, too few warps), blocks held in registers (94 to 104 us: the loads of several blocks end
// up waiting for one another), f16 operands (3 to 5 % faster for one row, slower for 16: h has to be converted), h as two
// e4m3 pieces (3 instructions for 8 codes, a nibble's byte being an e4m3 number; 79 us, mma.sync being slow on them).
// Which blocks a warp adds, and in which order the warps' sums are added, depends on N and K only: a row's result does
// not depend on how many rows share the pass.
template <int NG, int NT, int W, int D, int CB, bool HS, int TG>
__global__ void __launch_bounds__(W * 32, 1)
linear_w4_kernel(const unsigned char* __restrict__ packed, const uint16_t* __restrict__ h, int M, int N, int K,
                 int kblocks, int n_tiles, int lks, float* __restrict__ out, int residual)
{
    constexpr int BB = w4_block_bytes(NG);
    extern __shared__ __align__(128) unsigned char w4_smem[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int KS = 1 << lks, ks = warp & (KS - 1), team = warp >> lks;
    float4* part = reinterpret_cast<float4*>(w4_smem) + (team << lks) * 32 * NT;  // [warp of the team][NT][lane]; a tile at a time
    const uint32_t ring = smem_u32(w4_smem) + w4_part_bytes<NT, W>() + warp * D * BB;
    pdl_launch_dependents();

    const int kb0 = kblocks * ks >> lks, nkb = (kblocks * (ks + 1) >> lks) - kb0;
    const int n_groups = (n_tiles + TG - 1) / TG, group0 = team * gridDim.x + blockIdx.x, group_step = (W >> lks) * gridDim.x;
    // the sequence of stages, kDepth - 1 ahead of their use: CB consecutive blocks of a tile, or (TG = 2) one of each
    constexpr int kStage = CB * TG, kDepth = D / kStage;
    static_assert(D % kStage == 0 && (TG == 1 || CB == 1), "whole stages");
    int in_group = nkb ? group0 : n_groups, in_left = nkb;
    uint32_t in_at = ring + lane * 16;
    const long long tile_bytes = (long long)kblocks * BB;
    const unsigned char* src = packed + group0 * TG * tile_bytes + (long long)kb0 * BB + lane * 16;
    const long long jump = group_step * TG * tile_bytes - (long long)nkb * BB;
    auto copy = [&](uint32_t to, const unsigned char* from, auto blocks) {  // a lane's 16-byte pieces of consecutive blocks
        constexpr int kBytes = decltype(blocks)::value * BB;
#pragma unroll
        for (int i = 0; i < kBytes / 512; ++i) cp_async16_cg(to + 512 * i, from + 512 * i, 16);
        if (lane < kBytes % 512 / 16) cp_async16_cg(to + kBytes / 512 * 512, from + kBytes / 512 * 512, 16);
    };
    auto fetch = [&]() {
        if (in_group < n_groups) {
            if (TG == 2) {  // a last group of fewer tiles reads its first one again
                copy(in_at, src, std::integral_constant<int, 1>());
                copy(in_at + BB, src + (in_group * 2 + 1 < n_tiles ? tile_bytes : 0), std::integral_constant<int, 1>());
            } else if (CB == 1 || in_left >= CB) {
                copy(in_at, src, std::integral_constant<int, CB>());
            } else {
                copy(in_at, src, std::integral_constant<int, 1>());
            }
            src += CB * BB;
            in_left -= CB;
            if (CB == 1 ? in_left == 0 : in_left <= 0)
                src += CB == 1 ? jump : jump + in_left * BB, in_left = nkb, in_group += group_step;
            in_at += kStage * BB;
            if (in_at == ring + D * BB + lane * 16) in_at = ring + lane * 16;
        }
        cp_async_commit();
    };
#pragma unroll
    for (int i = 0; i < kDepth - 1; ++i) fetch();  // weights: no kernel before this one writes them
    pdl_wait();

    const uint32_t hs = smem_u32(w4_smem) + w4_part_bytes<NT, W>() + w4_ring_bytes<NG, W>(D);
    const int stride = w4_h_stride(kblocks);
    if (HS) {
        for (int i = threadIdx.x; i < kblocks * 16; i += W * 32) {
            const int bytes = 8 * i < K ? 16 : 0;
            const uint16_t* s = h + (bytes ? 8 * i : 0);
            uint32_t d = hs + i * 16;
            for (int m = 0; m < M; ++m, s += K, d += stride) cp_async16_ca(d, s, bytes);
        }
        cp_async_commit();
        cp_async_wait<0>();
        __syncthreads();
    }
    // B operand of a block: rows nt * 8 + g of h, columns 32 j + 8 t.  Rows beyond M repeat the last one (their
    // columns of the product are not stored).
    uint32_t hoff[NT];
    const uint16_t* hrow[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int m = min(nt * 8 + g, M - 1);
        hoff[nt] = hs + m * stride + t * 16;
        hrow[nt] = h + (long long)m * K + 8 * t;
    }

    uint32_t at = ring;
    for (int group = group0; group < n_groups; group += group_step) {
        float acc[TG][NT][4] = {};
        for (int kb = kb0; kb < kb0 + nkb; kb += CB) {
            fetch();
            cp_async_wait<kDepth - 1>();  // the oldest of the stages in flight
            __syncwarp();
#pragma unroll
            for (int i = 0; i < CB; ++i) {
                if (i && kb + i >= kb0 + nkb) break;
                uint4 b[NT][4];
                if (HS) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int j = 0; j < 4; ++j) b[nt][j] = lds16(hoff[nt] + (kb + i) * 256 + j * 64);
                } else {
                    const bool whole = (kb + i + 1) * kQ4Cols <= K;  // only the last block has columns beyond K
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            b[nt][j] = whole || (kb + i) * kQ4Cols + 32 * j + 8 * t < K
                                           ? ld_reuse16(hrow[nt] + (kb + i) * kQ4Cols + 32 * j)
                                           : make_uint4(0, 0, 0, 0);
                }
#pragma unroll
                for (int u = 0; u < TG; ++u) {
                    W4Regs<NG> w;
                    w.load(at + (i + u) * BB, lane);
                    w4_block_mma<NG, NT>(w, b, acc[u]);
                }
            }
            at += kStage * BB;
            if (at == ring + D * BB) at = ring;
            __syncwarp();  // every lane has read the stage before the ring comes round to it
        }
#pragma unroll
        for (int u = 0; u < TG; ++u) {
            const int tile = group * TG + u;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
                part[(ks * NT + nt) * 32 + lane] = make_float4(acc[u][nt][0], acc[u][nt][1], acc[u][nt][2], acc[u][nt][3]);
            asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "r"(KS * 32) : "memory");
            const float* sums = reinterpret_cast<const float*>(part);
            for (int x = ks * 32 + lane; x < 128 * NT && tile < n_tiles; x += KS * 32) {
                const int e = x & 3, l = x >> 2 & 31, m = (x >> 7) * 8 + 2 * (l & 3) + (e & 1);
                const int n = tile * kQ4Rows + (l >> 2) + 8 * (e >> 1);
                if (m >= M || n >= N) continue;
                float s = 0.f;
                for (int v = 0; v < KS; ++v) s += sums[v * 128 * NT + x];
                float* o = out + (long long)m * N + n;
                *o = residual ? *o + s : s;
            }
            __syncwarp();  // the barrier wants whole warps
            asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "r"(KS * 32) : "memory");  // the sums are read
        }
    }
}

}  // namespace ls
