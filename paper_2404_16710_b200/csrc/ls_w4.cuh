// Linear layer of the decode loop on 4-bit weights: out[m, n] (+)= sum_k c[n, k] s[n, k / group] h[m, k] for
// M <= 16 rows (LayerSkip Sec. 4.3: a draft pass has one row, a verify pass num_draft + 1).  Format and
// block layout: ls_q4.cuh.
#pragma once
#include "ls_q4.cuh"

namespace ls {

constexpr int kW4Warps = 8;

// D = A * B + C on one tile; with C a constant zero the first product of a group starts a new sum
__device__ __forceinline__ void mma_bf16_16816_new(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                                   uint32_t b0, uint32_t b1)
{
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
        "{%10,%10,%10,%10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}

// One CTA per 16 weight rows; its warps take the 128-column blocks in turn.  The codes are the A operand
// (exact small integers in bf16), the rows of h the B operand; a group's products are summed on the tensor
// cores in fp32 and multiplied by the group's scale (per weight row: a lane holds rows g and g + 8) when
// they join the running sum.  Which blocks a warp adds, and in which order the warps' sums are added,
// depends on K only, so a row's result does not depend on how many rows share the pass.
template <int NG, int NT>
__global__ void __launch_bounds__(kW4Warps * 32)
linear_w4_kernel(const unsigned char* __restrict__ packed, const uint16_t* __restrict__ h, int M, int N, int K,
                 int kblocks, float* __restrict__ out, int residual)
{
    __shared__ float part[kW4Warps][NT * 8][17];
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const unsigned char* rows = packed + (long long)blockIdx.x * kblocks * w4_block_bytes(NG);
    float acc[NT][4] = {};
    for (int kb = warp; kb < kblocks; kb += kW4Warps) {
        const unsigned char* blk = rows + (long long)kb * w4_block_bytes(NG);
        const uint4 lo = ld_stream16(blk + lane * 16), hi = ld_stream16(blk + kQ4CodeBytes / 2 + lane * 16);
        uint32_t s_lo[NG], s_hi[NG];
        q4_row_scales<NG>(blk + kQ4CodeBytes + g * NG * 2, s_lo);
        q4_row_scales<NG>(blk + kQ4CodeBytes + (g + 8) * NG * 2, s_hi);
        const uint32_t wl[4] = {lo.x, lo.y, lo.z, lo.w}, wh[4] = {hi.x, hi.y, hi.z, hi.w};
        float c[NT][4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int k = kb * kQ4Cols + 32 * j + 8 * t;
            uint32_t a[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) a[2 * i] = q4_bf16x2(wl[j], i), a[2 * i + 1] = q4_bf16x2(wh[j], i);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                uint4 b = make_uint4(0, 0, 0, 0);
                if (nt * 8 + g < M && k < K) b = ld_reuse16(h + (long long)(nt * 8 + g) * K + k);
                if (j % (4 / NG) == 0)
                    mma_bf16_16816_new(c[nt], a[0], a[1], a[2], a[3], b.x, b.y);
                else
                    mma_bf16_16816(c[nt], a[0], a[1], a[2], a[3], b.x, b.y);
                mma_bf16_16816(c[nt], a[4], a[5], a[6], a[7], b.z, b.w);
                if ((j + 1) % (4 / NG) == 0) {
                    const float s0 = bf16lo(s_lo[j * NG / 4]), s1 = bf16lo(s_hi[j * NG / 4]);
                    acc[nt][0] = fmaf(s0, c[nt][0], acc[nt][0]);
                    acc[nt][1] = fmaf(s0, c[nt][1], acc[nt][1]);
                    acc[nt][2] = fmaf(s1, c[nt][2], acc[nt][2]);
                    acc[nt][3] = fmaf(s1, c[nt][3], acc[nt][3]);
                }
            }
        }
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        part[warp][nt * 8 + 2 * t][g] = acc[nt][0];
        part[warp][nt * 8 + 2 * t + 1][g] = acc[nt][1];
        part[warp][nt * 8 + 2 * t][g + 8] = acc[nt][2];
        part[warp][nt * 8 + 2 * t + 1][g + 8] = acc[nt][3];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < NT * 8 * 16; i += kW4Warps * 32) {
        const int m = i / 16, r = i % 16;
        const long long n = (long long)blockIdx.x * kQ4Rows + r;
        if (m >= M || n >= N) continue;
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < kW4Warps; ++w) s += part[w][m][r];
        float* o = out + (long long)m * N + n;
        *o = residual ? *o + s : s;
    }
}

}  // namespace ls
