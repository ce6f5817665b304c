// Matrix product in 8 bits with a scale for each block of 128: out[m, n] (+)= sum_k h[m, k] w[n, k], both operands in the
// format of ls_f8.cuh, any number of rows.
//
// The 128 columns of a block are one row of a 128B-swizzled tile and four tcgen05.mma (kind f8f6f4, K = 32).  Their
// sum goes to a tensor-memory buffer of its own; four warps read it back, multiply by the product of the two scales
// and add it to fp32 registers, so what the tensor cores sum is never longer than 128 and the rest is plain fp32.
#pragma once
#include "ls_f8.cuh"
#include "ls_prefill_attn.cuh"

namespace ls {

// D[tmem] (+)= A[smem desc] * B[smem desc]^T, e4m3 inputs, fp32 accumulate
__device__ __forceinline__ void tc_mma_f8(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// 16 columns of the thread's lane; the caller waits (tc_wait_ld)
__device__ __forceinline__ void tc_ld16(uint32_t taddr, uint32_t (&v)[16])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
          "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
        : "r"(taddr));
}

struct F8Linear {
    const unsigned char *ws, *hs;  // scale bytes of weights and tokens
    int M, N, K;
    void* out;
    const void* add;  // null or of out's type
    int64_t ldo, lda;
    int bf16;
    int32_t* status;
};

// value (+ add) to out[m, n]
__device__ __forceinline__ void f8_put(const F8Linear& p, long long m, int n, float v)
{
    if (p.bf16) {
        if (p.add) v += bf16f(__ldcg(reinterpret_cast<const uint16_t*>(p.add) + m * p.lda + n));
        reinterpret_cast<uint16_t*>(p.out)[m * p.ldo + n] = f2bf(v);
    } else {
        if (p.add) v += __ldcg(reinterpret_cast<const float*>(p.add) + m * p.lda + n);
        reinterpret_cast<float*>(p.out)[m * p.ldo + n] = v;
    }
}

// ------------------------------------------------------------------ weights in the lanes, tokens in the columns
// A CTA computes 128 rows of weights x NT tokens: the weights are the 128-row operand, so that few tokens leave no part
// of the tensor core's rows idle, and a warp's stores of a token are 32 neighbouring outputs.  The S CTAs of a cluster
// share a tile, each taking a stretch of the blocks along K; their sums meet in the CTA that owns the token, in order.
constexpr int kF8Threads = 224;  // warps 0-3: sums and stores, 4: TMA, 5: MMA, 6: scales
constexpr int kF8WBytes = kF8Block * kF8Block;
constexpr int kF8SmemMax = 227 * 1024;
constexpr int kF8Slots = 4;  // slots of scales, one word of scale bytes (four blocks) each

template <int NT>
struct F8Cfg {
    static constexpr int kStage = kF8WBytes + NT * kF8Block;
    static constexpr int kScale = kF8Slots * 4 * NT * 4;      // floats [slot][block][token]
    static constexpr int kPart = NT * kF8Block * 4;           // what the cluster's CTAs send: [rank][token][row]
    static constexpr int kFixed = 1024 + kScale + kPart + 512;
    static constexpr int kFit = (kF8SmemMax - kFixed) / kStage;
    static constexpr int kStages = kFit < 10 ? kFit : 10;
    static constexpr int kBufs = NT <= 64 ? 4 : 2;            // tensor-memory buffers
    static constexpr int kCols = kBufs * NT < 32 ? 32 : kBufs * NT;
    static constexpr size_t kSmem = (size_t)kStages * kStage + kFixed;
};

// grid (S, tiles of 128 weight rows, tiles of NT tokens), clusters (S, 1, 1)
template <int NT>
__global__ void __launch_bounds__(kF8Threads, 1)
linear_f8_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_h, const F8Linear p)
{
    using C = F8Cfg<NT>;
    extern __shared__ unsigned char f8_raw[];
    __shared__ int failed;
    const uint32_t base = (smem_u32(f8_raw) + 1023u) & ~1023u;
    const uint32_t sc0 = base + C::kStages * C::kStage, part0 = sc0 + C::kScale, bars = part0 + C::kPart;
    auto full = [&](int s) { return bars + 8u * s; };
    auto empty = [&](int s) { return bars + 8u * (C::kStages + s); };
    auto tfull = [&](int b) { return bars + 8u * (2 * C::kStages + b); };
    auto tempty = [&](int b) { return bars + 8u * (2 * C::kStages + 4 + b); };
    auto sfull = [&](int b) { return bars + 8u * (2 * C::kStages + 8 + b); };
    auto sempty = [&](int b) { return bars + 8u * (2 * C::kStages + 12 + b); };
    const uint32_t tslot = bars + 8u * (2 * C::kStages + 16);
    static_assert(8 * (2 * C::kStages + 17) <= 512, "barriers");

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int S = gridDim.x, rank = blockIdx.x;
    const int n0 = blockIdx.y * kF8Block;
    const long long m0 = (long long)blockIdx.z * NT;
    const int nkb = (p.K + kF8Block - 1) / kF8Block;
    const int kb0 = (int)((long long)nkb * rank / S), kb1 = (int)((long long)nkb * (rank + 1) / S);

    if (tid == 0) {
        for (int s = 0; s < C::kStages; ++s) {
            mbar_init(full(s), 1);
            mbar_init(empty(s), 1);
        }
        for (int b = 0; b < C::kBufs; ++b) {
            mbar_init(tfull(b), 1);
            mbar_init(tempty(b), 4);
        }
        for (int b = 0; b < kF8Slots; ++b) {
            mbar_init(sfull(b), 1);
            mbar_init(sempty(b), 4);
        }
        failed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tslot), "r"(C::kCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    pdl_launch_dependents();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    uint32_t tmem;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(tmem) : "r"(tslot));
    if (S > 1) cluster_sync_all();  // every CTA of the cluster runs before any sends to it

    float acc[NT];
    if (warp == 4) {
        if (lane == 0) {  // TMA: the weights of the first stages before the wait for the operation ahead
            const int ahead = min(kb1 - kb0, C::kStages);
            for (int i = 0; i < ahead; ++i) {
                mbar_expect_tx(full(i), C::kStage);
                tma_load_2d(base + i * C::kStage, &map_w, (kb0 + i) * kF8Block, n0, full(i));
            }
            pdl_wait();
            for (int i = 0; i < ahead; ++i)
                tma_load_2d(base + i * C::kStage + kF8WBytes, &map_h, (kb0 + i) * kF8Block, (int)m0, full(i));
            for (int i = ahead; i < kb1 - kb0; ++i) {
                const int s = i % C::kStages;
                if (!mbar_wait(empty(s), (i / C::kStages - 1) & 1)) {
                    failed = 1;
                    break;
                }
                mbar_expect_tx(full(s), C::kStage);
                tma_load_2d(base + s * C::kStage, &map_w, (kb0 + i) * kF8Block, n0, full(s));
                tma_load_2d(base + s * C::kStage + kF8WBytes, &map_h, (kb0 + i) * kF8Block, (int)m0, full(s));
            }
        }
    } else if (warp == 5) {
        if (lane == 0) {
            // instruction descriptor: D fp32, A and B e4m3, both K-major, N = NT, M = 128
            const uint32_t idesc = (1u << 4) | ((uint32_t)(NT >> 3) << 17) | ((uint32_t)(kF8Block >> 4) << 24);
            for (int i = 0; i < kb1 - kb0; ++i) {
                const int s = i % C::kStages, b = i % C::kBufs;
                if ((i >= C::kBufs && !mbar_wait(tempty(b), (i / C::kBufs - 1) & 1)) || !mbar_wait(full(s), (i / C::kStages) & 1)) {
                    failed = 1;
                    break;
                }
                tc_fence_after();
                const uint64_t da = umma_desc_sw128(base + s * C::kStage), db = umma_desc_sw128(base + s * C::kStage + kF8WBytes);
#pragma unroll
                for (int k4 = 0; k4 < 4; ++k4)  // 32 bytes further along K per MMA
                    tc_mma_f8(tmem + (uint32_t)(b * NT), da + 2 * k4, db + 2 * k4, idesc, k4 != 0);
                tc_commit(empty(s));
                tc_commit(tfull(b));
            }
        }
    } else if (warp == 6) {
        // products of the scales of four blocks at a time, as floats
        const int width = (int)f8_scale_width(p.K);
        pdl_wait();
        for (int g = kb0 / 4, i = 0; g * 4 < kb1; ++g, ++i) {
            const int s = i % kF8Slots;
            if (i >= kF8Slots && !mbar_wait(sempty(s), (i / kF8Slots - 1) & 1)) {
                failed = 1;
                break;
            }
            const uint32_t w = __ldcg(reinterpret_cast<const uint32_t*>(p.ws + (long long)blockIdx.y * width + 4 * g));
#pragma unroll
            for (int t = lane; t < NT; t += 32) {
                const uint32_t h = m0 + t < p.M ? __ldcg(reinterpret_cast<const uint32_t*>(p.hs + (m0 + t) * width + 4 * g)) : 0u;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float f = f8_scale(w >> (8 * j) & 255u) * f8_scale(h >> (8 * j) & 255u);
                    asm volatile("st.shared.f32 [%0], %1;" ::"r"(sc0 + 4u * ((s * 4 + j) * NT + t)), "f"(f) : "memory");
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(sfull(s));
        }
    } else {
        // lane 32 w + l of tensor memory is row n0 + 32 w + l of the weights
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[j] = 0.f;
        bool ok = true;
#pragma unroll 1
        for (int kb = kb0; kb < kb1; ++kb) {
            const int i = kb - kb0, b = i % C::kBufs, gi = kb / 4 - kb0 / 4, s = gi % kF8Slots;
            if (i == 0 || kb % 4 == 0) ok = mbar_wait(sfull(s), (gi / kF8Slots) & 1);
            ok = ok && mbar_wait(tfull(b), (i / C::kBufs) & 1);
            if (!ok) {
                failed = 1;
                break;
            }
            tc_fence_after();
            const uint32_t t0 = tmem + ((uint32_t)(warp * 32) << 16) + (uint32_t)(b * NT);
            const uint32_t s0 = sc0 + 4u * ((s * 4 + kb % 4) * NT);
#pragma unroll
            for (int c = 0; c < NT; c += 16) {
                uint32_t t[16];
                tc_ld16(t0 + c, t);
                tc_wait_ld();
#pragma unroll
                for (int j = 0; j < 16; j += 4) {
                    const uint4 f = lds16(s0 + 4u * (c + j));
                    acc[c + j] = fmaf(__uint_as_float(t[j]), __uint_as_float(f.x), acc[c + j]);
                    acc[c + j + 1] = fmaf(__uint_as_float(t[j + 1]), __uint_as_float(f.y), acc[c + j + 1]);
                    acc[c + j + 2] = fmaf(__uint_as_float(t[j + 2]), __uint_as_float(f.z), acc[c + j + 2]);
                    acc[c + j + 3] = fmaf(__uint_as_float(t[j + 3]), __uint_as_float(f.w), acc[c + j + 3]);
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(tempty(b));
                if (kb % 4 == 3) mbar_arrive(sempty(s));
            }
        }
        pdl_wait();
        if (S > 1) {
            // token j belongs to CTA j / (NT / S): send it there
            const int per = NT / S;
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const uint32_t to = cluster_map(part0 + 4u * ((rank * per + j % per) * kF8Block + tid), j / per);
                asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to), "f"(acc[j]) : "memory");
            }
        }
    }
    __syncwarp();
    if (S > 1) cluster_sync_all();
    else __syncthreads();
    if (failed) {
        if (tid == 0) {
            if (p.status) *p.status = DEV_TIMEOUT;
            __nanosleep(1000000);  // let copies that may still be in flight land before the CTA goes away
        }
    } else if (warp < 4 && n0 + tid < p.N) {
        if (S > 1) {
            const int per = NT / S;
            for (int j = 0; j < per; ++j) {
                const long long m = m0 + rank * per + j;
                if (m >= p.M) break;
                float v = 0.f;
                for (int r = 0; r < S; ++r) {
                    float u;
                    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(u) : "r"(part0 + 4u * ((r * per + j) * kF8Block + tid)) : "memory");
                    v += u;
                }
                f8_put(p, m, n0 + tid, v);
            }
        } else {
#pragma unroll
            for (int j = 0; j < NT; ++j)
                if (m0 + j < p.M) f8_put(p, m0 + j, n0 + tid, acc[j]);
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 0)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(C::kCols) : "memory");
}

}  // namespace ls
