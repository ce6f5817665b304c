// Matrix product in 8 bits with a scale for each block of 128: out[m, n] = (add[m, n] +) sum_k h[m, k] w[n, k], both operands
// in the format of ls_f8.cuh, any number of rows m ("tokens").
//
// The 128 codes of a block's row are a row of a 128B-swizzled tile, as TMA writes it and four tcgen05.mma of K = 32 read it.
// In both kernels the weights are the operand in the lanes and the tokens the columns: few tokens then leave no lanes idle, tiles
// follow the tokens' number in steps of 16, and a warp's store of a token is 32 neighbouring outputs.
//   up to 128 tokens   linear_f8_kernel: bound by reading the weights, so 128 rows a CTA, two CTAs an SM, K split over a cluster
//                      where there are few tiles.  Scales multiply the sums of 128 columns in fp32 registers.
//   more               linear_f8_pair_kernel: bound by the products (and, through them, by the power limit), so CTA pairs, 256 rows
//                      x 240 tokens, and the scales multiplied in the tensor cores.
// Why not one for both: at 16 tokens the pair kernel's start (tensor memory, a cluster, scales through shared memory and tensor memory)
// costs what the products do not (4096 x 4096: 18.7 us, 7.5 - 10 without); at 4096 the first form reads back 128 x 128 sums for each
// block along K and stops at 584 TFLOP/s (2650 with pairs).
// Measured (B200, 1965 MHz until the power limit, inputs not in L2): 4096 x 4096, one token 7.5 us (5.6 chained); 4096 x 11008, 7 tokens
// with add 12.4; 128256 x 4096, 16 tokens 83 - 88 (6.0 - 6.4 TB/s); 12288 x 4096, 1030 tokens 47 (2.2 PFLOP/s); 22016 x 4096, 4096 tokens
// 276 - 282 (2.65 PFLOP/s; at 1.18 GHz under the power limit 84 % of what the tensor cores can do).
// Rows of K = 16 mod 32 bytes begin inside a 32-byte sector: the loads of every second row then cost more (2334 x 7600, 2108 tokens:
// 49.3 us, K = 7616 40.4).  The layout is the caller's, and both operands have to agree on the columns of a step.
#pragma once
#include <type_traits>

#include "ls_f8.cuh"
#include "ls_attention.cuh"
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
// true in one lane of a converged warp
__device__ __forceinline__ bool elect_one()
{
    uint32_t one;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one));
    return one != 0;
}
// 16 columns of the thread's lane; the caller waits (tc_wait_ld)
__device__ __forceinline__ void tc_ld16(uint32_t taddr, uint32_t* v)
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
          "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
        : "r"(taddr));
}

// acc[j] += t[j] * scale[j], scales in shared memory
template <int N>
__device__ __forceinline__ void f8_add_scaled(float* acc, const uint32_t* t, uint32_t scales)
{
#pragma unroll
    for (int j = 0; j < N; j += 4) {
        const uint4 f = lds16(scales + 4u * j);
        acc[j] = fmaf(__uint_as_float(t[j]), __uint_as_float(f.x), acc[j]);
        acc[j + 1] = fmaf(__uint_as_float(t[j + 1]), __uint_as_float(f.y), acc[j + 1]);
        acc[j + 2] = fmaf(__uint_as_float(t[j + 2]), __uint_as_float(f.z), acc[j + 2]);
        acc[j + 3] = fmaf(__uint_as_float(t[j + 3]), __uint_as_float(f.w), acc[j + 3]);
    }
}

struct F8Linear {
    const unsigned char *ws, *hs;  // scale bytes of weights and tokens
    int M, N, K;
    void* out;
    const void* add;  // null or of out's type
    int64_t ldo, lda;
    int32_t* status;
};

// out[m, n] = v (+ add)
template <bool BF16>
__device__ __forceinline__ void f8_put(const F8Linear& p, long long m, int n, float v)
{
    if constexpr (BF16) {
        if (p.add) v += bf16f(__ldcg(reinterpret_cast<const uint16_t*>(p.add) + m * p.lda + n));
        reinterpret_cast<uint16_t*>(p.out)[m * p.ldo + n] = f2bf(v);
    } else {
        if (p.add) v += __ldcg(reinterpret_cast<const float*>(p.add) + m * p.lda + n);
        reinterpret_cast<float*>(p.out)[m * p.ldo + n] = v;
    }
}
__device__ __forceinline__ float lds_f32(uint32_t addr)
{
    float v;
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}
// out of up to 16 tokens from m on
template <bool BF16>
__device__ __forceinline__ void f8_store16(const F8Linear& p, long long m, int n, int rows, const float* sum)
{
    using T = std::conditional_t<BF16, uint16_t, float>;
    T* dst = reinterpret_cast<T*>(p.out) + m * p.ldo + n;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        if (j < rows) {
            if constexpr (BF16) *dst = f2bf(sum[j]);
            else *dst = sum[j];
        }
        dst += p.ldo;
    }
}
// add of N tokens from m on, those below rows
template <bool BF16, int N>
__device__ __forceinline__ void f8_fetch_add(const F8Linear& p, long long m, int n, int rows, float* a)
{
    using T = std::conditional_t<BF16, uint16_t, float>;
    const T* src = reinterpret_cast<const T*>(p.add) + m * p.lda + n;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        if (j < rows) {
            if constexpr (BF16) a[j] = bf16f(__ldcg(src));
            else a[j] = __ldcg(src);
        }
        src += p.lda;
    }
}

// ------------------------------------------------------------------ up to 128 tokens
// A CTA takes 128 rows of weights and up to NT tokens.  A block's four MMAs (kind f8f6f4) leave their sum in tensor-memory columns
// of its own; four warps read them back, multiply by the product of the two scales (laid out ahead as floats by a warp of its own)
// and add to fp32 registers.  kUnit blocks change hands at a time: a hand-over takes some 400 cycles, a block's weights 700 at the
// copy rate.  The S CTAs of a cluster share a tile, each a stretch of the blocks along K; their sums meet in the CTA
// that owns the token, in order.  S is a function of the matrix alone: up to 16 tokens a row's bits do not depend on how many there are.
// Steps (4096 x 4096, one token / 128256 x 4096, 16): first form 11.8 / 130 us; 256-byte sectors asked of L2 - / 122; scale words
// asked for 12 blocks ahead and two CTAs an SM 10.1 / 79; hand-overs of four blocks 8.8; relaxed arrival at the cluster's first barrier (a
// release waits 1.9 us), barriers set up by a warp, sums sent without divisions 7.5.  With mma.sync on f16 (cvt from e4m3, registers straight
// from global memory) one token took 7.2 us and 16 took 11.2 (10.0 here), larger matrices up to twice as long: not kept.
constexpr int kF8Threads = 224;  // warps 0-3: sums and stores, 4: TMA, 5: MMA, 6: scales
constexpr int kF8WBytes = kF8Block * kF8Block;
constexpr int kF8SmemMax = 227 * 1024;
constexpr int kF8Slots = 4;  // slots of scales, one word of scale bytes (four blocks) each
constexpr int kF8MaxStages = 11;
template <int NT, int CTAS>  // CTAs that fit an SM
struct F8Cfg {
    static constexpr int kStage = kF8WBytes + NT * kF8Block;
    static constexpr int kScale = kF8Slots * 4 * NT * 4;      // floats [slot][block][token]
    static constexpr int kPart = NT * kF8Block * 4;           // what the cluster's CTAs send: [token / S][rank][row]
    static constexpr int kUnit = NT <= 16 ? 4 : NT <= 32 ? 2 : 1;  // blocks along K that change hands together
    static constexpr int kBufs = NT == 64 ? 4 : 2;            // tensor-memory buffers of kUnit * NT columns
    static constexpr int kCols = kBufs * kUnit * NT;
    static constexpr int fixed(int S) { return 1024 + kScale + (S > 1 ? kPart : 0) + 512; }
    static constexpr int stages(int S)
    {
        const int fit = (kF8SmemMax / CTAS - 1024 - fixed(S)) / kStage;
        return fit < kF8MaxStages ? fit : kF8MaxStages;
    }
    static constexpr size_t smem(int S) { return (size_t)stages(S) * kStage + fixed(S); }
};

// sums of the first `rows` tokens to the CTAs that own them: token j is the (j / S)-th of CTA j % S
template <int NT, int S>
__device__ __forceinline__ void f8_send(const float* acc, uint32_t row, int rows)
{
#pragma unroll
    for (int r = 0; r < S; ++r) {
        const uint32_t to = cluster_map(row, r);
#pragma unroll
        for (int j = r; j < NT; j += S)
            if (j < rows)
                asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to + 4u * (j / S * S * kF8Block)), "f"(acc[j]) : "memory");
    }
}
// the tokens m, m + S, ... of this CTA: sums of the cluster's CTAs in order
template <int NT, int S, bool BF16>
__device__ __forceinline__ void f8_join(const F8Linear& p, long long m, int n, uint32_t row)
{
#pragma unroll 1
    for (int j = 0; j < NT / S && m < p.M; ++j, m += S) {
        float u[S], v = 0.f;
#pragma unroll
        for (int r = 0; r < S; ++r) u[r] = lds_f32(row + 4u * ((j * S + r) * kF8Block));
#pragma unroll
        for (int r = 0; r < S; ++r) v += u[r];
        f8_put<BF16>(p, m, n, v);
    }
}

// grid (S, tiles of 128 weight rows), clusters (S, 1, 1); at most NT tokens
template <int NT, bool BF16, int CTAS>
__global__ void __launch_bounds__(kF8Threads, CTAS)
linear_f8_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_h, const F8Linear p, const int stages)
{
    using C = F8Cfg<NT, CTAS>;
    extern __shared__ unsigned char f8_raw[];
    __shared__ int failed;
    const uint32_t base = (smem_u32(f8_raw) + 1023u) & ~1023u;
    const int S = gridDim.x, rank = blockIdx.x;  // S: 1, 2, 4 or 8
    const uint32_t sc0 = base + stages * C::kStage, part0 = sc0 + C::kScale, bars = part0 + (S > 1 ? C::kPart : 0);
    auto full = [&](int s) { return bars + 8u * s; };
    auto empty = [&](int s) { return bars + 8u * (kF8MaxStages + s); };
    auto tfull = [&](int b) { return bars + 8u * (2 * kF8MaxStages + b); };
    auto tempty = [&](int b) { return bars + 8u * (2 * kF8MaxStages + 4 + b); };
    auto sfull = [&](int b) { return bars + 8u * (2 * kF8MaxStages + 8 + b); };
    auto sempty = [&](int b) { return bars + 8u * (2 * kF8MaxStages + 12 + b); };
    const uint32_t tslot = bars + 8u * (2 * kF8MaxStages + 16);
    static_assert(8 * (2 * kF8MaxStages + 17) <= 512, "barriers");

    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    const int n0 = blockIdx.y * kF8Block;
    const int nkb = (p.K + kF8Block - 1) / kF8Block;
    const int kb0 = (int)((long long)nkb * rank / S), kb1 = (int)((long long)nkb * (rank + 1) / S);

    const int ahead = min(kb1 - kb0, stages);
    if (warp == 4) {  // barriers, and at once the weights of the first stages: they need not wait for the operation ahead
        if (lane < 2 * kF8MaxStages) mbar_init(bars + 8u * lane, 1);
        if (lane < C::kBufs) {
            mbar_init(tfull(lane), 1);
            mbar_init(tempty(lane), 4);
        }
        if (lane < kF8Slots) {
            mbar_init(sfull(lane), 1);
            mbar_init(sempty(lane), 4);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) {
            failed = 0;
            for (int i = 0; i < ahead; ++i) {
                mbar_expect_tx(full(i), C::kStage);
                tma_load_2d(base + i * C::kStage, &map_w, (kb0 + i) * kF8Block, n0, full(i));
            }
        }
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
    if (S > 1) cluster_arrive_relaxed();  // "this CTA runs": a release here takes 1.9 us

    pdl_wait();  // before any bounded wait: the operation ahead may take its time

    float acc[NT];
    if (warp == 4) {
        if (lane == 0) {
            for (int i = 0; i < ahead; ++i)
                tma_load_2d(base + i * C::kStage + kF8WBytes, &map_h, (kb0 + i) * kF8Block, 0, full(i));
            for (int i = ahead; i < kb1 - kb0; ++i) {
                const int s = i % stages;
                if (!mbar_wait(empty(s), (i / stages - 1) & 1)) {
                    failed = 1;
                    break;
                }
                mbar_expect_tx(full(s), C::kStage);
                tma_load_2d(base + s * C::kStage, &map_w, (kb0 + i) * kF8Block, n0, full(s));
                tma_load_2d(base + s * C::kStage + kF8WBytes, &map_h, (kb0 + i) * kF8Block, 0, full(s));
            }
        }
    } else if (warp == 5) {
        // the whole warp walks the loop and one lane issues: what an instruction names stays in uniform registers
        // instruction descriptor: D fp32, A and B e4m3, both K-major, N = NT, M = 128
        constexpr uint32_t idesc = (1u << 4) | ((uint32_t)(NT >> 3) << 17) | ((uint32_t)(kF8Block >> 4) << 24);
        const uint64_t desc0 = umma_desc_sw128(0);
        const bool one = elect_one();
        uint32_t s = 0, s_phase = 0, b = 0, b_phase = 1;  // a buffer that was never used counts as read
        bool ok = true;
        for (int kb = kb0; kb < kb1 && ok;) {
            ok = mbar_wait(tempty(b), b_phase);
            // blocks up to the next multiple of kUnit, block q of it in columns q * NT
            do {
                ok = ok && mbar_wait(full(s), s_phase);
                if (!ok) break;
                tc_fence_after();
                const uint64_t da = desc0 + ((base + s * C::kStage) >> 4), db = da + (kF8WBytes >> 4);
                if (one) {
#pragma unroll
                    for (int k4 = 0; k4 < 4; ++k4)  // 32 bytes further along K per MMA
                        tc_mma_f8(tmem + (b * C::kUnit + kb % C::kUnit) * NT, da + 2 * k4, db + 2 * k4, idesc, k4 != 0);
                    tc_commit(empty(s));
                }
                if (++s == stages) s = 0, s_phase ^= 1u;
                ++kb;
            } while (kb < kb1 && kb % C::kUnit);
            if (one && ok) tc_commit(tfull(b));
            if (++b == C::kBufs) b = 0, b_phase ^= 1u;
        }
        if (!ok) failed = 1;
    } else if (warp == 6) {
        // products of the scales of four blocks at a time, as floats; words are asked for AHEAD times four blocks before
        constexpr int AHEAD = 3, R = (NT + 31) / 32;
        const int width = (int)f8_scale_width(p.K), g0 = kb0 / 4, gn = (kb1 + 3) / 4;
        uint32_t w[AHEAD + 1], h[AHEAD + 1][R];
        auto fetch = [&](int g, uint32_t& fw, uint32_t (&fh)[R]) {
            if (g >= gn) return;
            fw = __ldcg(reinterpret_cast<const uint32_t*>(p.ws + (long long)blockIdx.y * width + 4 * g));
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int t = 32 * r + lane;
                fh[r] = t < p.M ? __ldcg(reinterpret_cast<const uint32_t*>(p.hs + (long long)t * width + 4 * g)) : 0u;
            }
        };
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) fetch(g0 + i, w[i], h[i]);
        for (int g = g0, i = 0; g < gn; ++g, ++i) {
            const int s = i % kF8Slots;
            fetch(g + AHEAD, w[AHEAD], h[AHEAD]);
            if (i >= kF8Slots && !mbar_wait(sempty(s), (i / kF8Slots - 1) & 1)) {
                failed = 1;
                break;
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int t = 32 * r + lane;
                if (t < NT) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float f = f8_scale(w[0] >> (8 * j) & 255u) * f8_scale(h[0][r] >> (8 * j) & 255u);
                        asm volatile("st.shared.f32 [%0], %1;" ::"r"(sc0 + 4u * ((s * 4 + j) * NT + t)), "f"(f) : "memory");
                    }
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(sfull(s));
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                w[k] = w[k + 1];
#pragma unroll
                for (int r = 0; r < R; ++r) h[k][r] = h[k + 1][r];
            }
        }
    } else {
        // lane 32 w + l of tensor memory is row n0 + 32 w + l of the weights
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[j] = 0.f;
        bool ok = true;
        uint32_t b = 0, b_phase = 0;
#pragma unroll 1
        for (int kb = kb0; kb < kb1;) {
            const int gi = kb / 4 - kb0 / 4, s = gi % kF8Slots, end = min(kb1, (kb / C::kUnit + 1) * C::kUnit);
            if (kb == kb0 || kb % 4 == 0) ok = mbar_wait(sfull(s), (gi / kF8Slots) & 1);
            ok = ok && mbar_wait(tfull(b), b_phase);
            if (!ok) {
                failed = 1;
                break;
            }
            tc_fence_after();
            const uint32_t t0 = tmem + ((uint32_t)(warp * 32) << 16) + b * (C::kUnit * NT);
            const uint32_t s0 = sc0 + 4u * (s * 4 * NT);
            if constexpr (C::kUnit > 1) {
                uint32_t t[C::kUnit][NT];
#pragma unroll
                for (int q = 0; q < C::kUnit; ++q)
#pragma unroll
                    for (int c = 0; c < NT; c += 16) tc_ld16(t0 + q * NT + c, &t[q][c]);
                tc_wait_ld();
                const int q0 = kb % C::kUnit, q1 = q0 + end - kb, g0 = kb / C::kUnit * C::kUnit % 4;
#pragma unroll
                for (int q = 0; q < C::kUnit; ++q)
                    if (q >= q0 && q < q1) f8_add_scaled<NT>(acc, t[q], s0 + 4u * ((g0 + q) * NT));
            } else {
#pragma unroll
                for (int c = 0; c < NT; c += 16) {
                    uint32_t t[16];
                    tc_ld16(t0 + c, t);
                    tc_wait_ld();
                    f8_add_scaled<16>(acc + c, t, s0 + 4u * (kb % 4 * NT + c));
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(tempty(b));
                if (end % 4 == 0) mbar_arrive(sempty(s));
            }
            if (++b == C::kBufs) b = 0, b_phase ^= 1u;
            kb = end;
        }
    }
    __syncwarp();
    if (S > 1) {
        cluster_wait();  // every CTA of the cluster runs
        // token j belongs to CTA j % S: send it there, as its (j / S)-th, beside those of the other CTAs
        if (warp < 4) {
            const uint32_t row = part0 + 4u * (rank * kF8Block + tid);
            if (S == 2) f8_send<NT, 2>(acc, row, p.M);
            else if (S == 4) f8_send<NT, 4>(acc, row, p.M);
            else f8_send<NT, 8>(acc, row, p.M);
        }
        cluster_sync_all();
    } else {
        __syncthreads();
    }
    if (failed) {
        if (tid == 0) {
            if (p.status) *p.status = DEV_TIMEOUT;
            __nanosleep(1000000);  // let copies that may still be in flight land before the CTA goes away
        }
    } else if (warp < 4 && n0 + tid < p.N) {
        if (S > 1) {
            const uint32_t row = part0 + 4u * tid;
            if (S == 2) f8_join<NT, 2, BF16>(p, rank, n0 + tid, row);
            else if (S == 4) f8_join<NT, 4, BF16>(p, rank, n0 + tid, row);
            else f8_join<NT, 8, BF16>(p, rank, n0 + tid, row);
        } else {
#pragma unroll
            for (int j = 0; j < NT; j += 16) {
                float a[16];
                if (p.add) {  // all of it is asked for before anything is stored: out may be add
#pragma unroll
                    for (int i = 0; i < 16; ++i) a[i] = 0.f;
                    f8_fetch_add<BF16, 16>(p, j, n0 + tid, p.M - j, a);
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[j + i] += a[i];
                }
                f8_store16<BF16>(p, j, n0 + tid, p.M - j, acc + j);
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 0)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(C::kCols) : "memory");
}

// ------------------------------------------------------------------ many tokens: CTA pairs, scales in the tensor cores
// Two CTAs of a cluster compute 256 rows of weights x nt tokens (nt a multiple of 16, at most 240) with
// tcgen05.mma.cta_group::2 of kind mxf8f6f4: the tensor cores multiply each 32 columns' products by 2^(ew + eh) as they add
// them up, so a block's four MMAs name the same scale byte and no sum leaves tensor memory before the tile is
// done.  Scales go to tensor memory 512 columns at a time: a warp lays the words of 128 rows out as [row % 32][row / 32]
// in shared memory, tcgen05.cp spreads them over the lanes; byte i of a word is the i-th block's, which the instruction
// descriptor picks.  Weights are the 256-row operand, so that tiles follow the tokens' number in steps of 16 and a warp
// stores 32 neighbouring outputs; at 240 tokens two accumulators and the scales fit the 512 columns of tensor memory:
// a tile's sums are read while the next one's are made.  Every 16 blocks (2048 columns) sums move to fp32 registers: the tensor
// cores truncate as they add, and 11008 columns at once are off by 1.1e-6 of the result's norm, 2048 at a time by 1.6e-7.
// Persistent: pair p takes tiles p, p + P, ..., tokens fastest (pairs that run side by side share weights in L2).
// A block takes 480 cycles of products at 240 tokens and 500 in all; its loads are 31 KB a CTA, 60 bytes a cycle from L2, which is near what
// an SM gets.  Steps (22016 x 4096, 4096 tokens): one lane alone issuing 400 us; the whole warp walking the loop, so that
// descriptors stay in uniform registers, 338; eight storing warps with 120 tokens of straight code each 438, sixteen with 60 319 (instruction fetch);
// 256-byte sectors 312; scales by two warps, each asking for its next words behind its fence (which waits for loads under way) 290;
// the next stage's barrier asked ahead 277.  From there the power limit sets the clock.
constexpr int kF8PairTokens = 240;
constexpr int kF8PairRing = 7 * (kF8WBytes + kF8PairTokens / 2 * kF8Block);  // as many stages as fit, 7 at 240 tokens
constexpr int kF8PairMaxStages = 12;
// a stage: a CTA's weights, and half of the tokens
__host__ __device__ constexpr int f8_pair_stage(int nt) { return kF8WBytes + nt / 2 * kF8Block; }
__host__ __device__ constexpr int f8_pair_stages(int nt)
{
    return kF8PairRing / f8_pair_stage(nt) < kF8PairMaxStages ? kF8PairRing / f8_pair_stage(nt) : kF8PairMaxStages;
}
constexpr int kF8PairSlots = 4;
constexpr int kF8PairChunk = 16;             // blocks along K that are summed in tensor memory
constexpr int kF8PairSlot = 3 * 512;         // scale words of 128 rows of weights, of 256 tokens
constexpr int kF8PairScaleCols = 2 * kF8PairTokens;  // two sets of 16 columns behind the accumulators
constexpr int kF8PairThreads = 640;          // warps 0-15: sums and stores, 16: TMA, 17: MMA, 18, 19: scales
constexpr size_t kF8PairSmem = (size_t)kF8PairRing + kF8PairSlots * kF8PairSlot + 1024 + 512;
static_assert(f8_pair_stage(16) % 1024 == 0 && kF8PairSmem <= kF8SmemMax && kF8PairScaleCols + 32 <= 512, "shared and tensor memory");

// D[tmem] (+)= (A * scales)(B * scales)^T, e4m3, a scale for 32 columns of a row
__device__ __forceinline__ void tc_mma_f8_scaled_pair(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t sa,
                                                      uint32_t sb, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate)
        : "memory");
}
// 32 rows of 16 bytes of either CTA's shared memory -> 4 columns of its tensor memory, in all four groups of 32 lanes
__device__ __forceinline__ void tc_cp_scales_pair(uint32_t taddr, uint32_t smem)
{
    // rows 16 bytes apart, groups of 8 of them 128; no swizzle, descriptor version 1
    const uint64_t d = (uint64_t)((smem >> 4) & 0x3fff) | (uint64_t)(128 >> 4) << 32 | (uint64_t)1 << 46;
    asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(d) : "memory");
}

// mbar_wait for a barrier that the peer CTA arrives on too, after it has written what is read behind the wait
__device__ __forceinline__ bool mbar_wait_cluster(uint32_t bar, uint32_t parity)
{
    for (uint32_t it = 0; it < (1u << 22); ++it) {
        uint32_t done;
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(done)
            : "r"(bar), "r"(parity)
            : "memory");
        if (done) return true;
        if (it > 1024) __nanosleep(200);
    }
    return false;
}

__device__ __forceinline__ void tc_commit_to(uint32_t bar, uint16_t ctas)  // arrives on `bar` in these CTAs of the cluster
{
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(bar), "h"(ctas)
                 : "memory");
}
// whether the phase is complete, without waiting
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity)
{
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done)
        : "r"(bar), "r"(parity)
        : "memory");
    return done != 0;
}

// SPLIT: a cluster of sk pairs shares a tile, each taking a stretch along K; a pair's sums of 16 tokens go to the pair that
// owns them, through the rings, which by then are idle.  Every cluster has one tile then.
template <bool BF16, bool SPLIT>
__global__ void __launch_bounds__(kF8PairThreads, 1)
linear_f8_pair_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_h, const F8Linear p,
                      const int nt, const int token_tiles, const int n_tiles, const int sk)
{
    extern __shared__ unsigned char f8_raw[];
    __shared__ int failed;
    const uint32_t base = (smem_u32(f8_raw) + 1023u) & ~1023u;
    const uint32_t sc0 = base + kF8PairRing, bars = sc0 + kF8PairSlots * kF8PairSlot;
    const int stages = f8_pair_stages(nt), stage = f8_pair_stage(nt);
    auto full = [&](int s) { return bars + 8u * s; };
    auto empty = [&](int s) { return bars + 8u * (kF8PairMaxStages + s); };
    auto accf = [&](int b) { return bars + 8u * (2 * kF8PairMaxStages + b); };
    auto acce = [&](int b) { return bars + 8u * (2 * kF8PairMaxStages + 2 + b); };
    auto sfull = [&](int b) { return bars + 8u * (2 * kF8PairMaxStages + 4 + b); };
    auto sempty = [&](int b) { return bars + 8u * (2 * kF8PairMaxStages + 4 + kF8PairSlots + b); };
    const uint32_t tslot = bars + 8u * (2 * kF8PairMaxStages + 4 + 2 * kF8PairSlots);

    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    uint32_t cluster_rank;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(cluster_rank));
    const uint32_t rank = cluster_rank & 1u, leader = cluster_rank & ~1u;
    // tiles of this pair, and its blocks along K
    const int first = SPLIT ? (int)blockIdx.x / (2 * sk) : (int)blockIdx.x / 2, step = SPLIT ? n_tiles : (int)gridDim.x / 2;
    const int nkb = (p.K + kF8Block - 1) / kF8Block, all = (nkb + 3) / 4, own = SPLIT ? (int)cluster_rank / 2 : 0;
    const int g0 = SPLIT ? all * own / sk : 0, groups = SPLIT ? all * (own + 1) / sk - g0 : all;
    const int kb0 = 4 * g0, kb1 = min(nkb, kb0 + 4 * groups);

    if (warp == 16) {
        if (lane < kF8PairMaxStages) {
            mbar_init(full(lane), 1);
            mbar_init(empty(lane), 1);
        }
        if (lane < 2) {
            mbar_init(accf(lane), 1);
            mbar_init(acce(lane), 32);  // sixteen storing warps in each CTA of the pair
        }
        if (lane < kF8PairSlots) {
            mbar_init(sfull(lane), 2);  // the scale warps of both
            mbar_init(sempty(lane), 1);
        }
        if (lane == 0) failed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        __syncwarp();
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tslot), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    cluster_arrive_relaxed();  // behind the fence above: the peer's barriers exist before anything signals them
    cluster_wait();
    tc_fence_after();
    uint32_t tmem;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(tmem) : "r"(tslot));

    // Of a tile, warp w < 16 reads lanes 32 (w % 4) .. of this CTA's accumulators, rows of weights, and a quarter of the tokens.
    // Sixteen warps, as each runs through its tokens once a tile: longer straight code waits for its instructions.
    const int quarter = (nt / 4 + 15) / 16 * 16, c0 = (warp >> 2 & 3) * quarter, cols = min(quarter, nt - c0);
    auto row_of = [&](int t) { return (t / token_tiles * 2 + (int)rank) * kF8Block + (warp & 3) * 32 + lane; };
    float sum[64];
    if (warp == 16) {
        if (lane == 0) {
            const uint32_t bytes = 2u * (uint32_t)(kF8WBytes + nt / 2 * kF8Block);
            uint32_t s = 0, phase = 1;  // a stage that was never used counts as free
            bool ok = true;
            for (int t = first; t < n_tiles && ok; t += step) {
                const int w_row = (t / token_tiles * 2 + (int)rank) * kF8Block, h_row = t % token_tiles * nt + (int)rank * (nt / 2);
                for (int kb = kb0; kb < kb1; ++kb) {
                    if (!mbar_wait(empty(s), phase)) {
                        failed = 1;
                        ok = false;
                        break;
                    }
                    if (rank == 0) mbar_expect_tx(full(s), bytes);
                    const uint32_t lead = full(s) & kPeerBitMask;
                    tma_load_2d_pair(base + s * stage, &map_w, kb * kF8Block, w_row, lead);
                    tma_load_2d_pair(base + s * stage + kF8WBytes, &map_h, kb * kF8Block, h_row, lead);
                    if (++s == stages) s = 0, phase ^= 1u;
                }
            }
        }
    } else if (warp == 17) {
        if (rank == 0) {
            // The whole warp walks the loop and one lane issues: what an instruction names stays in uniform registers.
            // instruction descriptor: scales 2^(e - 127), A and B e4m3, both K-major, N = nt, M = 256 (128 per CTA)
            const uint32_t idesc = ((uint32_t)(nt >> 3) << 17) | (1u << 23) | (2u << 27);
            const uint64_t desc0 = umma_desc_sw128(0);
            const bool one = elect_one();
            const uint16_t both = (uint16_t)(3u << leader);  // the pair's CTAs in the cluster
            uint32_t s = 0, s_phase = 0, slot = 0, slot_phase = 0, old_phase = 1;
            uint32_t b = 0, b_phase = 1;  // an accumulator that was never used counts as read
            bool ok = true, ready = false;
            for (int t = first; t < n_tiles && ok; t += step) {
                for (int kb = kb0; kb < kb1 && ok; kb += 4) {
                    const uint32_t d = tmem + b * kF8PairTokens;
                    if ((kb - kb0) % kF8PairChunk == 0) {
                        if (!mbar_wait(acce(b), b_phase)) {
                            failed = 1;
                            ok = false;
                            break;
                        }
                        tc_fence_after();
                    }
                    // four blocks' scales; copies and products of a thread run in order
                    if (!mbar_wait_cluster(sfull(slot), slot_phase)) {
                        failed = 1;
                        ok = false;
                        break;
                    }
                    // the columns that the copies overwrite: the products of the group before the last have read them
                    if (!mbar_wait(sempty((slot + kF8PairSlots - 2) % kF8PairSlots), old_phase)) {
                        failed = 1;
                        ok = false;
                        break;
                    }
                    tc_fence_after();
                    const uint32_t sf = tmem + kF8PairScaleCols + (slot & 1u) * 16u, src = sc0 + slot * kF8PairSlot;
                    if (one) {
                        tc_cp_scales_pair(sf, src);
                        tc_cp_scales_pair(sf + 8, src + 512);
                        if (nt > 128) tc_cp_scales_pair(sf + 12, src + 1024);
                    }
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        if (kb + q >= kb1) break;
                        if (!ready && !mbar_wait(full(s), s_phase)) {
                            failed = 1;
                            ok = false;
                            break;
                        }
                        tc_fence_after();
                        const uint64_t da = desc0 + ((base + s * stage) >> 4), db = da + (kF8WBytes >> 4);
                        const uint32_t s_now = s;
                        if (++s == stages) s = 0, s_phase ^= 1u;
                        ready = mbar_test(full(s), s_phase);  // the next stage: its answer comes while the products are issued
                        if (one) {
                            const uint32_t id = idesc | (uint32_t)q << 4 | (uint32_t)q << 29;
#pragma unroll
                            for (int k4 = 0; k4 < 4; ++k4)
                                tc_mma_f8_scaled_pair(d, da + 2 * k4, db + 2 * k4, id, sf, sf + 8, ((kb - kb0) % kF8PairChunk | q | k4) != 0);
                            tc_commit_to(empty(s_now), both);
                        }
                    }
                    if (one && ok) tc_commit_to(sempty(slot), both);  // copies and products of these four blocks are done
                    if (++slot == kF8PairSlots) slot = 0, slot_phase ^= 1u;
                    if (slot == 2) old_phase ^= 1u;
                    if (ok && ((kb - kb0 + 4) % kF8PairChunk == 0 || kb + 4 >= kb1)) {
                        if (one) tc_commit_to(accf(b), both);
                        b ^= 1u;
                        if (b == 0) b_phase ^= 1u;
                    }
                }
            }
        }
    } else if (warp >= 18) {
        // Scale words of this CTA's weights (one for all its 128 rows) and of all the tile's tokens, four blocks at a time, the two warps
        // in turn.  The fence waits for the warp's loads too, so the next words are asked for behind it, and two
        // warps leave them the time of eight blocks (one warp: 2200 cycles for four, whatever the tile).
        const int width = (int)f8_scale_width(p.K), w_rows = (p.N + kF8Block - 1) / kF8Block;
        int t = first, gi = warp - 18;  // next group to ask for
        uint32_t w = 0, h[8];
        auto settle = [&] {
            while (gi >= groups) gi -= groups, t += step;
        };
        auto fetch = [&] {
            const int wb = t / token_tiles * 2 + (int)rank;
            const long long m0 = (long long)(t % token_tiles) * nt;
            w = wb < w_rows ? __ldcg(reinterpret_cast<const uint32_t*>(p.ws + (long long)wb * width + 4 * (g0 + gi))) : 0x7f7f7f7fu;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const long long m = m0 + 32 * j + lane;
                h[j] = 32 * j + lane < nt && m < p.M ? __ldcg(reinterpret_cast<const uint32_t*>(p.hs + m * width + 4 * (g0 + gi))) : 0x7f7f7f7fu;
            }
        };
        uint32_t slot = warp - 18, phase = 1;  // a slot that was never used counts as free
        settle();
        if (t < n_tiles) fetch();
        while (t < n_tiles) {
            if (!mbar_wait(sempty(slot), phase)) {
                failed = 1;
                break;
            }
            const uint32_t dst = sc0 + slot * kF8PairSlot + lane * 16;
            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(dst), "r"(w) : "memory");
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst + 512), "r"(h[0]), "r"(h[1]), "r"(h[2]), "r"(h[3]) : "memory");
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst + 1024), "r"(h[4]), "r"(h[5]), "r"(h[6]), "r"(h[7]) : "memory");
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // tcgen05.cp reads what was just stored
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(cluster_map(sfull(slot), leader));
            slot += 2;
            if (slot >= kF8PairSlots) slot -= kF8PairSlots, phase ^= 1u;
            gi += 2;
            settle();
            if (t < n_tiles) fetch();
        }
    } else {
        const uint32_t acce_leader[2] = {cluster_map(acce(0), leader), cluster_map(acce(1), leader)};
        uint32_t b = 0, b_phase = 0;
        bool ok = true;
        for (int t = first; t < n_tiles && ok; t += step) {
            const int n = row_of(t);
            const long long m0 = (long long)(t % token_tiles) * nt + c0;
            const int rows = (int)min((long long)cols, p.M - m0);
            // sums begin with add, which comes while the first products are made
#pragma unroll
            for (int j = 0; j < 64; ++j) sum[j] = 0.f;
            if (p.add && n < p.N && own == 0) f8_fetch_add<BF16, 64>(p, m0, n, rows, sum);
            for (int kb = kb0; kb < kb1; kb += kF8PairChunk) {
                if (!mbar_wait(accf(b), b_phase)) {
                    failed = 1;
                    ok = false;
                    break;
                }
                tc_fence_after();
                const uint32_t tacc = tmem + ((uint32_t)((warp & 3) * 32) << 16) + b * kF8PairTokens + c0;
#pragma unroll
                for (int c = 0; c < 64; c += 16) {
                    if (c < cols) {
                        uint32_t v[16];
                        tc_ld16(tacc + c, v);
                        tc_wait_ld();
#pragma unroll
                        for (int j = 0; j < 16; ++j) sum[c + j] += __uint_as_float(v[j]);
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(acce_leader[b]);
                b ^= 1u;
                if (b == 0) b_phase ^= 1u;
            }
            if (!SPLIT && ok && n < p.N) {
#pragma unroll
                for (int c = 0; c < 64; c += 16)
                    if (c < rows) f8_store16<BF16>(p, m0 + c, n, rows - c, sum + c);
            }
        }
    }
    if constexpr (SPLIT) {
        // the 16 tokens from c on belong to pair c / 16 % sk; part [pair][c / 16 / sk][warp][token][lane]
        __syncwarp();
        // every pair's products are made: nothing uses the rings any more (reads that are complete need no release, which takes 0.4 us)
        cluster_arrive_relaxed();
        cluster_wait();
        const uint32_t part = base + 4u * (uint32_t)(warp * 512 + lane), each = 4u * (uint32_t)(4 / sk) * 8192u;
        if (warp < 16) {
#pragma unroll
            for (int c = 0; c < 64; c += 16) {
                const int to = c / 16 % sk;
                if (c < cols && to != own) {
                    const uint32_t dst = cluster_map(part + (uint32_t)own * each + 4u * (uint32_t)(c / 16 / sk) * 8192u, 2u * to + rank);
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(dst + 128u * j), "f"(sum[c + j]) : "memory");
                }
            }
        }
        cluster_sync_all();
        const int n = row_of(first);
        const long long m0 = (long long)(first % token_tiles) * nt + c0;
        const int rows = (int)min((long long)cols, p.M - m0);
        if (warp < 16 && !failed) {
#pragma unroll
            for (int c = 0; c < 64; c += 16) {
                if (c < rows && c / 16 % sk == own) {
                    for (int from = 0; from < sk; ++from) {
                        if (from == own) continue;
                        const uint32_t src = part + (uint32_t)from * each + 4u * (uint32_t)(c / 16 / sk) * 8192u;
#pragma unroll
                        for (int j = 0; j < 16; ++j) sum[c + j] += lds_f32(src + 128u * j);
                    }
                    if (n < p.N) f8_store16<BF16>(p, m0 + c, n, rows - c, sum + c);
                }
            }
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (failed && tid == 0) {
        if (p.status) *p.status = DEV_TIMEOUT;
        __nanosleep(1000000);  // let copies that may still be in flight land before the CTA goes away
    }
    cluster_arrive_relaxed();  // both CTAs are done with tensor memory, and the MMAs with both shared memories
    cluster_wait();
    if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
}

}  // namespace ls
