// A layer's matrix product with what follows it, Y = act(X W^T + b) + R, in one kernel (cat_linear).
//
// Mathematics.  acc[n][t] = sum_k W[n][k] X[t][k] on the 5th-generation tensor cores (operands bf16 or fp16, products exact, sums in
// fp32 in TMEM); z = acc + b[n], y = act(z) + R[t][n] in fp32, rounded once to the type of Y.
//
// Layout.  The rows of W take the 128 lanes of an accumulator and the tokens its columns, whatever the number of tokens: one token fills
// an accumulator of 16 columns, and a thread of the epilogue owns one output column n -- its bias is one register, and the 32 lanes of a
// warp write 32 neighbouring columns of Y, so outputs, strides and residuals need no alignment at all.  Both operands arrive by TMA in
// 64-column slabs (128-byte swizzle, zero fill past the matrix, so K, N and M may be anything); rows that TMA cannot address (stride or base
// not a multiple of 16 bytes) are copied to the workspace first.
//
// Forms.  Many tokens: CTA pairs (cta_group::2) on tiles of 256 columns of Y x up to 256 tokens, persistent, accumulators double buffered so
// that one tile's epilogue passes under the next one's MMAs.  Few tokens: one CTA per 128 columns, and where those leave SMs idle the inner
// dimension is split over the CTAs of a cluster, whose partial sums meet in distributed shared memory in a fixed order (no atomics: the
// same call gives the same bits).
#include "cat_tc.cuh"

#include <cuda_bf16.h>

namespace cat {
namespace {

constexpr int LN_BK = 64;                       // inner columns per slab (128 bytes)
constexpr int LN_MAX_STAGES = 12;
constexpr int LN_EPI_WARPS = 16;                // warps of the epilogue at most: four per quarter of the TMEM lanes
constexpr int LN_MAX_THREADS = 32 * (2 + LN_EPI_WARPS);
constexpr int LN_RUN = 12;                      // slabs per run of an accumulator at most, where the result is fp32 (see linear_kernel) ...
constexpr int LN_RUN_16 = 24;                   // ... and where it is rounded to 16 bits
constexpr int LN_TWO = 32;                      // single CTAs of up to that many tokens fit two to an SM: 320 threads of 96 registers, half the shared memory
constexpr int LN_GROUP = 8;                     // token tiles that share a sweep over the weights

struct LinearParams {
    const void *bias;
    const void *residual;
    void *Y;
    Control *ctl;
    int64_t ldr, ldy;
    int64_t M;
    int N, K;
    int nt;            // tokens per tile
    int nt_cta;        // of which this CTA stages that many
    int tiles_w;       // tiles along N
    int tiles_t;       // tiles along M
    int splits;        // CTAs (or pairs of them) of a cluster that share a tile's inner dimension (1: none)
    int stages;
    int tmem_cols;
    uint32_t idesc;
    int32_t act, bias_type;
};

struct LinearShared {
    uint64_t full[LN_MAX_STAGES];
    uint64_t empty[LN_MAX_STAGES];
    uint64_t tmem_full[2];
    uint64_t tmem_empty[2];
    uint64_t drain;
    uint32_t tmem_base;
    int abort_flag;
};

__device__ __forceinline__ float load_as_float(const void *p, int64_t i, int type)
{
    if (type == CAT_F32) return reinterpret_cast<const float *>(p)[i];
    if (type == CAT_BF16) return __bfloat162float(reinterpret_cast<const __nv_bfloat16 *>(p)[i]);
    return __half2float(reinterpret_cast<const __half *>(p)[i]);
}
template <int T>
struct Elem;
template <>
struct Elem<CAT_F32> {
    using type = float;
    static __device__ __forceinline__ float up(float v) { return v; }
    static __device__ __forceinline__ float down(float v) { return v; }
};
template <>
struct Elem<CAT_BF16> {
    using type = __nv_bfloat16;
    static __device__ __forceinline__ float up(__nv_bfloat16 v) { return __bfloat162float(v); }
    static __device__ __forceinline__ __nv_bfloat16 down(float v) { return __float2bfloat16_rn(v); }
};
template <>
struct Elem<CAT_F16> {
    using type = __half;
    static __device__ __forceinline__ float up(__half v) { return __half2float(v); }
    static __device__ __forceinline__ __half down(float v) { return __float2half_rn(v); }
};

__device__ __forceinline__ float fast_exp2(float x)
{
    float e;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(x));
    return e;
}
__device__ __forceinline__ float fast_rcp(float x)
{
    float e;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(x));
    return e;
}

// gelu is z Phi(z) = max(z, 0) - |z| erfc(|z| / sqrt 2) / 2, which keeps its relative accuracy where 1 + erf(z) cancels; silu and gelu_tanh are
// z / (1 + e^-x), the tanh form 0.5 z (1 + tanh u) being z / (1 + e^-2u).  Where the result is rounded to 16 bits (FAST), the special function
// unit evaluates them (2 ulp each), and erfc(x) / 2 = t 2^(Q(t) - x^2 log2 e), t = 1 / (1 + x / 2), with Q of degree seven fitted to the
// logarithm of erfc for the smallest largest error over 0 <= x <= 9.5: 6.3e-7 of the value.
template <int ACT, bool FAST>
__device__ __forceinline__ float activate(float z)
{
    if (ACT == CAT_ACT_RELU) return z < 0.f ? 0.f : z;   // (a NaN stays one)
    if (ACT == CAT_ACT_GELU) {
        if (!FAST) return 0.5f * z * erfcf(-0.70710678f * z);
        const float a = fabsf(z), t = fast_rcp(fmaf(a, 0.35355339f, 1.f));
        float q = -0.26331830f;
        q = fmaf(q, t, 1.05167462f);
        q = fmaf(q, t, -1.38636313f);
        q = fmaf(q, t, 0.45006013f);
        q = fmaf(q, t, -0.02762734f);
        q = fmaf(q, t, 0.55924359f);
        q = fmaf(q, t, 1.44212111f);
        q = fmaf(q, t, -2.82579157f);
        const float r = a * t * fast_exp2(fmaf(a * a, -0.72134752f, q));
        return z > 20.f ? z : fmaxf(z, 0.f) - r;         // (of a NaN r is one)
    }
    if (ACT == CAT_ACT_GELU_TANH) {
        const float u = 0.7978845608f * z * fmaf(0.044715f * z, z, 1.f);
        return FAST ? z * fast_rcp(1.f + fast_exp2(-2.8853901f * u)) : z / (1.f + expf(-2.f * u));
    }
    if (ACT == CAT_ACT_SILU) return FAST ? z * fast_rcp(1.f + fast_exp2(-1.44269504f * z)) : z / (1.f + expf(-z));
    return z;
}

// 16 tokens of this thread's output column: y = act(acc + b) + r.  `count` tokens are there.
template <int OT, int ACT>
__device__ __forceinline__ void finish16(const float (&acc)[16], float bias, bool has, const typename Elem<OT>::type (&r)[16],
                                         typename Elem<OT>::type *out, int64_t ldy, int count)
{
    using E = Elem<OT>;
    constexpr bool FAST = OT != CAT_F32;
    if (count >= 16) {
        if (has) {
#pragma unroll
            for (int j = 0; j < 16; ++j, out += ldy) *out = E::down(activate<ACT, FAST>(acc[j] + bias) + E::up(r[j]));
        } else {
#pragma unroll
            for (int j = 0; j < 16; ++j, out += ldy) *out = E::down(activate<ACT, FAST>(acc[j] + bias));
        }
    } else {
#pragma unroll
        for (int j = 0; j < 16; ++j)
            if (j < count) {
                float y = activate<ACT, FAST>(acc[j] + bias);
                if (has) y += E::up(r[j]);
                out[j * ldy] = E::down(y);
            }
    }
}

template <int OT>
__device__ __forceinline__ void finish(int act, const float (&acc)[16], float bias, bool has, const typename Elem<OT>::type (&r)[16],
                                       typename Elem<OT>::type *out, int64_t ldy, int count)
{
    switch (act) {
    case CAT_ACT_RELU: finish16<OT, CAT_ACT_RELU>(acc, bias, has, r, out, ldy, count); break;
    case CAT_ACT_GELU: finish16<OT, CAT_ACT_GELU>(acc, bias, has, r, out, ldy, count); break;
    case CAT_ACT_GELU_TANH: finish16<OT, CAT_ACT_GELU_TANH>(acc, bias, has, r, out, ldy, count); break;
    case CAT_ACT_SILU: finish16<OT, CAT_ACT_SILU>(acc, bias, has, r, out, ldy, count); break;
    default: finish16<OT, CAT_ACT_NONE>(acc, bias, has, r, out, ldy, count); break;
    }
}

// the residual's entries for them
template <typename T>
__device__ __forceinline__ void load16(T (&r)[16], const T *from, int64_t ld, int64_t count)
{
    if (count >= 16) {
#pragma unroll
        for (int j = 0; j < 16; ++j, from += ld) r[j] = *from;
    } else {
#pragma unroll
        for (int j = 0; j < 16; ++j)
            if (j < count) r[j] = from[j * ld];
    }
}

template <bool FAST>
__device__ __forceinline__ float activate_any(int act, float z)
{
    switch (act) {
    case CAT_ACT_RELU: return activate<CAT_ACT_RELU, FAST>(z);
    case CAT_ACT_GELU: return activate<CAT_ACT_GELU, FAST>(z);
    case CAT_ACT_GELU_TANH: return activate<CAT_ACT_GELU_TANH, FAST>(z);
    case CAT_ACT_SILU: return activate<CAT_ACT_SILU, FAST>(z);
    default: return z;
    }
}

__device__ __forceinline__ void tmem_st16(uint32_t taddr, const float (&v)[16])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(taddr), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]), "f"(v[8]), "f"(v[9]), "f"(v[10]),
        "f"(v[11]), "f"(v[12]), "f"(v[13]), "f"(v[14]), "f"(v[15])
        : "memory");
}
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, float (&v)[8])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];\n\ttcgen05.wait::ld.sync.aligned;"
        : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// arrives on the barrier at this shared-memory offset in both CTAs of the pair whose first one has this rank
__device__ __forceinline__ void commit_to_pair(uint32_t bar, uint32_t leader)
{
    asm volatile(
        "{\n\t.reg .b16 m;\n\tcvt.u16.u32 m, %1;\n\t"
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], m;\n\t}"
        ::"r"(bar), "r"(3u << leader)
        : "memory");
}

__device__ __forceinline__ float ld_cluster_f32(uint32_t addr)
{
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}

// Unit -> tile.  LN_GROUP token tiles at a time sweep the weights, the tokens running fastest: the tiles in flight at a time are then
// about as many of either operand, and what they read comes out of L2.
__device__ __forceinline__ void tile_of(const LinearParams &p, int unit, int &tw, int &tt)
{
    const int full = LN_GROUP * p.tiles_w;
    const int g = unit / full, rem = unit - g * full;
    const int gs = min(LN_GROUP, p.tiles_t - g * LN_GROUP);
    tw = rem / gs;
    tt = g * LN_GROUP + rem - tw * gs;
}

// RUNS: a 16-bit result's accumulator may take several runs.  (With one the epilogue has the registers to itself: 4999 x 2047 x 1001 38 us, 40 with
// the code for several.)
template <bool PAIR, int OT, bool RUNS>
__global__ void __launch_bounds__(LN_MAX_THREADS, 1)
linear_kernel(const __grid_constant__ CUtensorMap mapW, const __grid_constant__ CUtensorMap mapX, const __grid_constant__ LinearParams p)
{
    extern __shared__ unsigned char smem_raw[];
    // (operand tiles start on 1024 bytes, as the swizzle wants)
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t ring = (raw + 1023u) & ~1023u;
    unsigned char *ring_ptr = smem_raw + (ring - raw);
    const int x_bytes = p.nt_cta * TC_SLAB_BYTES;
    const int stage_bytes = TC_A_BYTES + x_bytes;
    LinearShared &sh = *reinterpret_cast<LinearShared *>(ring_ptr + (size_t)p.stages * stage_bytes);

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, warps = (int)blockDim.x >> 5;
    const uint32_t crank = (PAIR || p.splits > 1) ? cluster_ctarank() : 0u;
    const uint32_t rank = PAIR ? crank & 1u : 0u;         // 0 = the CTA that issues the MMAs
    const uint32_t leader = PAIR ? crank & ~1u : crank;   // that CTA's rank in the cluster
    const uint32_t split = PAIR ? crank >> 1 : crank;     // part of the inner dimension
    volatile int *abort_flag = &sh.abort_flag;
    constexpr int TW = PAIR ? 256 : 128;                  // output columns per tile
    const int units = p.tiles_w * p.tiles_t;
    const int per_cluster = (PAIR ? 2 : 1) * p.splits;
    const int unit_first = blockIdx.x / per_cluster, unit_step = gridDim.x / per_cluster;
    const int slabs = (p.K + LN_BK - 1) / LN_BK;
    const int slab0 = (int)((int64_t)slabs * split / p.splits), slab1 = (int)((int64_t)slabs * (split + 1) / p.splits);

    // An accumulator runs over at most LN_RUN (LN_RUN_16) slabs at a time: the tensor cores truncate it at every step, always towards zero, and
    // what that costs grows with the length of the run.  The epilogue adds the runs up in registers, rounding to nearest.
    // fp32 results: relative error at 2048 inner columns (2-norm; fp32 sums in another order: 3.7e-7), time of 50 000 x 1000 under the power cap: one
    // run 1.9e-6, 192 us; 16 slabs 9.1e-7, 194 us; 12 slabs 6.1e-7, 196 us; 8 slabs 4.3e-7, 201 us.
    // 16-bit results: how far they are from those of fp32 sums in another order (2-norm; numbers that round to the other neighbour) at 8192 and at 4096
    // inner columns, time of 16384 x 16384 x 4096 under the power cap: one run 1.7e-4 and 1.5e-4, 1736 us; 32 slabs 8e-5 and 1.0e-4, 1753 us; 24 slabs 7e-5 and
    // 8e-5, 1779 us; 16 slabs 6e-5 and 7e-5, 1801 us.
    const int in_split = slab1 - slab0, longest = OT == CAT_F32 ? LN_RUN : LN_RUN_16;
    const int runs = RUNS ? (in_split + longest - 1) / longest : 1, run = (in_split + runs - 1) / runs;

    if (tid == 0) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&mapW)) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&mapX)) : "memory");
        for (int s = 0; s < p.stages; ++s) {
            mbar_init(smem_u32(&sh.full[s]), PAIR ? 2 : 1);   // one expect_tx arrival per CTA
            mbar_init(smem_u32(&sh.empty[s]), 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(smem_u32(&sh.tmem_full[b]), 1);
            mbar_init(smem_u32(&sh.tmem_empty[b]), (PAIR ? 2 : 1) * (warps - 2));
        }
        mbar_init(smem_u32(&sh.drain), 1);
        sh.abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    pdl_enter();   // (before the TMEM allocation: the previous kernel of the stream has given its own back by then)
    if (blockIdx.x == 0 && tid == 0) p.ctl->device_status = CAT_OK;   // (a wait that gives up does so seconds later)
    if (warp == 1) {
        if (PAIR) {
            tmem_alloc_pair(smem_u32(&sh.tmem_base), (uint32_t)p.tmem_cols);
            tmem_relinquish_pair();
        } else {
            tmem_alloc(smem_u32(&sh.tmem_base), (uint32_t)p.tmem_cols);
            tmem_relinquish();
        }
    }
    tc_fence_before();
    __syncthreads();
    if (PAIR) cluster_sync();   // the peer's barriers exist before anything arrives on them
    tc_fence_after();
    const uint32_t tmem_base = sh.tmem_base;

    if (warp == 0) {
        // ---------------------------------------------------------------- TMA producer of both operands
        if (lane == 0) {
            int s = 0;
            uint32_t ph = 0;
            bool ok = true;
            for (int unit = unit_first; unit < units && ok; unit += unit_step) {
                int tw, tt;
                tile_of(p, unit, tw, tt);
                const int n0 = tw * TW + (int)rank * 128;
                const int t0 = tt * p.nt + (int)rank * p.nt_cta;
                for (int sl = slab0; sl < slab1; ++sl) {
                    if (!mbar_wait(smem_u32(&sh.empty[s]), ph ^ 1u, abort_flag, p.ctl)) { ok = false; break; }
                    const uint32_t dst = ring + (uint32_t)(s * stage_bytes);
                    if (PAIR) {
                        const uint32_t full = mapa_cluster(smem_u32(&sh.full[s]), leader);
                        mbar_arrive_expect_tx_cluster(full, (uint32_t)stage_bytes);
                        tma_load_2d_pair(dst, &mapW, full, sl * LN_BK, n0);
                        tma_load_2d_pair(dst + TC_A_BYTES, &mapX, full, sl * LN_BK, t0);
                    } else {
                        const uint32_t full = smem_u32(&sh.full[s]);
                        mbar_arrive_expect_tx(full, (uint32_t)stage_bytes);
                        tma_load_2d(dst, &mapW, full, sl * LN_BK, n0);
                        tma_load_2d(dst + TC_A_BYTES, &mapX, full, sl * LN_BK, t0);
                    }
                    if (++s == p.stages) { s = 0; ph ^= 1u; }
                }
            }
            if (!ok && rank == 0) {
                // give copies that are still in flight a bounded time to land
                for (int i = 0; i < p.stages; ++i)
                    for (int tries = 0; tries < 100000; ++tries)
                        if (mbar_try_wait(smem_u32(&sh.full[i]), 0) || mbar_try_wait(smem_u32(&sh.full[i]), 1)) break;
            }
        }
    } else if (warp == 1) {
        // ---------------------------------------------------------------- MMA issuer
        if (lane == 0 && rank == 0) {
            const uint64_t wdesc0 = make_smem_desc(ring), xdesc0 = make_smem_desc(ring + TC_A_BYTES);
            int s = 0;
            uint32_t ph = 0, ti = 0;
            bool ok = true;
            for (int unit = unit_first; unit < units && ok; unit += unit_step)
                for (int first = slab0; first < slab1 && ok; first += run, ++ti) {
                    const int b = ti & 1, last = min(first + run, slab1);
                    if (!mbar_wait(smem_u32(&sh.tmem_empty[b]), ((ti >> 1) & 1u) ^ 1u, abort_flag, p.ctl)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t acc = tmem_base + (uint32_t)(b * p.nt);
                    for (int sl = first; sl < last; ++sl) {
                        if (!mbar_wait(smem_u32(&sh.full[s]), ph, abort_flag, p.ctl)) { ok = false; break; }
                        tc_fence_after();
                        const uint64_t at = (uint64_t)(uint32_t)(s * (stage_bytes >> 4));
#pragma unroll
                        for (int kk = 0; kk < 4; ++kk) {   // 16 inner columns = 32 B per MMA: +2 in 16-byte units
                            const uint32_t accum = (sl > first || kk > 0) ? 1u : 0u;
                            if (PAIR) mma_f16_pair(acc, wdesc0 + at + 2 * kk, xdesc0 + at + 2 * kk, p.idesc, accum);
                            else mma_f16(acc, wdesc0 + at + 2 * kk, xdesc0 + at + 2 * kk, p.idesc, accum);
                        }
                        if (PAIR) commit_to_pair(smem_u32(&sh.empty[s]), leader);
                        else tc_commit(smem_u32(&sh.empty[s]));
                        if (++s == p.stages) { s = 0; ph ^= 1u; }
                    }
                    if (ok) {
                        if (PAIR) commit_to_pair(smem_u32(&sh.tmem_full[b]), leader);
                        else tc_commit(smem_u32(&sh.tmem_full[b]));
                    }
                }
            // all MMAs issued by this thread have completed once this commit arrives
            if (PAIR) tc_commit_pair_local(smem_u32(&sh.drain));
            else tc_commit(smem_u32(&sh.drain));
            for (int tries = 0; tries < 4000000; ++tries)
                if (mbar_try_wait(smem_u32(&sh.drain), 0)) break;
        }
    } else {
        // ---------------------------------------------------------------- epilogue
        using E = Elem<OT>;
        using T = typename E::type;
        const int quarter = warp & 3, part = (warp - 2) >> 2;   // TMEM lanes this warp may read; which 16-column chunks it takes
        uint32_t ti = 0;
        bool ok = true;
        for (int unit = unit_first; unit < units && ok; unit += unit_step) {
            int tw, tt;
            tile_of(p, unit, tw, tt);
            const int n = tw * TW + (int)rank * 128 + quarter * 32 + lane;
            const bool inside = n < p.N;
            const int64_t t0 = (int64_t)tt * p.nt;
            const float bias = p.bias && inside && p.splits == 1 ? load_as_float(p.bias, n, p.bias_type) : 0.f;
            // 16-bit results: the residual of a chunk is on its way while the accumulator, or the chunk before, is waited for
            constexpr bool AHEAD = OT != CAT_F32;
            const bool has = p.residual && inside && p.splits == 1;
            T ahead[16];
            auto fetch = [&](T (&r)[16], int c) {
                if (has && c < p.nt && t0 + c < p.M)
                    load16<T>(r, reinterpret_cast<const T *>(p.residual) + (t0 + c) * p.ldr + n, p.ldr, p.M - t0 - c);
            };
            // accumulator buffer b may be overwritten from here on
            auto release = [&](int b) {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    if (PAIR) mbar_arrive_cluster(mapa_cluster(smem_u32(&sh.tmem_empty[b]), leader));
                    else mbar_arrive(smem_u32(&sh.tmem_empty[b]));
                }
            };
            auto accumulator = [&](int b) { return tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(b * p.nt); };
            if (AHEAD && runs == 1) fetch(ahead, part * 16);
            uint32_t raw16[16];
            if (RUNS && runs > 1) {
                // Runs are added up in registers, eight columns at a time: the sums take 64 of 96, and with sixteen at a time the loop spills (50 000 x 1000
                // x 2048: 211 us against 198).
                float sum[4][16];
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll
                    for (int j = 0; j < 16; ++j) sum[k][j] = 0.f;
#pragma unroll 1
                for (int left = runs;; ++ti) {
                    const int b = ti & 1;
                    ok = mbar_wait_warp(smem_u32(&sh.tmem_full[b]), (ti >> 1) & 1u, abort_flag, p.ctl);
                    if (!ok) break;
                    tc_fence_after();
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int c = ((warps - 2) / 4 * k + part) * 16;
                        if (c < p.nt) {
#pragma unroll
                            for (int h = 0; h < 16; h += 8) {
                                float v[8];
                                tmem_ld8(accumulator(b) + (uint32_t)(c + h), v);
#pragma unroll
                                for (int j = 0; j < 8; ++j) sum[k][h + j] += v[j];
                            }
                        }
                    }
                    if (--left == 0) break;
                    release(b);
                }
                if (OT == CAT_F32 && ok && p.splits == 1 && !p.residual && p.act == CAT_ACT_NONE) {
                    // Nothing but the bias follows: out of the registers, the accumulator free before that (192 us; more work here would spill again).
                    release(ti & 1);
                    ++ti;
                    if (inside) {
                        T *out = reinterpret_cast<T *>(p.Y) + (t0 + part * 16) * p.ldy + n;
                        const int rest = (int)min((int64_t)p.nt, p.M - t0) - part * 16;
                        const int64_t step = (int64_t)(warps - 2) * 4 * p.ldy;
#pragma unroll
                        for (int k = 0; k < 4; ++k, out += step) {
                            const int count = rest - (warps - 2) * 4 * k;
                            T *o = out;
                            if (count >= 16) {
#pragma unroll
                                for (int j = 0; j < 16; ++j, o += p.ldy) *o = E::down(sum[k][j] + bias);
                            } else {
#pragma unroll
                                for (int j = 0; j < 16; ++j, o += p.ldy)
                                    if (j < count) *o = E::down(sum[k][j] + bias);
                            }
                        }
                    }
                    continue;
                }
                // The last run's accumulator takes the sums, and one loop finishes either kind.
                if (ok) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int c = ((warps - 2) / 4 * k + part) * 16;
                        if (c < p.nt) tmem_st16(accumulator(ti & 1) + (uint32_t)c, sum[k]);
                    }
                    tmem_st_wait();
                }
                if (AHEAD) fetch(ahead, part * 16);
            } else {
                ok = mbar_wait_warp(smem_u32(&sh.tmem_full[ti & 1]), (ti >> 1) & 1u, abort_flag, p.ctl);
                tc_fence_after();
            }
            if (!ok) break;
            const int b = ti & 1;
#pragma unroll 1
            for (int c = part * 16; c < p.nt; c += (warps - 2) * 4) {
                tmem_ld16_issue(accumulator(b) + (uint32_t)c, raw16);
                tmem_ld_wait16(raw16);
                float acc[16];
#pragma unroll
                for (int j = 0; j < 16; ++j) acc[j] = __uint_as_float(raw16[j]);
                if (p.splits > 1) {
                    // [token][output column] of this CTA's part, in the ring (every slab has been consumed)
                    float *to = reinterpret_cast<float *>(ring_ptr) + (size_t)c * 128 + quarter * 32 + lane;
#pragma unroll
                    for (int j = 0; j < 16; ++j) to[j * 128] = acc[j];
                } else if (inside && t0 + c < p.M) {
                    const int64_t row = t0 + c;
                    const int count = (int)min((int64_t)16, p.M - row);
                    T r[16];
                    if (AHEAD) {
#pragma unroll
                        for (int j = 0; j < 16; ++j) r[j] = ahead[j];
                        fetch(ahead, c + (warps - 2) * 4);
                    } else {
                        fetch(r, c);
                    }
                    finish<OT>(p.act, acc, bias, has, r, reinterpret_cast<T *>(p.Y) + row * p.ldy + n, p.ldy, count);
                }
            }
            release(b);
            ++ti;
        }
    }

    tc_fence_before();
    __syncthreads();
    if (!PAIR && warp == 1) {
        // Given back before this CTA waits for the others of its cluster: a CTA of theirs may be waiting for TMEM that another stream's kernel
        // holds, which in turn waits for this SM's.  (Pairs have their SMs to themselves: their rings leave no other kernel with TMEM room.)
        __syncwarp();
        tc_fence_after();
        tmem_dealloc(tmem_base, (uint32_t)p.tmem_cols);
    }
    if (p.splits > 1) {
        // The parts meet: split q of the cluster finishes every q-th token of the tile, the parts in order.  A warp takes a token, a lane four of its
        // 128 output columns.
        using E = Elem<OT>;
        using T = typename E::type;
        cluster_sync();
        int tw, tt;
        tile_of(p, unit_first, tw, tt);
        const int64_t t0 = (int64_t)tt * p.nt;
        const int tokens = (int)min((int64_t)p.nt, p.M - t0), n0 = tw * TW + (int)rank * 128 + lane;
        float bias[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) bias[i] = p.bias && n0 + 32 * i < p.N ? load_as_float(p.bias, n0 + 32 * i, p.bias_type) : 0.f;
        if (*abort_flag == 0)
            for (int t = (int)split + p.splits * warp; t < tokens; t += p.splits * warps) {
                const int64_t row = t0 + t;
                float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 2
                for (int q = 0; q < p.splits; ++q) {
                    const uint32_t from = mapa_cluster(ring + (uint32_t)((t * 128 + lane) * 4), PAIR ? 2u * q + rank : (uint32_t)q);
                    float u[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) u[i] = ld_cluster_f32(from + 128u * i);
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] += u[i];
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int n = n0 + 32 * i;
                    if (n < p.N) {
                        float y = activate_any<OT != CAT_F32>(p.act, v[i] + bias[i]);
                        if (p.residual) y += E::up(reinterpret_cast<const T *>(p.residual)[row * p.ldr + n]);
                        reinterpret_cast<T *>(p.Y)[row * p.ldy + n] = E::down(y);
                    }
                }
            }
    }
    if (PAIR || p.splits > 1) cluster_sync();   // no CTA's shared memory or TMEM goes away under another
    if (PAIR && warp == 1) {
        __syncwarp();
        tc_fence_after();
        tmem_dealloc_pair(tmem_base, (uint32_t)p.tmem_cols);
    }
}

// Rows that TMA cannot address, copied to rows of `pitch` elements (zeros behind column K), for X and W in one launch.  A thread makes 16 bytes
// at a time, from aligned words and a shift between neighbours (the words at a row's ends element by element).
struct PadJob {
    const uint16_t *src;
    uint16_t *dst;
    int64_t ld, units;    // units: 16-byte pieces of the copy (0: nothing to do)
};
__global__ void __launch_bounds__(256) linear_pad_kernel(const __grid_constant__ PadJob x, const __grid_constant__ PadJob w, int K, int pitch)
{
    pdl_enter();
    const int per_row = pitch / 8;
    for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < x.units + w.units; u += (int64_t)gridDim.x * 256) {
        const bool of_x = u < x.units;
        const int64_t at = of_x ? u : u - x.units;
        const int64_t row = at / per_row;
        const int k = (int)(at - row * per_row) * 8;
        const uint16_t *src = (of_x ? x.src : w.src) + row * (of_x ? x.ld : w.ld) + k;
        uint32_t v[4];
        const uint32_t off = (uint32_t)reinterpret_cast<uintptr_t>(src) & 3u;
        if (k >= 1 && k + 8 < K) {      // (one element before and one behind are in the row)
            const uint32_t *words = reinterpret_cast<const uint32_t *>(reinterpret_cast<const unsigned char *>(src) - off);
            uint32_t a[5];
#pragma unroll
            for (int q = 0; q < 4; ++q) a[q] = __ldg(words + q);
            a[4] = off ? __ldg(words + 4) : 0u;
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] = __funnelshift_r(a[q], a[q + 1], 8 * off);
        } else {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const uint32_t lo = k + 2 * q < K ? src[2 * q] : 0u, hi = k + 2 * q + 1 < K ? src[2 * q + 1] : 0u;
                v[q] = lo | (hi << 16);
            }
        }
        reinterpret_cast<uint4 *>(of_x ? x.dst : w.dst)[at] = make_uint4(v[0], v[1], v[2], v[3]);
    }
}

bool tma_rows(const void *base, int64_t ld) { return (reinterpret_cast<uintptr_t>(base) & 15u) == 0 && ld % 8 == 0; }
int padded(int K) { return (K + 7) & ~7; }

struct LinearPlan {
    bool pair;
    int nt, splits;
};

LinearPlan plan(int64_t M, int N, int K, int sms)
{
    // Estimated times in microseconds of the forms that suit the shape; the shortest is taken.  A slab of 64 inner columns takes what is in the
    // table (measured on 200 to 1024 rows, N = 4096 and 8192, K = 2048 and 4096, all CTAs at work), splitting the inner dimension about a microsecond and
    // what the parts' exchange takes.
    static const struct { int nt; float single, pair; } table[] = {{16, 0.22f, 0.f}, {32, 0.22f, 0.f}, {64, 0.23f, 0.f}, {128, 0.25f, 0.25f}, {192, 0.30f, 0.29f}, {256, 0.38f, 0.33f}};
    const int slabs = (K + LN_BK - 1) / LN_BK;
    LinearPlan best{};
    float least = 1e30f;
    for (const auto &row : table) {
        if (row.nt > 16 && row.nt >= 2 * M) break;
        for (int pair = 0; pair < 2; ++pair) {
            const float slab = pair ? row.pair : row.single;
            if (slab == 0.f) continue;
            const int64_t tiles = (int64_t)((N + (pair ? 255 : 127)) / (pair ? 256 : 128)) * ((M + row.nt - 1) / row.nt);
            // (two CTAs share an SM where they fit)
            const int64_t slots = sms / (pair ? 2 : 1), most = row.nt <= LN_TWO && !pair ? 2 * slots : slots;
            for (int splits = 1; splits <= (pair ? 2 : row.nt <= 64 ? 8 : 4) && splits * 2 <= (slabs > 1 ? slabs : 2); splits *= 2) {
                if (splits > 1 && tiles * splits > most) break;
                const float waves = (float)((tiles * splits + slots - 1) / slots);
                const float t = waves * (float)((slabs + splits - 1) / splits) * (row.nt == 16 && waves > 1.f ? slab - 0.03f : slab) +
                                (splits > 1 ? 0.6f + 0.2f * splits + 2.5f * row.nt / 256.f : 0.f);
                if (t < least) {
                    least = t;
                    best.pair = pair;
                    best.nt = row.nt;
                    best.splits = splits;
                }
            }
        }
    }
    return best;
}

}  // namespace

size_t linear_workspace_bytes(const void *X, int64_t ldx, const void *W, int64_t ldw, int64_t M, int N, int K)
{
    size_t n = 256;
    if (!tma_rows(X, ldx)) n += align_up((size_t)M * padded(K) * 2, 256);
    if (!tma_rows(W, ldw)) n += align_up((size_t)N * padded(K) * 2, 256);
    return n;
}

cudaError_t launch_linear(const LinearArgs &a, void *workspace, cudaStream_t s)
{
    const int sms = tc_sm_count();
    unsigned char *room = reinterpret_cast<unsigned char *>(workspace) + 256;
    const void *X = a.X, *W = a.W;
    int64_t ldx = a.ldx, ldw = a.ldw;
    cudaError_t e;
    auto pad = [&](const void *&src, int64_t &ld, int64_t rows, PadJob &job) {
        if (tma_rows(src, ld)) return;
        job.src = reinterpret_cast<const uint16_t *>(src);
        job.dst = reinterpret_cast<uint16_t *>(room);
        job.ld = ld;
        job.units = rows * (padded(a.K) / 8);
        src = room;
        ld = padded(a.K);
        room += align_up((size_t)rows * padded(a.K) * 2, 256);
    };
    PadJob pad_x{}, pad_w{};
    pad(X, ldx, a.M, pad_x);
    pad(W, ldw, a.N, pad_w);
    if (pad_x.units + pad_w.units) {
        const int64_t blocks = (pad_x.units + pad_w.units + 255) / 256;
        if ((e = launch_pdl(linear_pad_kernel, dim3((unsigned)(blocks < 16 * sms ? blocks : 16 * sms)), dim3(256), 0, s, pad_x, pad_w, a.K, padded(a.K))) !=
            cudaSuccess)
            return e;
        count_launch();
    }

    const LinearPlan pl = plan(a.M, a.N, a.K, sms);
    LinearParams p{};
    p.bias = a.bias;
    p.residual = a.residual;
    p.Y = a.Y;
    p.ctl = reinterpret_cast<Control *>(workspace);
    p.ldr = a.ldr;
    p.ldy = a.ldy;
    p.M = a.M;
    p.N = a.N;
    p.K = a.K;
    p.nt = pl.nt;
    p.nt_cta = pl.pair ? pl.nt / 2 : pl.nt;
    p.tiles_w = (a.N + (pl.pair ? 255 : 127)) / (pl.pair ? 256 : 128);
    p.tiles_t = (int)((a.M + pl.nt - 1) / pl.nt);
    p.splits = pl.splits;
    p.act = a.act;
    p.bias_type = a.bias_type;
    int cols = 32;
    while (cols < 2 * pl.nt) cols <<= 1;
    p.tmem_cols = cols;
    p.idesc = make_idesc(pl.pair ? 256 : 128, pl.nt, a.in_type == CAT_BF16 ? 1u : 0u);

    CUtensorMap mapW, mapX;
    if (!tc_make_map16(&mapW, W, a.in_type == CAT_BF16, a.N, a.K, ldw, TC_BM) ||
        !tc_make_map16(&mapX, X, a.in_type == CAT_BF16, a.M, a.K, ldx, p.nt_cta))
        return cudaErrorInvalidValue;

    const int stage_bytes = TC_A_BYTES + p.nt_cta * TC_SLAB_BYTES;
    const int64_t units = (int64_t)p.tiles_w * p.tiles_t;
    // With few tokens half an SM's shared memory holds more than enough slabs in flight (100 KB; the memory wants about 45), and the next call's
    // CTAs can settle in beside these.  From 33 tokens on (576 threads) they cannot, and the whole of it is taken: 64 x 28672 x 4096 48.5 us, 54.9 with half
    // of it.
    const int room_smem = (pl.nt <= LN_TWO && !pl.pair ? 113 : 227) * 1024 - 2048 - (int)sizeof(LinearShared);
    p.stages = room_smem / stage_bytes;
    if (p.stages > LN_MAX_STAGES) p.stages = LN_MAX_STAGES;
    if (pl.splits > 1 && (size_t)p.stages * stage_bytes < (size_t)pl.nt * 512) return cudaErrorInvalidValue;   // (the parts of a split tile lie in the ring)
    const size_t smem = 1024 + (size_t)p.stages * stage_bytes + sizeof(LinearShared);
    const int per_cluster = (pl.pair ? 2 : 1) * pl.splits;
    int64_t clusters = (pl.nt <= LN_TWO && !pl.pair ? 2 : 1) * sms / per_cluster;
    if (units < clusters) clusters = units;
    if (pl.splits > 1 && clusters < units) return cudaErrorInvalidValue;   // (a split tile is a cluster's only one)

    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(clusters * per_cluster), 1, 1);
    cfg.blockDim = dim3((unsigned)(64 + 32 * (pl.nt / 4 < LN_EPI_WARPS ? pl.nt / 4 : LN_EPI_WARPS)), 1, 1);   // (a warp of the epilogue per 16 tokens and quarter)
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)per_cluster;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;   // (the kernel calls pdl_enter)
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;

    int dev = 0;
    if ((e = cudaGetDevice(&dev)) != cudaSuccess) return e;
    const uint64_t dev_bit = dev < 64 ? (uint64_t)1 << dev : 0;
#define CAT_LINEAR_LAUNCH(PAIR, OT, RUNS)                                                                                       \
    do {                                                                                                                        \
        auto kern = linear_kernel<PAIR, OT, RUNS>;                                                                              \
        static std::atomic<uint64_t> ready{0};      /* (a bit per device: the attribute is set once) */                           \
        if (!(dev_bit & ready.load(std::memory_order_relaxed))) {                                                                \
            if ((e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024)) != cudaSuccess) return e; \
            ready.fetch_or(dev_bit, std::memory_order_relaxed);                                                                  \
        }                                                                                                                        \
        e = cudaLaunchKernelEx(&cfg, kern, mapW, mapX, p);                                                                      \
    } while (0)
    const bool several = ((a.K + LN_BK - 1) / LN_BK + pl.splits - 1) / pl.splits > LN_RUN_16;
    if (pl.pair) {
        if (a.out_type == CAT_F32) CAT_LINEAR_LAUNCH(true, CAT_F32, true);
        else if (a.out_type == CAT_BF16 && several) CAT_LINEAR_LAUNCH(true, CAT_BF16, true);
        else if (a.out_type == CAT_BF16) CAT_LINEAR_LAUNCH(true, CAT_BF16, false);
        else if (several) CAT_LINEAR_LAUNCH(true, CAT_F16, true);
        else CAT_LINEAR_LAUNCH(true, CAT_F16, false);
    } else {
        if (a.out_type == CAT_F32) CAT_LINEAR_LAUNCH(false, CAT_F32, true);
        else if (a.out_type == CAT_BF16 && several) CAT_LINEAR_LAUNCH(false, CAT_BF16, true);
        else if (a.out_type == CAT_BF16) CAT_LINEAR_LAUNCH(false, CAT_BF16, false);
        else if (several) CAT_LINEAR_LAUNCH(false, CAT_F16, true);
        else CAT_LINEAR_LAUNCH(false, CAT_F16, false);
    }
#undef CAT_LINEAR_LAUNCH
    count_launch();
    return e;
}

}  // namespace cat
