// Verification of drafted tokens against the target network's probabilities (cat_verify_drafts).
//
// Mathematics.  p_j = softmax(target_j / T), q_j = softmax(draft_j / T).  Draft x_j is accepted while u_j q_j(x_j) < p_j(x_j); at the
// first refusal the next token is drawn from max(p_j - q_j, 0), after the last draft from the row behind it: the first index whose
// cumulated mass exceeds u times the whole.  Outputs are tokens, so they have to be those of exact arithmetic whatever the order of
// the sums.
#include "cat_internal.cuh"

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math_constants.h>

namespace cat {
namespace {

constexpr int VF_THREADS = 512;
constexpr int VF_WARPS = VF_THREADS / 32;
constexpr int VF_MAX_CLUSTER = 16;
constexpr double VF_NO_RESIDUAL = 9.094947017729282e-13;   // 2^-40: a residual of less mass is what rounding left of none
constexpr float VF_LARGEST = 3.4028234663852886e38f;

__device__ __forceinline__ uint32_t cta_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void sync_cluster()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// address of the same shared-memory location in the CTA of the given rank
__device__ __forceinline__ uint32_t peer(const void *p, uint32_t rank)
{
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    return a;
}
__device__ __forceinline__ double peer_f64(const double *p, uint32_t rank)
{
    double v;
    asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(v) : "r"(peer(p, rank)) : "memory");
    return v;
}
__device__ __forceinline__ int peer_s32(const int *p, uint32_t rank)
{
    int v;
    asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(peer(p, rank)) : "memory");
    return v;
}

// A logit as the definitions take it: NaN counts as -inf, +inf as the largest number.
__device__ __forceinline__ float clean(float x) { return fminf(x != x ? -CUDART_INF_F : x, VF_LARGEST); }

__device__ __forceinline__ float logit(const void *row, int i, int type)
{
    if (type == CAT_F32) return clean(reinterpret_cast<const float *>(row)[i]);
    if (type == CAT_BF16) return clean(__bfloat162float(reinterpret_cast<const __nv_bfloat16 *>(row)[i]));
    return clean(__half2float(reinterpret_cast<const __half *>(row)[i]));
}

// A uniform number as the definitions take it, in [0, 1 - 2^-24]; NaN: 0.
__device__ __forceinline__ double uniform(float u) { return (double)fminf(fmaxf(u, 0.f), 0.99999994f); }

struct VerifyParams {
    VerifyArgs a;
    Control *ctl;
};

__device__ __forceinline__ const void *row_of(const void *base, int type, int64_t seq, int64_t row, int64_t seq_stride, int64_t row_stride)
{
    return reinterpret_cast<const unsigned char *>(base) + (seq * seq_stride + row * row_stride) * (type == CAT_F32 ? 4 : 2);
}

// ---------------------------------------------------------------- in 64 bits
struct ExactShared {
    double sum[2][VF_WARPS];     // per-warp sums; two sets in turn, so that one exchange is one barrier
    double cta[2];
    int at[2][VF_WARPS];
    double prefix[VF_MAX_CLUSTER * VF_WARPS];
};

// One cluster on one sequence: CTA r takes the r-th contiguous part of a row, warp w the w-th part of that.
struct ExactCluster {
    ExactShared &sh;
    uint32_t rank, size;
    int V, i0, i1, warp, lane;
    int turn = 0;

    __device__ ExactCluster(ExactShared &s, uint32_t r, uint32_t n, int vocab) : sh(s), rank(r), size(n), V(vocab)
    {
        warp = threadIdx.x >> 5;
        lane = threadIdx.x & 31;
        const int parts = (int)size * VF_WARPS, part = (int)rank * VF_WARPS + warp;
        i0 = (int)((int64_t)V * part / parts);
        i1 = (int)((int64_t)V * (part + 1) / parts);
    }
    // sum over the cluster in a fixed order
    __device__ double sum(double v)
    {
        turn ^= 1;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        if (lane == 0) sh.sum[turn][warp] = v;
        sync_cluster();
        v = 0;
        for (uint32_t q = 0; q < size; ++q)
            for (int w = 0; w < VF_WARPS; ++w) v += peer_f64(&sh.sum[turn][w], q);
        return v;
    }
    // largest logit of a row and the first place that has it
    __device__ float top(const void *row, int type, int &at)
    {
        turn ^= 1;
        float m = -CUDART_INF_F;
        int best = 0x7fffffff;
        for (int i = i0 + lane; i < i1; i += 32) {
            const float x = logit(row, i, type);
            if (x > m) { m = x; best = i; }
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            const float om = __shfl_xor_sync(0xffffffffu, m, o);
            const int ob = __shfl_xor_sync(0xffffffffu, best, o);
            if (om > m || (om == m && ob < best)) { m = om; best = ob; }
        }
        if (lane == 0) {
            sh.sum[turn][warp] = m;
            sh.at[turn][warp] = best;
        }
        sync_cluster();
        m = -CUDART_INF_F;
        best = 0x7fffffff;
        for (uint32_t q = 0; q < size; ++q)
            for (int w = 0; w < VF_WARPS; ++w) {
                const float om = (float)peer_f64(&sh.sum[turn][w], q);
                const int ob = peer_s32(&sh.at[turn][w], q);
                if (om > m || (om == m && ob < best)) { m = om; best = ob; }
            }
        at = best;
        return m;
    }
};

// exp((x - m) / T); m is finite
__device__ __forceinline__ double weight(float x, float m, double T) { return x == -CUDART_INF_F ? 0.0 : exp(((double)x - (double)m) / T); }

__global__ void __launch_bounds__(VF_THREADS, 1) verify_exact_kernel(const __grid_constant__ VerifyParams p, int size)
{
    __shared__ ExactShared sh;
    pdl_enter();
    const VerifyArgs &a = p.a;
    const uint32_t rank = cta_rank();
    ExactCluster c(sh, rank, (uint32_t)size, a.V);
    const bool writer = rank == 0 && threadIdx.x == 0;
    for (int b = (int)(blockIdx.x / size); b < a.B; b += (int)(gridDim.x / size)) {
        const int length = a.lengths ? min(a.lengths[b], a.S) : a.S;
        if (length < 0) continue;
        const double T = a.temperature ? (double)a.temperature[b] : 1.0;
        const bool greedy = !(T > 0.0);
        int j = 0, best = 0;
        const void *t_row, *q_row = nullptr;
        float mt, mq = 0.f;
        double zt = 0, zq = 0;
        int x = -1;
        bool refused = false;
        for (;; ++j) {
            t_row = row_of(a.target, a.target_type, b, j, a.target_seq, a.target_row);
            mt = c.top(t_row, a.target_type, best);
            if (!greedy && mt > -CUDART_INF_F) {
                double z = 0;
                for (int i = c.i0 + c.lane; i < c.i1; i += 32) z += weight(logit(t_row, i, a.target_type), mt, T);
                zt = c.sum(z);
            }
            if (j == length) break;
            x = a.tokens[(int64_t)b * a.S + j];
            const bool inside = x >= 0 && x < a.V;
            if (greedy) {
                refused = !(mt > -CUDART_INF_F && x == best);
            } else {
                double px = 0, qx = 0;
                if (inside && mt > -CUDART_INF_F) px = weight(logit(t_row, x, a.target_type), mt, T) / zt;
                if (a.draft) {
                    q_row = row_of(a.draft, a.draft_type, b, j, a.draft_seq, a.draft_row);
                    int at;
                    mq = c.top(q_row, a.draft_type, at);
                    zq = 0;
                    if (mq > -CUDART_INF_F) {
                        double z = 0;
                        for (int i = c.i0 + c.lane; i < c.i1; i += 32) z += weight(logit(q_row, i, a.draft_type), mq, T);
                        zq = c.sum(z);
                        if (inside) qx = weight(logit(q_row, x, a.draft_type), mq, T) / zq;
                    }
                } else if (inside) {
                    qx = 1;
                }
                refused = !(uniform(a.u_accept[(int64_t)b * a.S + j]) * qx < px);
            }
            if (refused) break;
            if (writer) a.tokens_out[(int64_t)b * (a.S + 1) + j] = x;
        }
        int token = -1;
        if (greedy) {
            if (mt > -CUDART_INF_F) token = best;
        } else if (mt > -CUDART_INF_F) {
            const double u = uniform(a.u_sample[b]);
            bool residual = refused;
            auto mass = [&](int i) {
                const double pi = weight(logit(t_row, i, a.target_type), mt, T) / zt;
                if (!residual) return pi;
                double qi = 0;
                if (!a.draft) qi = i == x ? 1.0 : 0.0;
                else if (mq > -CUDART_INF_F) qi = weight(logit(q_row, i, a.draft_type), mq, T) / zq;
                return fmax(pi - qi, 0.0);
            };
            double part = 0, total = 0;
            for (int attempt = 0; attempt < 2; ++attempt) {
                part = 0;
                for (int i = c.i0 + c.lane; i < c.i1; i += 32) part += mass(i);
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) part += __shfl_xor_sync(0xffffffffu, part, o);
                total = c.sum(c.lane == 0 ? part : 0.0);
                if (!residual || total >= VF_NO_RESIDUAL) break;
                residual = false;
            }
            // the part of the row in which the sum passes u * total, and its place there
            const double goal = u * total;
            double below = 0;
            int owner = -1, last = -1;
            double last_below = 0;
            for (int q = 0; q < size * VF_WARPS; ++q) {
                const double s = peer_f64(&sh.sum[c.turn][q % VF_WARPS], (uint32_t)(q / VF_WARPS));
                if (s > 0) { last = q; last_below = below; }
                if (owner < 0 && below + s > goal) { owner = q; break; }
                below += s;
            }
            if (owner < 0) { owner = last; below = last_below; }
            if (owner == (int)rank * VF_WARPS + c.warp) {
                int found = -1, some = -1;
                for (int base = c.i0; base < c.i1 && found < 0; base += 32) {
                    const int i = base + c.lane;
                    const double w = i < c.i1 ? mass(i) : 0.0;
                    double run = w;
#pragma unroll
                    for (int o = 1; o < 32; o <<= 1) {
                        const double v = __shfl_up_sync(0xffffffffu, run, o);
                        if (c.lane >= o) run += v;
                    }
                    const unsigned over = __ballot_sync(0xffffffffu, w > 0 && below + run > goal);
                    const unsigned any = __ballot_sync(0xffffffffu, w > 0);
                    if (any) some = base + 31 - __clz(any);
                    if (over) found = base + __ffs(over) - 1;
                    below += __shfl_sync(0xffffffffu, run, 31);
                }
                if (c.lane == 0) a.tokens_out[(int64_t)b * (a.S + 1) + j] = found >= 0 ? found : some;
            }
            sync_cluster();   // (the sums have been read)
        }
        if (rank == 0) {
            for (int k = threadIdx.x; k <= a.S; k += VF_THREADS)
                if (k > j || (k == j && (greedy || !(mt > -CUDART_INF_F)))) a.tokens_out[(int64_t)b * (a.S + 1) + k] = k == j ? token : -1;
            if (threadIdx.x == 0) a.accepted_out[b] = j;
        }
    }
    sync_cluster();   // no CTA's shared memory goes away under another
}

}  // namespace

cudaError_t launch_verify(const VerifyArgs &a, void *workspace, cudaStream_t s)
{
    VerifyParams p{a, reinterpret_cast<Control *>(workspace)};
    cudaError_t e;
    const int size = a.V >= 4096 ? 8 : 1;
    int clusters = 148 / size;
    if (a.B < clusters) clusters = a.B;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(clusters * size), 1, 1);
    cfg.blockDim = dim3(VF_THREADS, 1, 1);
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)size;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;   // (the kernel starts with pdl_enter)
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    e = cudaLaunchKernelEx(&cfg, verify_exact_kernel, p, size);
    count_launch();
    return e;
}

}  // namespace cat
