// Verification of drafted tokens against the target network's probabilities (cat_verify_drafts).
//
// Mathematics.  p_j = softmax(target_j / T), q_j = softmax(draft_j / T).  Draft x_j is accepted while u_j q_j(x_j) < p_j(x_j); at the
// first refusal the next token is drawn from max(p_j - q_j, 0), after the last draft from the row behind it: the first index whose
// cumulated mass exceeds u times the whole.  Outputs are tokens, so they have to be those of exact arithmetic whatever the order of
// the sums.  The library's way with such decisions: fast fp32 weights whose errors are bounded, and an fp64 pass for what is closer
// than the bound.
//
// verify_kernel.  A cluster of 1 to 8 CTAs takes a sequence, every CTA a contiguous part of the vocabulary, every warp chunks of 32 or 128
// 16-byte granules (one or four per lane, in flight together).  A chunk leaves its largest exponent (an integer in units of log 2) and its
// sum of weights, so one read of a row gives its normaliser and, where the row itself is drawn from, the chunk that holds the token; only a
// residual reads its two rows again, out of L2.  `group` rows and their drafts go through between two exchanges: few where reading the rows
// behind a refusal for nothing costs more than an exchange, up to eight where it does not.  What bounds it: the latency of a
// sequence's phases -- load, sums, exchange, decision, draw -- one after the other (8 sequences of 4 drafts over 32 000: 16 us, the bytes 2.8); with a large
// batch that of its loads too, which stop between the phases (cold, alone: 256 rows of 50 001 25 us at 0.25 instructions a cycle and scheduler; 64
// sequences of 7 drafts over 128 000 84 us for the 130 MB that it reads, 0.45).
//
// verify_settle_kernel, and the same in verify_kernel: what the sums leave undecided, in fp64.  Bound by latency: 14 us a sequence of 32 000.
//
// A weight 2^(x c - M), c = log2(e) / T, M an integer: n = rint(x c), f = x c - n in two fused steps on c as a sum of two floats, 2^f
// from the special function unit, n - M added to the exponent.  Its relative error does not grow with |x c|: f is off by at most
// 2^-26 + 2^-25 + 2^-28 (the roundings of x hi - n, at most 1/2, and of f, at most 1/2 + 2^-4, c's low float being worth up to 2^-4 where |x c| = 2^20; what
// the two floats leave of x c), the unit's 2^f by 1.46e-7 of itself (the largest over every float of [-0.57, 0.57], counted on the device):
// VF_EPS_WEIGHT.
#include "cat_tc.cuh"

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math_constants.h>

namespace cat {
namespace {

constexpr int VF_THREADS = 512;
constexpr int VF_SETTLE_CLUSTER = 16;                      // (largest cluster there is)
constexpr double VF_NO_RESIDUAL = 9.094947017729282e-13;   // 2^-40: a residual of less mass is what rounding left of none

// address of the same shared-memory location in the CTA of the given rank
__device__ __forceinline__ uint32_t peer(const void *p, uint32_t rank) { return mapa_cluster((uint32_t)__cvta_generic_to_shared(p), rank); }
__device__ __forceinline__ double peer_f64(const double *p, uint32_t rank)
{
    double v;
    asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(v) : "r"(peer(p, rank)) : "memory");
    return v;
}
__device__ __forceinline__ float peer_f32(const float *p, uint32_t rank)
{
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(peer(p, rank)) : "memory");
    return v;
}
__device__ __forceinline__ int peer_s32(const int *p, uint32_t rank)
{
    int v;
    asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(peer(p, rank)) : "memory");
    return v;
}

// A logit as the definitions take it: NaN counts as -inf, +inf as the largest number.
__device__ __forceinline__ float clean(float x)
{
    const uint32_t u = __float_as_uint(x), size = u & 0x7fffffffu;
    return __uint_as_float(size > 0x7f800000u ? 0xff800000u : u == 0x7f800000u ? 0x7f7fffffu : u);
}

__device__ __forceinline__ float logit(const void *row, int i, int type)
{
    if (type == CAT_F32) return clean(reinterpret_cast<const float *>(row)[i]);
    if (type == CAT_BF16) return clean(__bfloat162float(reinterpret_cast<const __nv_bfloat16 *>(row)[i]));
    return clean(__half2float(reinterpret_cast<const __half *>(row)[i]));
}

// A uniform number as the definitions take it, in [0, 1 - 2^-24]; NaN: 0.
__device__ __forceinline__ double uniform(float u) { return (double)fminf(fmaxf(u, 0.f), 0.99999994f); }

__device__ __forceinline__ float warp_max(float m)
{
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(m));
    return r;
}
__device__ __forceinline__ double warp_sum(double v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
// sums over the lanes up to this one
__device__ __forceinline__ double warp_scan(double v, int lane)
{
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const double w = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += w;
    }
    return v;
}

struct VerifyParams {
    VerifyArgs a;
    Control *ctl;
    int size;        // CTAs per cluster
    int group;       // target rows (and their drafts) before the first exchange; twice as many before each further one ...
    int max_group;   // ... up to this
    int vecs;        // granules of 16 bytes per lane and chunk
    int chunks_t, chunks_q;   // chunks of a target row, of a draft row
    int slots;       // chunk sums a CTA holds between two exchanges
    int settle;      // undecided sequences are settled in the same kernel
    int keep;        // there is room for the weights of two rows while they are
};

__device__ __forceinline__ const void *row_of(const void *base, int type, int64_t seq, int64_t row, int64_t seq_stride, int64_t row_stride)
{
    return reinterpret_cast<const unsigned char *>(base) + (seq * seq_stride + row * row_stride) * (type == CAT_F32 ? 4 : 2);
}

// ---------------------------------------------------------------- in 32 bits, with a bound
constexpr int VF_MAX_GROUP = 8;
constexpr int VF_MAX_ROWS = 2 * VF_MAX_GROUP;            // rows between two exchanges
constexpr int VF_EMPTY = -(1 << 28);                     // exponent of a part without mass
constexpr int VF_WILD = 1 << 28;                         // exponent of a part that fp32 cannot hold (|x c| > 2^20)
constexpr float VF_U = 5.9604645e-8f;                    // 2^-24
// relative errors: of a weight; of the sum of a chunk (three roundings where a granule's weights are added, the rest in fp64); of a probability
constexpr float VF_EPS_WEIGHT = 1.46e-7f + 0.6931472f * (1.4901161e-8f + 2.9802322e-8f + 3.7252903e-9f);
constexpr float VF_EPS_SUM = VF_EPS_WEIGHT + 3.f * VF_U;
constexpr float VF_EPS_P = VF_EPS_WEIGHT + VF_EPS_SUM + 4.f * VF_U;

template <int TYPE>
struct Logits;
template <>
struct Logits<CAT_F32> {
    static constexpr int PER = 4, SIZE = 4;
    static __device__ __forceinline__ float get(const uint4 &v, int k)
    {
        const uint32_t w = k == 0 ? v.x : k == 1 ? v.y : k == 2 ? v.z : v.w;
        return __uint_as_float(w);
    }
    static __device__ __forceinline__ uint32_t bits(const void *p, int64_t i) { return reinterpret_cast<const uint32_t *>(p)[i]; }
    static constexpr uint32_t MASKED = 0xff800000u;
    static __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) { return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b))); }
    static __device__ __forceinline__ float top(uint32_t a) { return fmaxf(__uint_as_float(a), -CUDART_INF_F); }
};
template <>
struct Logits<CAT_BF16> {
    static constexpr int PER = 8, SIZE = 2;
    static __device__ __forceinline__ float get(const uint4 &v, int k)
    {
        const uint32_t w = (k >> 1) == 0 ? v.x : (k >> 1) == 1 ? v.y : (k >> 1) == 2 ? v.z : v.w;
        return __uint_as_float(k & 1 ? w & 0xffff0000u : w << 16);
    }
    static __device__ __forceinline__ uint32_t bits(const void *p, int64_t i) { return reinterpret_cast<const uint16_t *>(p)[i]; }
    static constexpr uint32_t MASKED = 0xff80u;
    static __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b)
    {
        uint32_t d;
        asm("max.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
        return d;
    }
    static __device__ __forceinline__ float top(uint32_t a)
    {
        const uint4 v = make_uint4(a, a, a, a);
        return fmaxf(fmaxf(get(v, 0), get(v, 1)), -CUDART_INF_F);
    }
};
template <>
struct Logits<CAT_F16> {
    static constexpr int PER = 8, SIZE = 2;
    static __device__ __forceinline__ float get(const uint4 &v, int k)
    {
        const uint32_t w = (k >> 1) == 0 ? v.x : (k >> 1) == 1 ? v.y : (k >> 1) == 2 ? v.z : v.w;
        return __half2float(__ushort_as_half((unsigned short)(k & 1 ? w >> 16 : w & 0xffffu)));
    }
    static __device__ __forceinline__ uint32_t bits(const void *p, int64_t i) { return reinterpret_cast<const uint16_t *>(p)[i]; }
    static constexpr uint32_t MASKED = 0xfc00u;
    static __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b)
    {
        uint32_t d;
        asm("max.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
        return d;
    }
    static __device__ __forceinline__ float top(uint32_t a)
    {
        const uint4 v = make_uint4(a, a, a, a);
        return fmaxf(fmaxf(get(v, 0), get(v, 1)), -CUDART_INF_F);
    }
};

// PER entries of a row from `i` on as one granule, -inf outside [0, V).  One load where the granule lies in the row on 16 bytes.
template <int TYPE>
__device__ __forceinline__ uint4 granule(const void *row, int i, int V)
{
    using L = Logits<TYPE>;
    const unsigned char *at = reinterpret_cast<const unsigned char *>(row) + (int64_t)i * L::SIZE;
    uint4 v;
    if (i >= 0 && i + L::PER <= V && (reinterpret_cast<uintptr_t>(at) & 15u) == 0) {
        asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(at));
        return v;
    }
    uint32_t w[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if (L::SIZE == 4) {
            w[q] = i + q >= 0 && i + q < V ? L::bits(row, i + q) : L::MASKED;
        } else {
            const int k = i + 2 * q;
            const uint32_t lo = k >= 0 && k < V ? L::bits(row, k) : L::MASKED, hi = k + 1 >= 0 && k + 1 < V ? L::bits(row, k + 1) : L::MASKED;
            w[q] = lo | (hi << 16);
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// entries between the 16-byte boundary before the row and the row
template <int TYPE>
__device__ __forceinline__ int row_offset(const void *row)
{
    return (int)(reinterpret_cast<uintptr_t>(row) & 15u) / Logits<TYPE>::SIZE;
}

__device__ __forceinline__ uint64_t pack2(float a, float b)
{
    uint64_t v;
    asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b));
    return v;
}
__device__ __forceinline__ void unpack2(uint64_t v, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ float ex2(float f)
{
    float e;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(f));
    return e;
}

// c = log2(e) / T as a sum of two floats; `fits` where |x c| of ordinary logits and the shifts below are ordinary numbers too
struct Scale {
    double c;
    uint64_t hi, lo;
    float high, inv;
    bool fits;
    __device__ explicit Scale(double T)
    {
        c = 1.4426950408889634 / T;
        const float h = (float)c, l = (float)(c - (double)h);
        high = h;
        hi = pack2(h, h);
        lo = pack2(l, l);
        fits = h > 1e-15f && h < 1e15f;
        inv = fits ? 1.f / h : 1.f;
    }
};

// Weights 2^(x c - M) of two entries.  Entries below (M - 100) / c -- masked ones among them, and NaN -- count as that: they are 2^-100 of
// the sum at most.
struct Weights {
    uint64_t magic, back;
    float floor;
    __device__ Weights(const Scale &s, int M)
    {
        const float m = 12582912.f - (float)M;      // 1.5 2^23 - M: what is added to it is rounded to a whole number
        magic = pack2(m, m);
        back = magic;
        floor = ((float)M - 100.f) * s.inv;
    }
    __device__ __forceinline__ void operator()(const Scale &s, float a, float b, float &wa, float &wb) const
    {
        const uint64_t x = pack2(fmaxf(a, floor), fmaxf(b, floor));
        const uint64_t r = fma2(x, s.hi, magic);                                   // n - M in its low bits
        const uint64_t minus_n = fma2(r, 0xbf800000bf800000ull, back);             // magic - r = -n, exactly
        const uint64_t f = fma2(x, s.lo, fma2(x, s.hi, minus_n));
        float fa, fb, ra, rb;
        unpack2(f, fa, fb);
        unpack2(r, ra, rb);
        wa = __uint_as_float(__float_as_uint(ex2(fa)) + (__float_as_uint(ra) << 23));
        wb = __uint_as_float(__float_as_uint(ex2(fb)) + (__float_as_uint(rb) << 23));
    }
};

// sum of N weights in pairs: as many roundings as a tree over them has levels
template <int N>
__device__ __forceinline__ float sum_of(const float (&w)[N])
{
    uint64_t v[N / 2];
#pragma unroll
    for (int k = 0; k < N / 2; ++k) v[k] = pack2(w[2 * k], w[2 * k + 1]);
#pragma unroll
    for (int h = N / 4; h > 0; h >>= 1)
#pragma unroll
        for (int k = 0; k < h; ++k) asm("add.rn.f32x2 %0, %1, %2;" : "=l"(v[k]) : "l"(v[k]), "l"(v[k + h]));
    float a, b;
    unpack2(v[0], a, b);
    return a + b;
}

// What a sequence's control flow hangs on is read once, by its cluster's first CTA, and reaches the others through shared memory: whatever a
// caller does to its inputs meanwhile, all take the same way and meet at the same barriers.
struct Head {
    float T, u_sample;
    int length;
};
__device__ __forceinline__ Head read_head(const VerifyArgs &a, int b)
{
    return Head{a.temperature ? a.temperature[b] : 1.f, a.u_sample[b], a.lengths ? min(a.lengths[b], a.S) : a.S};
}
__device__ __forceinline__ Head peer_head(const Head *h, uint32_t rank)
{
    return Head{peer_f32(&h->T, rank), peer_f32(&h->u_sample, rank), peer_s32(&h->length, rank)};
}
// A draft, its uniform number, and its logits in the target's and in the draft's row (-inf for a token outside the vocabulary).
struct Draft {
    int x;
    float u, xt, xq;
};
__device__ __forceinline__ Draft read_draft(const VerifyArgs &a, int64_t b, int j, int target_type, int draft_type)
{
    Draft d{*(const volatile int32_t *)&a.tokens[b * a.S + j], a.u_accept[b * a.S + j], -CUDART_INF_F, -CUDART_INF_F};      // (x: read once, checked, used)
    if (d.x >= 0 && d.x < a.V) {
        d.xt = logit(row_of(a.target, target_type, b, j, a.target_seq, a.target_row), d.x, target_type);
        if (a.draft) d.xq = logit(row_of(a.draft, draft_type, b, j, a.draft_seq, a.draft_row), d.x, draft_type);
    }
    return d;
}
__device__ __forceinline__ Draft peer_draft(const Draft *d, uint32_t rank)
{
    return Draft{peer_s32(&d->x, rank), peer_f32(&d->u, rank), peer_f32(&d->xt, rank), peer_f32(&d->xq, rank)};
}

struct SettleShared {
    double table[64];                       // 2^(i / 64)
    int claim[2];                           // the sequence that the cluster works on, and the row it goes on from ...
    Head head;                              // ... and what it hangs on (the first CTA's)
    Draft draft[2];                         // the draft of the row at work (likewise; two sets in turn)
    double part[2][VF_THREADS / 32];        // the warps' parts of two sums over the cluster ...
    double cta[2][2];                       // ... and the CTA's (two sets in turn: an exchange is one barrier)
    float top[VF_THREADS / 32];             // the warps' largest logits of a row ...
    float cta_top[2];                       // ... and the CTA's (two sets in turn; apart from the sums, which a draw goes on from)
};

struct VerifyShared {
    SettleShared settle;
    Head head;                        // (the first CTA's, as are the drafts of a round: two sets in turn)
    Draft draft[2][VF_MAX_GROUP];
    double row_z[2][VF_MAX_ROWS];     // this CTA's part of the rows between two exchanges (two sets in turn) ...
    int row_m[2][VF_MAX_ROWS];        // ... and their exponents; greedy: value and place of the largest entry
    double total_z[VF_MAX_ROWS];      // over the cluster
    int total_m[VF_MAX_ROWS];
    int verdict, at, x;               // what the round decided, for which row, and the draft there;
    int source, token;                // what the token behind the accepted drafts is drawn from, or (VF_FROM_NOTHING) the token
    int owner, open;                  // the CTA that draws; there: the draw came too close to a border
};
enum { VF_GO_ON = 0, VF_REFUSED = 1, VF_ALL_STAND = 2, VF_UNDECIDED = 3 };
enum { VF_FROM_NOTHING = 0, VF_FROM_ROW = 1, VF_FROM_DIFFERENCE = 2 /* p - q */, VF_FROM_OTHERS = 3 /* p without a refused draft from a lookup */ };

// z 2^(m - M), m <= M
__device__ __forceinline__ double scaled(double z, int m, int M)
{
    const int d = m - M;
    return d < -1000 ? 0.0 : z * __hiloint2double((1023 + d) << 20, 0);
}

// the sum of a lane's granules' sums
template <int VECS>
__device__ __forceinline__ double lane_sum(const float (&v)[VECS])
{
    double d = (double)v[0];
#pragma unroll
    for (int q = 1; q < VECS; ++q) d += (double)v[q];
    return d;
}

// The granules of a chunk; chunks start on the 16-byte boundary before the row.
template <int TYPE, int VECS>
__device__ __forceinline__ void load_chunk(const void *row, int chunk, int V, int lane, uint4 (&v)[VECS])
{
    using L = Logits<TYPE>;
    const int first = chunk * ((32 * VECS) * L::PER) - row_offset<TYPE>(row);
    if (first >= 0 && first + (32 * VECS) * L::PER <= V) {
        const unsigned char *at = reinterpret_cast<const unsigned char *>(row) + (int64_t)first * L::SIZE + lane * 16;
#pragma unroll
        for (int q = 0; q < VECS; ++q)
            asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                         : "=r"(v[q].x), "=r"(v[q].y), "=r"(v[q].z), "=r"(v[q].w) : "l"(at + q * 512));
    } else {
#pragma unroll
        for (int q = 0; q < VECS; ++q) v[q] = granule<TYPE>(row, first + (q * 32 + lane) * L::PER, V);
    }
}

// largest entry of the granules (pairs at a time in 16 bits), NaN left out
template <int TYPE>
__device__ __forceinline__ uint32_t granule_max2(const uint4 &v)
{
    using L = Logits<TYPE>;
    return L::max2(L::max2(v.x, v.y), L::max2(v.z, v.w));
}
template <int TYPE, int VECS>
__device__ __forceinline__ float chunk_max(const uint4 (&v)[VECS])
{
    using L = Logits<TYPE>;
    uint32_t m = granule_max2<TYPE>(v[0]);
#pragma unroll
    for (int q = 1; q < VECS; ++q) m = L::max2(m, granule_max2<TYPE>(v[q]));
    return warp_max(L::top(m));
}

// Largest exponent and sum of weights of a chunk.
template <int TYPE, int VECS>
__device__ __forceinline__ void chunk_stats(const uint4 (&v)[VECS], const Scale &sc, int &M, double &Z)
{
    using L = Logits<TYPE>;
    const float m = chunk_max<TYPE, VECS>(v);
    const float mc = m * sc.high;
    Z = 0;
    M = VF_EMPTY;
    if (m == -CUDART_INF_F) return;
    M = VF_WILD;
    if (!(fabsf(mc) <= 1048576.f)) return;
    M = __float2int_rn(mc);
    const Weights weights(sc, M);
    float sum[VECS];
#pragma unroll
    for (int q = 0; q < VECS; ++q) {
        float w[L::PER];
#pragma unroll
        for (int k = 0; k < L::PER; k += 2) weights(sc, L::get(v[q], k), L::get(v[q], k + 1), w[k], w[k + 1]);
        sum[q] = sum_of<L::PER>(w);
    }
    Z = warp_sum(lane_sum(sum));
}

// Largest entry and its first place in a chunk that starts at entry `first` (greedy decoding).
template <int TYPE, int VECS>
__device__ __forceinline__ void chunk_top(const uint4 (&v)[VECS], int first, int lane, double &value, int &place)
{
    using L = Logits<TYPE>;
    const float m = clean(chunk_max<TYPE, VECS>(v));
    place = 0x7fffffff;
#pragma unroll
    for (int q = VECS - 1; q >= 0; --q)
#pragma unroll
        for (int k = L::PER - 1; k >= 0; --k)
            if (L::get(v[q], k) >= m) place = first + (q * 32 + lane) * L::PER + k;
    place = __reduce_min_sync(0xffffffffu, place);
    value = (double)m;
}

// What a draw is from: one row, or what is left of it less another.
struct Source {
    const void *t_row, *q_row;      // q_row: null where the draft is a point, or nothing is subtracted
    float t_scale, q_scale;         // 1 / normaliser
    int t_m, q_m;                   // exponents of the rows
    int point;                      // entry without mass (a refused draft from a lookup), or -1
};

// N entries of a row from `i` on as words, any alignment: whole 32-bit words and a shift between neighbours where the row allows it.
template <int N>
struct Words {
    uint32_t w[N];
};
template <int TYPE, int N>
__device__ __noinline__ Words<N * Logits<TYPE>::SIZE / 4> unaligned_words(const void *row, int i, int V)
{
    using L = Logits<TYPE>;
    constexpr int WORDS = N * L::SIZE / 4;
    const unsigned char *at = reinterpret_cast<const unsigned char *>(row) + (int64_t)i * L::SIZE;
    Words<WORDS> r;
    if (i >= 1 && i + N < V) {
        if ((reinterpret_cast<uintptr_t>(at) & 3u) == 0) {
#pragma unroll
            for (int q = 0; q < WORDS; ++q) asm volatile("ld.global.nc.u32 %0, [%1];" : "=r"(r.w[q]) : "l"(at + 4 * q));
        } else {
            // (one entry before and one behind these are in the row)
            uint32_t u[WORDS + 1];
#pragma unroll
            for (int q = 0; q <= WORDS; ++q) asm volatile("ld.global.nc.u32 %0, [%1];" : "=r"(u[q]) : "l"(at - 2 + 4 * q));
#pragma unroll
            for (int q = 0; q < WORDS; ++q) r.w[q] = __funnelshift_r(u[q], u[q + 1], 16);
        }
    } else {
#pragma unroll
        for (int q = 0; q < WORDS; ++q) {
            const int k = i + q * (4 / L::SIZE);
            r.w[q] = k >= 0 && k < V ? L::bits(row, k) : L::MASKED;
            if (L::SIZE == 2) r.w[q] |= (k + 1 >= 0 && k + 1 < V ? L::bits(row, k + 1) : L::MASKED) << 16;
        }
    }
    return r;
}
template <int TYPE, int N>
__device__ __forceinline__ Words<N * Logits<TYPE>::SIZE / 4> words_of(const void *row, int i, int V)
{
    using L = Logits<TYPE>;
    constexpr int WORDS = N * L::SIZE / 4;
    const unsigned char *at = reinterpret_cast<const unsigned char *>(row) + (int64_t)i * L::SIZE;
    if (i < 0 || i + N > V || (reinterpret_cast<uintptr_t>(at) & (WORDS >= 4 ? 15u : 7u)) != 0) return unaligned_words<TYPE, N>(row, i, V);
    Words<WORDS> r;
    if constexpr (WORDS == 2) {
        asm volatile("ld.global.nc.v2.u32 {%0, %1}, [%2];" : "=r"(r.w[0]), "=r"(r.w[1]) : "l"(at));
    } else {
#pragma unroll
        for (int q = 0; q < WORDS; q += 4)
            asm volatile("ld.global.nc.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.w[q]), "=r"(r.w[q + 1]), "=r"(r.w[q + 2]), "=r"(r.w[q + 3]) : "l"(at + 4 * q));
    }
    return r;
}
template <int TYPE, int N>
__device__ __forceinline__ void entries(const Words<N * Logits<TYPE>::SIZE / 4> &r, float (&x)[N])
{
    using L = Logits<TYPE>;
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const uint32_t one = r.w[k * L::SIZE / 4];
        x[k] = L::get(make_uint4(one, one, one, one), L::SIZE == 4 ? 0 : k & 1);
    }
}

// entries between the boundary of four entries' bytes before the row and the row
template <int TYPE>
__device__ __forceinline__ int fours_offset(const void *row)
{
    return (int)(reinterpret_cast<uintptr_t>(row) & (4 * Logits<TYPE>::SIZE - 1)) / Logits<TYPE>::SIZE;
}

// The masses of PER entries of the target's chunk grid, entry i on: p, or p - q where that is positive (x: the draft's logits there).
template <int TT>
__device__ __forceinline__ void masses_of(const Source &src, const Scale &sc, const Weights &wt, const Weights &wq, int i, int V, const uint4 &tv,
                                          const float (&x)[Logits<TT>::PER], float (&w)[Logits<TT>::PER])
{
    using L = Logits<TT>;
#pragma unroll
    for (int k = 0; k < L::PER; k += 2) wt(sc, L::get(tv, k), L::get(tv, k + 1), w[k], w[k + 1]);
#pragma unroll
    for (int k = 0; k < L::PER; ++k) w[k] *= src.t_scale;
    if (src.q_row) {
#pragma unroll
        for (int k = 0; k < L::PER; k += 2) {
            float a, b;
            wq(sc, x[k], x[k + 1], a, b);
            w[k] = fmaxf(w[k] - a * src.q_scale, 0.f);
            w[k + 1] = fmaxf(w[k + 1] - b * src.q_scale, 0.f);
        }
    }
    if (i < 0 || i + L::PER > V || (uint32_t)(src.point - i) < (uint32_t)L::PER) {
#pragma unroll
        for (int k = 0; k < L::PER; ++k)
            if (i + k == src.point || i + k < 0 || i + k >= V) w[k] = 0.f;
    }
}
// ... of a chunk's granules of this lane, added up
template <int TT, int QT, int VECS>
__device__ __forceinline__ void chunk_masses(const Source &src, const Scale &sc, const Weights &wt, const Weights &wq, int chunk, int V, int lane,
                                             float (&sum)[VECS])
{
    using L = Logits<TT>;
    uint4 tv[VECS];
    load_chunk<TT, VECS>(src.t_row, chunk, V, lane, tv);
    const int first = (chunk * (32 * VECS) + lane) * L::PER - row_offset<TT>(src.t_row);
    Words<L::PER * Logits<QT>::SIZE / 4> qv[VECS];
    float x[L::PER], w[L::PER];     // (qv and x are looked at where there is a draft's row only)
    if (src.q_row) {
#pragma unroll
        for (int q = 0; q < VECS; ++q) qv[q] = words_of<QT, L::PER>(src.q_row, first + q * 32 * L::PER, V);
    }
#pragma unroll
    for (int q = 0; q < VECS; ++q) {
        if (src.q_row) entries<QT, L::PER>(qv[q], x);
        masses_of<TT>(src, sc, wt, wq, first + q * 32 * L::PER, V, tv[q], x, w);
        sum[q] = sum_of<L::PER>(w);
    }
}

// One warp finds the token in a chunk: `below` is the mass before the chunk, `goal` what has to be exceeded, `err` how far either may be off
// together.  Returns the token, or -1 where it is not certain.
template <int TT, int QT, int VECS>
__device__ __forceinline__ int find_in_chunk(const Source &src, const Scale &sc, const Weights &wt, const Weights &wq, int chunk, int V, double below,
                                             double goal, double err, int lane)
{
    using L = Logits<TT>;
    float sum[VECS];
    chunk_masses<TT, QT, VECS>(src, sc, wt, wq, chunk, V, lane, sum);
    double run[VECS];
#pragma unroll
    for (int q = 0; q < VECS; ++q) run[q] = (double)sum[q];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1)
#pragma unroll
        for (int q = 0; q < VECS; ++q) {
            const double v = __shfl_up_sync(0xffffffffu, run[q], o);
            if (lane >= o) run[q] += v;
        }
    // the granule in which the sum passes the goal
    int at = -1;
    double before = 0;
#pragma unroll
    for (int q = 0; q < VECS; ++q) {
        const unsigned over = __ballot_sync(0xffffffffu, below + run[q] > goal);
        if (over && at < 0) {
            const int l = __ffs(over) - 1;
            at = q * 32 + l;
            before = below + __shfl_sync(0xffffffffu, run[q] - (double)sum[q], l);
        }
        below += __shfl_sync(0xffffffffu, run[q], 31);
    }
    if (at < 0) return -1;
    const int i = (chunk * (32 * VECS) + at) * L::PER - row_offset<TT>(src.t_row);
    const uint4 tv = granule<TT>(src.t_row, i, V);
    float x[L::PER], w[L::PER];
    if (src.q_row) entries<QT, L::PER>(words_of<QT, L::PER>(src.q_row, i, V), x);
    masses_of<TT>(src, sc, wt, wq, i, V, tv, x, w);
#pragma unroll
    for (int k = 0; k < L::PER; ++k) {
        const double after = before + (double)w[k];
        if (after > goal) return goal - before >= err && after - goal >= err ? i + k : -1;
        before = after;
    }
    return -1;
}

// ---------------------------------------------------------------- in 64 bits
// The weights 2^((x - m) c) of N logits in fp64, logits as the definitions take them: 2^(n / 64) from a table, the rest by the Taylor series of
// e^(r ln 2) up to the fourth power (|r| <= 1 / 128 leaves 4e-14).  Ten fp64 operations each (floats are made doubles by moving their bits
// where c leaves ordinary logits ordinary numbers: the conversion unit is slower).  Step by step across the entries, and so that the
// compiler keeps it that way: one alone is a chain of dependent steps.
template <int N>
__device__ __forceinline__ void weights_f64(const double *table, const float (&x)[N], float m, double c, double (&w)[N])
{
    double e[N], t[N], r[N];
    int beyond[N];
    const float cf = (float)c;
    const bool ordinary = cf > 1e-15f && cf < 1e15f;
    // (z - m) c in three steps, none of which overflows before the product would pass 1000 (c from 1e-300 to 2^150, z and m over all of fp32) or gives a
    // number where z = m but nought; a masked z gives -inf, or NaN
    const float before = c < 1.0 ? 0.5f : 1.f, between = c > 0x1p100 ? 0x1p40f : 1.f, after = (float)(c / ((double)before * (double)between));
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const float z = clean(x[k]), at = fmaf(z, before, -m * before) * between * after;
        const bool fits = at > -1001.f && at < 1000.f;
        beyond[k] = fits ? 0 : at >= 1000.f ? 2 : 1;      // (a reference that does not suit the row shows in the sum)
        const float y = fits ? z : m;
        const uint32_t f = __float_as_uint(y);
        if (ordinary) e[k] = __hiloint2double((int)((f & 0x80000000u) | (((f & 0x7fffffffu) >> 3) + 0x38000000u)), (int)(f << 29));
        else e[k] = (double)y;
    }
    const uint32_t fm = __float_as_uint(m);
    const double md = ordinary ? __hiloint2double((int)((fm & 0x80000000u) | (((fm & 0x7fffffffu) >> 3) + 0x38000000u)), (int)(fm << 29)) : (double)m;
#pragma unroll
    for (int k = 0; k < N; ++k) asm volatile("sub.rn.f64 %0, %0, %1;" : "+d"(e[k]) : "d"(md));
#pragma unroll
    for (int k = 0; k < N; ++k) asm volatile("mul.rn.f64 %0, %0, %1;" : "+d"(e[k]) : "d"(c));
#pragma unroll
    for (int k = 0; k < N; ++k)
        if (e[k] < -1000.0) beyond[k] = 1;
#pragma unroll
    for (int k = 0; k < N; ++k) asm volatile("fma.rn.f64 %0, %1, %2, %3;" : "=d"(t[k]) : "d"(e[k]), "d"(64.0), "d"(6755399441055744.0));   // 1.5 2^52: rounded
#pragma unroll
    for (int k = 0; k < N; ++k) asm volatile("sub.rn.f64 %0, %1, %2;" : "=d"(r[k]) : "d"(t[k]), "d"(6755399441055744.0));
#pragma unroll
    for (int k = 0; k < N; ++k) asm volatile("fma.rn.f64 %0, %1, %2, %0;" : "+d"(e[k]) : "d"(r[k]), "d"(-0.015625));      // (exact)
#pragma unroll
    for (int k = 0; k < N; ++k) asm volatile("fma.rn.f64 %0, %1, %2, %3;" : "=d"(r[k]) : "d"(e[k]), "d"(0.009618129107628477), "d"(0.05550410866482158));
    const double coef[3] = {0.2402265069591007, 0.6931471805599453, 1.0};      // (ln 2)^i / i!
#pragma unroll
    for (int i = 0; i < 3; ++i)
#pragma unroll
        for (int k = 0; k < N; ++k) asm volatile("fma.rn.f64 %0, %0, %1, %2;" : "+d"(r[k]) : "d"(e[k]), "d"(coef[i]));
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const int n = __double2loint(t[k]);
        const double s = table[n & 63];
        w[k] = beyond[k] == 0 ? r[k] * __hiloint2double(__double2hiint(s) + ((n >> 6) << 20), __double2loint(s)) : beyond[k] == 2 ? 1e300 : 0.0;
    }
}
__device__ __forceinline__ void fill_table(double *table)
{
    if (threadIdx.x < 64) table[threadIdx.x] = exp2((double)threadIdx.x * 0.015625);
}

// One cluster settles a sequence in fp64.  Its rows are taken four entries at a time, both on the grid of the target's addresses: CTA r, warp w have
// the (warps r + w)-th part, in order.
template <int TT, int QT>
struct Settle {
    const VerifyArgs &a;
    SettleShared &sh;
    double *kept;                    // [row][entry of four][unit]: the weights, where they find room (else null)
    const void *t_row, *q_row;       // q_row: null where there is none
    int rank, size, warps, warp, lane, turn = 0, top_turn = 0;
    int offset, g_cta, room, g_first, g_end;
    float m[2] = {0.f, 0.f};         // what the weights of the rows are relative to
    double c;

    __device__ Settle(const VerifyArgs &args, SettleShared &s, double *k, int n, double T) : a(args), sh(s), kept(k), size(n)
    {
        rank = size > 1 ? (int)cluster_ctarank() : 0;
        warps = (int)blockDim.x >> 5;
        warp = threadIdx.x >> 5;
        lane = threadIdx.x & 31;
        c = fmax(1.4426950408889634 / T, 1e-300);       // (T infinite: all entries that are there weigh the same)
    }
    __device__ void rows(const void *t, const void *q)
    {
        t_row = t;
        q_row = q;
        offset = fours_offset<TT>(t);
        const int64_t units = (a.V + offset + 3) / 4, parts = (int64_t)size * warps;
        g_cta = (int)(units * rank / size);
        room = (int)((units + size - 1) / size);
        g_first = (int)(units * (rank * warps + warp) / parts);
        g_end = (int)(units * (rank * warps + warp + 1) / parts);
        m[0] = m[1] = 0.f;
    }
    __device__ __forceinline__ double weight(float x, float ref) const
    {
        const float xs[1] = {x};
        double w[1];
        weights_f64<1>(sh.table, xs, ref, c, w);
        return w[0];
    }
    // two sums over the cluster, in a fixed order; their parts stay in sh.part and sh.cta[turn]
    __device__ void sums(double &v0, double &v1)
    {
        turn ^= 1;
        const double s0 = warp_sum(v0), s1 = warp_sum(v1);
        if (lane == 0) {
            sh.part[0][warp] = s0;
            sh.part[1][warp] = s1;
        }
        __syncthreads();
        if (warp < 2) {
            const double s = warp_sum(lane < warps ? sh.part[warp][lane] : 0.0);
            if (lane == 0) sh.cta[turn][warp] = s;
        }
        cluster_sync();
        v0 = warp_sum(lane < size ? peer_f64(&sh.cta[turn][0], (uint32_t)lane) : 0.0);
        v1 = warp_sum(lane < size ? peer_f64(&sh.cta[turn][1], (uint32_t)lane) : 0.0);
    }
    // the weights of one unit of both rows
    __device__ __forceinline__ void weights_at(int g, double (&wt)[4], double (&wq)[4]) const
    {
        const int i = g * 4 - offset;
        const Words<Logits<TT>::SIZE> tv = words_of<TT, 4>(t_row, i, a.V);
        Words<Logits<QT>::SIZE> qv;
        if (q_row) qv = words_of<QT, 4>(q_row, i, a.V);
        float x[4];
        entries<TT, 4>(tv, x);
        weights_f64<4>(sh.table, x, m[0], c, wt);
        if (q_row) {
            entries<QT, 4>(qv, x);
            weights_f64<4>(sh.table, x, m[1], c, wq);
        } else {
            wq[0] = wq[1] = wq[2] = wq[3] = 0;
        }
    }
    __device__ __forceinline__ void weights_kept(int g, double (&wt)[4], double (&wq)[4]) const
    {
        if (!kept) {
            weights_at(g, wt, wq);
            return;
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            wt[k] = kept[k * room + g - g_cta];
            wq[k] = q_row ? kept[(4 + k) * room + g - g_cta] : 0.0;
        }
    }
    // Sums of the rows' weights.  `exact_end`: entries below 2^-1000 of their row's largest, and only those, weigh nothing.
    __device__ void normalisers(double &zt, double &zq, bool exact_end)
    {
        for (bool looked_up = false;; looked_up = true) {
            if (looked_up || exact_end) {
                m[0] = largest<TT>(t_row);
                m[1] = q_row ? largest<QT>(q_row) : 0.f;
                if (m[0] == -CUDART_INF_F) m[0] = 0.f;
                if (m[1] == -CUDART_INF_F) m[1] = 0.f;
            }
            zt = zq = 0;
#pragma unroll 1
            for (int g = g_first + lane; g < g_end; g += 32) {
                double wt[4], wq[4];
                weights_at(g, wt, wq);
                zt += (wt[0] + wt[1]) + (wt[2] + wt[3]);
                zq += (wq[0] + wq[1]) + (wq[2] + wq[3]);
                if (kept) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        kept[k * room + g - g_cta] = wt[k];
                        if (q_row) kept[(4 + k) * room + g - g_cta] = wq[k];
                    }
                }
            }
            sums(zt, zq);
            // With logits / T within some hundreds of zero, nought is as good a reference as the row's largest: what either drops is less than any
            // u times the mass, u = 0 apart.  Else they are looked up.
            const bool suits = zt > 1e-200 && zt < 1e270 && (!q_row || (zq > 1e-200 && zq < 1e270));
            if (suits || looked_up || exact_end) return;
        }
    }
    // whether a logit's weight is less than 2^-1000 of its row's largest, which is between the row's sum and a V-th (2^-22) of it
    template <int TYPE>
    __device__ bool vanishes(const void *row, float x, double log_mass)
    {
        if (log_mass > -1000.0 || log_mass < -1023.0) return log_mass < -1000.0;
        return ((double)x - (double)largest<TYPE>(row)) * c < -1000.0;
    }
    template <int TYPE>
    __device__ float largest(const void *row)
    {
        float top = -CUDART_INF_F;
#pragma unroll 1
        for (int g = g_first + lane; g < g_end; g += 32) {
            float x[4];
            entries<TYPE, 4>(words_of<TYPE, 4>(row, g * 4 - offset, a.V), x);
            top = fmaxf(top, fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])));
        }
        top = clean(warp_max(top));
        if (lane == 0) sh.top[warp] = top;
        top_turn ^= 1;
        __syncthreads();
        if (warp == 0) {
            const float t = warp_max(lane < warps ? sh.top[lane] : -CUDART_INF_F);
            if (lane == 0) sh.cta_top[top_turn] = t;
        }
        cluster_sync();
        return warp_max(lane < size ? peer_f32(&sh.cta_top[top_turn], (uint32_t)lane) : -CUDART_INF_F);
    }
};

// Sequence b from its row j on (the drafts before stand), by the whole cluster.  Greedy sequences never come here.
template <int TT, int QT>
__device__ __noinline__ void settle_sequence(const VerifyParams &p, SettleShared &sh, double *kept, int size, int b, int j, Head head)
{
    const VerifyArgs &a = p.a;
    const int length = head.length;
    Settle<TT, QT> c(a, sh, kept, size, (double)head.T);
    const int lane = c.lane;
    const bool writer = c.rank == 0 && threadIdx.x == 0;
    const double u_sample = uniform(head.u_sample);       // (0: the draw is the first entry with any mass)
    if (writer) atomicAdd(reinterpret_cast<unsigned long long *>(&p.ctl->refined_total), 1ull);
    int32_t *out = a.tokens_out + (int64_t)b * (a.S + 1);
    double zt, zq;
    int x = -1;
    bool refused = false;
    for (;; ++j) {
        c.rows(row_of(a.target, TT, b, j, a.target_seq, a.target_row),
               a.draft && j < length ? row_of(a.draft, QT, b, j, a.draft_seq, a.draft_row) : nullptr);
        if (writer && j < length) sh.draft[j & 1] = read_draft(a, b, j, TT, QT);
        c.normalisers(zt, zq, u_sample == 0.0);
        if (j >= length) break;
        const Draft d = peer_draft(&sh.draft[j & 1], 0);
        x = d.x;
        const bool inside = x >= 0 && x < a.V;
        // u q < p by logarithms: either may be smaller than any number of fp64
        const float xt = zt > 0 ? d.xt : -CUDART_INF_F, xq = zq > 0 ? d.xq : -CUDART_INF_F;
        const double log_p = ((double)xt - (double)c.m[0]) * c.c - log2(zt), log_q = a.draft ? ((double)xq - (double)c.m[1]) * c.c - log2(zq) : 0.0;
        const bool no_p = xt == -CUDART_INF_F || c.template vanishes<TT>(c.t_row, xt, log_p);
        const bool no_q = a.draft ? xq == -CUDART_INF_F || c.template vanishes<QT>(c.q_row, xq, log_q) : !inside;
        refused = no_p || !(no_q || log2(uniform(d.u)) + log_q < log_p);
        if (refused) break;
        if (writer) out[j] = x;
    }
    int token = -1;
    bool mine = writer;
    if (zt > 0) {
        // Masses: the target's weights as they are, or (residual) what the draft's row leaves of p; the sums of the former are there.
        const double per_t = 1.0 / zt, per_q = zq > 0 ? 1.0 / zq : 0.0;
        bool residual = refused && (zq > 0 || !a.draft);
        auto masses = [&](int g, double (&w)[4]) {
            double wq[4];
            c.weights_kept(g, w, wq);
            if (!residual) return;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                w[k] = fma(wq[k], -per_q, w[k] * per_t);
                if (__double2hiint(w[k]) < 0 || (!a.draft && g * 4 - c.offset + k == x)) w[k] = 0.0;
            }
        };
        double total = zt;
        if (residual) {
            double none = 0;
            total = 0;
#pragma unroll 1
            for (int g = c.g_first + lane; g < c.g_end; g += 32) {
                double w[4];
                masses(g, w);
                total += (w[0] + w[1]) + (w[2] + w[3]);
            }
            c.sums(total, none);
            if (total < VF_NO_RESIDUAL) {
                residual = false;
                total = 0;
#pragma unroll 1
                for (int g = c.g_first + lane; g < c.g_end; g += 32) {
                    double w[4];
                    masses(g, w);
                    total += (w[0] + w[1]) + (w[2] + w[3]);
                }
                c.sums(total, none);
            }
        }
        // the CTA, the warp, the entry at which the sum passes u times the whole; roundings apart: the last with mass
        const double goal = u_sample * total;
        auto passes = [&](double v, double &below) {
            const double run = warp_scan(v, lane);
            const unsigned over = __ballot_sync(0xffffffffu, v > 0 && below + run > goal), any = __ballot_sync(0xffffffffu, v > 0);
            const int l = over ? __ffs(over) - 1 : 31 - __clz(any);
            below += __shfl_sync(0xffffffffu, run - v, l);
            return l;
        };
        double below = 0;
        const int owner = passes(lane < size ? peer_f64(&sh.cta[c.turn][0], (uint32_t)lane) : 0.0, below);
        mine = false;
        if (owner == c.rank) {
            const int owner_warp = passes(lane < c.warps ? sh.part[0][lane] : 0.0, below);
            if (owner_warp == c.warp) {
                int some = -1;
#pragma unroll 1
                for (int base = c.g_first; base < c.g_end && token < 0; base += 32) {
                    const int g = base + lane, i = g * 4 - c.offset;
                    double w[4] = {0, 0, 0, 0};
                    if (g < c.g_end) masses(g, w);
                    const double sum = (w[0] + w[1]) + (w[2] + w[3]), run = warp_scan(sum, lane);
                    int here = -1, last = -1;
                    double at = below + run - sum;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        at += w[k];
                        if (w[k] > 0) {
                            last = i + k;
                            if (here < 0 && at > goal) here = i + k;
                        }
                    }
                    const unsigned over = __ballot_sync(0xffffffffu, here >= 0), any = __ballot_sync(0xffffffffu, last >= 0);
                    if (over) token = __shfl_sync(0xffffffffu, here, __ffs(over) - 1);
                    if (any) some = __shfl_sync(0xffffffffu, last, 31 - __clz(any));
                    below += __shfl_sync(0xffffffffu, run, 31);
                }
                if (token < 0) token = some;
                mine = lane == 0;
            }
        }
    }
    if (mine) out[j] = token;
    if (c.rank == 0) {
        for (int k = j + 1 + (int)threadIdx.x; k <= a.S; k += (int)blockDim.x) out[k] = -1;
        if (threadIdx.x == 0) a.accepted_out[b] = j;
    }
    cluster_sync();   // (everything shared has been read)
}

// The sequences that verify_kernel left undecided (accepted_out[b] = -2 - row to go on from).  A cluster claims one after the other -- who
// settles a sequence makes no difference to it -- and starts to look for them at its own part of the batch.
constexpr int VF_CLAIMED = -(1 << 30);
template <int TT, int QT>
__global__ void __launch_bounds__(VF_THREADS, 1) verify_settle_kernel(const __grid_constant__ VerifyParams p)
{
    extern __shared__ double kept[];
    __shared__ SettleShared sh;
    fill_table(sh.table);     // (while the kernel before this one ends)
    pdl_enter();
    const VerifyArgs &a = p.a;
    const int clusters = (int)gridDim.x / p.size, own = (int)blockIdx.x / p.size, lane = threadIdx.x & 31;
    const bool chooses = cluster_ctarank() == 0 && threadIdx.x < 32;
    const int64_t start = (int64_t)a.B * own / clusters;
    int64_t looked = 0;
    for (;;) {
        if (chooses) {
            int claim = -1, row = 0;
            while (looked < a.B && claim < 0) {
                const int64_t i = start + looked + lane;
                const int b = (int)(i < a.B ? i : i - a.B);
                const bool there = looked + lane < a.B && !(a.lengths && a.lengths[b] < 0);
                const int mark = there ? *(volatile int32_t *)&a.accepted_out[b] : 0;
                unsigned open = __ballot_sync(0xffffffffu, mark <= -2 && mark > VF_CLAIMED);
                while (open && claim < 0) {
                    const int l = __ffs(open) - 1;
                    open &= open - 1;
                    const bool mine = lane == l && atomicCAS(&a.accepted_out[b], mark, VF_CLAIMED) == mark;
                    if (__any_sync(0xffffffffu, mine)) {
                        claim = __shfl_sync(0xffffffffu, b, l);
                        row = __shfl_sync(0xffffffffu, -2 - mark, l);
                    }
                }
                if (claim < 0) looked += 32;
            }
            if (lane == 0) {
                sh.claim[0] = claim;
                sh.claim[1] = min(row, a.S);
                if (claim >= 0) sh.head = read_head(a, claim);
            }
        }
        cluster_sync();
        const int b = peer_s32(&sh.claim[0], 0), row = peer_s32(&sh.claim[1], 0);
        if (b < 0) break;
        settle_sequence<TT, QT>(p, sh, p.keep ? kept : nullptr, p.size, b, row, peer_head(&sh.head, 0));      // (its barriers lie between this claim's reading and the next one's writing)
    }
    cluster_sync();
}

template <int TT, int QT, int VECS>
__global__ void __launch_bounds__(VF_THREADS, 2) verify_kernel(const __grid_constant__ VerifyParams p)
{
    extern __shared__ double chunk_z[];     // the chunks' sums, then their exponents
    __shared__ VerifyShared sh;
    pdl_enter();
    const VerifyArgs &a = p.a;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, warps = (int)blockDim.x >> 5;
    const int size = p.size;
    const uint32_t rank = size > 1 ? cluster_ctarank() : 0u;
    const int b = (int)blockIdx.x / size;
    if (blockIdx.x == 0 && tid == 0) p.ctl->device_status = CAT_OK;      // (nothing here waits for long)
    if (rank == 0 && tid == 0) sh.head = read_head(a, b);
    if (size > 1) cluster_sync();
    else __syncthreads();
    const Head head = peer_head(&sh.head, 0);
    const int length = head.length;
    if (length < 0) {                       // (all CTAs of the cluster)
        if (size > 1) cluster_sync();       // (all have read the first one's shared memory)
        return;
    }
    const bool greedy = !(head.T > 0.f), decides = warp == warps - 1, drafts = a.draft != nullptr && !greedy;
    // chunks of this CTA: of target rows, of draft rows
    const int c0 = (int)((int64_t)p.chunks_t * rank / size), mine = (int)((int64_t)p.chunks_t * (rank + 1) / size) - c0;
    const int d0 = (int)((int64_t)p.chunks_q * rank / size), mine_q = (int)((int64_t)p.chunks_q * (rank + 1) / size) - d0;
    int *chunk_m = reinterpret_cast<int *>(chunk_z + p.slots);
    auto target_row = [&](int j) { return row_of(a.target, TT, b, j, a.target_seq, a.target_row); };
    auto draft_row = [&](int j) { return row_of(a.draft, QT, b, j, a.draft_seq, a.draft_row); };
    const Scale sc(greedy ? 1.0 : (double)head.T);

    int verdict = sc.fits ? VF_GO_ON : VF_UNDECIDED, j = 0, turn = 0, rows_t = 0, j0 = 0, group = p.group;
    if (tid == 0) sh.owner = sh.open = 0;
    while (verdict == VF_GO_ON) {
        j0 = j;
        turn ^= 1;
        // rows of this round: targets j0 .. j0 + rows_t - 1 (the one behind the last draft among them where the round gets there), then drafts
        rows_t = min(group, length + 1 - j0);
        group = min(2 * group, p.max_group);
        const int pairs = min(rows_t, length - j0), rows = rows_t + (drafts ? pairs : 0);
        const int tasks_t = rows_t * mine, tasks = tasks_t + (rows - rows_t) * mine_q;
        // What the decisions take besides the sums is read by the warp that decides, the last one: it has the fewest chunks.
        if (rank == 0 && decides && lane < pairs) sh.draft[turn][lane] = read_draft(a, b, j0 + lane, TT, QT);
        // a warp's tasks are every warps-th chunk of the rows, one after the other
        int row_at = 0, per = mine, c = warp;
        const void *row = target_row(j0);
#pragma unroll 1
        for (int task = warp; task < tasks; task += warps, c += warps) {
            while (c >= per) {
                c -= per;
                ++row_at;
                per = row_at < rows_t ? mine : mine_q;
                row = row_at < rows_t ? target_row(j0 + row_at) : draft_row(j0 + row_at - rows_t);
            }
            double z;
            int m;
            uint4 v[VECS];
            if (greedy) {
                load_chunk<TT, VECS>(row, c0 + c, a.V, lane, v);
                chunk_top<TT, VECS>(v, (c0 + c) * ((32 * VECS) * Logits<TT>::PER) - row_offset<TT>(row), lane, z, m);
            } else if (TT == QT || row_at < rows_t) {
                load_chunk<TT, VECS>(row, c + (row_at < rows_t ? c0 : d0), a.V, lane, v);
                chunk_stats<TT, VECS>(v, sc, m, z);
            } else {
                load_chunk<QT, VECS>(row, d0 + c, a.V, lane, v);
                chunk_stats<QT, VECS>(v, sc, m, z);
            }
            if (lane == 0) {
                chunk_z[task] = z;
                chunk_m[task] = m;
            }
        }
        __syncthreads();
        // the lanes' (exponent, sum) pairs -- greedy: (place, value) -- joined
        auto join = [&](int &m, double &z) {
            if (greedy) {
                const float top = warp_max((float)z);
                m = __reduce_min_sync(0xffffffffu, (float)z == top ? m : 0x7fffffff);
                z = (double)top;
            } else {
                const int M = __reduce_max_sync(0xffffffffu, m);
                z = warp_sum(scaled(z, m, M));
                m = M;
            }
        };
        const int no_m = greedy ? 0x7fffffff : VF_EMPTY;
        const double no_z = greedy ? -CUDART_INF : 0.0;
        // each row: the CTA's part, then the whole
        double *part_z = size > 1 ? sh.row_z[turn] : sh.total_z;
        int *part_m = size > 1 ? sh.row_m[turn] : sh.total_m;
        for (int r = warp; r < rows; r += warps) {
            const int count = r < rows_t ? mine : mine_q, base = r < rows_t ? r * mine : tasks_t + (r - rows_t) * mine_q;
            double z = no_z;
            int m = no_m;
            for (int c = 0; c < count; c += 32) {
                double oz = c + lane < count ? chunk_z[base + c + lane] : no_z;
                int om = c + lane < count ? chunk_m[base + c + lane] : no_m;
                join(om, oz);
                if (greedy) {
                    if (oz > z) { z = oz; m = om; }      // (chunks in order: the first of equals)
                } else {
                    const int M = max(m, om);
                    z = scaled(z, m, M) + scaled(oz, om, M);
                    m = M;
                }
            }
            if (lane == 0) {
                part_z[r] = z;
                part_m[r] = m;
            }
        }
        if (size > 1) {
            cluster_sync();
            for (int r = warp; r < rows; r += warps) {
                double z = lane < size ? peer_f64(&sh.row_z[turn][r], (uint32_t)lane) : no_z;
                int m = lane < size ? peer_s32(&sh.row_m[turn][r], (uint32_t)lane) : no_m;
                join(m, z);
                if (lane == 0) {
                    sh.total_z[r] = z;
                    sh.total_m[r] = m;
                }
            }
        }
        __syncthreads();
        if (decides) {
            // lane i: draft j0 + i; every CTA of the cluster decides the same from the same numbers
            int how = VF_ALL_STAND, x = -1;      // (nothing left to decide)
            if (lane < pairs) {
                const Draft d = peer_draft(&sh.draft[turn][lane], 0);
                const float ua = d.u, xt = d.xt, xq = d.xq;
                x = d.x;
                const double zt = sh.total_z[lane];
                const int mt = sh.total_m[lane];
                if (greedy) {
                    how = zt > -CUDART_INF && x == mt ? VF_GO_ON : VF_REFUSED;
                } else {
                    bool clear = mt < VF_WILD;
                    double zq = 1;
                    int mq = 0;
                    if (drafts && sh.total_m[rows_t + lane] > VF_EMPTY) {
                        zq = sh.total_z[rows_t + lane];
                        mq = sh.total_m[rows_t + lane];
                        clear = clear && mq < VF_WILD;
                    }
                    float w[2], none;
                    const Weights wt(sc, clear ? mt : 0), wq(sc, clear ? mq : 0);
                    wt(sc, xt, xt, w[0], none);
                    wq(sc, xq, xq, w[1], none);
                    if (xt == -CUDART_INF_F) w[0] = 0.f;
                    if (xq == -CUDART_INF_F) w[1] = 0.f;
                    if (!drafts) w[1] = x >= 0 && x < a.V ? 1.f : 0.f;
                    // u q < p, both sides times both normalisers
                    const double u = uniform(ua), left = u * (double)w[1] * zt, right = (double)w[0] * zq;
                    if (!clear) {
                        how = VF_UNDECIDED;
                    } else if (w[0] == 0.f) {
                        how = VF_REFUSED;
                    } else if (w[0] < 1e-27f || (w[1] > 0.f && w[1] < 1e-27f)) {
                        // entries far below their rows' largest, where weights have a floor: by their exponents
                        const bool has_q = w[1] > 0.f;
                        const double et = (double)xt * sc.c - (double)mt, eq = drafts && has_q ? (double)xq * sc.c - (double)mq : 0.0;
                        const double by = et + (double)log2f((float)zq) - eq - (double)log2f((float)(u * zt));
                        // (what is below 2^-1000 of its row's largest has no mass; the exponents here are relative to that rounded)
                        if (fabs(et + 1000.0) < 1.0 || fabs(eq + 1000.0) < 1.0) how = VF_UNDECIDED;
                        else if (et < -1000.0) how = VF_REFUSED;
                        else if (!has_q || eq < -1000.0) how = VF_GO_ON;
                        else how = !(fabs(by) > 1e-3) ? VF_UNDECIDED : by > 0 ? VF_GO_ON : VF_REFUSED;
                    } else {
                        how = fabs(left - right) < 2.0 * VF_EPS_P * (left + right) ? VF_UNDECIDED : left < right ? VF_GO_ON : VF_REFUSED;
                    }
                }
            }
            const unsigned stops = __ballot_sync(0xffffffffu, how != VF_GO_ON);    // (lane `pairs` says that there is nothing left)
            const int first = __ffs(stops) - 1;
            how = __shfl_sync(0xffffffffu, how, first);
            if (first == pairs) how = rows_t > pairs ? VF_ALL_STAND : VF_GO_ON;
            if (rank == 0 && lane < first) a.tokens_out[(int64_t)b * (a.S + 1) + j0 + lane] = x;
            x = __shfl_sync(0xffffffffu, x, first);
            if (lane == 0) {
                sh.verdict = how;
                sh.at = j0 + first;
                sh.x = x;
                if (how == VF_REFUSED || how == VF_ALL_STAND) {
                    const int mt = sh.total_m[first];
                    if (greedy || mt <= VF_EMPTY) {
                        sh.source = VF_FROM_NOTHING;
                        sh.token = greedy && sh.total_z[first] > -CUDART_INF ? mt : -1;      // (no mass: no token)
                    } else if (mt >= VF_WILD) {
                        sh.verdict = VF_UNDECIDED;
                    } else if (how == VF_REFUSED && !drafts) {
                        sh.source = VF_FROM_OTHERS;
                    } else {
                        sh.source = how == VF_REFUSED && sh.total_m[rows_t + first] > VF_EMPTY ? VF_FROM_DIFFERENCE : VF_FROM_ROW;
                    }
                }
            }
        }
        __syncthreads();
        verdict = sh.verdict;
        j = sh.at;
    }

    // the token behind the accepted drafts
    int32_t *out = a.tokens_out + (int64_t)b * (a.S + 1);
    if (verdict != VF_UNDECIDED) {
        const int source = sh.source;
        if (source == VF_FROM_NOTHING) {
            if (rank == 0 && tid == 0) {
                out[j] = sh.token;
                a.accepted_out[b] = j;
            }
        } else {
            const int r = j - j0, mt = sh.total_m[r];
            const double zt = sh.total_z[r];
            Source src{target_row(j), nullptr, 1.f, 1.f, mt, 0, -1};
            int slot = r;                                   // where the masses of the CTAs and of the chunks are
            double err = 1.01 * 2.0 * VF_EPS_SUM * zt;
            const bool residual = source != VF_FROM_ROW;
            if (residual) {
                // from what the refused draft's row leaves of it: both rows once more.  (Of the row itself the chunks' sums are known.)
                src.t_scale = 1.f / (float)zt;
                if (source == VF_FROM_DIFFERENCE) {
                    src.q_row = draft_row(j);
                    src.q_m = sh.total_m[rows_t + r];
                    src.q_scale = 1.f / (float)sh.total_z[rows_t + r];
                } else {
                    src.point = sh.x;
                }
            }
            const Weights wt(sc, src.t_m), wq(sc, src.q_m);
            if (residual) {
                __syncthreads();            // (the chunks' sums have been read)
#pragma unroll 1
                for (int c = warp; c < mine; c += warps) {
                    float sum[VECS];
                    chunk_masses<TT, QT, VECS>(src, sc, wt, wq, c0 + c, a.V, lane, sum);
                    const double z = warp_sum(lane_sum(sum));
                    if (lane == 0) {
                        chunk_z[c] = z;
                        chunk_m[c] = mt;
                    }
                }
                __syncthreads();
                turn ^= 1;
                slot = 0;
                if (warp == 0) {
                    double z = 0;
                    for (int c = lane; c < mine; c += 32) z += chunk_z[c];
                    z = warp_sum(z);
                    if (lane == 0) {
                        sh.row_z[turn][0] = z;
                        sh.row_m[turn][0] = mt;
                    }
                }
                if (size > 1) cluster_sync();
            }
            if (warp == 0) {
                // the CTA, the chunk, the entry at which the sum passes u times the whole
                double v;
                if (size > 1) v = lane < size ? scaled(peer_f64(&sh.row_z[turn][slot], (uint32_t)lane), peer_s32(&sh.row_m[turn][slot], (uint32_t)lane), mt) : 0.0;
                else v = lane == 0 ? (residual ? sh.row_z[turn][0] : zt) : 0.0;
                double run = warp_scan(v, lane);
                const double total = __shfl_sync(0xffffffffu, run, 31), goal = uniform(head.u_sample) * total;
                // sums of p - q: p and q are off by VF_EPS_P of themselves, and the sums round
                if (residual) err = 1.01 * 2.0 * (2.0 * VF_EPS_P + 5.0 * VF_U * total);
                unsigned over = __ballot_sync(0xffffffffu, run > goal);
                if (!(total > 2.0 * err)) over = 0;
                const int owner = over ? __ffs(over) - 1 : 0;
                double below = __shfl_sync(0xffffffffu, run - v, owner);
                if (owner == (int)rank) {
                    int token = -1, chunk = -1;
#pragma unroll 1
                    for (int base = 0; over && base < mine && chunk < 0; base += 32) {
                        const int c = base + lane;
                        v = c < mine ? scaled(chunk_z[slot * mine + c], chunk_m[slot * mine + c], mt) : 0.0;
                        run = warp_scan(v, lane);
                        const unsigned here = __ballot_sync(0xffffffffu, below + run > goal);
                        const int l = here ? __ffs(here) - 1 : 31;
                        below += __shfl_sync(0xffffffffu, here ? run - v : run, l);
                        if (here) chunk = base + l;
                    }
                    if (chunk >= 0) token = find_in_chunk<TT, QT, VECS>(src, sc, wt, wq, c0 + chunk, a.V, below, goal, err, lane);
                    if (lane == 0) {
                        sh.open = token < 0;
                        out[j] = token;
                        a.accepted_out[b] = token < 0 ? -2 - j : j;       // (or the mark of a sequence that is not decided)
                    }
                }
                if (lane == 0) sh.owner = owner;
            }
        }
    }
    if (verdict == VF_UNDECIDED && rank == 0 && tid == 0) a.accepted_out[b] = -2 - j;
    if (rank == 0)
        for (int k = j + 1 + tid; k <= a.S; k += (int)blockDim.x) out[k] = -1;
    if (size > 1) cluster_sync();   // no CTA's shared memory goes away under another
    else __syncthreads();
    if (p.settle) {
        const bool open = verdict == VF_UNDECIDED || peer_s32(&sh.open, (uint32_t)sh.owner) != 0;
        if (size > 1) cluster_sync();
        if (open) {
            fill_table(sh.settle.table);
            __syncthreads();
            settle_sequence<TT, QT>(p, sh.settle, p.keep ? chunk_z : nullptr, size, b, j, head);
        }
    }
}

// The limit of a kernel's dynamic shared memory is the kernel's, not the call's: every call sets the same, or one from another thread could find a
// smaller one than it needs.
constexpr int VF_MAX_SMEM = 200 * 1024;

template <int TT, int QT>
cudaError_t launch_fast(const VerifyParams &p, cudaLaunchConfig_t &cfg)
{
    auto kern = p.vecs == 4 ? verify_kernel<TT, QT, 4> : verify_kernel<TT, QT, 1>;
    cudaError_t e;
    if (cfg.dynamicSmemBytes > 40 * 1024 && (e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, VF_MAX_SMEM)) != cudaSuccess)
        return e;
    return cudaLaunchKernelEx(&cfg, kern, p);
}

template <int TT, int QT>
cudaError_t launch_settle(const VerifyParams &p, cudaLaunchConfig_t &cfg)
{
    cudaError_t e;
    if ((e = cudaFuncSetAttribute(verify_settle_kernel<TT, QT>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1)) != cudaSuccess) return e;
    if ((e = cudaFuncSetAttribute(verify_settle_kernel<TT, QT>, cudaFuncAttributeMaxDynamicSharedMemorySize, VF_MAX_SMEM)) != cudaSuccess) return e;
    return cudaLaunchKernelEx(&cfg, verify_settle_kernel<TT, QT>, p);
}

}  // namespace

cudaError_t launch_verify(const VerifyArgs &a, void *workspace, cudaStream_t s)
{
    VerifyParams p{};
    p.a = a;
    p.ctl = reinterpret_cast<Control *>(workspace);
    const int draft_type = a.draft ? a.draft_type : a.target_type;
    const int sms = tc_sm_count();
    const int64_t entries = a.V;
    // CTAs per sequence: two resident on every SM, each with something to read
    p.size = 1;
    while (p.size < 8 && (int64_t)a.B * p.size <= sms && entries >= 1024 * p.size) p.size *= 2;
    while (p.size < 8 && entries > (int64_t)(1 << 19) * p.size) p.size *= 2;
    // One granule per lane and chunk where no SM has a second CTA to hide a long chunk's latency behind (8 sequences, 4 drafts, V = 32 000: 16 us
    // against 19); four, with a quarter of the sums over the warp, where it has (64 sequences, 7 drafts, V = 128 000: 107 us against 164).
    p.vecs = (int64_t)a.B * p.size <= sms ? 1 : 4;
    auto chunks = [&](int type) {
        const int per = type == CAT_F32 ? 4 : 8, chunk = 32 * p.vecs * per;
        return (a.V + per - 1 + chunk - 1) / chunk;
    };
    p.chunks_t = chunks(a.target_type);
    p.chunks_q = chunks(draft_type);
    const int per_t = (p.chunks_t + p.size - 1) / p.size, per_q = a.draft ? (p.chunks_q + p.size - 1) / p.size : 0;
    // Target rows before the first exchange: about 40 MB of rows over the batch take as long to read as the exchange does.
    const int64_t pair_bytes = (int64_t)a.B * a.V * ((a.target_type == CAT_F32 ? 4 : 2) + (a.draft ? (draft_type == CAT_F32 ? 4 : 2) : 0));
    p.max_group = VF_MAX_GROUP;
    while (p.max_group > 1 && p.max_group * (per_t + per_q) * 12 > 40 * 1024) p.max_group /= 2;
    if (p.max_group > a.S + 1) p.max_group = a.S + 1;
    p.group = (int)((((int64_t)40 << 20) + pair_bytes - 1) / pair_bytes);
    if (p.group > p.max_group) p.group = p.max_group;
    p.slots = p.max_group * (per_t + per_q);
    // An undecided sequence is settled by the CTAs that have it where every thread has sixteen entries of a row at most; else by a cluster of 16 in a
    // launch of its own (64 sequences, V = 128 000: 107 us against 143; 256 sequences, V = 50 001: 32 us against 61).
    p.settle = entries <= (int64_t)16 * VF_THREADS * p.size;
    // (the weights of two rows in fp64: where a CTA has an SM to itself, or they are small)
    auto kept_bytes = [&](int size) { return ((entries + 6) / 4 / size + 1) * 64; };
    size_t smem = (size_t)p.slots * 12;
    p.keep = p.settle && (kept_bytes(p.size) <= 16 * 1024 || ((int64_t)a.B * p.size <= sms && kept_bytes(p.size) <= VF_MAX_SMEM));
    if (p.keep && smem < (size_t)kept_bytes(p.size)) smem = (size_t)kept_bytes(p.size);

    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(a.B * p.size), 1, 1);
    cfg.blockDim = dim3(VF_THREADS, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)p.size;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;   // (the kernels start with pdl_enter)
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    using Launch = cudaError_t (*)(const VerifyParams &, cudaLaunchConfig_t &);
#define CAT_VERIFY_FORMS(F) \
    {{F<CAT_F32, CAT_F32>, F<CAT_F32, CAT_BF16>, F<CAT_F32, CAT_F16>}, {F<CAT_BF16, CAT_F32>, F<CAT_BF16, CAT_BF16>, F<CAT_BF16, CAT_F16>}, \
     {F<CAT_F16, CAT_F32>, F<CAT_F16, CAT_BF16>, F<CAT_F16, CAT_F16>}}
    static const Launch fast[3][3] = CAT_VERIFY_FORMS(launch_fast), settle[3][3] = CAT_VERIFY_FORMS(launch_settle);
#undef CAT_VERIFY_FORMS
    cudaError_t e = fast[a.target_type][draft_type](p, cfg);
    count_launch();
    if (e != cudaSuccess || p.settle) return e;

    p.size = VF_SETTLE_CLUSTER;
    p.keep = kept_bytes(p.size) <= VF_MAX_SMEM;
    const int clusters = a.B < sms / p.size ? a.B : sms / p.size;
    cfg.gridDim = dim3((unsigned)(clusters * p.size), 1, 1);
    cfg.blockDim = dim3(VF_THREADS, 1, 1);
    cfg.dynamicSmemBytes = p.keep ? (size_t)kept_bytes(p.size) : 0;
    attr[0].val.clusterDim.x = (unsigned)p.size;
    e = settle[a.target_type][draft_type](p, cfg);
    count_launch();
    return e;
}

}  // namespace cat
