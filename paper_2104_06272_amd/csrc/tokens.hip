// Operators of token policies on rows of logits: log-probabilities and their backward pass, the clipped policy loss, and
// the loss over pairs of sequences.  The mathematics of a row stands in tokens.h, that of the losses at policy_row and
// pair_sums.  Three things are done with a row -- its sums, its gradient from given coefficients, and both with the clipped
// loss between them -- and each comes in three forms by the length of a row:
//   lanes_rows short rows: 1 to 32 lanes hold a row in registers, 64 / lanes rows to a wavefront
//   block_sums, block_gradients   a workgroup streams a row
//   block_policy                  a workgroup holds a row in registers between its sums and its gradient
// and   weight_sums   partial sums of the rows' (pairs') weights
//       pair_sums     the pairs: summed log ratios, coefficients of their rows
//       fold_stats, finish_stats  add the workgroups' sums in a fixed order
#include <math.h>
#include "tokens.h"

namespace ank {

struct Partial { double v[STATS]; };

// ---- sums in a fixed order ---------------------------------------------------------------------------------------
__device__ __forceinline__ double wave_sum(double v)
{
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
    return v;
}
__device__ __forceinline__ double block_sum(double v, double* lds)      // every thread gets it
{
    v = wave_sum(v);
    const int waves = blockDim.x >> 6;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    double s = 0.0;
    for (int w = 0; w < waves; ++w) s += lds[w];
    return s;
}
// Eight sums at once: in three steps every lane gives half of what it holds to its partner and adds what it is given, in three
// more the lanes of one sum join.  The lane's sum is number stat_of(lane).
__device__ __forceinline__ int stat_of(int lane) { return ((lane >> 5) & 1) * 4 + ((lane >> 4) & 1) * 2 + ((lane >> 3) & 1); }
__device__ __forceinline__ double wave_stats(const double (&v)[STATS])
{
    const int lane = threadIdx.x & 63;
    double w[4], x[2];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = (lane & 32 ? v[4 + i] : v[i]) + __shfl_xor(lane & 32 ? v[i] : v[4 + i], 32, 64);
#pragma unroll
    for (int i = 0; i < 2; ++i) x[i] = (lane & 16 ? w[2 + i] : w[i]) + __shfl_xor(lane & 16 ? w[i] : w[2 + i], 16, 64);
    double y = (lane & 8 ? x[1] : x[0]) + __shfl_xor(lane & 8 ? x[0] : x[1], 8, 64);
    for (int off = 4; off > 0; off >>= 1) y += __shfl_xor(y, off, 64);
    return y;
}
// the workgroup's eight sums in `out` (LDS): y is this lane's share of sum k, and lanes `first` speak for theirs
__device__ __forceinline__ void block_stats(double y, int k, bool first, double (*lds)[STATS], double (&out)[STATS])
{
    const int waves = blockDim.x >> 6;
    __syncthreads();
    if (first) lds[threadIdx.x >> 6][k] = y;
    __syncthreads();
    if (threadIdx.x < STATS) {
        double s = 0.0;
        for (int w = 0; w < waves; ++w) s += lds[w][threadIdx.x];
        out[threadIdx.x] = s;
    }
    __syncthreads();
}

// What a mean is taken over: the given norm, or the sum of the weights -- of parts that weight_sums left, or of the rows
// themselves where they are few enough for every workgroup to add them up beside its first loads (a launch less).
struct Norm { double norm; const double* parts; int n_parts; const float* weight; int inline_rows; };
constexpr int INLINE_ROWS = 2048;                // (20480 x 3, 16 targets of 8 bits at a time: 15.5 us in a graph, 10.6 with weight_sums)
__device__ __forceinline__ double weight_of(const Rows& r, const float* weight, int64_t n) { return row_target(r, n) < 0 ? 0.0 : weight ? (double)weight[n] : 1.0; }
// of the rows themselves, 2 to 4 targets at a time (2048 x 700 fp32, a wavefront each: 17.6 us in a graph, one at a time 20.6)
template <class I>
__device__ __forceinline__ double weights_of(const Rows& r, const Norm& w, int thread, int threads)
{
    constexpr int N = sizeof(I) == 8 ? 2 : 4;
    typedef I targets __attribute__((ext_vector_type(N), aligned(sizeof(I))));
    const I* target = static_cast<const I*>(r.target);
    const int V = r.V, whole = w.inline_rows - w.inline_rows % N;
    double s = 0.0;
    int count = 0;
#pragma unroll 4
    for (int i = thread * N; i < whole; i += threads * N) {
        const targets t = *reinterpret_cast<const targets*>(target + i);
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (t[k] >= 0 && t[k] < V) { if (w.weight) s += (double)w.weight[i + k]; else count += 1; }
    }
    if (whole + thread < w.inline_rows) s += weight_of(r, w.weight, whole + thread);
    return s + count;
}
// the share of it that this thread of `threads` adds up; the sum over all threads is W
__device__ __forceinline__ double weight_share(const Norm& w, const Rows& r, int thread, int threads)
{
    if (w.norm != 0.0) return thread == 0 ? w.norm : 0.0;
    double s = 0.0;
    for (int i = thread; i < w.n_parts; i += threads) s += w.parts[i];
    if (w.inline_rows == 0) return s;
    if (r.target_type == ANAKIN_INDEX_U8) return weights_of<uint8_t>(r, w, thread, threads);
    return r.target_type == ANAKIN_INDEX_I32 ? weights_of<int32_t>(r, w, thread, threads) : weights_of<int64_t>(r, w, thread, threads);
}

// partial sums of the weights of the rows (target in range) or pairs that take part
__global__ __launch_bounds__(WG) void weight_sums(const Rows r, const int64_t n, const float* weight, const bool pairs, double* parts)
{
    __shared__ double lds[WG / 64];
    double s = 0.0;
#pragma unroll 4
    for (int64_t i = (int64_t)blockIdx.x * WG + threadIdx.x; i < n; i += (int64_t)gridDim.x * WG)
        s += pairs ? (double)weight[i] : weight_of(r, weight, i);
    s = block_sum(s, lds);
    if (threadIdx.x == 0) parts[blockIdx.x] = s;
}

// means over W of the summed statistics; slot 0 becomes the loss
struct FinishArgs { const Partial* parts; int n_parts; Rows r; Norm norm; float* stats; double kl, ent; int policy; };
struct FinishLds { double waves[16][STATS], sums[STATS], weights[16]; };
__device__ __forceinline__ void finish(const FinishArgs& a, FinishLds& lds)
{
    // lane l adds sum l % 8 of partials l / 8, l / 8 + threads / 8, ...: whole cache lines
    const int k = threadIdx.x & 7;
    double y = 0.0;
#pragma unroll 4
    for (int i = threadIdx.x >> 3; i < a.n_parts; i += blockDim.x >> 3) y += a.parts[i].v[k];
    for (int off = 8; off < 64; off <<= 1) y += __shfl_xor(y, off, 64);
    const double share = weight_share(a.norm, a.r, threadIdx.x, blockDim.x);
    block_stats(y, k, (threadIdx.x & 63) < STATS, lds.waves, lds.sums);
    const double W = block_sum(share, lds.weights), inv = W != 0.0 ? reciprocal(W) : 0.0;
    if (threadIdx.x >= STATS) return;
    const double* v = lds.sums;
    double m = W != 0.0 ? v[k] * inv : 0.0;
    if (a.policy) {
        if (k == 0) m = W != 0.0 ? (v[1] + (a.kl != 0.0 ? a.kl * v[2] : 0.0) - (a.ent != 0.0 ? a.ent * v[3] : 0.0)) * inv : 0.0;
        if (k == 6) m = W;
    } else {                                                            // loss, [h > 0], first, second, h, W (broken pairs), pairs, tokens
        if (k == 0 && v[5] != 0.0) m = (double)NAN;
        if (k == 5) m = W;
        if (k == 6) m = v[6];
    }
    if (k == 7) m = v[7];
    a.stats[k] = (float)m;
}
// many partial sums (one of every long row): FOLDED workgroups make as many of them
constexpr int FOLDED = 64, FOLD_FROM = 512;
__global__ __launch_bounds__(WG) void fold_stats(const Partial* parts, const int n, Partial* out)
{
    __shared__ FinishLds lds;
    const int k = threadIdx.x & 7;
    double y = 0.0;
#pragma unroll 4
    for (int i = blockIdx.x * (WG / 8) + (threadIdx.x >> 3); i < n; i += FOLDED * (WG / 8)) y += parts[i].v[k];
    for (int off = 8; off < 64; off <<= 1) y += __shfl_xor(y, off, 64);
    block_stats(y, k, (threadIdx.x & 63) < STATS, lds.waves, lds.sums);
    if (threadIdx.x < STATS) out[blockIdx.x].v[k] = lds.sums[k];
}
constexpr int FINISH_WG = 512;
__global__ __launch_bounds__(FINISH_WG) void finish_stats(const FinishArgs a)
{
    __shared__ FinishLds lds;
    finish(a, lds);
}

// ---- what becomes of a row's sums -----------------------------------------------------------------------------------
// what the first pass over pairs leaves of a row for the second
struct RowWs { double lp; Shift k; float inv_s; int target; };

struct SumArgs {
    Rows r;
    float *logp, *lse, *entropy;                 // each may be null
    RowWs* ws;                                   // may be null
    float* coef;                                 // may be null: set to 0 (pair_sums fills in the rows of its sequences)
};
template <bool FINE>
__device__ __forceinline__ void store_sums(const SumArgs& a, int64_t n, const Sums& p, int target, float chosen)
{
    RowSum x{};
    double lp = 0.0;
    if (target >= 0) { x = finish_row<FINE>(p, a.r); lp = logp_of<FINE>(x, chosen, a.r); }
    if (a.logp) a.logp[n] = (float)lp;
    if (a.lse) a.lse[n] = (float)x.lse;
    if (a.entropy) a.entropy[n] = (float)x.entropy;
    if (a.ws) a.ws[n] = RowWs{lp, x.k, x.empty ? 0.0f : x.inv_s, target};
    if (a.coef) a.coef[n] = 0.0f;
}

struct GradArgs {
    Rows r;
    void* out; int64_t out_stride;
    const RowWs* ws;                             // of the first pass; null: from the caller's lse
    const float *lse, *entropy, *to_logp, *to_entropy;   // the caller's (to_entropy may be null); to_logp also with ws
    FinishArgs fin;                              // stats not null: a workgroup more finishes the statistics
    int shares;                                  // long rows: workgroups to a row
};
// from the row's numbers (all but its entropy) and the caller's coefficients
__device__ __forceinline__ RowGrad row_gradient_to(const GradArgs& a, int64_t n, RowSum x, int target)
{
    const double e = a.to_entropy ? a.to_entropy[n] : 0.0;
    x.entropy = e != 0.0 ? (double)a.entropy[n] : 0.0;
    return row_gradient(x, a.to_logp[n], e, target, a.r.scale);
}
__device__ __forceinline__ RowGrad grad_of_row(const GradArgs& a, int64_t n)
{
    RowSum x{};
    if (a.ws) {
        // (a coefficient of 0 -- a row in no pair, or of a pair of weight 0 -- is a row without a target: its logits, which may
        // be anything, are not read)
        const RowWs w = a.ws[n];
        const float g = a.to_logp[n];
        if (w.target < 0 || g == 0.0f) { RowGrad q{}; q.target = -1; return q; }
        x.k = w.k; x.inv_s = w.inv_s;
        x.empty = w.inv_s == 0.0f;                                      // (all of it minus infinity)
        return row_gradient(x, g, 0.0, w.target, a.r.scale);
    }
    const int target = row_target(a.r, n);
    if (target < 0) { RowGrad q{}; q.target = -1; return q; }
    // p_j = 2^(c z - K) / s with K = fl(lse log2 e) and the rest of lse in s
    const double k = (double)a.lse[n] * LOG2E;
    x.k = Shift{a.r.c, (float)k};
    x.log_s = (k - (double)x.k.K) * LN2;
    x.inv_s = (float)exp_of(-x.log_s);
    return row_gradient_to(a, n, x, target);
}
// A log-sum-exp in binary32 is off by up to 2^-15 below LSE_MOST, and so is p of itself.  What lies beyond, up to rows of a type's
// lowest value, whose log-sum-exp has no room for the logarithm of their length or overflows, takes p from the row's own sums.
constexpr float LSE_MOST = 1024.0f;
__device__ __forceinline__ bool by_own_sums(const GradArgs& a, int64_t n)
{
    return !a.ws && fabsf(a.lse[n]) >= LSE_MOST && row_target(a.r, n) >= 0;
}

// ---------------------------------------------------------------------------
// The clipped loss of one row.  Which side of a clipping border a ratio lies on hangs on lp, so the difference of the
// log-probabilities is compared with the borders' logarithms in 64 bits.
//   dL/dlp = w (-A r [r A <= clipped A] + kl_coef (1 - e^d)),  dL/dH = -entropy_coef w    (both without 1 / W)
// ---------------------------------------------------------------------------
struct PolicyCfg {
    const float *old, *adv, *ref, *weight;
    double log_low, log_high;                    // ln(1 - clip_low), ln(1 + clip_high)
    double low, high, kl, ent, grad_scale;       // low = 1 - clip_low, high = 1 + clip_high
};
struct PolicyIn { float old, adv, ref, w; };      // what a row's loss reads, asked for before its logits
__device__ __forceinline__ PolicyIn policy_in(const PolicyCfg& a, int64_t n)
{
    return PolicyIn{a.old[n], a.adv[n], a.ref ? a.ref[n] : 0.0f, a.weight ? a.weight[n] : 1.0f};
}
struct PolicyRow { double g, e, policy, kl, entropy, clipped, ratio, w; };
__device__ __forceinline__ PolicyRow policy_row(const PolicyCfg& a, const PolicyIn& in, double lp, double entropy, bool empty)
{
    PolicyRow x{};
    x.w = (double)in.w;
    if (empty) return x;
    const double A = in.adv, diff = lp - (double)in.old, r = exp_of(diff);
    const bool clipped = (A > 0.0 && diff > a.log_high) || (A < 0.0 && diff < a.log_low);      // (a NaN stays in the gradient)
    x.policy = clipped ? -(A > 0.0 ? a.high : a.low) * A : -r * A;
    x.clipped = clipped ? 1.0 : 0.0; x.ratio = r; x.entropy = entropy;
    x.g = clipped ? 0.0 : -r * A;
    if (a.ref) {
        // e^d - 1 and e^d - 1 - d: their series where they would cancel
        const double d = (double)in.ref - lp;
        double e1, e2;
        if (fabs(d) < 0.5) {
            double p = 1.0 / 39916800;
            p = fma(p, d, 1.0 / 3628800); p = fma(p, d, 1.0 / 362880); p = fma(p, d, 1.0 / 40320); p = fma(p, d, 1.0 / 5040);
            p = fma(p, d, 1.0 / 720); p = fma(p, d, 1.0 / 120); p = fma(p, d, 1.0 / 24); p = fma(p, d, 1.0 / 6); p = fma(p, d, 0.5);
            e2 = p * d * d; e1 = e2 + d;
        } else { e1 = exp_of(d) - 1.0; e2 = e1 - d; }
        x.kl = e2;
        if (a.kl != 0.0) x.g -= a.kl * e1;
    }
    x.g *= x.w; x.e = -a.ent * x.w;
    return x;
}
__device__ __forceinline__ void add_stats(double (&v)[STATS], const PolicyRow& x)
{
    v[1] += x.w * x.policy; v[2] += x.w * x.kl; v[3] += x.w * x.entropy; v[4] += x.w * x.clipped; v[5] += x.w * x.ratio; v[6] += x.w; v[7] += 1.0;
}
struct PolicyArgs {
    Rows r;
    PolicyCfg p;
    Norm norm;
    float* logp;                                 // may be null
    void* out; int64_t out_stride;               // out null: the loss alone
    Partial* parts;
};
__device__ __forceinline__ int policy_target(const PolicyArgs& a, int64_t n)
{
    const int t = row_target(a.r, n);
    return a.p.weight && a.p.weight[n] == 0.0f ? -1 : t;
}

// ---------------------------------------------------------------------------
// Short rows.  `lanes` lanes (a power of two up to 32) hold a row: PIECES of 16 bytes each, piece k lanes + l at lane l, and a
// loose element (8 lanes: pieces from column 0 on, which leaves no more than 7 loose); or (PIECES 0) four single elements, element
// k of lane l in column k lanes + l.  Everything of a row happens in registers; all its lanes carry out the row's 64-bit
// arithmetic together, so that a row should have few of them.
// ---------------------------------------------------------------------------
enum { DO_SUMS, DO_GRADIENT, DO_POLICY };
template <int DO> struct LaneArgs;
template <> struct LaneArgs<DO_SUMS> { SumArgs s; int lanes; __device__ const Rows& rows() const { return s.r; } };
template <> struct LaneArgs<DO_GRADIENT> { GradArgs g; int lanes; __device__ const Rows& rows() const { return g.r; } };
template <> struct LaneArgs<DO_POLICY> { PolicyArgs p; int lanes; __device__ const Rows& rows() const { return p.r; } };

// what a lane holds of a row: `slots` of its P groups of W elements are in use (the same in all of a wavefront, which passes over
// the others), and VECTOR a loose element
template <class E, int PIECES>
struct LaneRow {
    typedef typename E::T T;
    static constexpr bool VECTOR = PIECES > 0;
    static constexpr int P = VECTOR ? PIECES : 1, W = VECTOR ? E::N : 4;
    float z[P][W], loose[1];

    static __device__ __forceinline__ int slots(int V, int lanes) { return VECTOR ? (V / W + lanes - 1) / lanes : 1; }
    __device__ __forceinline__ void load(const T* row, const Cut& cut, int V, int lanes, int l, int slots)
    {
        loose[0] = -INFINITY;
        if constexpr (VECTOR && W == 8) {
            // all loads before the first use: a million rows of 256 bf16, sums 169 -> 140 us (fp32 as below: 116, so 168)
            u32x4_any w[P];
#pragma unroll
            for (int k = 0; k < P; ++k) if (k * lanes + l < cut.pieces) w[k] = *reinterpret_cast<const u32x4_any*>(row + cut.head + (k * lanes + l) * W);
#pragma unroll
            for (int k = 0; k < P; ++k) {
                if (k >= slots) continue;
                E::unpack(w[k], z[k]);
                if (k == slots - 1 && k * lanes + l >= cut.pieces)
#pragma unroll
                    for (int i = 0; i < W; ++i) z[k][i] = -INFINITY;
            }
        } else if constexpr (VECTOR) {
#pragma unroll
            for (int k = 0; k < P; ++k) {
                const int v = k * lanes + l;
                if (k < slots && v < cut.pieces) E::unpack(*reinterpret_cast<const u32x4_any*>(row + cut.head + v * W), z[k]);
                else {
#pragma unroll
                    for (int i = 0; i < W; ++i) z[k][i] = -INFINITY;
                }
            }
        }
        if constexpr (VECTOR) {
            if (l < cut.loose) loose[0] = E::get(row + loose_column<E>(cut, l));
        } else {
#pragma unroll
            for (int k = 0; k < W; ++k) { const int j = k * lanes + l; z[0][k] = j < V ? E::get(row + j) : -INFINITY; }
        }
    }
    template <bool FINE>
    __device__ __forceinline__ Sums sums(const Rows& r, int lanes, int slots) const
    {
        float m = loose[0];
#pragma unroll
        for (int k = 0; k < P; ++k) if (k < slots) m = max_of(z[k], m);
        for (int off = 1; off < lanes; off <<= 1) m = fmaxf(m, __shfl_xor(m, off, 64));
        Part p{m, 0.0f, 0.0f};
        const Shift s = shift_of(m, r.c);
        const float m0 = m == -INFINITY ? 0.0f : m;
#pragma unroll
        for (int k = 0; k < P; ++k) if (k < slots) add_at<FINE>(p, z[k], m0, s, r.c, r.c_lo);
        if constexpr (VECTOR) add_at<FINE>(p, loose, m0, s, r.c, r.c_lo);
        if (FINE) {
            double d = fma(LN2, (double)p.u, (double)p.s);
            for (int off = 1; off < lanes; off <<= 1) d += __shfl_xor(d, off, 64);
            return Sums{m, d, 0.0};
        }
        for (int off = 1; off < lanes; off <<= 1) { p.s += __shfl_xor(p.s, off, 64); p.u += __shfl_xor(p.u, off, 64); }
        return Sums{m, (double)p.s, (double)p.u};
    }
    // the row's gradient to `out` (of a row without a target z is all zeros, as are the coefficients)
    template <bool ALL>                                                 // all of it before the first store (more registers)
    __device__ __forceinline__ void put_gradient(const RowGrad& q, T* out, const Cut& cut, int V, int lanes, int l, int slots) const
    {
        if constexpr (VECTOR) {
            const int tp = q.target - cut.head, tv = tp >= 0 ? tp / W : -1, ti = tp % W;
            float d[ALL ? P : 1][W];
#pragma unroll
            for (int k = 0; k < P; ++k) {
                if (k >= slots) continue;
                float (&dk)[W] = d[ALL ? k : 0];
                const int v = k * lanes + l;
                gradient_of<true>(q, z[k], dk);
#pragma unroll
                for (int i = 0; i < W; ++i) dk[i] += (ALL ? v * W + i == tp : v == tv && i == ti) ? q.to_target : 0.0f;
                if (!ALL && v < cut.pieces) *reinterpret_cast<u32x4_any*>(out + cut.head + v * W) = E::pack(dk);
            }
            if (ALL)
#pragma unroll
                for (int k = 0; k < P; ++k) if (k * lanes + l < cut.pieces) *reinterpret_cast<u32x4_any*>(out + cut.head + (k * lanes + l) * W) = E::pack(d[k]);
            if (l < cut.loose) {
                const int j = loose_column<E>(cut, l);
                float d[1];
                gradient_of<true>(q, loose, d);
                E::put(out + j, d[0] + (j == q.target ? q.to_target : 0.0f));
            }
        } else {
            float d[W];
            gradient_of<true>(q, z[0], d);
#pragma unroll
            for (int k = 0; k < W; ++k) { const int j = k * lanes + l; if (j < V) E::put(out + j, d[k] + (j == q.target ? q.to_target : 0.0f)); }
        }
    }
};

// The gradient of a row of by_own_sums, element by element, after the others.  (Beside them, with the row in registers, they would
// pay for it in registers of their own: a million rows of 256 bf16 260 us, not 215.)
template <class E>
__device__ __forceinline__ void lanes_own_sums(const GradArgs& a, int64_t n, int lanes, int l)
{
    const int V = a.r.V, target = row_target(a.r, n);
    const typename E::T* row = static_cast<const typename E::T*>(a.r.logits) + n * a.r.stride;
    typename E::T* out = static_cast<typename E::T*>(a.out) + n * a.out_stride;
    Part p{-INFINITY, 0.0f, 0.0f};
#pragma unroll 1
    for (int j = l; j < V; j += lanes) { const float z[1] = {E::get(row + j)}; add_elements<false>(p, z, a.r.c, a.r.c_lo); }
    float m = p.m;
    for (int off = 1; off < lanes; off <<= 1) m = fmaxf(m, __shfl_xor(m, off, 64));
    rescale<false>(p, m, a.r.c, a.r.c_lo);
    Sums q{m, (double)p.s, (double)p.u};
    for (int off = 1; off < lanes; off <<= 1) { q.s += __shfl_xor(q.s, off, 64); q.u += __shfl_xor(q.u, off, 64); }
    const RowGrad g = row_gradient_to(a, n, finish_row<false>(q, a.r), target);
#pragma unroll 1
    for (int j = l; j < V; j += lanes) {
        const float z[1] = {E::get(row + j)};
        float d[1];
        gradient_of<true>(g, z, d);
        E::put(out + j, d[0] + (j == target ? g.to_target : 0.0f));
    }
}

// Wavefronts to a SIMD at least.  16-bit gradients: as many as their common rows fit, where lanes_own_sums would have a few registers
// more (a million rows of 256 bf16 with three wavefronts 258 us, with four 217).
template <class E, int DO, int PIECES>
constexpr int lanes_waves()
{
    if (DO == DO_GRADIENT && E::N == 8) return PIECES == 4 ? 4 : PIECES == 2 ? 6 : 1;
    return PIECES == 4 && E::N == 4 ? 4 : 1;
}
template <class E, int DO, int PIECES, bool FINE>
__global__ __launch_bounds__(WG, (lanes_waves<E, DO, PIECES>())) void lanes_rows(const LaneArgs<DO> a)
{
    typedef typename E::T T;
    __shared__ FinishLds lds;
    const Rows& r = a.rows();
    const int lanes = a.lanes, l = threadIdx.x & (lanes - 1), per = WG / lanes, V = r.V, slots = LaneRow<E, PIECES>::slots(V, lanes);
    int64_t grid = gridDim.x;
    if constexpr (DO == DO_GRADIENT) {
        if (a.g.fin.stats && blockIdx.x == gridDim.x - 1) { finish(a.g.fin, lds); return; }
        if (a.g.fin.stats) grid -= 1;
    }
    double inv = 0.0, v[STATS] = {};
    bool left = false;                                                  // rows for lanes_own_sums
    if constexpr (DO == DO_POLICY) {
        const double W = block_sum(weight_share(a.p.norm, r, threadIdx.x, WG), lds.weights);
        inv = W != 0.0 ? a.p.p.grad_scale / W : 0.0;
    }
    for (int64_t base = (int64_t)blockIdx.x * per; base < r.rows; base += grid * per) {
        const int64_t n = base + threadIdx.x / lanes;
        const bool there = n < r.rows;
        const T* row = static_cast<const T*>(r.logits) + (there ? n : 0) * r.stride;
        const Cut cut = cut_at<E>(row, V, lanes >= 16);
        LaneRow<E, PIECES> x{};
        if constexpr (DO == DO_GRADIENT) {
            if (!there) continue;
            if (by_own_sums(a.g, n)) { left = true; continue; }
            const RowGrad q = grad_of_row(a.g, n);
            if (q.target >= 0) x.load(row, cut, V, lanes, l, slots);
            x.template put_gradient<E::N == 8>(q, static_cast<T*>(a.g.out) + n * a.g.out_stride, cut, V, lanes, l, slots);
        } else {
            int target = -1;
            PolicyIn in{};
            if constexpr (DO == DO_POLICY) {
                if (there) target = policy_target(a.p, n);
                if (target >= 0) in = policy_in(a.p.p, n);
            } else if (there) target = row_target(r, n);
            if (target >= 0) x.load(row, cut, V, lanes, l, slots);
            const float chosen = target >= 0 ? E::get(row + target) : 0.0f;
            const Sums p = x.template sums<FINE>(r, lanes, slots);
            if constexpr (DO == DO_SUMS) {
                if (there && l == 0) store_sums<FINE>(a.s, n, p, target, chosen);
            } else {
                RowGrad q{};
                double lp = 0.0;
                q.target = -1;
                if (target >= 0) {
                    const RowSum y = finish_row<false>(p, r);
                    lp = logp_of<false>(y, chosen, r);
                    const PolicyRow z = policy_row(a.p.p, in, lp, y.entropy, y.empty);
                    if (l == 0) add_stats(v, z);
                    if (inv != 0.0) q = row_gradient(y, z.g * inv, z.e * inv, target, r.scale);
                    else x = LaneRow<E, PIECES>{};                      // no weight, no gradient, of no matter what
                }
                if (there && l == 0 && a.p.logp) a.p.logp[n] = (float)lp;
                if (there && a.p.out) x.template put_gradient<false>(q, static_cast<T*>(a.p.out) + n * a.p.out_stride, cut, V, lanes, l, slots);
            }
        }
    }
    if constexpr (DO == DO_GRADIENT) {
        if (!left) return;
        for (int64_t n = (int64_t)blockIdx.x * per + threadIdx.x / lanes; n < r.rows; n += grid * per)
            if (by_own_sums(a.g, n)) lanes_own_sums<E>(a.g, n, lanes, l);
    }
    if constexpr (DO == DO_POLICY) {
        const int lane = threadIdx.x & 63;
        block_stats(wave_stats(v), stat_of(lane), (lane & 7) == 0, lds.waves, lds.sums);
        if (threadIdx.x < STATS) a.p.parts[blockIdx.x].v[threadIdx.x] = lds.sums[threadIdx.x];
    }
}

// ---------------------------------------------------------------------------
// Long rows, a workgroup each.  Sums: one pass with every thread's own running maximum; bound by the read.
// ---------------------------------------------------------------------------
// A wavefront's sums at its maximum, and those of a workgroup's wavefronts (a power of two of them) for the lanes of one.  Joined in
// 64 bits: the roundings of the last ten additions in 32 were most of what a log-probability was off by.
__device__ __forceinline__ Sums wave_joined(Part p, float c, float c_lo)
{
    float m = p.m;
    for (int off = 1; off < 64; off <<= 1) m = fmaxf(m, __shfl_xor(m, off, 64));
    rescale<false>(p, m, c, c_lo);
    return Sums{m, wave_sum((double)p.s), wave_sum((double)p.u)};
}
__device__ __forceinline__ Sums waves_joined(const Sums* lds, int waves, int lane, float c)
{
    Sums q = lds[lane < waves ? lane : 0];
    float m = q.m;
    for (int off = 1; off < waves; off <<= 1) m = fmaxf(m, __shfl_xor(m, off, 64));
    if (q.m != m && q.m != -INFINITY) {
        const float d = step_between(q.m, m, c);
        const double f = (double)__builtin_amdgcn_exp2f(d);
        q.u = f * fma(q.s, (double)d, q.u);
        q.s *= f;
    }
    for (int off = 1; off < waves; off <<= 1) { q.s += __shfl_xor(q.s, off, 64); q.u += __shfl_xor(q.u, off, 64); }
    return Sums{m, q.s, q.u};
}
// (lane 0 of the first wavefront has the result)
template <bool FINE>
__device__ __forceinline__ Sums block_joined(Part p, float c, float c_lo, Sums* lds, double* lds_s)
{
    const int waves = blockDim.x >> 6, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (!FINE) {
        const Sums q = wave_joined(p, c, c_lo);
        if (lane == 0) lds[wave] = q;
        __syncthreads();
        return waves_joined(lds, waves, lane, c);
    }
    float m = p.m;
    for (int off = 1; off < 64; off <<= 1) m = fmaxf(m, __shfl_xor(m, off, 64));
    if (lane == 0) lds[wave].m = m;
    __syncthreads();
    for (int w = 0; w < waves; ++w) m = fmaxf(m, lds[w].m);
    rescale<FINE>(p, m, c, c_lo);
    return Sums{m, block_sum(fma(LN2, (double)p.u, (double)p.s), lds_s), 0.0};
}
// U pieces of this thread, all loaded before the first is used
template <class E, bool FINE, int U>
__device__ __forceinline__ void add_pieces(Part& p, const typename E::T* in, int v, int nt, float c, float c_lo)
{
    u32x4_any w[U];
#pragma unroll
    for (int k = 0; k < U; ++k) w[k] = *reinterpret_cast<const u32x4_any*>(in + (int64_t)(v + k * nt) * E::N);
    float z[U][E::N], m = p.m;
#pragma unroll
    for (int k = 0; k < U; ++k) { E::unpack(w[k], z[k]); m = max_of(z[k], m); }
    if (m > p.m) rescale<FINE>(p, m, c, c_lo);
    const Shift s = shift_of(m, c);
    const float m0 = m == -INFINITY ? 0.0f : m;
#pragma unroll
    for (int k = 0; k < U; ++k) add_at<FINE>(p, z[k], m0, s, c, c_lo);
}
template <class E, bool FINE, int U>                                   // U: loads in flight
__global__ __launch_bounds__(1024) void block_sums(const SumArgs a)
{
    __shared__ Sums lds[16];
    __shared__ double lds_s[16];
    const int64_t n = blockIdx.x;
    const int target = row_target(a.r, n), V = a.r.V, nt = blockDim.x;
    const typename E::T* row = static_cast<const typename E::T*>(a.r.logits) + n * a.r.stride;
    const float chosen = target >= 0 ? E::get(row + target) : 0.0f;
    Part p{-INFINITY, 0.0f, 0.0f};
    Sums sums{};
    if (target >= 0) {
        const Cut cut = cut_at<E>(row, V);
        const typename E::T* in = row + cut.head;
        const float c = a.r.c, c_lo = a.r.c_lo;
        int v = threadIdx.x;
        for (; v + (U - 1) * nt < cut.pieces; v += U * nt) add_pieces<E, FINE, U>(p, in, v, nt, c, c_lo);
        if (U > 4 && v + 3 * nt < cut.pieces) { add_pieces<E, FINE, 4>(p, in, v, nt, c, c_lo); v += 4 * nt; }
        for (; v < cut.pieces; v += nt) {
            float z[E::N];
            E::unpack(*reinterpret_cast<const u32x4_any*>(in + (int64_t)v * E::N), z);
            add_elements<FINE>(p, z, c, c_lo);
        }
        if ((int)threadIdx.x < cut.loose) {
            const float z[1] = {E::get(row + loose_column<E>(cut, threadIdx.x))};
            add_elements<FINE>(p, z, c, c_lo);
        }
        sums = block_joined<FINE>(p, c, c_lo, lds, lds_s);
    }
    if (threadIdx.x == 0) store_sums<FINE>(a, n, sums, target, chosen);
}

// Zeros in all of a row of the gradient.  (Stored past the caches: with a fifth of the rows like that the backward pass of
// 1021 x 50001 fp32 takes 72 us, not 80.  The gradient itself is better off in them, 831 us and 857 for the largest case of the
// clipped loss -- but where the logits have just been read and are read again.)
template <class E, int NT>
__device__ __forceinline__ void zero_row(typename E::T* out, int V)
{
    const Cut cut = cut_at<E>(out, V);
    for (int v = threadIdx.x; v < cut.pieces; v += NT) __builtin_nontemporal_store(u32x4_any{0, 0, 0, 0}, reinterpret_cast<u32x4_any*>(out + cut.head + (int64_t)v * E::N));
    if ((int)threadIdx.x < cut.loose) E::put(out + loose_column<E>(cut, threadIdx.x), 0.0f);
}
template <class E, bool ENT, bool PAST = false>                         // PAST: past the caches
__device__ __forceinline__ void put_piece(const RowGrad& q, const u32x4_any& w, typename E::T* out)
{
    float z[E::N], d[E::N];
    E::unpack(w, z);
    gradient_of<ENT>(q, z, d);
    if (PAST) __builtin_nontemporal_store(E::pack(d), reinterpret_cast<u32x4_any*>(out));
    else *reinterpret_cast<u32x4_any*>(out) = E::pack(d);
}
template <class E, bool ENT>
__device__ __forceinline__ void put_element(const RowGrad& q, float x, float more, typename E::T* out)
{
    const float z[1] = {x};
    float d[1];
    gradient_of<ENT>(q, z, d);
    E::put(out, d[0] + more);
}
// whether this thread stores column `target` of a row whose piece v goes to thread v % NT: it stores it once more behind its
// pieces, with what the target gets beside the others (stores of one thread to one place keep their order)
template <class E, int NT>
__device__ __forceinline__ bool stores_target(const Cut& cut, int target)
{
    const int i = target - cut.head, v = i / E::N;
    if (i < 0) return (int)threadIdx.x == target;
    return v < cut.pieces ? (int)threadIdx.x == v % NT : (int)threadIdx.x == target - cut.pieces * E::N;
}

// ---------------------------------------------------------------------------
// d / d logits of a row, element by element, from its coefficients; bound by the read and the write.  AGAIN: a pass of sums over
// the same logits has just been made, and its last rows may still lie in the last-level cache.  So the rows are taken from the
// last to the first and the gradient is stored past the caches (6000 x 100003 fp16, all of the loss: 638 us without either, 645
// and 638 with one of them, 614 with both).
// ---------------------------------------------------------------------------
// (us with 4 and 8: 6000 x 100003 fp16 508 and 496, 4096 x 50001 fp32 345 and 337; 65536 x 2500 bf16, a wavefront each, 124 and 137)
constexpr int loads_in_flight(int threads) { return threads > 64 ? 8 : 4; }
// (q lies in scalar registers, whichever way it came)
__device__ __forceinline__ float uniform(float x) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x))); }
template <class E, bool ENT, bool AGAIN, int NT>
__global__ __launch_bounds__(NT) void block_gradients(const GradArgs a)
{
    typedef typename E::T T;
    __shared__ FinishLds lds;
    if (a.fin.stats && blockIdx.x == gridDim.x - 1) { finish(a.fin, lds); return; }
    const int64_t n = AGAIN ? a.r.rows - 1 - blockIdx.x / a.shares : blockIdx.x / a.shares;
    RowGrad q = grad_of_row(a, n);
    const T* row = static_cast<const T*>(a.r.logits) + n * a.r.stride;
    T* out = static_cast<T*>(a.out) + n * a.out_stride;
    constexpr int U = loads_in_flight(NT);
    int share = (int)(blockIdx.x % a.shares), shares = a.shares;        // of the row, in whole rounds of U pieces a thread
    if (q.target < 0) { if (share == 0) zero_row<E, NT>(out, a.r.V); return; }
    const Cut cut = cut_at<E>(row, a.r.V);
    const T* in = row + cut.head;
    T* to = out + cut.head;
    if (!AGAIN && by_own_sums(a, n)) {
        // (the first workgroup alone: the gradient may overwrite what others would still add up)
        if (share != 0) return;
        shares = 1;
        __shared__ Sums waves[NT / 64];
        __shared__ RowGrad own;
        Part p{-INFINITY, 0.0f, 0.0f};
        for (int v = threadIdx.x; v < cut.pieces; v += NT) {
            float z[E::N];
            E::unpack(*reinterpret_cast<const u32x4_any*>(in + (int64_t)v * E::N), z);
            add_elements<false>(p, z, a.r.c, a.r.c_lo);
        }
        if ((int)threadIdx.x < cut.loose) {
            const float z[1] = {E::get(row + loose_column<E>(cut, threadIdx.x))};
            add_elements<false>(p, z, a.r.c, a.r.c_lo);
        }
        const Sums sums = block_joined<false>(p, a.r.c, a.r.c_lo, waves, nullptr);
        if (threadIdx.x == 0) own = row_gradient_to(a, n, finish_row<false>(sums, a.r), q.target);
        __syncthreads();
        q = RowGrad{Shift{uniform(own.k.c), uniform(own.k.K)}, uniform(own.a0), uniform(own.a1), uniform(own.to_target), q.target};
    }
    const int rounds = (cut.pieces + U * NT - 1) / (U * NT), each = (rounds + shares - 1) / shares;
    const int begin = share * each * U * NT, end = begin + each * U * NT < cut.pieces ? begin + each * U * NT : cut.pieces;
    // (the target's logit before it is overwritten; of a row in shares, by the one that stores it)
    const int tp = q.target - cut.head, tv = tp >= 0 ? tp / E::N : 0;
    const bool loose = tp < 0 || tv >= cut.pieces, mine = loose ? share == 0 : tv >= begin && tv < end;
    const float chosen = mine ? E::get(row + q.target) : 0.0f;
    int v = begin + threadIdx.x;
    for (; v + (U - 1) * NT < end; v += U * NT) {
        u32x4_any w[U];
#pragma unroll
        for (int k = 0; k < U; ++k) w[k] = *reinterpret_cast<const u32x4_any*>(in + (int64_t)(v + k * NT) * E::N);
#pragma unroll
        for (int k = 0; k < U; ++k) put_piece<E, ENT, AGAIN>(q, w[k], to + (int64_t)(v + k * NT) * E::N);
    }
    for (; v < end; v += NT) put_piece<E, ENT, AGAIN>(q, *reinterpret_cast<const u32x4_any*>(in + (int64_t)v * E::N), to + (int64_t)v * E::N);
    if (share == 0 && (int)threadIdx.x < cut.loose) { const int j = loose_column<E>(cut, threadIdx.x); put_element<E, ENT>(q, E::get(row + j), 0.0f, out + j); }
    if (mine && stores_target<E, NT>(cut, q.target)) put_element<E, ENT>(q, chosen, q.to_target, out + q.target);
}

// ---------------------------------------------------------------------------
// The clipped loss over long rows: a workgroup of NT threads holds a row, VPT pieces of 16 bytes a thread in registers and LPT in
// LDS, from the one read to the one write; of a row longer than that the rest is read again, from the caches.  The pieces in LDS
// are loaded there past the registers, which have no room for them even for a moment (through registers 15 were spilled, and half
// of the gain was lost).
// ---------------------------------------------------------------------------
template <class E, int NT, int VPT, int LPT, bool ENT>
__global__ __launch_bounds__(NT, VPT <= 4 ? 7 : VPT <= 8 ? 5 : 4) void block_policy(const PolicyArgs a)
{
    typedef typename E::T T;
    constexpr int WAVES = NT / 64;
    __shared__ Sums lds[WAVES];
    __shared__ double weights[WAVES];
    __shared__ RowGrad row_grad;
    typedef uint32_t u32x4_whole __attribute__((ext_vector_type(4)));
    __shared__ u32x4_whole stash[LPT > 0 ? LPT : 1][LPT > 0 ? NT : 1];       // (a thread reads back what it loaded itself)
    constexpr int HELD = VPT + LPT;
    const int64_t n = blockIdx.x;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const int target = policy_target(a, n);
    const T* row = static_cast<const T*>(a.r.logits) + n * a.r.stride;
    T* out = static_cast<T*>(a.out) + n * a.out_stride;
    if (target < 0) {
        if (a.out) zero_row<E, NT>(out, a.r.V);
        if (tid == 0) {
            if (a.logp) a.logp[n] = 0.0f;
#pragma unroll
            for (int k = 0; k < STATS; ++k) a.parts[n].v[k] = 0.0;
        }
        return;
    }
    const Cut cut = cut_at<E>(row, a.r.V);
    const T* in = row + cut.head;
    // (loads return in order: the few small ones first)
    PolicyIn pin{};
    if (tid == 0) pin = policy_in(a.p, n);
    double share = weight_share(a.norm, a.r, tid, NT);
    const float chosen = E::get(row + target);
    u32x4_any w[VPT];
#pragma unroll
    for (int k = 0; k < LPT; ++k)                                      // (lane l of a wavefront at 16 l bytes)
        if (tid + (VPT + k) * NT < cut.pieces)
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(in + (int64_t)(tid + (VPT + k) * NT) * E::N),
                                             (__attribute__((address_space(3))) void*)&stash[k][__builtin_amdgcn_readfirstlane(wave) * 64], 16, 0, 0);
#pragma unroll
    for (int k = 0; k < VPT; ++k)
        if (tid + k * NT < cut.pieces) w[k] = *reinterpret_cast<const u32x4_any*>(in + (int64_t)(tid + k * NT) * E::N);
    const int j_loose = loose_column<E>(cut, tid);
    const float z_loose = tid < cut.loose ? E::get(row + j_loose) : -INFINITY;
    share = wave_sum(share);
    // maximum of the wavefront's pieces, then their sums at that shift
    const float c = a.r.c, c_lo = a.r.c_lo;
    float m = z_loose;
    if (LPT > 0) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
    for (int k = 0; k < LPT; ++k)
        if (tid + (VPT + k) * NT < cut.pieces) { float z[E::N]; E::unpack(stash[k][tid], z); m = max_of(z, m); }
#pragma unroll
    for (int k = 0; k < VPT; ++k)
        if (tid + k * NT < cut.pieces) { float z[E::N]; E::unpack(w[k], z); m = max_of(z, m); }
    for (int off = 1; off < 64; off <<= 1) m = fmaxf(m, __shfl_xor(m, off, 64));
    Part p{m, 0.0f, 0.0f};
    const Shift s = shift_of(m, c);
#pragma unroll
    for (int k = 0; k < VPT; ++k)
        if (tid + k * NT < cut.pieces) { float z[E::N]; E::unpack(w[k], z); add_at<false>(p, z, 0.0f, s, c, c_lo); }
#pragma unroll
    for (int k = 0; k < LPT; ++k)
        if (tid + (VPT + k) * NT < cut.pieces) { float z[E::N]; E::unpack(stash[k][tid], z); add_at<false>(p, z, 0.0f, s, c, c_lo); }
    if (tid < cut.loose) { const float z[1] = {z_loose}; add_at<false>(p, z, 0.0f, s, c, c_lo); }
    for (int v = tid + HELD * NT; v < cut.pieces; v += NT) {
        float z[E::N];
        E::unpack(*reinterpret_cast<const u32x4_any*>(in + (int64_t)v * E::N), z);
        add_elements<false>(p, z, c, c_lo);
    }
    const Sums of_wave = wave_joined(p, c, c_lo);
    if (lane == 0) { lds[wave] = of_wave; weights[wave] = share; }
    __syncthreads();
    if (wave == 0) {
        const Sums sums = waves_joined(lds, WAVES, lane, c);
        const double W = wave_sum(lane < WAVES ? weights[lane] : 0.0);
        if (lane == 0) {
            const RowSum x = finish_row<false>(sums, a.r);
            const double lp = logp_of<false>(x, chosen, a.r), inv = W != 0.0 ? a.p.grad_scale / W : 0.0;
            const PolicyRow y = policy_row(a.p, pin, lp, x.entropy, x.empty);
            row_grad = row_gradient(x, y.g * inv, y.e * inv, inv != 0.0 ? target : -1, a.r.scale);
            if (a.logp) a.logp[n] = (float)lp;
            double v[STATS] = {};
            add_stats(v, y);
#pragma unroll
            for (int k = 0; k < STATS; ++k) a.parts[n].v[k] = v[k];
        }
    }
    if (!a.out) return;
    __syncthreads();
    const RowGrad q = row_grad;
    if (q.target < 0) { zero_row<E, NT>(out, a.r.V); return; }          // no weight, no gradient, of no matter what
    T* to = out + cut.head;
#pragma unroll
    for (int k = 0; k < VPT; ++k)
        if (tid + k * NT < cut.pieces) put_piece<E, ENT>(q, w[k], to + (int64_t)(tid + k * NT) * E::N);
#pragma unroll
    for (int k = 0; k < LPT; ++k)
        if (tid + (VPT + k) * NT < cut.pieces) put_piece<E, ENT>(q, stash[k][tid], to + (int64_t)(tid + (VPT + k) * NT) * E::N);
    for (int v = tid + HELD * NT; v < cut.pieces; v += NT) put_piece<E, ENT>(q, *reinterpret_cast<const u32x4_any*>(in + (int64_t)v * E::N), to + (int64_t)v * E::N);
    if (tid < cut.loose) put_element<E, ENT>(q, z_loose, 0.0f, out + j_loose);
    if (stores_target<E, NT>(cut, target)) put_element<E, ENT>(q, chosen, q.to_target, out + target);
}

// ---------------------------------------------------------------------------
// A workgroup per pair: the summed log ratios of its two sequences, the loss of their difference h, and the coefficient
// of every row:  dL/dlp = +- w beta ((1 - y) sigmoid(h) - y sigmoid(-h)) (/ tokens)  (over W).
// ---------------------------------------------------------------------------
struct PairArgs {
    Rows r;
    Seqs q;
    const RowWs* ws;
    const float *ref, *label, *weight;
    double beta, margin, grad_scale;
    int mean;
    float *margins, *to_logp;
    Norm norm;
    Partial* parts;
};
__global__ __launch_bounds__(1024) void pair_sums(const PairArgs a)
{
    __shared__ FinishLds lds;
    const int64_t P = a.q.count / 2;
    const int lane = threadIdx.x & 63, nt = blockDim.x;
    const double W = block_sum(weight_share(a.norm, a.r, threadIdx.x, nt), lds.weights), inv = W != 0.0 ? a.grad_scale * reciprocal(W) : 0.0;
    double v[STATS] = {};
    for (int64_t k = blockIdx.x; k < P; k += gridDim.x) {
        const Seq s[2] = {sequence(a.q, k), sequence(a.q, k + P)};
        double t[STATS] = {};                                           // of the first and of the second: sum, tokens
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll 4
            for (int64_t j = threadIdx.x; j < s[i].n; j += nt) {
                const int64_t row = s[i].first + j * s[i].step;
                const RowWs w = a.ws[row];
                const float ref = a.ref ? a.ref[row] : 0.0f;
                if (w.target >= 0) { t[2 * i] += w.lp - (double)ref; t[2 * i + 1] += 1.0; }
            }
        block_stats(wave_stats(t), stat_of(lane), (lane & 7) == 0, lds.waves, lds.sums);
        double D[2], per[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            per[i] = a.mean && lds.sums[2 * i + 1] > 0.0 ? reciprocal(lds.sums[2 * i + 1]) : 1.0;
            D[i] = s[i].broken ? (double)NAN : lds.sums[2 * i] * per[i];
        }
        const double n = lds.sums[1] + lds.sums[3];
        const double h = a.beta * (D[0] - D[1]) - a.margin, y = a.label ? (double)a.label[k] : 1.0, w = a.weight ? (double)a.weight[k] : 1.0;
        if (a.margins && threadIdx.x == 0) a.margins[k] = (float)h;
        __syncthreads();                                                // (sums are read before the next pair's are written)
        if (s[0].broken || s[1].broken) v[5] += 1.0;
        if (w == 0.0) continue;
        const double e = exp_of(-fabs(h)), up = reciprocal(1.0 + e), down = e * up;         // sigmoid(|h|), sigmoid(-|h|)
        const double soft = e < 1e-4 ? e * (1.0 - 0.5 * e) : log_of_sum(1.0 + e);                   // ln(1 + e^-|h|)
        const double sig = h >= 0.0 ? up : down, gis = h >= 0.0 ? down : up;
        const double dh = inv != 0.0 ? w * a.beta * ((1.0 - y) * sig - y * gis) * inv : 0.0;    // (no weight, no gradient)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float g = (float)((i == 0 ? dh : -dh) * per[i]);
            for (int64_t j = threadIdx.x; j < s[i].n; j += nt) a.to_logp[s[i].first + j * s[i].step] = g;
        }
        if (threadIdx.x == 0) {
            const double nan = h != h ? (double)NAN : 0.0;
            const double lossy = y != 0.0 ? y * (soft + fmax(-h, 0.0)) : 0.0, lossn = y != 1.0 ? (1.0 - y) * (soft + fmax(h, 0.0)) : 0.0;
            v[0] += w * (lossy + lossn) + nan; v[1] += w * (h > 0.0 ? 1.0 : 0.0); v[2] += w * a.beta * D[0]; v[3] += w * a.beta * D[1]; v[4] += w * h;
            v[6] += 1.0; v[7] += n;
        }
    }
    if (threadIdx.x == 0)                                               // (the pairs' sums are that thread's alone)
#pragma unroll
        for (int k = 0; k < STATS; ++k) a.parts[blockIdx.x].v[k] = v[k];
}

// ---- host --------------------------------------------------------------------------------------------------------
int32_t fail(int32_t code, const char* what)
{
    try { call_error() = what; } catch (...) {}
    return code;
}
int32_t fail_hip(hipError_t e)
{
    try { call_error() = std::string("kernel launch: ") + hipGetErrorString(e); } catch (...) {}
    return ANAKIN_E_HIP;
}
static int type_bytes(int type) { return type == ANAKIN_TYPE_FP32 ? 4 : 2; }

struct LaneForm { int lanes; int pieces; };       // pieces 0: single elements; lanes 0: longer than that
static LaneForm lane_form(int type, int64_t V, bool policy);
constexpr int MAX_PARTS = 2048;                   // workgroups of short rows (8 for every compute unit) and of pairs that report sums at most

// log-probabilities need none; the clipped loss room for the weights' and the workgroups' sums; pairs rows of their own too
struct RowsWs { size_t weights, parts, folded, ws, to_logp, total; };
static RowsWs rows_workspace(int64_t rows, int64_t vocab, int64_t pairs)
{
    RowsWs w;
    size_t off = 0;
    auto take = [&](size_t bytes) { const size_t o = off; off += up256(bytes); return o; };
    w.weights = take(WEIGHT_PARTS * sizeof(double));
    const bool lanes = lane_form(ANAKIN_TYPE_FP32, vocab, true).lanes > 0 && lane_form(ANAKIN_TYPE_BF16, vocab, true).lanes > 0;
    w.parts = take((size_t)(!lanes && rows > MAX_PARTS ? rows : MAX_PARTS) * sizeof(Partial));
    w.folded = take(FOLDED * sizeof(Partial));
    w.ws = take(pairs ? (size_t)rows * sizeof(RowWs) : 0);
    w.to_logp = take(pairs ? (size_t)rows * 4 : 0);
    w.total = off;
    return w;
}

// A launch counts its threads in 32 bits.  Rows of more than 512 columns may take a workgroup each (and one that finishes): of
// so many threads at most, where there are more than 512 of them.
constexpr int64_t LANES_ALWAYS = 512;
static int most_threads(int type, int64_t V)
{
    const int64_t per = type == ANAKIN_TYPE_FP32 ? 4 : 8, pieces = (V + per - 1) / per;
    return pieces <= 256 ? 64 : pieces <= 512 ? 128 : pieces <= 2048 ? 256 : pieces <= 8192 ? 512 : 1024;
}
static bool fits(int64_t rows, int threads) { return (uint64_t)(rows + 1) * threads < ((uint64_t)1 << 32); }

// whether addresses of rows so far apart can be counted
static bool spans(int64_t rows, int64_t stride) { return rows <= 1 || stride <= ((int64_t)1 << 50) / rows; }

static int32_t check_rows(const anakin_rows* x, Rows& r)
{
    if (!x) return fail(ANAKIN_E_INVALID_ARG, "null rows");
    if (x->type < ANAKIN_TYPE_FP32 || x->type > ANAKIN_TYPE_FP16) return fail(ANAKIN_E_INVALID_ARG, "unknown type of the logits");
    if (x->target_type < ANAKIN_INDEX_U8 || x->target_type > ANAKIN_INDEX_I64) return fail(ANAKIN_E_INVALID_ARG, "unknown type of the targets");
    if (x->rows < 0 || x->rows > MAX_ROWS) return fail(ANAKIN_E_INVALID_ARG, "rows out of range");
    if (x->vocab < 1 || x->vocab > MAX_VOCAB) return fail(ANAKIN_E_INVALID_ARG, "vocab out of range");
    if (x->vocab > LANES_ALWAYS && !fits(x->rows, most_threads(x->type, x->vocab))) return fail(ANAKIN_E_INVALID_ARG, "more rows than a launch can count");
    if (x->row_stride < x->vocab && x->rows > 1) return fail(ANAKIN_E_INVALID_ARG, "row_stride is less than vocab");
    if (!spans(x->rows, x->row_stride)) return fail(ANAKIN_E_INVALID_ARG, "row_stride out of range");
    if (!(x->scale >= 1e-6 && x->scale <= 1e6)) return fail(ANAKIN_E_INVALID_ARG, "scale has to lie in [1e-6, 1e6]");
    if (x->rows > 0 && (!x->d_logits || !x->d_target)) return fail(ANAKIN_E_INVALID_ARG, "null logits or targets");
    if ((uintptr_t)x->d_logits % type_bytes(x->type)) return fail(ANAKIN_E_MISALIGNED, "logits are not aligned to their type");
    static const int index_bytes[3] = {1, 4, 8};
    if ((uintptr_t)x->d_target % index_bytes[x->target_type]) return fail(ANAKIN_E_MISALIGNED, "targets are not aligned to their type");
    r.logits = x->d_logits; r.target = x->d_target; r.rows = x->rows; r.stride = x->row_stride; r.V = (int)x->vocab;
    r.target_type = x->target_type; r.scale = x->scale;
    const double c = x->scale * LOG2E;
    r.c = (float)c; r.dc = c - (double)r.c; r.c_lo = (float)r.dc; r.inv_c = 1.0 / (double)r.c;
    return ANAKIN_OK;
}
static int32_t check_gradient(const anakin_rows* x, const void* out, int64_t stride)
{
    if (!out) return x->rows > 0 ? fail(ANAKIN_E_INVALID_ARG, "null gradient") : ANAKIN_OK;
    if (stride < x->vocab && x->rows > 1) return fail(ANAKIN_E_INVALID_ARG, "grad_stride is less than vocab");
    if (!spans(x->rows, stride)) return fail(ANAKIN_E_INVALID_ARG, "grad_stride out of range");
    const int64_t b = type_bytes(x->type);
    if ((uintptr_t)out % b) return fail(ANAKIN_E_MISALIGNED, "gradient is not aligned to its type");
    if (x->rows == 0) return ANAKIN_OK;
    const char *p = static_cast<const char*>(x->d_logits), *q = static_cast<const char*>(out);
    const char *pe = p + ((x->rows - 1) * x->row_stride + x->vocab) * b, *qe = q + ((x->rows - 1) * stride + x->vocab) * b;
    if (p < qe && q < pe && !(p == q && (stride == x->row_stride || x->rows == 1)))
        return fail(ANAKIN_E_INVALID_ARG, "the gradient overlaps the logits without being the same rows");
    return ANAKIN_OK;
}
int32_t check_workspace(const void* ws, size_t have, size_t need)
{
    if (!ws) return fail(ANAKIN_E_INVALID_ARG, "null workspace");
    if ((uintptr_t)ws & 255u) return fail(ANAKIN_E_MISALIGNED, "workspace must be 256-byte aligned");
    if (have < need) {
        try { call_error() = "workspace too small: need " + std::to_string(need) + " bytes"; } catch (...) {}
        return ANAKIN_E_WORKSPACE_TOO_SMALL;
    }
    return ANAKIN_OK;
}
static bool is_finite(double x) { return x - x == 0.0; }

// ---- which form a row takes ----------------------------------------------------------------------------------------
// Up to 32 columns: the fewest lanes that hold a row with 4 single elements each.  Up to 32 lanes of 4 pieces: the fewest of at
// least 8 lanes that hold it, with 1, 2 or 4 pieces.  (Wavefronts for rows of 256 columns, as once here, spend their time on
// one row's 64-bit arithmetic and its latencies: a million rows of bf16, sums 935 us against 173.)  Longer rows take a workgroup,
// of 64 threads at first: 131072 x 2048 bf16, clipped loss 196 us against 376 with 64 lanes of 4 pieces here, 65536 x 1024 fp32
// 200 and 250; the clipped loss over 16-bit rows does from 16 lanes of 4 pieces on (262144 x 1024 266 and 371; 524288 x 512 458
// and 368), for which it has too many registers.
static LaneForm lane_form(int type, int64_t V, bool policy)
{
    const int64_t per = type == ANAKIN_TYPE_FP32 ? 4 : 8;
    if (V <= 32) { int l = 1; while (l * 4 < V) l *= 2; return LaneForm{l, 0}; }
    for (int pieces = 1; pieces <= 2; pieces *= 2)
        if (V <= 8 * pieces * per) return LaneForm{8, pieces};
    for (int lanes = 8; lanes <= (policy && per == 8 ? 16 : 32); lanes *= 2)
        if (V <= lanes * 4 * per) return LaneForm{lanes, 4};
    return LaneForm{0, 0};
}
static unsigned lane_grid(const LaneForm& f, int64_t rows)
{
    const int64_t per = WG / f.lanes, g = (rows + per - 1) / per;
    return (unsigned)(g < 1 ? 1 : g > MAX_PARTS ? MAX_PARTS : g);
}
template <class E, int DO, bool FINE>
static void launch_lanes(const LaneForm& f, const LaneArgs<DO>& a, unsigned grid, hipStream_t s)
{
    auto k = f.pieces == 0 ? lanes_rows<E, DO, 0, FINE> : f.pieces == 1 ? lanes_rows<E, DO, 1, FINE> : f.pieces == 2 ? lanes_rows<E, DO, 2, FINE> : lanes_rows<E, DO, 4, FINE>;
    hipLaunchKernelGGL(k, dim3(grid), dim3(WG), 0, s, a);
}
#define BY_TYPE(type, f, ...) ((type) == ANAKIN_TYPE_FP32 ? f<Fp32, __VA_ARGS__> : (type) == ANAKIN_TYPE_BF16 ? f<Bf16, __VA_ARGS__> : f<Fp16, __VA_ARGS__>)

static hipError_t launch_sums(int type, const SumArgs& a, bool fine, hipStream_t s)
{
    if (a.r.rows == 0) return hipSuccess;
    const LaneForm f = lane_form(type, a.r.V, false);
    if (f.lanes) {
        LaneArgs<DO_SUMS> l{};
        l.lanes = f.lanes; l.s = a;
        if (fine) BY_TYPE(type, launch_lanes, DO_SUMS, true)(f, l, lane_grid(f, a.r.rows), s);
        else BY_TYPE(type, launch_lanes, DO_SUMS, false)(f, l, lane_grid(f, a.r.rows), s);
    } else {
        // Fewer rows than compute units: 16 pieces a thread (one row of 131072 bf16 with 256 threads 11.7 us, with 1024 10.2; 64 x 8192
        // 4.1 and 5.0).  Many rows: the shorter they are the fewer threads, so that more of them are on their way.  At the borders, bf16
        // from the caches, us with 128, 256, 512 and 1024 threads: 256 x 131072 25.3, 17.0, 15.9, 17.3 and 257 34.5, 20.5, 21.0, 24.3;
        // 256 x 32768 8.5, 6.5, 6.1, 6.4 and 257 10.8, 7.9, 7.4, 10.3; 512 x 131072 36.2, 23.9, 28.0, 31.6 and 513 36.1, 29.2, 29.8, 35.3;
        // 512 x 32768 11.6, 8.4, 8.1, 10.9; 512 x 8192 5.7, 5.0, 5.9, 7.6 and (64 threads 6.1) 513 5.7, 5.2, 6.5, 9.8.
        const int64_t pieces = a.r.V / (type == ANAKIN_TYPE_FP32 ? 4 : 8);
        const int few = pieces >= 12288 ? 1024 : pieces >= 6144 ? 512 : 256, many = pieces <= 1024 ? 64 : pieces <= 2048 ? 128 : 256;
        const dim3 grid((unsigned)a.r.rows), block(a.r.rows <= 256 ? few : a.r.rows <= 512 ? 256 : many);
        // Loads in flight of a thread: 8, but for rows of a wavefront, where more wavefronts to a compute unit are worth more (us with 4 and
        // 8, bf16: 4096 x 65536 101.7 and 97.4 (96.4 since), 16384 x 16384 100 and 94; 32768 x 6000 84 and 86, 65536 x 2500 80 and 93).
        auto k = pieces <= 1024 ? (fine ? BY_TYPE(type, block_sums, true, 4) : BY_TYPE(type, block_sums, false, 4))
                                : (fine ? BY_TYPE(type, block_sums, true, 8) : BY_TYPE(type, block_sums, false, 8));
        hipLaunchKernelGGL(k, grid, block, 0, s, a);
    }
    return hipGetLastError();
}
static hipError_t launch_gradients(int type, const GradArgs& a, bool ent, hipStream_t s)
{
    const unsigned more = a.fin.stats ? 1 : 0;
    const LaneForm f = lane_form(type, a.r.V, false);
    if (a.r.rows == 0 && !more) return hipSuccess;
    if (f.lanes) {
        LaneArgs<DO_GRADIENT> l{};
        l.lanes = f.lanes; l.g = a;
        BY_TYPE(type, launch_lanes, DO_GRADIENT, false)(f, l, lane_grid(f, a.r.rows) + more, s);
    } else {
        // short rows: a wavefront each, so that more of them are on their way
        const bool brief = a.r.V / (type == ANAKIN_TYPE_FP32 ? 4 : 8) <= 1024;
        auto k = brief ? (ent ? BY_TYPE(type, block_gradients, true, false, 64) : a.ws ? BY_TYPE(type, block_gradients, false, true, 64) : BY_TYPE(type, block_gradients, false, false, 64))
                       : (ent ? BY_TYPE(type, block_gradients, true, false, WG) : a.ws ? BY_TYPE(type, block_gradients, false, true, WG) : BY_TYPE(type, block_gradients, false, false, WG));
        // few rows: shares of them, until there are four workgroups to a compute unit (one row of 131072 bf16 10.3 -> 3.5 us; us with 1,
        // 2, 4 and 8 shares: 16 rows 10.5, 7.0, 5.1, 4.2; 64 12.2, 9.3, 7.5, 7.1; 256 22.8, 22.5, 22.3, 22.2; 512 42.5, 42.0, 42.1, 41.4;
        // 1500 153, 152, 150, 144)
        GradArgs b = a;
        const int64_t rounds = a.r.V / ((type == ANAKIN_TYPE_FP32 ? 4 : 8) * loads_in_flight(WG) * WG);
        b.shares = brief || a.r.rows >= 1024 || rounds < 2 ? 1 : (int)(1024 / (a.r.rows > 0 ? a.r.rows : 1) < rounds ? 1024 / (a.r.rows > 0 ? a.r.rows : 1) : rounds);
        hipLaunchKernelGGL(k, dim3((unsigned)(a.r.rows * b.shares) + more), dim3(brief ? 64 : WG), 0, s, b);
    }
    return hipGetLastError();
}
template <class E, bool ENT>
static void launch_block_policy(const PolicyArgs& a, hipStream_t s)
{
    // As few threads as hold a row: several rows share a compute unit, and one is loaded while another is added up.  GB/s read and
    // written (bf16) with these and with 1024 threads: 16384 x 12000 5000 and 1970, 16384 x 32768 5740 and 4250, 4096 x 65536 4800
    // and 4250; 65536 x 2500 with 128 threads 4030, with 256 2600.
    // Two rows of 29 pieces a thread fit a compute unit with 9 of them in LDS; where rows are fewer than that one of 1024 threads
    // is faster (us: fp32 512 x 50001 42 and 50, 256 x 50001 29 and 27; bf16 4096 x 100003 343 and 368, 1125 x 100003 119 and 134).
    // Three rows of 10 pieces in registers and 6 in LDS in place of two of 16 are not (bf16 4096 x 65536 243 and 224).
    // Longer rows: 16 pieces, and 9 in LDS, of 1024 threads, the rest read twice (without those 9: bf16 2048 x 200000 365 and 393,
    // fp32 256 x 100003 45 and 52).
    const int64_t pieces = (a.r.V + E::N - 1) / E::N;
    const dim3 grid((unsigned)a.r.rows);
    if (pieces <= 64 * 4) hipLaunchKernelGGL((block_policy<E, 64, 4, 0, ENT>), grid, dim3(64), 0, s, a);
    else if (pieces <= 128 * 4) hipLaunchKernelGGL((block_policy<E, 128, 4, 0, ENT>), grid, dim3(128), 0, s, a);
    else if (pieces <= 256 * 4) hipLaunchKernelGGL((block_policy<E, 256, 4, 0, ENT>), grid, dim3(256), 0, s, a);
    else if (pieces <= 256 * 8) hipLaunchKernelGGL((block_policy<E, 256, 8, 0, ENT>), grid, dim3(256), 0, s, a);
    else if (pieces <= 512 * 8) hipLaunchKernelGGL((block_policy<E, 512, 8, 0, ENT>), grid, dim3(512), 0, s, a);
    else if (pieces <= 512 * 16) hipLaunchKernelGGL((block_policy<E, 512, 16, 0, ENT>), grid, dim3(512), 0, s, a);
    else if (pieces <= 512 * 29 && a.r.rows > 256) hipLaunchKernelGGL((block_policy<E, 512, 20, 9, ENT>), grid, dim3(512), 0, s, a);
    else if (pieces <= 1024 * 16) hipLaunchKernelGGL((block_policy<E, 1024, 16, 0, ENT>), grid, dim3(1024), 0, s, a);
    else hipLaunchKernelGGL((block_policy<E, 1024, 16, 9, ENT>), grid, dim3(1024), 0, s, a);
}
// *parts: how many workgroups report sums
static hipError_t launch_policy(int type, const PolicyArgs& a, int* parts, hipStream_t s)
{
    *parts = 0;
    if (a.r.rows == 0) return hipSuccess;
    const LaneForm f = lane_form(type, a.r.V, true);
    if (f.lanes) {
        LaneArgs<DO_POLICY> l{};
        l.lanes = f.lanes; l.p = a;
        const unsigned grid = lane_grid(f, a.r.rows);
        *parts = (int)grid;
        BY_TYPE(type, launch_lanes, DO_POLICY, false)(f, l, grid, s);
    } else {
        *parts = (int)a.r.rows;
        if (a.p.ent != 0.0) BY_TYPE(type, launch_block_policy, true)(a, s);
        else BY_TYPE(type, launch_block_policy, false)(a, s);
    }
    return hipGetLastError();
}
// W: the given norm, the rows' own weights where they are few, or partial sums (of rows', or of `pairs` pairs' weights)
static hipError_t launch_weights(const Rows& r, int64_t n, const float* weight, bool pairs, double norm, double* parts, Norm& w, hipStream_t s)
{
    w = Norm{norm, parts, 0, weight, 0};
    if (norm != 0.0 || n == 0) return hipSuccess;
    if (pairs && !weight) { w.norm = (double)n; return hipSuccess; }
    if (!pairs && n <= INLINE_ROWS) { w.inline_rows = (int)n; return hipSuccess; }
    const int64_t g = (n + WG - 1) / WG;
    w.n_parts = (int)(g > WEIGHT_PARTS ? WEIGHT_PARTS : g);
    hipLaunchKernelGGL(weight_sums, dim3(w.n_parts), dim3(WG), 0, s, r, n, weight, pairs, parts);
    return hipGetLastError();
}

}  // namespace ank

using namespace ank;

#define TRY(call) do { const int32_t rc_ = (call); if (rc_ != ANAKIN_OK) return rc_; } while (0)
#define LAUNCH(call) do { const hipError_t e_ = (call); if (e_ != hipSuccess) return fail_hip(e_); } while (0)

extern "C" size_t anakin_rows_workspace_bytes(int64_t rows, int64_t vocab, int64_t pairs)
{
    if (rows < 0 || rows > MAX_ROWS || vocab < 1 || vocab > MAX_VOCAB || pairs < 0 || pairs > MAX_ROWS) return 0;
    return rows_workspace(rows, vocab, pairs).total;
}

extern "C" int32_t anakin_token_logprobs(const anakin_rows* x, float* d_logp, float* d_lse, float* d_entropy, void* hip_stream)
{
    SumArgs a{};
    TRY(check_rows(x, a.r));
    if (x->rows > 0 && !d_logp) return fail(ANAKIN_E_INVALID_ARG, "null logp");
    a.logp = d_logp; a.lse = d_lse; a.entropy = d_entropy;
    LAUNCH(launch_sums(x->type, a, false, static_cast<hipStream_t>(hip_stream)));
    return ANAKIN_OK;
}

extern "C" int32_t anakin_token_logprobs_backward(const anakin_rows* x, const float* d_lse, const float* d_entropy,
                                                  const float* d_grad_logp, const float* d_grad_entropy,
                                                  void* d_dlogits, int64_t grad_stride, void* hip_stream)
{
    GradArgs a{};
    TRY(check_rows(x, a.r));
    if (x->rows > 0 && (!d_lse || !d_grad_logp)) return fail(ANAKIN_E_INVALID_ARG, "null lse or grad_logp");
    if (d_grad_entropy && !d_entropy) return fail(ANAKIN_E_INVALID_ARG, "grad_entropy needs the entropy of the forward call");
    TRY(check_gradient(x, d_dlogits, grad_stride));
    a.out = d_dlogits; a.out_stride = grad_stride; a.lse = d_lse; a.entropy = d_entropy; a.to_logp = d_grad_logp; a.to_entropy = d_grad_entropy;
    LAUNCH(launch_gradients(x->type, a, d_grad_entropy != nullptr, static_cast<hipStream_t>(hip_stream)));
    return ANAKIN_OK;
}

extern "C" int32_t anakin_policy_loss(const anakin_rows* x, const anakin_policy_args* a, void* d_workspace, size_t workspace_bytes, void* hip_stream)
{
    Rows r;
    TRY(check_rows(x, r));
    if (!a) return fail(ANAKIN_E_INVALID_ARG, "null arguments");
    if (!a->d_stats) return fail(ANAKIN_E_INVALID_ARG, "null stats");
    if (x->rows > 0 && (!a->d_logp_old || !a->d_adv)) return fail(ANAKIN_E_INVALID_ARG, "null logp_old or adv");
    if (!(a->clip_low >= 0.0 && a->clip_low <= 1.0) || !(a->clip_high >= 0.0) || !is_finite(a->clip_high))
        return fail(ANAKIN_E_INVALID_ARG, "clip_low has to lie in [0, 1], clip_high not below 0");
    if (!is_finite(a->kl_coef) || !is_finite(a->entropy_coef) || !is_finite(a->grad_scale) || !is_finite(a->norm) || a->norm < 0.0)
        return fail(ANAKIN_E_INVALID_ARG, "a coefficient is not finite, or norm is negative");
    if (a->kl_coef != 0.0 && !a->d_logp_ref && x->rows > 0) return fail(ANAKIN_E_INVALID_ARG, "kl_coef needs logp_ref");
    if (a->d_dlogits) TRY(check_gradient(x, a->d_dlogits, a->grad_stride));
    const RowsWs w = rows_workspace(x->rows, x->vocab, 0);
    TRY(check_workspace(d_workspace, workspace_bytes, w.total));
    char* base = static_cast<char*>(d_workspace);
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    PolicyArgs p{};
    p.r = r;
    p.p = PolicyCfg{a->d_logp_old, a->d_adv, a->d_logp_ref, a->d_weight, log1p(-a->clip_low), log1p(a->clip_high), 1.0 - a->clip_low, 1.0 + a->clip_high,
                    a->kl_coef, a->entropy_coef, a->grad_scale};
    p.logp = a->d_logp; p.out = a->d_dlogits; p.out_stride = a->grad_stride;
    p.parts = reinterpret_cast<Partial*>(base + w.parts);
    LAUNCH(launch_weights(r, x->rows, a->d_weight, false, a->norm, reinterpret_cast<double*>(base + w.weights), p.norm, s));
    int parts = 0;
    LAUNCH(launch_policy(x->type, p, &parts, s));
    FinishArgs f{p.parts, parts, r, p.norm, a->d_stats, a->kl_coef, a->entropy_coef, 1};
    if (parts > FOLD_FROM) {
        Partial* folded = reinterpret_cast<Partial*>(base + w.folded);
        hipLaunchKernelGGL(fold_stats, dim3(FOLDED), dim3(WG), 0, s, p.parts, parts, folded);
        LAUNCH(hipGetLastError());
        f.parts = folded; f.n_parts = FOLDED;
    }
    hipLaunchKernelGGL(finish_stats, dim3(1), dim3(FINISH_WG), 0, s, f);
    LAUNCH(hipGetLastError());
    return ANAKIN_OK;
}

int32_t ank::check_sequences(const anakin_sequences* q, int64_t rows)
{
    if (!q) return fail(ANAKIN_E_INVALID_ARG, "null sequences");
    if (q->count < 0 || q->count > MAX_ROWS) return fail(ANAKIN_E_INVALID_ARG, "number of sequences out of range");
    if (q->layout == ANAKIN_LAYOUT_PACKED) {
        if (!q->d_offsets) return fail(ANAKIN_E_INVALID_ARG, "packed sequences need offsets");
        if ((uintptr_t)q->d_offsets & 7u) return fail(ANAKIN_E_MISALIGNED, "offsets are not aligned to their type");
    } else if (q->layout == ANAKIN_LAYOUT_BATCH || q->layout == ANAKIN_LAYOUT_TIME) {
        if (q->length < 0 || q->length > MAX_ROWS || (q->length > 0 && q->count > MAX_ROWS / q->length)) return fail(ANAKIN_E_INVALID_ARG, "length out of range");
        if (q->count * q->length != rows) return fail(ANAKIN_E_INVALID_ARG, "rows are not count x length");
    } else return fail(ANAKIN_E_INVALID_ARG, "unknown layout");
    return ANAKIN_OK;
}

extern "C" int32_t anakin_preference_loss(const anakin_rows* x, const anakin_sequences* q, const anakin_preference_args* a,
                                          void* d_workspace, size_t workspace_bytes, void* hip_stream)
{
    Rows r;
    TRY(check_rows(x, r));
    TRY(check_sequences(q, x->rows));
    if (q->count % 2) return fail(ANAKIN_E_INVALID_ARG, "pairs need an even number of sequences");
    if (!a) return fail(ANAKIN_E_INVALID_ARG, "null arguments");
    if (!a->d_stats) return fail(ANAKIN_E_INVALID_ARG, "null stats");
    if (!is_finite(a->beta) || !is_finite(a->margin) || !is_finite(a->grad_scale) || !is_finite(a->norm) || a->norm < 0.0)
        return fail(ANAKIN_E_INVALID_ARG, "a coefficient is not finite, or norm is negative");
    if (a->d_dlogits) TRY(check_gradient(x, a->d_dlogits, a->grad_stride));
    const int64_t P = q->count / 2;
    const RowsWs w = rows_workspace(x->rows, x->vocab, P > 0 ? P : 1);
    TRY(check_workspace(d_workspace, workspace_bytes, w.total));
    char* base = static_cast<char*>(d_workspace);
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    PairArgs p{};
    p.r = r;
    p.q = Seqs{q->layout, q->count, q->length, x->rows, q->d_offsets, q->d_lengths};
    p.ws = reinterpret_cast<RowWs*>(base + w.ws);
    p.ref = a->d_logp_ref; p.label = a->d_label; p.weight = a->d_weight; p.beta = a->beta; p.margin = a->margin; p.grad_scale = a->grad_scale;
    p.mean = a->mean; p.margins = a->d_margins; p.to_logp = reinterpret_cast<float*>(base + w.to_logp); p.parts = reinterpret_cast<Partial*>(base + w.parts);
    LAUNCH(launch_weights(r, P, a->d_weight, true, a->norm, reinterpret_cast<double*>(base + w.weights), p.norm, s));
    SumArgs sum{};
    sum.r = r; sum.logp = a->d_logp; sum.ws = reinterpret_cast<RowWs*>(base + w.ws); sum.coef = p.to_logp;
    LAUNCH(launch_sums(x->type, sum, true, s));
    const unsigned blocks = (unsigned)(P < 1 ? 1 : P > MAX_PARTS ? MAX_PARTS : P);
    // (long sequences: as many threads as there are; 2 x 500000 tokens 880 us with 256)
    hipLaunchKernelGGL(pair_sums, dim3(blocks), dim3(P > 0 && x->rows / (2 * P) > 512 ? 1024 : 256), 0, s, p);
    LAUNCH(hipGetLastError());
    const FinishArgs f{p.parts, (int)blocks, r, p.norm, a->d_stats, 0.0, 0.0, 0};
    if (a->d_dlogits && x->rows > 0) {
        // the gradient's launch finishes the statistics too
        GradArgs g{};
        g.r = r; g.out = a->d_dlogits; g.out_stride = a->grad_stride; g.ws = p.ws; g.to_logp = p.to_logp; g.fin = f;
        LAUNCH(launch_gradients(x->type, g, false, s));
    } else {
        hipLaunchKernelGGL(finish_stats, dim3(1), dim3(FINISH_WG), 0, s, f);
        LAUNCH(hipGetLastError());
    }
    return ANAKIN_OK;
}
