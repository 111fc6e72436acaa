// Operators of token policies on rows of logits: log-probabilities and their backward pass, the clipped policy loss, and
// the loss over pairs of sequences.  The mathematics stands in tokens.h (one row) and at the kernels below.
//   row_sums         a workgroup per row: log-sum-exp, entropy, log-probability of the target
//   row_gradients    a workgroup per row: d / d logits from a row's coefficients
//   weight_sums      partial sums of the rows' (pairs') weights
//   policy_rows      the clipped loss: coefficients of a row's gradient and the sums that are reported
//   pair_sums        the pairs: summed log ratios, coefficients of their rows
//   finish_stats     adds the workgroups' sums in a fixed order
#include <math.h>
#include "tokens.h"

namespace ank {

// what the first pass leaves of a row for the second
struct __align__(16) RowWs { double lp, entropy, log_s; float m, K, inv_s; int target; int empty, pad; };
struct Partial { double v[STATS]; };

__device__ __forceinline__ Part block_joined(Part p, float c, Part* lds)
{
    p = wave_joined(p, c);
    const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    if (waves == 1) return p;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[wave] = p;
    __syncthreads();
    Part q = lds[0];
    for (int w = 1; w < waves; ++w) q = joined(q, lds[w], c);
    return q;
}

// elements [begin, end) of a row, shared out over the workgroup
template <class E>
__device__ __forceinline__ Part row_part(const typename E::T* row, int begin, int end, float c)
{
    Part p{-INFINITY, 0.0f, 0.0f};
    const int vecs = (end - begin) / E::N;
    for (int v = threadIdx.x; v < vecs; v += blockDim.x) {
        float z[E::N];
        E::unpack(*reinterpret_cast<const u32x4_any*>(row + begin + v * E::N), z);
        add_elements(p, z, c);
    }
    for (int j = begin + vecs * E::N + threadIdx.x; j < end; j += blockDim.x) {
        const float z[1] = {E::get(row + j)};
        add_elements(p, z, c);
    }
    return p;
}

struct SumArgs {
    Rows r;
    const float* weight;                         // rows of weight 0 take no part (null: 1)
    float *logp, *lse, *entropy;                 // each may be null
    RowWs* ws;                                   // may be null
    float* coef;                                 // may be null: set to 0 (pair_sums fills in the rows of its sequences)
};

// ---------------------------------------------------------------------------
// One pass over a row with running maximum and sums.  Bound by the read.
// ---------------------------------------------------------------------------
template <class E>
__global__ __launch_bounds__(WG) void row_sums(const SumArgs a)
{
    __shared__ Part lds[WG / 64];
    for (int64_t n = blockIdx.x; n < a.r.rows; n += gridDim.x) {
        int target = row_target(a.r, n);
        if (a.weight && a.weight[n] == 0.0f) target = -1;
        const typename E::T* row = static_cast<const typename E::T*>(a.r.logits) + n * a.r.stride;
        Part p{-INFINITY, 0.0f, 0.0f};
        if (target >= 0) p = block_joined(row_part<E>(row, 0, a.r.V, a.r.c), a.r.c, lds);
        if (threadIdx.x == 0) {
            RowSum x{};
            double lp = 0.0;
            if (target >= 0) { x = finish_row(p, a.r); lp = logp_of(x, E::get(row + target), a.r); }
            if (a.logp) a.logp[n] = (float)lp;
            if (a.lse) a.lse[n] = (float)x.lse;
            if (a.entropy) a.entropy[n] = (float)x.entropy;
            if (a.ws) a.ws[n] = RowWs{lp, x.entropy, x.log_s, x.m, x.K, x.inv_s, target, x.empty, 0};
            if (a.coef) a.coef[n] = 0.0f;
        }
    }
}

// the coefficients of row n's gradient, and whether it has one
struct GradArgs {
    Rows r;
    void* out; int64_t out_stride;
    const RowWs* ws;                             // log-sum-exp and the like of the first pass; null: from the caller's lse
    const float *lse, *entropy, *to_logp, *to_entropy;   // the caller's (to_entropy may be null); to_logp also with ws
    const double* inv;                           // factor of to_logp and to_entropy (null: 1)
};
__device__ __forceinline__ RowGrad grad_of_row(const GradArgs& a, int64_t n)
{
    double g = a.to_logp[n], e = a.to_entropy ? a.to_entropy[n] : 0.0;
    if (a.inv) { g *= *a.inv; e *= *a.inv; }
    RowSum x;
    int target;
    if (a.ws) {
        const RowWs w = a.ws[n];
        x.entropy = w.entropy; x.log_s = w.log_s; x.m = w.m; x.K = w.K; x.inv_s = w.inv_s; x.empty = w.empty != 0;
        target = w.target;
    } else {
        // p_j = 2^(c z - K) (1 / s) with K = fl(lse log2 e) and the rest of lse in s
        target = row_target(a.r, n);
        const double lse = target >= 0 ? (double)a.lse[n] : 0.0, k = lse * LOG2E;
        x.empty = lse == -INFINITY;
        x.m = (float)(lse / a.r.scale); x.K = (float)k;
        x.log_s = x.empty || is_far(x.K) ? 0.0 : (k - (double)x.K) * LN2;
        x.inv_s = (float)exp(-x.log_s);
        x.entropy = e != 0.0 && target >= 0 ? (double)a.entropy[n] : 0.0;
    }
    return row_gradient(x, g, e, target, a.r.scale);
}

template <int N, bool ENT>
__device__ __forceinline__ void gradient_of(const RowGrad& q, float c, int j0, const float (&z)[N], float (&d)[N])
{
    if (is_far(q.K)) {
#pragma unroll
        for (int i = 0; i < N; ++i) { const float t = (z[i] - q.m) * c; d[i] = __builtin_amdgcn_exp2f(t) * (ENT ? fmaf(q.a1, fmaxf(t, T_MIN), q.a0) : q.a0); }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) { const float t = fmaf(z[i], c, -q.K); d[i] = __builtin_amdgcn_exp2f(t) * (ENT ? fmaf(q.a1, fmaxf(t, T_MIN), q.a0) : q.a0); }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) d[i] += j0 + i == q.target ? q.to_target : 0.0f;
}

// ---------------------------------------------------------------------------
// d / d logits of a row, element by element.  Bound by the read and the write.
// ---------------------------------------------------------------------------
template <class E, bool ENT>
__global__ __launch_bounds__(WG) void row_gradients(const GradArgs a)
{
    typedef typename E::T T;
    for (int64_t n = blockIdx.x; n < a.r.rows; n += gridDim.x) {
        const RowGrad q = grad_of_row(a, n);
        const T* row = static_cast<const T*>(a.r.logits) + n * a.r.stride;
        T* out = static_cast<T*>(a.out) + n * a.out_stride;
        const int V = a.r.V, vecs = V / E::N;
        const bool zero = q.target < 0;
        for (int v = threadIdx.x; v < vecs; v += blockDim.x) {
            float z[E::N], d[E::N] = {};
            if (!zero) {
                E::unpack(*reinterpret_cast<const u32x4_any*>(row + v * E::N), z);
                gradient_of<E::N, ENT>(q, a.r.c, v * E::N, z, d);
            }
            *reinterpret_cast<u32x4_any*>(out + v * E::N) = E::pack(d);
        }
        for (int j = vecs * E::N + threadIdx.x; j < V; j += blockDim.x) {
            float z[1], d[1] = {0.0f};
            if (!zero) { z[0] = E::get(row + j); gradient_of<1, ENT>(q, a.r.c, j, z, d); }
            E::put(out + j, d[0]);
        }
    }
}

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
__device__ __forceinline__ void block_partial(const double (&v)[STATS], double* lds, Partial* out)
{
    double s[STATS];
#pragma unroll
    for (int k = 0; k < STATS; ++k) s[k] = block_sum(v[k], lds);
    if (threadIdx.x == 0)
        for (int k = 0; k < STATS; ++k) out->v[k] = s[k];
}

// partial sums of the weights of the rows (target in range) or pairs that take part
__global__ __launch_bounds__(WG) void weight_sums(const Rows r, const int64_t n, const float* weight, const bool pairs, double* parts)
{
    __shared__ double lds[WG / 64];
    double s = 0.0;
    for (int64_t i = (int64_t)blockIdx.x * WG + threadIdx.x; i < n; i += (int64_t)gridDim.x * WG)
        if (pairs || row_target(r, i) >= 0) s += weight ? (double)weight[i] : 1.0;
    s = block_sum(s, lds);
    if (threadIdx.x == 0) parts[blockIdx.x] = s;
}

// what a mean is taken over: the given norm, or the sum of the weights
struct Norm { double norm; const double* parts; int n_parts; };
__device__ __forceinline__ double weight_total(const Norm& w)
{
    if (w.norm != 0.0) return w.norm;
    double s = 0.0;
    for (int i = threadIdx.x & 63; i < w.n_parts; i += 64) s += w.parts[i];
    return wave_sum(s);
}

// ---------------------------------------------------------------------------
// The clipped loss of one row, everything in 64 bits: which side of a clipping border a ratio lies on hangs on lp.
//   dL/dlp = w (-A r [r A <= clipped A] + kl_coef (1 - e^d)),  dL/dH = -entropy_coef w    (both without 1 / W)
// ---------------------------------------------------------------------------
struct PolicyCfg {
    const float *old, *adv, *ref, *weight;
    double low, high, kl, ent, grad_scale;
};
struct PolicyRow { double g, e, policy, kl, entropy, clipped, ratio, w; };
__device__ __forceinline__ PolicyRow policy_row(const PolicyCfg& a, int64_t n, double lp, double entropy, bool empty)
{
    PolicyRow x{};
    x.w = a.weight ? (double)a.weight[n] : 1.0;
    if (empty) return x;
    const double A = a.adv[n], r = exp(lp - (double)a.old[n]);
    const double plain = r * A, clip = fmin(fmax(r, 1.0 - a.low), 1.0 + a.high) * A;
    const bool inside = plain <= clip || plain != plain;                // a NaN stays in the gradient
    x.policy = -(inside ? plain : clip); x.clipped = inside ? 0.0 : 1.0; x.ratio = r; x.entropy = entropy;
    x.g = inside ? -plain : 0.0;
    if (a.ref) {
        const double d = (double)a.ref[n] - lp, e = exp(d);
        x.kl = e - d - 1.0;
        if (a.kl != 0.0) x.g += a.kl * (1.0 - e);
    }
    x.g *= x.w; x.e = -a.ent * x.w;
    return x;
}
__device__ __forceinline__ void add_stats(double (&v)[STATS], const PolicyRow& x)
{
    v[1] += x.w * x.policy; v[2] += x.w * x.kl; v[3] += x.w * x.entropy; v[4] += x.w * x.clipped; v[5] += x.w * x.ratio; v[6] += x.w; v[7] += 1.0;
}

struct PolicyArgs {
    PolicyCfg p;
    int64_t rows;
    const RowWs* ws;
    float *to_logp, *to_entropy;
    Norm norm;
    Partial* parts;
};
__global__ __launch_bounds__(WG) void policy_rows(const PolicyArgs a)
{
    __shared__ double lds[WG / 64];
    const double W = weight_total(a.norm), inv = W != 0.0 ? a.p.grad_scale / W : 0.0;
    double v[STATS] = {};
    for (int64_t n = (int64_t)blockIdx.x * WG + threadIdx.x; n < a.rows; n += (int64_t)gridDim.x * WG) {
        const RowWs w = a.ws[n];
        float g = 0.0f, e = 0.0f;
        if (w.target >= 0) {
            const PolicyRow x = policy_row(a.p, n, w.lp, w.entropy, w.empty != 0);
            add_stats(v, x);
            g = (float)(x.g * inv); e = (float)(x.e * inv);
        }
        a.to_logp[n] = g; a.to_entropy[n] = e;
    }
    block_partial(v, lds, a.parts + blockIdx.x);
}

// means over W of the summed statistics; slot 0 becomes the loss
struct FinishArgs { const Partial* parts; int n_parts; Norm norm; float* stats; double kl, ent; int policy; };
__global__ __launch_bounds__(WG) void finish_stats(const FinishArgs a)
{
    __shared__ double lds[WG / 64];
    double v[STATS] = {};
    for (int i = threadIdx.x; i < a.n_parts; i += WG)
        for (int k = 0; k < STATS; ++k) v[k] += a.parts[i].v[k];
    for (int k = 0; k < STATS; ++k) v[k] = block_sum(v[k], lds);
    const double W = weight_total(a.norm), inv = W != 0.0 ? 1.0 / W : 0.0;
    if (threadIdx.x != 0) return;
    double m[STATS];
    for (int k = 0; k < STATS; ++k) m[k] = W != 0.0 ? v[k] * inv : 0.0;
    if (a.policy) m[0] = m[1] + (a.kl != 0.0 ? a.kl * m[2] : 0.0) - (a.ent != 0.0 ? a.ent * m[3] : 0.0);
    m[5] = a.policy ? m[5] : W;                                         // pairs: loss, [h > 0], first, second, h, W, pairs, tokens
    m[6] = a.policy ? W : v[6];
    m[7] = v[7];
    for (int k = 0; k < STATS; ++k) a.stats[k] = (float)m[k];
}

// ---------------------------------------------------------------------------
// A workgroup per pair: the summed log ratios of its two sequences, the loss of their difference h, and the coefficient
// of every row:  dL/dlp = +- w beta ((1 - y) sigmoid(h) - y sigmoid(-h)) (/ tokens)  (without 1 / W).
// ---------------------------------------------------------------------------
struct PairArgs {
    Seqs q;
    const RowWs* ws;
    const float *ref, *label, *weight;
    double beta, margin, grad_scale;
    int mean;
    float *margins, *to_logp;
    Norm norm;
    Partial* parts;
};
__global__ __launch_bounds__(WG) void pair_sums(const PairArgs a)
{
    __shared__ double lds[WG / 64];
    const int64_t P = a.q.count / 2;
    const double W = weight_total(a.norm), inv = W != 0.0 ? a.grad_scale / W : 0.0;
    double v[STATS] = {};
    for (int64_t k = blockIdx.x; k < P; k += gridDim.x) {
        const Seq s[2] = {sequence(a.q, k), sequence(a.q, k + P)};
        double D[2], n[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            double d = 0.0, c = 0.0;
            for (int64_t j = threadIdx.x; j < s[i].n; j += WG) {
                const int64_t row = s[i].first + j * s[i].step;
                if (a.ws[row].target >= 0) { d += a.ws[row].lp - (a.ref ? (double)a.ref[row] : 0.0); c += 1.0; }
            }
            D[i] = block_sum(d, lds); n[i] = block_sum(c, lds);
            if (a.mean) D[i] = n[i] > 0.0 ? D[i] / n[i] : 0.0;
            if (s[i].broken) D[i] = NAN;
        }
        const double h = a.beta * (D[0] - D[1]) - a.margin, y = a.label ? (double)a.label[k] : 1.0, w = a.weight ? (double)a.weight[k] : 1.0;
        if (a.margins && threadIdx.x == 0) a.margins[k] = (float)h;
        if (w == 0.0) continue;
        const double e = exp(-fabs(h)), up = 1.0 / (1.0 + e), down = e / (1.0 + e);                 // sigmoid(|h|), sigmoid(-|h|)
        const double soft = log1p(e), sig = h >= 0.0 ? up : down, gis = h >= 0.0 ? down : up;
        const double lossy = y != 0.0 ? y * (soft + fmax(-h, 0.0)) : 0.0, lossn = y != 1.0 ? (1.0 - y) * (soft + fmax(h, 0.0)) : 0.0;
        const double dh = w * a.beta * ((1.0 - y) * sig - y * gis) * inv;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float g = (float)((i == 0 ? dh : -dh) / (a.mean ? (n[i] > 0.0 ? n[i] : 1.0) : 1.0));
            for (int64_t j = threadIdx.x; j < s[i].n; j += WG) a.to_logp[s[i].first + j * s[i].step] = g;
        }
        if (threadIdx.x == 0) {
            const double nan = h != h ? (double)NAN : 0.0;
            v[0] += w * (lossy + lossn) + nan; v[1] += w * (h > 0.0 ? 1.0 : 0.0); v[2] += w * a.beta * D[0]; v[3] += w * a.beta * D[1]; v[4] += w * h;
            v[6] += 1.0; v[7] += n[0] + n[1];
        }
    }
    block_partial(v, lds, a.parts + blockIdx.x);
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

constexpr int MAX_PARTS = 1024;                  // workgroups that report sums at most

struct RowsWs { size_t ws, to_logp, to_entropy, weights, parts, total; };
static RowsWs rows_workspace(int64_t rows)
{
    RowsWs w;
    size_t off = 0;
    auto take = [&](size_t bytes) { const size_t o = off; off += up256(bytes); return o; };
    w.ws = take((size_t)rows * sizeof(RowWs));
    w.to_logp = take((size_t)rows * 4); w.to_entropy = take((size_t)rows * 4);
    w.weights = take(WEIGHT_PARTS * sizeof(double));
    w.parts = take(MAX_PARTS * sizeof(Partial));
    w.total = off;
    return w;
}

static int32_t check_rows(const anakin_rows* x, Rows& r)
{
    if (!x) return fail(ANAKIN_E_INVALID_ARG, "null rows");
    if (x->type < ANAKIN_TYPE_FP32 || x->type > ANAKIN_TYPE_FP16) return fail(ANAKIN_E_INVALID_ARG, "unknown type of the logits");
    if (x->target_type < ANAKIN_INDEX_U8 || x->target_type > ANAKIN_INDEX_I64) return fail(ANAKIN_E_INVALID_ARG, "unknown type of the targets");
    if (x->rows < 0 || x->rows > MAX_ROWS) return fail(ANAKIN_E_INVALID_ARG, "rows out of range");
    if (x->vocab < 1 || x->vocab > MAX_VOCAB) return fail(ANAKIN_E_INVALID_ARG, "vocab out of range");
    if (x->row_stride < x->vocab && x->rows > 1) return fail(ANAKIN_E_INVALID_ARG, "row_stride is less than vocab");
    if (x->row_stride > ((int64_t)1 << 40)) return fail(ANAKIN_E_INVALID_ARG, "row_stride out of range");
    if (!(x->scale >= 1e-6 && x->scale <= 1e6)) return fail(ANAKIN_E_INVALID_ARG, "scale has to lie in [1e-6, 1e6]");
    if (x->rows > 0 && (!x->d_logits || !x->d_target)) return fail(ANAKIN_E_INVALID_ARG, "null logits or targets");
    if ((uintptr_t)x->d_logits % type_bytes(x->type)) return fail(ANAKIN_E_MISALIGNED, "logits are not aligned to their type");
    static const int index_bytes[3] = {1, 4, 8};
    if ((uintptr_t)x->d_target % index_bytes[x->target_type]) return fail(ANAKIN_E_MISALIGNED, "targets are not aligned to their type");
    r.logits = x->d_logits; r.target = x->d_target; r.rows = x->rows; r.stride = x->row_stride; r.V = (int)x->vocab;
    r.target_type = x->target_type; r.scale = x->scale;
    const double c = x->scale * LOG2E;
    r.c = (float)c; r.dc = c - (double)r.c;
    return ANAKIN_OK;
}
static int32_t check_gradient(const anakin_rows* x, const void* out, int64_t stride)
{
    if (!out) return x->rows > 0 ? fail(ANAKIN_E_INVALID_ARG, "null gradient") : ANAKIN_OK;
    if (stride < x->vocab && x->rows > 1) return fail(ANAKIN_E_INVALID_ARG, "grad_stride is less than vocab");
    if (stride > ((int64_t)1 << 40)) return fail(ANAKIN_E_INVALID_ARG, "grad_stride out of range");
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

static unsigned row_grid(int64_t rows) { return (unsigned)(rows < 65536 ? rows : 65536); }
static unsigned part_grid(int64_t n, int64_t per) { const int64_t g = (n + per - 1) / per; return (unsigned)(g < 1 ? 1 : g > MAX_PARTS ? MAX_PARTS : g); }

static hipError_t launch_row_sums(int type, const SumArgs& a, hipStream_t s)
{
    if (a.r.rows == 0) return hipSuccess;
    auto k = type == ANAKIN_TYPE_FP32 ? row_sums<Fp32> : type == ANAKIN_TYPE_BF16 ? row_sums<Bf16> : row_sums<Fp16>;
    hipLaunchKernelGGL(k, dim3(row_grid(a.r.rows)), dim3(WG), 0, s, a);
    return hipGetLastError();
}
static hipError_t launch_row_gradients(int type, const GradArgs& a, bool ent, hipStream_t s)
{
    if (a.r.rows == 0) return hipSuccess;
    auto k = ent ? (type == ANAKIN_TYPE_FP32 ? row_gradients<Fp32, true> : type == ANAKIN_TYPE_BF16 ? row_gradients<Bf16, true> : row_gradients<Fp16, true>)
                 : (type == ANAKIN_TYPE_FP32 ? row_gradients<Fp32, false> : type == ANAKIN_TYPE_BF16 ? row_gradients<Bf16, false> : row_gradients<Fp16, false>);
    hipLaunchKernelGGL(k, dim3(row_grid(a.r.rows)), dim3(WG), 0, s, a);
    return hipGetLastError();
}
// W: the given norm, or partial sums of the weights (of rows, or of `pairs` pairs)
static hipError_t launch_weights(const Rows& r, int64_t n, const float* weight, bool pairs, double norm, double* parts, Norm& w, hipStream_t s)
{
    w.norm = norm; w.parts = parts; w.n_parts = 0;
    if (norm != 0.0 || n == 0) return hipSuccess;
    if (pairs && !weight) { w.norm = (double)n; return hipSuccess; }
    const int64_t g = (n + 4 * WG - 1) / (4 * WG);
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
    return rows_workspace(rows).total;
}

extern "C" int32_t anakin_token_logprobs(const anakin_rows* x, float* d_logp, float* d_lse, float* d_entropy,
                                         void* d_workspace, size_t workspace_bytes, void* hip_stream)
{
    SumArgs a{};
    TRY(check_rows(x, a.r));
    if (x->rows > 0 && (!d_logp || !d_lse)) return fail(ANAKIN_E_INVALID_ARG, "null logp or lse");
    TRY(check_workspace(d_workspace, workspace_bytes, rows_workspace(x->rows).total));
    a.logp = d_logp; a.lse = d_lse; a.entropy = d_entropy;
    LAUNCH(launch_row_sums(x->type, a, static_cast<hipStream_t>(hip_stream)));
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
    LAUNCH(launch_row_gradients(x->type, a, d_grad_entropy != nullptr, static_cast<hipStream_t>(hip_stream)));
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
    const RowsWs w = rows_workspace(x->rows);
    TRY(check_workspace(d_workspace, workspace_bytes, w.total));
    char* base = static_cast<char*>(d_workspace);
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    PolicyArgs p{};
    p.p = PolicyCfg{a->d_logp_old, a->d_adv, a->d_logp_ref, a->d_weight, a->clip_low, a->clip_high, a->kl_coef, a->entropy_coef, a->grad_scale};
    p.rows = x->rows; p.ws = reinterpret_cast<RowWs*>(base + w.ws);
    p.to_logp = reinterpret_cast<float*>(base + w.to_logp); p.to_entropy = reinterpret_cast<float*>(base + w.to_entropy);
    p.parts = reinterpret_cast<Partial*>(base + w.parts);
    LAUNCH(launch_weights(r, x->rows, a->d_weight, false, a->norm, reinterpret_cast<double*>(base + w.weights), p.norm, s));
    SumArgs sum{};
    sum.r = r; sum.weight = a->d_weight; sum.logp = a->d_logp; sum.ws = reinterpret_cast<RowWs*>(base + w.ws);
    LAUNCH(launch_row_sums(x->type, sum, s));
    const unsigned blocks = part_grid(x->rows, WG);
    hipLaunchKernelGGL(policy_rows, dim3(blocks), dim3(WG), 0, s, p);
    LAUNCH(hipGetLastError());
    const FinishArgs f{p.parts, (int)blocks, p.norm, a->d_stats, a->kl_coef, a->entropy_coef, 1};
    hipLaunchKernelGGL(finish_stats, dim3(1), dim3(WG), 0, s, f);
    LAUNCH(hipGetLastError());
    if (a->d_dlogits) {
        GradArgs g{};
        g.r = r; g.out = a->d_dlogits; g.out_stride = a->grad_stride; g.ws = p.ws; g.to_logp = p.to_logp; g.to_entropy = p.to_entropy;
        LAUNCH(launch_row_gradients(x->type, g, a->entropy_coef != 0.0, s));
    }
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
    const RowsWs w = rows_workspace(x->rows);
    TRY(check_workspace(d_workspace, workspace_bytes, w.total));
    char* base = static_cast<char*>(d_workspace);
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    const int64_t P = q->count / 2;
    PairArgs p{};
    p.q = Seqs{q->layout, q->count, q->length, x->rows, q->d_offsets, q->d_lengths};
    p.ws = reinterpret_cast<RowWs*>(base + w.ws);
    p.ref = a->d_logp_ref; p.label = a->d_label; p.weight = a->d_weight; p.beta = a->beta; p.margin = a->margin; p.grad_scale = a->grad_scale;
    p.mean = a->mean; p.margins = a->d_margins; p.to_logp = reinterpret_cast<float*>(base + w.to_logp); p.parts = reinterpret_cast<Partial*>(base + w.parts);
    LAUNCH(launch_weights(r, P, a->d_weight, true, a->norm, reinterpret_cast<double*>(base + w.weights), p.norm, s));
    SumArgs sum{};
    sum.r = r; sum.logp = a->d_logp; sum.ws = reinterpret_cast<RowWs*>(base + w.ws); sum.coef = p.to_logp;
    LAUNCH(launch_row_sums(x->type, sum, s));
    const unsigned blocks = part_grid(P, 1);
    hipLaunchKernelGGL(pair_sums, dim3(blocks), dim3(WG), 0, s, p);
    LAUNCH(hipGetLastError());
    const FinishArgs f{p.parts, (int)blocks, p.norm, a->d_stats, 0.0, 0.0, 0};
    hipLaunchKernelGGL(finish_stats, dim3(1), dim3(WG), 0, s, f);
    LAUNCH(hipGetLastError());
    if (a->d_dlogits) {
        GradArgs g{};
        g.r = r; g.out = a->d_dlogits; g.out_stride = a->grad_stride; g.ws = p.ws; g.to_logp = p.to_logp;
        LAUNCH(launch_row_gradients(x->type, g, false, s));
    }
    return ANAKIN_OK;
}
