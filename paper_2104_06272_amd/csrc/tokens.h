// What the operators of token policies share: argument blocks, element types, and the arithmetic of one row of logits.
#pragma once
#include "internal.h"

namespace ank {

constexpr double LOG2E = 1.4426950408889634074, LN2 = 0.69314718055994530942;
constexpr int STATS = 8;                         // sums that a call reports
constexpr int WEIGHT_PARTS = 256;                // partial sums of the weights at most

std::string& call_error();                       // message of this thread's last failed call without a handle (anakin.hip)

// a matrix of logits as the kernels take it; c = scale log2 e: softmax(scale z) is 2^(c z) over its sum
struct Rows {
    const void* logits; const void* target;
    int64_t rows, stride;
    int V, target_type;
    float c;
    double scale, dc;                            // dc: the exact product minus c
};

// the column row n chose, -1 where it takes no part
__device__ __forceinline__ int row_target(const Rows& r, int64_t n)
{
    int64_t t;
    if (r.target_type == ANAKIN_INDEX_U8) t = static_cast<const uint8_t*>(r.target)[n];
    else if (r.target_type == ANAKIN_INDEX_I32) t = static_cast<const int32_t*>(r.target)[n];
    else t = static_cast<const int64_t*>(r.target)[n];
    return t >= 0 && t < r.V ? (int)t : -1;
}

// element types: 16 bytes are loaded at a time at the type's own alignment (global memory takes any), so that rows of odd
// lengths and strides run like others
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
struct Fp32 {
    typedef float T;
    static constexpr int N = 4;
    static __device__ __forceinline__ void unpack(const u32x4_any& w, float (&f)[4])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(w[i]);
    }
    static __device__ __forceinline__ u32x4_any pack(const float (&f)[4])
    {
        u32x4_any w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(f[i]);
        return w;
    }
    static __device__ __forceinline__ float get(const T* p) { return *p; }
    static __device__ __forceinline__ void put(T* p, float f) { *p = f; }
};
struct Bf16 {
    typedef uint16_t T;
    typedef __bf16 pair __attribute__((ext_vector_type(2)));
    static constexpr int N = 8;
    static __device__ __forceinline__ void unpack(const u32x4_any& w, float (&f)[8])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
    }
    static __device__ __forceinline__ u32x4_any pack(const float (&f)[8])
    {
        u32x4_any w;
#pragma unroll
        for (int i = 0; i < 4; ++i) { pair p; p[0] = (__bf16)f[2 * i]; p[1] = (__bf16)f[2 * i + 1]; w[i] = __builtin_bit_cast(uint32_t, p); }   // to nearest even
        return w;
    }
    static __device__ __forceinline__ float get(const T* p) { return __uint_as_float((uint32_t)*p << 16); }
    static __device__ __forceinline__ void put(T* p, float f) { *p = __builtin_bit_cast(uint16_t, (__bf16)f); }
};
struct Fp16 {
    typedef uint16_t T;
    typedef _Float16 pair __attribute__((ext_vector_type(2)));
    static constexpr int N = 8;
    static __device__ __forceinline__ void unpack(const u32x4_any& w, float (&f)[8])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) { const pair p = __builtin_bit_cast(pair, (uint32_t)w[i]); f[2 * i] = (float)p[0]; f[2 * i + 1] = (float)p[1]; }
    }
    static __device__ __forceinline__ u32x4_any pack(const float (&f)[8])
    {
        u32x4_any w;
#pragma unroll
        for (int i = 0; i < 4; ++i) { pair p; p[0] = (_Float16)f[2 * i]; p[1] = (_Float16)f[2 * i + 1]; w[i] = __builtin_bit_cast(uint32_t, p); }
        return w;
    }
    static __device__ __forceinline__ float get(const T* p) { return (float)__builtin_bit_cast(_Float16, *p); }
    static __device__ __forceinline__ void put(T* p, float f) { *p = __builtin_bit_cast(uint16_t, (_Float16)f); }
};

// ---------------------------------------------------------------------------
// Part of a row's softmax: m = max z, s = sum 2^t, u = sum t 2^t over the elements seen, t = c z - K with the shift
// K = fl(c m).  K need not be exact: every use takes the same K, and the error of c against scale log2 e (2^-24 of t at
// worst, the same sign all along a row) is made up for in the log-sum-exp to first order, ln 2 (exact c - c) E[z] with E[z]
// from u.  Over sums of thousands of log-probabilities it would otherwise show.
// Rows of nothing but values near the type's lowest would overflow c m; they are `far`: t = c (z - m).
// Elements of minus infinity add 0 (their t enters u clamped); a NaN stays in s.
// ---------------------------------------------------------------------------
struct Part { float m, s, u; };
constexpr float FAR = 1e30f, T_MIN = -1e4f;
__device__ __forceinline__ float shift_of(float m, float c) { return m == -INFINITY ? 0.0f : m * c; }
__device__ __forceinline__ bool is_far(float K) { return fabsf(K) > FAR; }
__device__ __forceinline__ float exponent_of(float z, float m, float K, float c) { return is_far(K) ? (z - m) * c : fmaf(z, c, -K); }

// p's sums moved to the shift of a larger maximum
__device__ __forceinline__ void rescale(Part& p, float m, float c)
{
    if (p.m == m || p.m == -INFINITY) { p.m = m; return; }
    const float K0 = shift_of(p.m, c), K1 = shift_of(m, c);
    const float d = fmaxf((is_far(K0) || is_far(K1)) ? (p.m - m) * c : K0 - K1, T_MIN);
    const float f = __builtin_amdgcn_exp2f(d);
    p.u = f * fmaf(p.s, d, p.u);
    p.s *= f;
    p.m = m;
}
__device__ __forceinline__ Part joined(Part a, Part b, float c)
{
    const float m = fmaxf(a.m, b.m);
    rescale(a, m, c); rescale(b, m, c);
    return Part{m, a.s + b.s, a.u + b.u};
}
template <int N>
__device__ __forceinline__ void add_elements(Part& p, const float (&z)[N], float c)
{
    float m = z[0];
#pragma unroll
    for (int i = 1; i < N; ++i) m = fmaxf(m, z[i]);
    m = fmaxf(m, p.m);                                                  // (fmaxf passes over a NaN)
    if (m > p.m) rescale(p, m, c);
    const float K = shift_of(p.m, c);
    if (is_far(K)) {
        const float m0 = p.m;
#pragma unroll
        for (int i = 0; i < N; ++i) { const float t = (z[i] - m0) * c, e = __builtin_amdgcn_exp2f(t); p.s += e; p.u = fmaf(e, fmaxf(t, T_MIN), p.u); }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) { const float t = fmaf(z[i], c, -K), e = __builtin_amdgcn_exp2f(t); p.s += e; p.u = fmaf(e, fmaxf(t, T_MIN), p.u); }
    }
}
__device__ __forceinline__ Part wave_joined(Part p, float c, int lanes = 64)
{
    for (int off = 1; off < lanes; off <<= 1) {
        Part q{__shfl_xor(p.m, off, 64), __shfl_xor(p.s, off, 64), __shfl_xor(p.u, off, 64)};
        p = joined(p, q, c);
    }
    return p;
}

// a whole row: log-sum-exp, entropy, log-probability of an element, and 1 / s for the gradient
struct RowSum {
    double lse, entropy, log_s;
    float m, K, inv_s;
    bool empty;                                                         // all of it minus infinity
};
__device__ __forceinline__ RowSum finish_row(const Part& p, const Rows& r)
{
    RowSum x;
    x.m = p.m; x.K = shift_of(p.m, r.c);
    x.empty = p.m == -INFINITY && p.s == 0.0f;
    const double s = (double)p.s, mean_t = (double)p.u / s;             // E[t]
    const double log_s = log(s);                                        // with c for scale log2 e, as the exponents have it
    if (is_far(x.K)) x.lse = r.scale * (double)p.m + log_s;
    else x.lse = LN2 * ((double)x.K + r.dc * ((mean_t + (double)x.K) / (double)r.c)) + log_s;
    x.entropy = log_s - LN2 * mean_t;
    x.log_s = log_s;
    x.inv_s = (float)exp(-log_s);
    if (x.empty) { x.lse = -INFINITY; x.entropy = 0.0; x.inv_s = 0.0f; x.log_s = 0.0; }
    return x;
}
__device__ __forceinline__ double logp_of(const RowSum& x, float z, const Rows& r)
{
    if (x.empty) return -INFINITY;
    if (is_far(x.K)) return r.scale * ((double)z - (double)x.m) - x.log_s;
    return r.scale * (double)z - x.lse;
}

// Gradient of one row: element j gets 2^t (a0 + a1 t), and the target `to_target` more.  From  g ([j = a] - p_j) - e p_j (log p_j + H)
// with p_j = 2^t / s, log p_j = ln 2 t - log s:  a0 = (-g - e (H - log s)) / s,  a1 = -e ln 2 / s.
struct RowGrad { float m, K, a0, a1, to_target; int target; };
__device__ __forceinline__ RowGrad row_gradient(const RowSum& x, double g, double e, int target, double scale)
{
    RowGrad q;
    q.m = x.m; q.K = x.K; q.target = target;
    const double k = scale * (double)x.inv_s;
    q.a0 = (float)(k * (-g - (e != 0.0 ? e * (x.entropy - x.log_s) : 0.0)));
    q.a1 = (float)(-k * e * LN2);
    q.to_target = (float)(scale * g);
    if (x.empty) q.a0 = q.a1 = q.to_target = 0.0f;
    return q;
}

// ---- sequences over rows -----------------------------------------------------------------------------------------
struct Seqs { int layout; int64_t count, length, rows; const int64_t* offsets; const int32_t* lengths; };
struct Seq { int64_t first, step, n; bool broken; };
__device__ __forceinline__ Seq sequence(const Seqs& q, int64_t s)
{
    Seq x;
    if (q.layout == ANAKIN_LAYOUT_PACKED) {
        const int64_t b = q.offsets[s], e = q.offsets[s + 1];
        const int64_t b1 = b < 0 ? 0 : b > q.rows ? q.rows : b, e1 = e < b1 ? b1 : e > q.rows ? q.rows : e;
        x.first = b1; x.step = 1; x.n = e1 - b1; x.broken = b1 != b || e1 != e;
        return x;
    }
    const int64_t n = q.lengths ? (int64_t)q.lengths[s] : q.length;
    x.n = n < 0 ? 0 : n > q.length ? q.length : n; x.broken = x.n != n;
    x.first = q.layout == ANAKIN_LAYOUT_BATCH ? s * q.length : s;
    x.step = q.layout == ANAKIN_LAYOUT_BATCH ? 1 : q.count;
    return x;
}

int32_t check_sequences(const anakin_sequences* q, int64_t rows);   // and the other refusals of calls without a handle (tokens.hip)
int32_t fail(int32_t code, const char* what);
int32_t fail_hip(hipError_t e);
int32_t check_workspace(const void* ws, size_t have, size_t need);
inline size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }
constexpr int64_t MAX_ROWS = ((int64_t)1 << 31) - 1, MAX_VOCAB = (1 << 28) - 1;

}  // namespace ank
