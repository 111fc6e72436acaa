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
    float c_lo;                                  // the exact product minus c
    double scale, dc, inv_c;                     // dc: c_lo in 64 bits; inv_c = 1 / c
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

// Element types.  16 bytes are loaded and stored at a time; global memory takes any alignment, so the type's own would do, but
// rows of 16-bit elements off their dwords cost a quarter (100003 columns, fp16: sums 200 us and 166 in place, the clipped
// loss 486 and 383) and stores off 16 bytes a tenth.  A row is therefore cut into loose elements up to a 16-byte border of the
// logits, pieces of 16 bytes, and loose elements behind them; a gradient of the same strides lies alike, and where it does not
// the result is the same all the same.
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

struct Cut { int head, pieces, loose; };         // loose: in front and behind, 14 at most
template <class E>
__device__ __forceinline__ Cut cut_at(const typename E::T* row, int V, bool at_border = true)      // false: pieces from column 0 on
{
    int head = at_border ? (int)((16 - ((uintptr_t)row & 15)) & 15) / (int)sizeof(typename E::T) : 0;
    head = head < V ? head : V;
    const int pieces = (V - head) / E::N;
    return Cut{head, pieces, V - pieces * E::N};
}
// column of loose element i
template <class E>
__device__ __forceinline__ int loose_column(const Cut& c, int i) { return i < c.head ? i : i + c.pieces * E::N; }

// ---------------------------------------------------------------------------
// The softmax of a row in powers of two:  2^t with t = c z - K,  K = fl(c m), m the maximum.  K need not be c m exactly: every
// use of the row takes the same K.  From |c m| = 2^30 on that would overflow; but there neighbouring numbers of any type
// are 64 apart in c z, so that only elements equal to the maximum count, and a power of two in place of c that puts c m at
// 2^31 makes K exact and keeps the others at 2^-128 (`far`).
// ---------------------------------------------------------------------------
struct Shift { float c, K; };
constexpr float FAR = 0x1p30f, T_MIN = -1e4f;
__device__ __forceinline__ bool is_far(float m, float c) { return !(fabsf(m * c) < FAR) && m != -INFINITY; }
__device__ __forceinline__ Shift shift_of(float m, float c)
{
    if (m == -INFINITY) return Shift{c, 0.0f};                          // nothing seen yet, or nothing allowed
    if (!is_far(m, c)) return Shift{c, m * c};
    if (m == INFINITY) return Shift{1.0f, m};                           // (inf - inf: the row becomes NaN)
    const int e = (int)((__float_as_uint(m) >> 23) & 0xff) - 127;
    const float p = __builtin_amdgcn_ldexpf(1.0f, 31 - e);
    return Shift{p, m * p};
}

// Sums over part of a row: s = sum 2^t, and beside it either u = sum t 2^t (the entropy) or, `fine`, u = sum r 2^t with r what
// rounding took from the exponents: there t = fl(c x), x = z - m, and r = c x - t with c to 48 bits.  r matters where thousands
// of log-probabilities are summed and two such sums subtracted.  Of 16-bit logits x is exact and r is all that was lost; of fp32
// logits x is rounded itself, which r does not hold (root mean square of what a log-sum of 3 to 1024 columns around 0 is off by,
// exponentials rounded to nearest: coarse 5 to 23e-9; fine 2 to 7e-9 with 16 bits, 3 to 9e-9 with fp32).  A number added to all of
// a row, where the type holds the sums, changes nothing.  Elements of minus infinity add 0 (their t or r enters u clamped); a NaN
// stays in s.
struct Part { float m, s, u; };
// what t changes by from one maximum to a larger one
__device__ __forceinline__ float step_between(float from, float to, float c)
{
    return fmaxf(is_far(from, c) || is_far(to, c) ? (from - to) * c : from * c - to * c, T_MIN);
}
template <bool FINE>
__device__ __forceinline__ void rescale(Part& p, float m, float c, float c_lo)      // to a larger maximum
{
    if (p.m == m || p.m == -INFINITY) { p.m = m; return; }
    float d, r = 0.0f;
    if (FINE) { const float x = p.m - m; d = fmaxf(x * c, T_MIN); r = __builtin_amdgcn_fmed3f(fmaf(x, c_lo, fmaf(x, c, -d)), -1.0f, 1.0f); }
    else d = step_between(p.m, m, c);
    const float f = __builtin_amdgcn_exp2f(d);
    p.u = f * fmaf(p.s, FINE ? r : d, p.u);
    p.s *= f;
    p.m = m;
}
// elements at shift k (coarse) or maximum m (fine); s grows by their sum, which is a tree: a thread of a long row adds a few
// dozen times and not a few hundred
template <bool FINE, int N>
__device__ __forceinline__ void add_at(Part& p, const float (&z)[N], float m, const Shift& k, float c, float c_lo)
{
    float e[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (FINE) {
            const float x = z[i] - m, t = x * c;
            e[i] = __builtin_amdgcn_exp2f(t);
            p.u = fmaf(e[i], __builtin_amdgcn_fmed3f(fmaf(x, c_lo, fmaf(x, c, -t)), -1.0f, 1.0f), p.u);
        } else {
            const float t = fmaf(z[i], k.c, -k.K);
            e[i] = __builtin_amdgcn_exp2f(t);
            p.u = fmaf(e[i], fmaxf(t, T_MIN), p.u);
        }
    }
#pragma unroll
    for (int w = 1; w < N; w *= 2)
#pragma unroll
        for (int i = 0; i + w < N; i += 2 * w) e[i] += e[i + w];
    p.s += e[0];
}
template <int N>
__device__ __forceinline__ float max_of(const float (&z)[N], float m)   // (passes over a NaN)
{
#pragma unroll
    for (int i = 0; i < N; ++i) m = fmaxf(m, z[i]);
    return m;
}
template <bool FINE, int N>
__device__ __forceinline__ void add_elements(Part& p, const float (&z)[N], float c, float c_lo)
{
    const float m = max_of(z, p.m);
    if (m > p.m) rescale<FINE>(p, m, c, c_lo);
    add_at<FINE>(p, z, m == -INFINITY ? 0.0f : m, shift_of(m, c), c, c_lo);
}

// ---- one row's numbers in 64 bits --------------------------------------------------------------------------------
__device__ __forceinline__ double reciprocal(double x)
{
    double r = __builtin_amdgcn_rcp(x);
    r = fma(fma(-x, r, 1.0), r, r);
    return fma(fma(-x, r, 1.0), r, r);
}
// ln x of a sum of exponentials: mantissa in (sqrt 1/2, sqrt 2], 2 atanh((m - 1) / (m + 1)) as a series to the 15th power
// (off by 1e-14 at most).  Other x (zero, NaN, infinite) as log has it.
__device__ __forceinline__ double log_of_sum(double x)
{
    if (!(x > 1e-30 && x < 1e30)) return x == 0.0 ? -INFINITY : x == INFINITY ? INFINITY : NAN;
    const uint64_t b = __double_as_longlong(x);
    int e = (int)(b >> 52) - 1023;
    double m = __longlong_as_double((b & 0xfffffffffffffull) | 0x3ff0000000000000ull);
    if (m > 1.4142135623730951) { m *= 0.5; e += 1; }
    const double f = (m - 1.0) * reciprocal(m + 1.0), g = f * f;
    double p = 1.0 / 15;
    p = fma(p, g, 1.0 / 13); p = fma(p, g, 1.0 / 11); p = fma(p, g, 1.0 / 9); p = fma(p, g, 1.0 / 7);
    p = fma(p, g, 1.0 / 5); p = fma(p, g, 1.0 / 3); p = fma(p, g, 1.0);
    return fma((double)e, LN2, 2.0 * f * p);
}
// e^x, its Taylor series to the 9th power around the nearest power of two (off by 1e-11 of it at most).  (A
// ratio with the roundings of single precision is what the loss of few rows was off by.)
__device__ __forceinline__ double exp_of(double x)
{
    double t = x * LOG2E;
    t = t > 1100.0 ? 1100.0 : t < -1100.0 ? -1100.0 : t;                // infinity and 0 (NaN stays)
    const double i = rint(t), f = (t - i) * LN2;
    double p = 1.0 / 362880;
    p = fma(p, f, 1.0 / 40320); p = fma(p, f, 1.0 / 5040); p = fma(p, f, 1.0 / 720); p = fma(p, f, 1.0 / 120);
    p = fma(p, f, 1.0 / 24); p = fma(p, f, 1.0 / 6); p = fma(p, f, 0.5); p = fma(p, f, 1.0); p = fma(p, f, 1.0);
    return __builtin_amdgcn_ldexp(p, (int)i);
}

// A row's sums as its workgroup or its lanes have them together, joined in 64 bits where they are long or `fine`: the roundings of
// the last few additions in 32 would be most of what is left (of `fine` ones u is in s then).
struct Sums { float m; double s, u; };

struct RowSum {
    double lse, entropy, log_s;                  // log_s: with the shift's own c
    float m; Shift k;
    float inv_s;
    bool far, empty;                             // empty: all of it minus infinity
};
template <bool FINE>
__device__ __forceinline__ RowSum finish_row(const Sums& p, const Rows& r)
{
    RowSum x{};
    const double s = p.s;
    x.m = p.m; x.far = is_far(p.m, r.c);
    x.empty = p.m == -INFINITY && s == 0.0;
    x.k = shift_of(p.m, r.c);
    if (x.empty) { x.lse = -INFINITY; return x; }
    if (FINE) {
        x.log_s = log_of_sum(s);
        x.lse = fma(r.scale, (double)p.m, x.log_s);
        // the shift of the gradient: 2^(c z - K) / s' with K = fl(c m)
        x.inv_s = (float)(reciprocal(s) * (x.far ? 1.0 : exp_of(((double)x.k.K - (double)r.c * (double)p.m) * LN2)));
        return x;
    }
    const double inv = reciprocal(s), mean_t = p.u * inv;               // E[t]
    x.log_s = log_of_sum(s);
    // c stands for scale log2 e (off by 2^-25 of it): to first order that adds  ln 2 (exact c - c) E[z]  to the log-sum-exp
    if (x.far) x.lse = fma(r.scale, (double)p.m, x.log_s);
    else x.lse = LN2 * ((double)x.k.K + r.dc * ((mean_t + (double)x.k.K) * r.inv_c)) + x.log_s;
    x.entropy = x.log_s - LN2 * fmax(mean_t, (double)T_MIN);
    x.inv_s = (float)inv;
    return x;
}
template <bool FINE>
__device__ __forceinline__ double logp_of(const RowSum& x, float z, const Rows& r)
{
    if (x.empty) return -INFINITY;
    if (FINE || x.far) return r.scale * ((double)z - (double)x.m) - x.log_s;
    return r.scale * (double)z - x.lse;
}

// Gradient of one row: element j gets 2^t (a0 + a1 t), and the target `to_target` more.  From  g ([j = a] - p_j) - e p_j (log p_j + H)
// with p_j = 2^t / s, log p_j = ln 2 t - log s:  a0 = (-g - e (H - log s)) / s,  a1 = -e ln 2 / s.
struct RowGrad { Shift k; float a0, a1, to_target; int target; };
__device__ __forceinline__ RowGrad row_gradient(const RowSum& x, double g, double e, int target, double scale)
{
    RowGrad q;
    q.k = x.k; q.target = target;
    const double k = scale * (double)x.inv_s;
    q.a0 = (float)(k * (-g - (e != 0.0 ? e * (x.entropy - x.log_s) : 0.0)));
    q.a1 = (float)(-k * e * LN2);
    q.to_target = (float)(scale * g);
    if (x.empty) q.a0 = q.a1 = q.to_target = 0.0f;
    return q;
}
template <bool ENT, int N>
__device__ __forceinline__ void gradient_of(const RowGrad& q, const float (&z)[N], float (&d)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float t = fmaf(z[i], q.k.c, -q.k.K);
        d[i] = __builtin_amdgcn_exp2f(t) * (ENT ? fmaf(q.a1, fmaxf(t, T_MIN), q.a0) : q.a0);
    }
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
