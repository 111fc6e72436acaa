// lambda-returns and advantages over sequences of unequal length:
//   G_t = r_t + disc_t ((1 - lambda) V_{t+1} + lambda G_{t+1}),  A_t = G_t - V_t,  which is the recursion
//   A_t = b_t + a_t A_{t+1},  b_t = r_t + disc_t V_{t+1} - V_t,  a_t = disc_t lambda,  0 at a sequence's last token.
// The maps x -> b + a x compose, so a long axis is cut into pieces: every thread composes the maps of 8 tokens, the
// workgroup scans them, and workgroups hand over one map each.  An a of 0 cuts: what stands behind it is never looked at,
// so sequences that lie one behind the other are one scan, and a NaN of one does not reach another.  All in 64 bits: the
// sum of a sequence cancels against its values, and the maps cost nothing beside the 16 bytes a token that are moved.
//
// returns_rows: packed and batch-major sequences are runs of rows; 2048 rows a workgroup of 256 threads.
// returns_columns: time-major; up to 32 columns (128 bytes: whole cache lines) by as many pieces of 8 steps as 1024 threads
// make, 256 steps with 32 columns.
// Where the maps of other workgroups are needed they come from a first launch of the same kernel that only composes
// (APPLY false); where they are many, carry_maps composes them in between.  Columns that fill the device by themselves walk their tiles one after another in one launch instead.
#include <math.h>
#include <initializer_list>
#include "tokens.h"

namespace ank {

constexpr int STEPS = 8;                         // tokens of a thread
constexpr int ROWS_TILE = WG * STEPS;            // rows of a workgroup
constexpr int COLS_WG = 1024, COLS_MAX = 32;     // threads of a workgroup of columns; columns at most

struct Map { double a, b; };                     // x -> b + a x
// first `l` (the earlier tokens), then `r` behind it
__device__ __forceinline__ Map composed(const Map& l, const Map& r) { return l.a == 0.0 ? l : Map{l.a * r.a, fma(l.a, r.b, l.b)}; }
__device__ __forceinline__ double applied(const Map& l, double x) { return l.a == 0.0 ? l.b : fma(l.a, x, l.b); }

struct ReturnsArgs {
    Seqs q;
    const float* reward; const void* value; const uint8_t* done; const float* bootstrap;
    double gamma, lambda;
    float *adv, *ret;
    Map* maps;                                   // of every tile: [tiles] of rows, [tiles][count] of columns
    int tiles;                                   // of the rows, or of the time axis
    int width; unsigned groups;                  // columns: of a workgroup, and how many such groups
    int walk;                                    // columns: one workgroup takes all tiles of its columns in turn
    int carried;                                 // a tile's map is that of all tiles behind it (carry_maps)
};

// The map of everything behind this thread's piece in its column of the workgroup (threads piece * W + column), and of the
// whole column from piece 0 on.  lds: [waves][W]
template <bool WHOLE>
__device__ __forceinline__ void block_maps(const Map& own, int W, Map* lds, Map& behind, Map& whole)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    Map inc = own;                                                     // this piece and those behind it in the wavefront
    for (int d = W; d < 64; d <<= 1) {
        const Map o{__shfl_down(inc.a, d, 64), __shfl_down(inc.b, d, 64)};
        if (lane + d < 64) inc = composed(inc, o);
    }
    Map next{__shfl_down(inc.a, W, 64), __shfl_down(inc.b, W, 64)};
    if (lane + W >= 64) next = Map{1.0, 0.0};
    __syncthreads();
    if (lane < W) lds[wave * W + lane] = inc;                          // the wavefront's column
    __syncthreads();
    const int col = lane % W;
    Map later{1.0, 0.0};
    for (int w = wave + 1; w < waves && later.a != 0.0; ++w) later = composed(later, lds[w * W + col]);
    behind = composed(next, later);
    if (!WHOLE) return;
    whole = lds[col];
    for (int w = 1; w < waves && whole.a != 0.0; ++w) whole = composed(whole, lds[w * W + col]);
}

// In place of every tile's map that of everything behind the tile: each tile would compose them by itself otherwise, which is
// quadratic in their number.  W columns a workgroup; a thread takes a run of tiles of one column, from the last to the first.
__global__ __launch_bounds__(COLS_WG) void carry_maps(Map* maps, const int tiles, const int64_t S, const int W)
{
    __shared__ Map lds[(COLS_WG / 64) * COLS_MAX];
    const int piece = threadIdx.x / W, pieces = blockDim.x / W, per = (tiles + pieces - 1) / pieces;
    const int64_t col = (int64_t)blockIdx.x * W + threadIdx.x % W;
    const int first = piece * per < tiles ? piece * per : tiles, end = first + per < tiles ? first + per : tiles, n = col < S ? end - first : 0;
    Map own{1.0, 0.0};
#pragma unroll 8
    for (int k = 0; k < n; ++k) own = composed(own, maps[(int64_t)(first + k) * S + col]);
    Map behind, whole;
    block_maps<false>(own, W, lds, behind, whole);
#pragma unroll 8
    for (int k = n - 1; k >= 0; --k) {
        const int64_t i = (int64_t)(first + k) * S + col;
        const Map m = maps[i];
        maps[i] = behind;
        behind = composed(m, behind);
    }
}

template <class E>
__device__ __forceinline__ void load_steps(const void* value, int64_t i0, float (&v)[STEPS])
{
    const typename E::T* p = static_cast<const typename E::T*>(value) + i0;
#pragma unroll
    for (int k = 0; k < STEPS; k += E::N) {
        float z[E::N];
        E::unpack(*reinterpret_cast<const u32x4_any*>(p + k), z);
#pragma unroll
        for (int i = 0; i < E::N; ++i) v[k + i] = z[i];
    }
}

// first sequence of packed ones that ends behind row `row`: 64 places are looked at in each round.  Offsets that do not
// ascend give some sequence, and callers check what it is.
__device__ __forceinline__ int64_t first_ending_behind(const Seqs& q, int64_t row)
{
    int64_t lo = 0, n = q.count;                                       // the answer lies in [lo, lo + n]
    const int lane = threadIdx.x & 63;
    while (n > 0) {
        const int64_t step = (n + 63) / 64, s = lo + (int64_t)(lane + 1) * step - 1;
        const bool before = s < lo + n && q.offsets[s + 1] <= row;
        const int k = __popcll(__ballot(before));                      // so many steps lie in front, if they ascend
        const int64_t at = lo + (int64_t)k * step, end = lo + n;
        if (step == 1) return at;
        lo = at < end ? at : end;
        n = end - lo < step - 1 ? end - lo : step - 1;                 // the last place of the next step is behind already
    }
    return lo;
}

template <class E, bool APPLY>
__global__ __launch_bounds__(WG) void returns_rows(const ReturnsArgs a)
{
    __shared__ Map lds[WG / 64];
    __shared__ int32_t ends[ROWS_TILE];                                // 1 + the sequence that a row is the last of, else 0
    const int64_t start = (int64_t)blockIdx.x * ROWS_TILE, i0 = start + (int64_t)threadIdx.x * STEPS, N = a.q.rows;
    const bool full = i0 + STEPS <= N;
    float r[STEPS], v[STEPS], vn = 0.0f;
    uint8_t d[STEPS];
    const typename E::T* value = static_cast<const typename E::T*>(a.value);
    if (full) {
        load_steps<Fp32>(a.reward, i0, r);
        load_steps<E>(a.value, i0, v);
    }
#pragma unroll
    for (int k = 0; k < STEPS; ++k) {
        if (!full) { r[k] = i0 + k < N ? a.reward[i0 + k] : 0.0f; v[k] = i0 + k < N ? E::get(value + i0 + k) : 0.0f; }
        d[k] = a.done && i0 + k < N ? a.done[i0 + k] : 0;
    }
    if (i0 + STEPS < N) vn = E::get(value + i0 + STEPS);
    int64_t from = 0, to = N;                                          // rows of sequences (packed)
    if (a.q.layout == ANAKIN_LAYOUT_PACKED) {
        for (int k = threadIdx.x; k < ROWS_TILE; k += WG) ends[k] = 0;
        if (a.q.count > 0) { from = a.q.offsets[0]; to = a.q.offsets[a.q.count]; } else to = 0;
        const int64_t s0 = first_ending_behind(a.q, start);
        __syncthreads();
        for (int64_t s = s0 + threadIdx.x; s < a.q.count && a.q.offsets[s] < start + ROWS_TILE; s += WG) {
            const Seq x = sequence(a.q, s);
            const int64_t e = x.first + x.n - 1 - start;
            if (x.n > 0 && e >= 0 && e < ROWS_TILE) ends[e] = (int32_t)(s + 1);
        }
        __syncthreads();
    }
    Map m[STEPS];
    float member[STEPS];
    uint32_t s = 0, j = 0;
    if (a.q.layout != ANAKIN_LAYOUT_PACKED) { s = (uint32_t)i0 / (uint32_t)a.q.length; j = (uint32_t)i0 % (uint32_t)a.q.length; }
    int64_t n = a.q.length;
    uint32_t n_of = ~0u;
    Map own{1.0, 0.0};
#pragma unroll
    for (int k = 0; k < STEPS; ++k) {
        const int64_t i = i0 + k;
        bool in, last;
        int64_t seq;
        if (a.q.layout == ANAKIN_LAYOUT_PACKED) {
            const int32_t e = ends[threadIdx.x * STEPS + k];
            in = i >= from && i < to && i < N; last = e != 0; seq = e - 1;
        } else {
            if (i < N && a.q.lengths && s != n_of) { n = sequence(a.q, s).n; n_of = s; }
            in = i < N && j < n; last = j + 1 == n; seq = s;
            if (++j == (uint32_t)a.q.length) { j = 0; ++s; }
        }
        const double disc = d[k] ? 0.0 : a.gamma, next = k + 1 < STEPS ? v[k + 1 < STEPS ? k + 1 : k] : vn;
        const double vnext = last ? (a.bootstrap && in ? (double)a.bootstrap[seq] : 0.0) : next;
        m[k].a = in && !last ? disc * a.lambda : 0.0;
        m[k].b = in ? ((double)r[k] - (double)v[k]) + (disc != 0.0 ? disc * vnext : 0.0) : 0.0;
        member[k] = in ? v[k] : 0.0f;
        own = composed(own, m[k]);
    }
    Map behind, whole;
    block_maps<!APPLY>(own, 1, lds, behind, whole);
    if (!APPLY) {
        if (threadIdx.x == 0) a.maps[blockIdx.x] = whole;
        return;
    }
    // what reaches the end of this tile: the maps of the tiles behind it, 64 at a time until one of them cuts
    Map later{1.0, 0.0};
    if (a.carried) later = a.maps[blockIdx.x];
    else for (int64_t base = (int64_t)blockIdx.x + 1; base < gridDim.x && later.a != 0.0; base += 64) {
        const int64_t t = base + (threadIdx.x & 63);
        Map c = t < gridDim.x ? a.maps[t] : Map{0.0, 0.0};             // nothing behind the last row
        for (int dist = 1; dist < 64; dist <<= 1) {
            const Map o{__shfl_down(c.a, dist, 64), __shfl_down(c.b, dist, 64)};
            if ((threadIdx.x & 63) + dist < 64) c = composed(c, o);
        }
        later = composed(later, Map{__shfl(c.a, 0, 64), __shfl(c.b, 0, 64)});
    }
    double A = applied(behind, applied(later, 0.0));
    float adv[STEPS], ret[STEPS];
#pragma unroll
    for (int k = STEPS - 1; k >= 0; --k) {
        A = applied(m[k], A);
        adv[k] = (float)A; ret[k] = (float)(A + (double)member[k]);
    }
    if (full) {
#pragma unroll
        for (int k = 0; k < STEPS; k += 4) {
            *reinterpret_cast<u32x4_any*>(a.adv + i0 + k) = Fp32::pack({adv[k], adv[k + 1], adv[k + 2], adv[k + 3]});
            *reinterpret_cast<u32x4_any*>(a.ret + i0 + k) = Fp32::pack({ret[k], ret[k + 1], ret[k + 2], ret[k + 3]});
        }
    } else {
#pragma unroll
        for (int k = 0; k < STEPS; ++k) if (i0 + k < N) { a.adv[i0 + k] = adv[k]; a.ret[i0 + k] = ret[k]; }
    }
}

// what a thread reads of its piece of a column
struct Steps { float r[STEPS], v[STEPS + 1]; uint8_t d[STEPS]; };
template <class E>
__device__ __forceinline__ void load_column(const ReturnsArgs& a, int64_t j0, int64_t n, int64_t col, Steps& x)
{
    const typename E::T* value = static_cast<const typename E::T*>(a.value);
    const int64_t S = a.q.count;
#pragma unroll
    for (int k = 0; k < STEPS; ++k) {
        const bool in = j0 + k < n;
        const int64_t i = (j0 + k) * S + col;
        x.r[k] = in ? a.reward[i] : 0.0f; x.v[k] = in ? E::get(value + i) : 0.0f; x.d[k] = in && a.done ? a.done[i] : 0;
    }
    x.v[STEPS] = j0 + STEPS < n ? E::get(value + (j0 + STEPS) * S + col) : 0.0f;
}

template <class E, bool APPLY>
__global__ __launch_bounds__(COLS_WG) void returns_columns(const ReturnsArgs a)
{
    __shared__ Map lds[(COLS_WG / 64) * COLS_MAX];
    const int W = a.width, lane_col = threadIdx.x % W, piece = threadIdx.x / W, pieces = blockDim.x / W;
    const int64_t S = a.q.count, T = a.q.length, col = (int64_t)(blockIdx.x % a.groups) * W + lane_col, tile_steps = (int64_t)pieces * STEPS;
    const int64_t my_tile = a.walk ? a.tiles - 1 : blockIdx.x / a.groups;
    const bool mine = col < S;
    const int64_t n = mine ? sequence(a.q, col).n : 0;                 // (0: nothing of a column that is not there is read)
    const double end = mine && a.bootstrap ? (double)a.bootstrap[col] : 0.0;
    Map later{1.0, 0.0};                                               // of the tiles behind
    Steps next;
    load_column<E>(a, my_tile * tile_steps + (int64_t)piece * STEPS, n, col, next);
    if (APPLY && a.carried) { if (mine) later = a.maps[my_tile * S + col]; }
    else if (APPLY && !a.walk && a.tiles > 1) {
        // of the other workgroups' maps: every piece takes its share of the tiles behind this one
        const int64_t rest = a.tiles - 1 - my_tile, per = (rest + pieces - 1) / pieces, t0 = my_tile + 1 + piece * per;
        Map c{1.0, 0.0}, behind;
        for (int64_t t = t0; t < t0 + per && t < a.tiles && mine && c.a != 0.0; ++t) c = composed(c, a.maps[t * S + col]);
        block_maps<true>(c, W, lds, behind, later);
    }
    for (int64_t tile = my_tile; tile >= 0; --tile) {
        const int64_t j0 = tile * tile_steps + (int64_t)piece * STEPS;
        const Steps x = next;
        Map m[STEPS], own{1.0, 0.0};
#pragma unroll
        for (int k = 0; k < STEPS; ++k) {
            const bool in = j0 + k < n, last = j0 + k + 1 == n;
            const double disc = x.d[k] ? 0.0 : a.gamma, vnext = last ? end : (double)x.v[k + 1];
            m[k].a = in && !last ? disc * a.lambda : 0.0;
            m[k].b = in ? ((double)x.r[k] - (double)x.v[k]) + (disc != 0.0 ? disc * vnext : 0.0) : 0.0;
            own = composed(own, m[k]);
        }
        if (a.walk && tile > 0) load_column<E>(a, j0 - tile_steps, n, col, next);      // on its way while this tile is scanned
        Map behind, whole;
        if (APPLY && !a.walk) block_maps<false>(own, W, lds, behind, whole);
        else block_maps<true>(own, W, lds, behind, whole);
        if (!APPLY) {
            if (mine && piece == 0) a.maps[tile * S + col] = whole;
            return;
        }
        double A = applied(behind, applied(later, 0.0));
#pragma unroll
        for (int k = STEPS - 1; k >= 0; --k) {
            A = applied(m[k], A);
            if (mine && j0 + k < T) { const int64_t i = (j0 + k) * S + col; a.adv[i] = (float)A; a.ret[i] = (float)(A + (double)x.v[k]); }
        }
        if (!a.walk) return;
        later = composed(whole, later);
    }
}

// Columns of a workgroup, and pieces of 8 steps: what the time axis takes, up to 32 of them where that is all of it, else 16
// (two workgroups to a compute unit).
struct ColumnForm { int width, pieces; int64_t groups, tiles; bool walk; };
static ColumnForm column_form(int64_t count, int64_t length)
{
    ColumnForm f{1, 1, 0, 0, false};
    while (f.width < COLS_MAX && f.width < count) f.width *= 2;
    const int most = length <= 32 * STEPS ? 32 : 16;
    while (f.pieces * f.width < 64 || (f.pieces < most && f.pieces * STEPS < length) || (f.width < COLS_MAX && f.pieces * f.width < 256)) f.pieces *= 2;
    f.groups = (count + f.width - 1) / f.width;
    f.tiles = (length + f.pieces * STEPS - 1) / (f.pieces * STEPS);
    // columns that give every compute unit a workgroup walk their tiles in one launch; fewer share the tiles out in two
    f.walk = f.tiles > 1 && f.groups >= 256;
    return f;
}

// A tile looks at the maps behind it in rounds, of 64 of them or of as many as a column has pieces; above so many rounds a launch
// more that looks at them once is faster (us without and with: one sequence of 2^21 tokens 32 and 31, of 2^22 72 and 37, of 2^26 9600
// and 380; time-major, 64 columns: 2^22 tokens 42 and 45, 2^24 243 and 131; 1024 columns, 2^26 tokens 611 and 487)
constexpr int CARRY_FROM = 16;
static hipError_t launch_carry(const ReturnsArgs& a, int64_t columns, int W, hipStream_t s)
{
    hipLaunchKernelGGL(carry_maps, dim3((unsigned)((columns + W - 1) / W)), dim3(COLS_WG), 0, s, a.maps, a.tiles, columns, W);
    return hipGetLastError();
}

template <class E>
static hipError_t launch_returns_of(ReturnsArgs& a, hipStream_t s)
{
    if (a.q.layout == ANAKIN_LAYOUT_TIME) {
        const ColumnForm f = column_form(a.q.count, a.q.length);
        a.width = f.width; a.tiles = (int)f.tiles; a.walk = f.walk; a.groups = (unsigned)f.groups;
        const dim3 grid(a.groups * (f.walk ? 1u : (unsigned)f.tiles)), block(f.width * f.pieces);
        if (!f.walk && f.tiles > 1) {
            hipLaunchKernelGGL((returns_columns<E, false>), grid, block, 0, s, a);
            hipError_t e = hipGetLastError();
            a.carried = f.tiles > CARRY_FROM * f.pieces;
            if (e == hipSuccess && a.carried) e = launch_carry(a, a.q.count, f.width, s);
            if (e != hipSuccess) return e;
        }
        hipLaunchKernelGGL((returns_columns<E, true>), grid, block, 0, s, a);
        return hipGetLastError();
    }
    a.tiles = (int)((a.q.rows + ROWS_TILE - 1) / ROWS_TILE);
    if (a.tiles > 1) {
        hipLaunchKernelGGL((returns_rows<E, false>), dim3(a.tiles), dim3(WG), 0, s, a);
        hipError_t e = hipGetLastError();
        a.carried = a.tiles > CARRY_FROM * 64;
        if (e == hipSuccess && a.carried) e = launch_carry(a, 1, 1, s);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((returns_rows<E, true>), dim3(a.tiles), dim3(WG), 0, s, a);
    return hipGetLastError();
}

}  // namespace ank

using namespace ank;

static bool overlaps(const void* p, size_t np, const void* q, size_t nq)
{
    const uintptr_t a = (uintptr_t)p, b = (uintptr_t)q;
    return p && q && np && nq && a < b + nq && b < a + np;
}

extern "C" size_t anakin_returns_workspace_bytes(int64_t rows, int64_t count)
{
    if (rows < 0 || rows > MAX_ROWS || count < 0 || count > MAX_ROWS) return 0;
    // a map for every tile of rows, or for every tile of every column (time-major: rows / count steps)
    const size_t by_rows = (size_t)((rows + ROWS_TILE - 1) / ROWS_TILE);
    size_t by_columns = 0;
    if (count > 0 && rows % count == 0) { const ColumnForm f = column_form(count, rows / count); by_columns = f.walk ? 0 : (size_t)(f.tiles * count); }
    return up256((by_rows > by_columns ? by_rows : by_columns) * sizeof(Map)) + 256;
}

extern "C" int32_t anakin_lambda_returns(const anakin_sequences* q, const anakin_returns_args* a, void* d_workspace, size_t workspace_bytes, void* hip_stream)
{
    if (!a) return fail(ANAKIN_E_INVALID_ARG, "null arguments");
    if (a->rows < 0 || a->rows > MAX_ROWS) return fail(ANAKIN_E_INVALID_ARG, "rows out of range");
    const int32_t rc = check_sequences(q, a->rows);
    if (rc != ANAKIN_OK) return rc;
    if (a->value_type < ANAKIN_TYPE_FP32 || a->value_type > ANAKIN_TYPE_FP16) return fail(ANAKIN_E_INVALID_ARG, "unknown type of the values");
    if (!(a->gamma >= 0.0 && a->gamma <= 1.0) || !(a->lambda_ >= 0.0 && a->lambda_ <= 1.0)) return fail(ANAKIN_E_INVALID_ARG, "gamma and lambda have to lie in [0, 1]");
    if (a->rows > 0 && (!a->d_reward || !a->d_value || !a->d_adv || !a->d_ret)) return fail(ANAKIN_E_INVALID_ARG, "null rewards, values, adv or ret");
    const size_t n = (size_t)a->rows;
    for (const float* out : {a->d_adv, a->d_ret})
        if (overlaps(out, n * 4, a->d_reward, n * 4) || overlaps(out, n * 4, a->d_value, n * (a->value_type == ANAKIN_TYPE_FP32 ? 4 : 2)) || overlaps(out, n * 4, a->d_done, n) ||
            overlaps(out, n * 4, a->d_bootstrap, (size_t)q->count * 4) || overlaps(a->d_adv, n * 4, a->d_ret, n * 4))
            return fail(ANAKIN_E_INVALID_ARG, "adv and ret have to be apart from the inputs and from each other");
    const int32_t rw = check_workspace(d_workspace, workspace_bytes, anakin_returns_workspace_bytes(a->rows, q->count));
    if (rw != ANAKIN_OK) return rw;
    if (a->rows == 0) return ANAKIN_OK;
    ReturnsArgs k{};
    k.q = Seqs{q->layout, q->count, q->length, a->rows, q->d_offsets, q->d_lengths};
    if (q->layout == ANAKIN_LAYOUT_TIME && (q->count == 1 || q->length == 1)) k.q.layout = ANAKIN_LAYOUT_BATCH;      // the same rows
    k.reward = a->d_reward; k.value = a->d_value; k.done = a->d_done; k.bootstrap = a->d_bootstrap; k.gamma = a->gamma; k.lambda = a->lambda_;
    k.adv = a->d_adv; k.ret = a->d_ret; k.maps = static_cast<Map*>(d_workspace);
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    const hipError_t e = a->value_type == ANAKIN_TYPE_FP32 ? launch_returns_of<Fp32>(k, s) : a->value_type == ANAKIN_TYPE_BF16 ? launch_returns_of<Bf16>(k, s) : launch_returns_of<Fp16>(k, s);
    return e == hipSuccess ? ANAKIN_OK : fail_hip(e);
}
