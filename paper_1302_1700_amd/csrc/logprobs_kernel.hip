// Log probabilities of labels, entropy and best classes of rows of scores, and
// their gradient.
//
// With m the row's maximum, d_j = (x_j - m) / T <= 0, S = sum exp(d_j) and
// D = sum exp(d_j) d_j: log p_j = d_j - ln S and the entropy is ln S - D / S,
// two terms >= 0, so nothing cancels where the scores are far from 0.  The
// kernels keep d in units of log2 (one factor k = log2(e) / T, the hardware's
// exp2) and D with it.  Every row is read once; of a long row whose best classes
// are listed, the scores of the threads that may hold them a second time.
//
// A score of -inf has exp 0; its d is held at -1e30 where it multiplies that 0.
// Maxima start from the lowest finite float, so -inf never meets -inf; S = 0
// then says that a row is empty, and a NaN or +inf makes S a NaN by itself.
#include <algorithm>
#include <type_traits>

#include "rows.h"

namespace fs {
namespace {

constexpr float kLowest = -3.402823466e38f;
constexpr double kLog2eExact = 1.4426950408889634;  // log2(e) = 1 / ln 2, to 53 bits
constexpr float kLog2e = (float)kLog2eExact, kLn2 = 0.693147180559945f;
constexpr float kLog2eRest = (float)(kLog2eExact - (double)kLog2e);  // what float32 leaves of it
constexpr float kFar = -1e30f;

// Elements per 16-byte load: rows start anywhere their element type may.
template <typename T>
constexpr int kVec = 16 / sizeof(T);

template <typename T, int N>
__device__ __forceinline__ void load_run(const T *p, float *v)
{
    unpack<T, N>(load_words<N * sizeof(T)>(p), v);
}

// Scores in the order of their values, equal ones by their class: the float as
// an unsigned number that compares alike (-0 as 0), then the class reversed.
// 0 stands for no class.
__device__ __forceinline__ uint64_t score_key(float v, uint32_t id)
{
    const uint32_t u = __float_as_uint(v + 0.0f);
    const uint32_t s = u & 0x80000000u ? ~u : u | 0x80000000u;
    return ((uint64_t)s << 32) | (0xffffffffu - id);
}
__device__ __forceinline__ float key_score(uint64_t k)
{
    const uint32_t s = (uint32_t)(k >> 32);
    return __uint_as_float(s & 0x80000000u ? s & 0x7fffffffu : ~s);
}
__device__ __forceinline__ int key_id(uint64_t k) { return (int)(0xffffffffu - (uint32_t)k); }

template <int G, typename T>
__device__ __forceinline__ T group_max(T v)
{
#pragma unroll
    for (int d = G / 2; d; d >>= 1) {
        const T o = __shfl_xor(v, d);
        v = o > v ? o : v;
    }
    return v;
}
template <int G>
__device__ __forceinline__ float group_sum(float v)
{
#pragma unroll
    for (int d = G / 2; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

// What is known of a part of a row: maximum, S and D relative to it.
struct Part {
    float m, s, d;
};

// A part seen from a larger maximum.
__device__ __forceinline__ void move_to(Part &p, float m, float k)
{
    const float t = fmaxf((p.m - m) * k, kFar);
    const float c = __builtin_amdgcn_exp2f(t);
    p.d = c * fmaf(p.s, t, p.d);
    p.s *= c;
    p.m = m;
}

template <int G>
__device__ __forceinline__ Part group_join(Part p, float k)
{
    move_to(p, group_max<G>(p.m), k);
    p.s = group_sum<G>(p.s);
    p.d = group_sum<G>(p.d);
    return p;
}

// A row's statistics as they are stored.
struct RowStats {
    float m, log_s, entropy;
    bool bad, empty;
};

__device__ __forceinline__ RowStats finish(const Part &p)
{
    RowStats r;
    r.bad = !(p.s >= 0.f);
    r.empty = p.s == 0.f;
    r.m = r.bad ? NAN : r.empty ? -INFINITY : p.m;
    r.log_s = r.bad ? NAN : r.empty ? 0.f : logf(p.s);
    r.entropy = r.bad ? NAN : r.empty ? 0.f : r.log_s - p.d * kLn2 / p.s;
    return r;
}

__device__ __forceinline__ float label_logp(const RowStats &r, int y, int V, float xy, float inv_t)
{
    if (y < 0) return 0.f;
    if (y >= V || r.bad) return NAN;
    return r.empty ? -INFINITY : (xy - r.m) * inv_t - r.log_s;
}

__device__ __forceinline__ void store_stats(const LogprobArgs &a, int64_t row, const RowStats &r, int y, float xy)
{
    if (a.norm) {
        const float v[2] = {r.m, r.log_s};
        store_words<8>(a.norm + 2 * row, pack<float, 2>(v));
    }
    if (a.entropy) a.entropy[row] = r.entropy;
    if (a.logp) a.logp[row] = label_logp(r, y, a.V, xy, a.inv_t);
}

__device__ __forceinline__ void store_top(const LogprobArgs &a, int64_t row, int place, const RowStats &r, uint64_t key)
{
    const bool none = r.bad || key == 0;
    if (a.top_id) a.top_id[row * a.n_top + place] = none ? -1 : key_id(key);
    if (a.top_logp)
        a.top_logp[row * a.n_top + place] =
            r.bad ? NAN : none ? -INFINITY : (key_score(key) - r.m) * a.inv_t - r.log_s;
}

// Short rows: G lanes hold a row in registers, C chunks of N scores each (lane
// l of the group: chunks l, l + G, ...), 64 / G rows a wave.  The best classes
// are taken out one after the other, a group maximum each.
template <typename T, int G, int C, int N>
__global__ __launch_bounds__(256) void logprobs_short(LogprobArgs a)
{
    const int sub = threadIdx.x % G;
    const int V = a.V;
    const float k = a.inv_t * kLog2e;
    for (int64_t row = (int64_t)blockIdx.x * (256 / G) + threadIdx.x / G; row < a.rows;
         row += (int64_t)gridDim.x * (256 / G)) {
        const T *x = reinterpret_cast<const T *>(a.x) + row * a.stride;
        const int y = a.logp ? a.labels[row] : -1;
        float v[C * N];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int j = (c * G + sub) * N;
            if (j + N <= V) load_run<T, N>(x + j, v + c * N);
            else {
#pragma unroll
                for (int e = 0; e < N; ++e) v[c * N + e] = j + e < V ? to_f32(x[j + e]) : -INFINITY;
            }
        }
        const float xy = y >= 0 && y < V ? to_f32(x[y]) : 0.f;
        Part p{kLowest, 0.f, 0.f};
#pragma unroll
        for (int e = 0; e < C * N; ++e) p.m = fmaxf(p.m, v[e]);
        p.m = group_max<G>(p.m);
#pragma unroll
        for (int e = 0; e < C * N; ++e) {
            const float t = (v[e] - p.m) * k, w = __builtin_amdgcn_exp2f(t);
            p.s += w;
            p.d = fmaf(w, fmaxf(t, kFar), p.d);
        }
        p.s = group_sum<G>(p.s);
        p.d = group_sum<G>(p.d);
        const RowStats r = finish(p);
        if (sub == 0) store_stats(a, row, r, y, xy);
        for (int place = 0; place < a.n_top; ++place) {
            uint64_t best = 0;
#pragma unroll
            for (int e = 0; e < C * N; ++e) {
                const uint64_t key = score_key(v[e], (uint32_t)((e / N * G + sub) * N + e % N));
                if (v[e] != -INFINITY && key > best) best = key;
            }
            best = group_max<G>(best);
            if (sub == 0) store_top(a, row, place, r, best);
            const int id = best ? key_id(best) : -1;
#pragma unroll
            for (int e = 0; e < C * N; ++e)
                if ((e / N * G + sub) * N + e % N == id) v[e] = -INFINITY;
        }
    }
}

__device__ __forceinline__ float lane_value(float v, int lane)
{
    return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), lane));
}

// The n-th and the k-th largest of the wave's values (n, k <= 64), equal ones
// counted each: the smallest value that fewer than n (k) exceed.
__device__ __forceinline__ void nth_largest(float v, int n, int k, float *nth, float *kth)
{
    int above = 0;
#pragma unroll
    for (int o = 0; o < 64; ++o) above += lane_value(v, o) > v ? 1 : 0;
    float a = above < n ? v : INFINITY, b = above < k ? v : INFINITY;
#pragma unroll
    for (int d = 32; d; d >>= 1) {
        a = fminf(a, __shfl_xor(a, d));
        b = fminf(b, __shfl_xor(b, d));
    }
    *nth = a;
    *kth = b;
}

// Joins sorted lists of n keys each (in LDS, `lists` of them, 0 past their
// ends): a key's place is its own index plus the number of larger keys in each
// other list.  Threads of the block take keys in turn; writes the n best.
__device__ __forceinline__ void join_lists(const LogprobArgs &a, int64_t row, const RowStats &r, const uint64_t *keys,
                                           int lists)
{
    const int n = a.n_top;
    for (int q = threadIdx.x; q < lists * n; q += blockDim.x) {
        const int mine = q / n;
        const uint64_t key = keys[q];
        int place = q - mine * n;
        if (key == 0) {
            // nobody's: the places behind all classes that are listed anywhere
            if (mine != 0) continue;
            for (int l = 1; l < lists; ++l) {
                int lo = 0, hi = n;
                while (lo < hi) {
                    const int mid = (lo + hi) / 2;
                    if (keys[l * n + mid] != 0) lo = mid + 1;
                    else hi = mid;
                }
                place += lo;
            }
            if (place < n) store_top(a, row, place, r, 0);
            continue;
        }
        for (int l = 0; l < lists && place < n; ++l) {
            if (l == mine) continue;
            int lo = 0, hi = n;
            while (lo < hi) {
                const int mid = (lo + hi) / 2;
                if (keys[l * n + mid] > key) lo = mid + 1;
                else hi = mid;
            }
            place += lo;
        }
        if (place < n) store_top(a, row, place, r, key);
    }
}

// The best classes of a long row, or of a run of it, that the threads of a
// workgroup have just gone through (element (i W + wave) U + u, times 64, plus
// lane, is the i U + u-th run of N scores of a thread).  Every thread knows its
// largest score.  n scores reach the n-th largest of these in a wave, and n / W
// of every wave the (n / W)-th largest of its own: the larger of the best of the
// first and the worst of the second bounds the n best from below, so only the
// few threads whose largest reaches it hold any of them.  Their scores are read
// once more, a run a thread, and those that reach the bound are listed as keys
// and placed by counting larger keys.  Where more than the list holds reach it (equal scores,
// or many of the best in one thread's hands) the list is cut to its n best and
// its last key is the new bound, as often as it takes.
constexpr int kList = 1024;  // a wave's runs hold up to 512

template <int W>
struct TopLds {
    uint64_t list[kList + 64], sorted[64];
    int flagged[64 * W], counts[W];
    float one[W], all[W];  // the waves' bounds
};

template <typename T, int W, int U>
__device__ __forceinline__ int find_top(TopLds<W> &l, const T *x, int first, int V, float largest, int n)
{
    constexpr int N = kVec<T>, NT = 64 * W;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    __syncthreads();  // the unit before has been read
    float nth, share;
    nth_largest(largest, n, (n + W - 1) / W, &nth, &share);
    if (lane == 0) {
        l.one[wave] = nth;
        l.all[wave] = share;
    }
    __syncthreads();
    nth = l.one[0];
    share = l.all[0];
#pragma unroll
    for (int w = 1; w < W; ++w) {
        nth = fmaxf(nth, l.one[w]);
        share = fminf(share, l.all[w]);
    }
    const float t = fmaxf(nth, share);
    const uint64_t mine = __ballot(largest >= t && largest > -INFINITY);
    if (lane == 0) l.counts[wave] = __popcll(mine);
    __syncthreads();
    int holders = 0, before = 0;
    for (int w = 0; w < W; ++w) {
        before += w < wave ? l.counts[w] : 0;
        holders += l.counts[w];
    }
    if (mine >> lane & 1) l.flagged[before + __popcll(mine & ((1ull << lane) - 1))] = threadIdx.x;
    // keys above `cut` are wanted: scores of at least t, none of -inf
    uint64_t cut = t == -INFINITY ? score_key(-INFINITY, 0) : score_key(t, 0xffffffffu) - 1;
    const int batches = (V - first + U * 64 * N - 1) / (U * 64 * N), runs = (batches + W - 1) / W * U;
    int length = 0;
    // places of the list's keys among all; keeps the n best
    auto shorten = [&]() {
        __syncthreads();
        for (int q = threadIdx.x; q < length; q += NT) {
            const uint64_t key = l.list[q];
            int place = 0;
#pragma unroll 8
            for (int o = 0; o < length; ++o) place += l.list[o] > key ? 1 : 0;
            if (place < n) l.sorted[place] = key;
        }
        __syncthreads();
        length = min(length, n);
        if ((int)threadIdx.x < length) l.list[threadIdx.x] = l.sorted[threadIdx.x];
        __syncthreads();
        if (length == n) cut = max(cut, l.list[n - 1]);
    };
    __syncthreads();
    for (int at = 0; at < holders * runs; at += NT) {
        const int item = at + (int)threadIdx.x;
        int j = V;
        if (item < holders * runs) {
            const int run = item / holders, who = l.flagged[item - run * holders];
            const int64_t piece = (int64_t)(run / U * W + (who >> 6)) * U + run % U;
            j = (int)min((int64_t)V, first + (piece * 64 + (who & 63)) * N);
        }
        float v[N];
        if (j + N <= V) load_run<T, N>(x + j, v);
        else {
#pragma unroll
            for (int e = 0; e < N; ++e) v[e] = j + e < V ? to_f32(x[j + e]) : -INFINITY;
        }
        bool pending = true;  // this wave's runs still have to be listed
        for (;;) {
            int found = 0;
#pragma unroll
            for (int e = 0; e < N; ++e) found += __popcll(__ballot(pending && score_key(v[e], (uint32_t)(j + e)) > cut));
            if (lane == 0) l.counts[wave] = found;
            __syncthreads();
            int start = length, to = length, left = 0;
            for (int w = 0; w < W; ++w) {
                const int c = l.counts[w];
                if (to + c <= kList) {  // as many waves as fit, in order
                    start += w < wave ? c : 0;
                    to += c;
                } else {
                    left = 1;
                    if (w <= wave) start = -1;
                    break;
                }
            }
            __syncthreads();
            if (start >= 0 && pending) {
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const uint64_t key = score_key(v[e], (uint32_t)(j + e));
                    const uint64_t hit = __ballot(key > cut);
                    if (hit >> lane & 1) l.list[start + __popcll(hit & ((1ull << lane) - 1))] = key;
                    start += __popcll(hit);
                }
                pending = false;
            }
            length = to;
            if (!left) break;
            shorten();
        }
    }
    shorten();
    return length;
}

// What a split of a row leaves for the join: its part, then its keys.
__host__ __device__ __forceinline__ size_t split_bytes(int n_top) { return 16 + 8 * (size_t)n_top; }

// Long rows: W waves to a row, or to one of `splits` runs of it, each going
// through batches of U * 64 * N scores, W batches apart, the next batch's
// loads in flight.  A lane keeps its own maximum and sums, moved to the larger
// maximum once a batch.
template <typename T, int W, int U, bool TOP>
__global__ __launch_bounds__(64 * W) void logprobs_long(LogprobArgs a, int splits, int per_split, char *parts)
{
    constexpr int N = kVec<T>, BATCH = U * 64 * N;
    __shared__ Part lds_part[W];
    __shared__ TopLds<TOP ? W : 1> top;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const float k = a.inv_t * kLog2e;
    const int n = TOP ? a.n_top : 0;
    const int64_t units = a.rows * splits;
    for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
        int64_t row = unit;
        int first = 0;
        if (splits > 1) {
            row = unit / splits;
            first = (int)(unit - row * splits) * per_split;
        }
        const int V = min(a.V, first + per_split);  // this run's end
        const T *x = reinterpret_cast<const T *>(a.x) + row * a.stride;
        const int y = a.logp ? a.labels[row] : -1;
        const float xy = y >= 0 && y < a.V ? to_f32(x[y]) : 0.f;

        Part p{kLowest, 0.f, 0.f};
        float largest = -INFINITY;
        typename Words<16>::type next[U];
        auto fetch = [&](int at) {
            if (at + BATCH <= V) {
#pragma unroll
                for (int u = 0; u < U; ++u) next[u] = load_words<16>(x + at + (u * 64 + lane) * N);
                return;
            }
            for (int u = 0; u < U; ++u) {
                const int j = at + (u * 64 + lane) * N;
                typename Words<16>::type w;
                if (j + N <= V) w = load_words<16>(x + j);
                else {
                    float part[N];
#pragma unroll
                    for (int e = 0; e < N; ++e) part[e] = j + e < V ? to_f32(x[j + e]) : -INFINITY;
                    w = pack<T, N>(part);
                }
#pragma unroll
                for (int o = 0; o < U; ++o) next[o] = o == u ? w : next[o];
            }
        };
        int at = first + wave * BATCH;
        if (at < V) fetch(at);
        for (; at < V; at += W * BATCH) {
            float v[U * N];
#pragma unroll
            for (int u = 0; u < U; ++u) unpack<T, N>(next[u], v + u * N);
            if (at + W * BATCH < V) fetch(at + W * BATCH);
#pragma unroll
            for (int e = 0; e < U * N; ++e) largest = fmaxf(largest, v[e]);
            move_to(p, fmaxf(p.m, largest), k);
#pragma unroll
            for (int e = 0; e < U * N; ++e) {
                const float t = (v[e] - p.m) * k, w = __builtin_amdgcn_exp2f(t);
                p.s += w;
                p.d = fmaf(w, fmaxf(t, kFar), p.d);
            }
        }
        p = group_join<64>(p, k);
        if constexpr (W > 1) {
            __syncthreads();  // the unit before has been read
            if (lane == 0) lds_part[wave] = p;
            __syncthreads();
            Part q{kLowest, 0.f, 0.f};
            if (lane < W) q = lds_part[lane];
            p = group_join<64>(q, k);
        }
        RowStats r = finish(p);
        int listed = 0;
        if constexpr (TOP)
            if (!r.bad && !r.empty) listed = find_top<T, W, U>(top, x, first, V, largest, n);
        if (splits > 1) {
            char *to = parts + unit * split_bytes(a.n_top);
            if (threadIdx.x == 0) *reinterpret_cast<Part *>(to) = p;
            if constexpr (TOP)
                if ((int)threadIdx.x < n)
                    reinterpret_cast<uint64_t *>(to + 16)[threadIdx.x] =
                        (int)threadIdx.x < listed ? top.list[threadIdx.x] : 0;
            continue;
        }
        if (threadIdx.x == 0) store_stats(a, row, r, y, xy);
        if constexpr (TOP)
            if ((int)threadIdx.x < n)
                store_top(a, row, threadIdx.x, r, (int)threadIdx.x < listed ? top.list[threadIdx.x] : 0);
    }
}

// Joins the splits of a row (at most 64).
template <typename T>
__global__ __launch_bounds__(256) void logprobs_join(LogprobArgs a, int splits, const char *parts)
{
    extern __shared__ uint64_t lds_keys[];  // [splits][n_top]
    const float k = a.inv_t * kLog2e;
    const int lane = threadIdx.x & 63, n = a.n_top;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const char *from = parts + row * splits * split_bytes(n);
        Part p{kLowest, 0.f, 0.f};
        if (lane < splits) p = *reinterpret_cast<const Part *>(from + lane * split_bytes(n));
        __syncthreads();  // the row before has been read
        for (int q = threadIdx.x; q < splits * n; q += 256)
            lds_keys[q] = reinterpret_cast<const uint64_t *>(from + q / n * split_bytes(n) + 16)[q % n];
        __syncthreads();
        const RowStats r = finish(group_join<64>(p, k));
        if (threadIdx.x == 0) {
            const T *x = reinterpret_cast<const T *>(a.x) + row * a.stride;
            const int y = a.logp ? a.labels[row] : -1;
            store_stats(a, row, r, y, y >= 0 && y < a.V ? to_f32(x[y]) : 0.f);
        }
        if (n) join_lists(a, row, r, lds_keys, splits);
    }
}

// -- gradient ------------------------------------------------------------------
// e^x = 2^(x log2 e) = 2^t 2^r for any t + r = x log2 e.  t is the product as
// float32 rounds it and r what that leaves: the product's own error, which a
// fused multiply-add gives exactly (Ogita, Rump, Oishi 2005, TwoProductFMA), plus x
// times what float32 leaves of log2 e.  |r| is below 2^-15 at |x| <= 200, so
// 2^r is 1 + r ln 2, the first terms of its series, to 2^-31.  The result is
// off by its own roundings, not by |x| times them as exp2 of t alone is.
__device__ __forceinline__ float exp_exact(float x)
{
    const float y = fmaxf(x, -200.f), t = y * kLog2e;
    const float r = fmaf(y, kLog2e, -t) + y * kLog2eRest;
    const float e = __builtin_amdgcn_exp2f(t);
    return x != x ? x : fmaf(e, r * kLn2, e);
}

// What the elements of a row's gradient share.
struct GradRow {
    float m, log_s, gl, ge, ent, inv_t;
    int y;
    bool zero;
    __device__ __forceinline__ GradRow(const LogprobGradArgs &a, int64_t row)
    {
        float nm[2];
        load_run<float, 2>(a.norm + 2 * row, nm);
        y = a.labels ? a.labels[row] : -1;
        gl = y >= 0 ? a.g_logp[row] : 0.f;
        ge = a.g_entropy ? a.g_entropy[row] : 0.f;
        ent = a.g_entropy ? a.entropy[row] : 0.f;
        inv_t = a.inv_t;
        m = y >= a.V ? NAN : nm[0];
        log_s = nm[1];
        zero = m == -INFINITY;
    }
    template <bool EXACT>
    __device__ __forceinline__ float at(float x, int j) const
    {
        const float lp = (x - m) * inv_t - log_s;
        const float p = EXACT ? exp_exact(lp) : __expf(lp);
        const float v = gl * ((j == y ? 1.f : 0.f) - p) - ge * p * (fmaxf(lp, kFar) + ent);
        return zero ? 0.f : v * inv_t;
    }
};

template <typename T, int N>
__device__ __forceinline__ void grad_run(const GradRow &r, const T *x, T *g, int j, int V)
{
    if (j + N <= V) {
        float v[N];
        load_run<T, N>(x + j, v);
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = r.at<sizeof(T) == 4>(v[e], j + e);
        store_words<N * sizeof(T)>(g + j, pack<T, N>(v));
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (j + e < V) store_as(g + j + e, r.at<sizeof(T) == 4>(to_f32(x[j + e]), j + e));
    }
}

// Short rows: G lanes to a row, a chunk of N scores each.
template <typename T, int G, int N>
__global__ __launch_bounds__(256) void logprobs_grad_short(LogprobGradArgs a)
{
    for (int64_t row = (int64_t)blockIdx.x * (256 / G) + threadIdx.x / G; row < a.rows;
         row += (int64_t)gridDim.x * (256 / G)) {
        const GradRow r(a, row);
        const T *x = reinterpret_cast<const T *>(a.x) + row * a.stride;
        T *g = reinterpret_cast<T *>(a.g) + row * a.g_stride;
        for (int j = threadIdx.x % G * N; j < a.V; j += G * N) grad_run<T, N>(r, x, g, j, a.V);
    }
}

// Long rows: a workgroup to a piece of kU chunks a thread.
constexpr int kU = 4;

template <typename T>
__global__ __launch_bounds__(256) void logprobs_grad_long(LogprobGradArgs a, int pieces)
{
    constexpr int N = kVec<T>;
    const int64_t units = a.rows * pieces;
    for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
        const int64_t row = unit / pieces;
        const int j0 = (int)(unit - row * pieces) * kU * 256 * N;
        const GradRow r(a, row);
        const T *x = reinterpret_cast<const T *>(a.x) + row * a.stride;
        T *g = reinterpret_cast<T *>(a.g) + row * a.g_stride;
#pragma unroll
        for (int u = 0; u < kU; ++u) grad_run<T, N>(r, x, g, j0 + (u * 256 + (int)threadIdx.x) * N, a.V);
    }
}

int capped(int64_t blocks) { return (int)std::max<int64_t>(1, std::min<int64_t>(blocks, 1 << 22)); }

// -- choices -------------------------------------------------------------------
// Classes a wave's registers hold at 8 a lane.  20,000 x 500 float32: 12 us, as
// long rows of one wave 18; the best one 16 and 35, the 5 best 30 and 37, the 64
// best, a group maximum each, 242 and 198 (20,000 x 400 bf16: 239 and 412).
constexpr int kShort = 512;

struct LongPlan {
    int waves, splits, per_split;
};

constexpr int kBatch = 4;  // chunks of a batch

// One wave to a row where its share of the row's fixed costs weighs more than
// the wait for it: 4000 x 8192 bf16, 5 best: 22 us, with four waves 37; 4000 x
// 32768: 65 and 57.  Where rows are few and long, runs of eight batches joined by
// a second launch (4 x 131072 float32, 5 best: 15.5 us, whole 22.6; shorter ones
// do not repay it: 64 x 16384 float32 12 us, whole 8.7).
LongPlan long_plan(int64_t rows, int V, int dtype)
{
    const int batch = kBatch * 64 * (dtype == DT_BF16 ? 8 : 4);
    LongPlan p{V <= 2 * batch || (rows > 512 && V <= 8192) ? 1 : 4, 1, V};
    if (rows <= 512 && V > 24 * batch) {
        const int most = (int)std::min<int64_t>(64, std::max<int64_t>(1, 512 / rows));
        p.splits = std::min(most, (V + 8 * batch - 1) / (8 * batch));
        if (p.splits > 1) {
            p.per_split = ((V + p.splits - 1) / p.splits + 7) / 8 * 8;
            p.splits = (V + p.per_split - 1) / p.per_split;
        }
    }
    return p;
}

template <typename T, int G, int C, int N>
hipError_t go_short(const LogprobArgs &a, hipStream_t s)
{
    hipLaunchKernelGGL((logprobs_short<T, G, C, N>), dim3(capped((a.rows + 256 / G - 1) / (256 / G))), dim3(256), 0, s, a);
    return hipGetLastError();
}

template <typename T, int W, int U>
hipError_t go_long(const LogprobArgs &a, const LongPlan &p, char *parts, hipStream_t s)
{
    const dim3 grid(capped(a.rows * p.splits)), block(64 * W);
    if (a.n_top) hipLaunchKernelGGL((logprobs_long<T, W, U, true>), grid, block, 0, s, a, p.splits, p.per_split, parts);
    else hipLaunchKernelGGL((logprobs_long<T, W, U, false>), grid, block, 0, s, a, p.splits, p.per_split, parts);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.splits == 1) return e;
    hipLaunchKernelGGL(logprobs_join<T>, dim3(capped(a.rows)), dim3(256), (size_t)p.splits * a.n_top * 8, s, a, p.splits,
                       (const char *)parts);
    return hipGetLastError();
}

template <typename T>
hipError_t run(const LogprobArgs &a, int dtype, char *parts, hipStream_t s)
{
    constexpr int N = kVec<T>, C = 8 / N;  // 8 scores a lane
    const int V = a.V;
    if (V <= 2) return go_short<T, 1, 1, 2>(a, s);
    if (V <= 4) return go_short<T, 1, 1, 4>(a, s);
    if (V <= 8) return go_short<T, 1, C, N>(a, s);
    if (V <= 16) return go_short<T, 2, C, N>(a, s);
    if (V <= 32) return go_short<T, 4, C, N>(a, s);
    if (V <= 64) return go_short<T, 8, C, N>(a, s);
    if (V <= 128) return go_short<T, 16, C, N>(a, s);
    if (V <= 256) return go_short<T, 32, C, N>(a, s);
    if (V <= kShort) return go_short<T, 64, C, N>(a, s);
    const LongPlan p = long_plan(a.rows, V, dtype);
    if (p.waves == 1) return go_long<T, 1, kBatch>(a, p, parts, s);
    return go_long<T, 4, kBatch>(a, p, parts, s);
}

template <typename T, int G, int N>
hipError_t go_grad(const LogprobGradArgs &a, hipStream_t s)
{
    hipLaunchKernelGGL((logprobs_grad_short<T, G, N>), dim3(capped((a.rows + 256 / G - 1) / (256 / G))), dim3(256), 0, s, a);
    return hipGetLastError();
}

template <typename T>
hipError_t run_grad(const LogprobGradArgs &a, hipStream_t s)
{
    constexpr int N = kVec<T>;
    const int V = a.V;
    if (V <= 2) return go_grad<T, 1, 2>(a, s);
    if (V <= 4) return go_grad<T, 1, 4>(a, s);
    if (V <= 2 * N) return go_grad<T, 2, N>(a, s);
    if (V <= 4 * N) return go_grad<T, 4, N>(a, s);
    if (V <= 8 * N) return go_grad<T, 8, N>(a, s);
    if (V <= 32 * N) return go_grad<T, 16, N>(a, s);
    if (V <= 256 * N) return go_grad<T, 64, N>(a, s);
    const int pieces = (V + kU * 256 * N - 1) / (kU * 256 * N);
    hipLaunchKernelGGL(logprobs_grad_long<T>, dim3(capped(a.rows * pieces)), dim3(256), 0, s, a, pieces);
    return hipGetLastError();
}

}  // namespace

size_t logprobs_workspace(int64_t rows, int V, int dtype, int n_top)
{
    if (V <= kShort) return 0;
    const LongPlan p = long_plan(rows, V, dtype);
    return p.splits > 1 ? (size_t)rows * p.splits * split_bytes(n_top) : 0;
}

hipError_t launch_logprobs(const LogprobArgs &a, int dtype, void *ws, hipStream_t s)
{
    return dtype == DT_BF16 ? run<uint16_t>(a, dtype, (char *)ws, s) : run<float>(a, dtype, (char *)ws, s);
}

hipError_t launch_logprobs_grad(const LogprobGradArgs &a, int dtype, hipStream_t s)
{
    return dtype == DT_BF16 ? run_grad<uint16_t>(a, s) : run_grad<float>(a, s);
}

}  // namespace fs
