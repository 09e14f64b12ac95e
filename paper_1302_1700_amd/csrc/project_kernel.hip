// A fully connected layer on rows with a low-rank adapter of each row's own
// choice, and its gradient:  y = W x + bias + s_i B_i (A_i x), i = ids[row].
//
// Few outputs (m + rank up to 64): one kernel, in which the rows of W and of A_i
// are the columns of one product (project_narrow; rows of more adapters than the
// columns have room for are multiplied again, from the caches); more: the
// rows times A_i first (rank_rows), then a tiled product that adds B_i's part
// (project_tiles_wide.hip).  The factors' gradients: per adapter, sums over its rows
// of outer products, in runs of rows joined by a second launch in the order of
// the runs (factor_grad, factor_join).
#include <algorithm>

#include "project.h"

namespace fs {
namespace {

// Rows [16 RB] of a wave times `cols` columns, column c from src(c) (null: 0),
// summed over [c0, c1) of the shared axis.
template <bool GATHER, typename T, int RB, int NB>
__device__ __forceinline__ void row_products(const T *const (&row)[RB], const T *const (&col)[NB], int64_t col_step,
                                             int c0, int c1, f4 (&acc)[RB][NB])
{
    constexpr int E = Operand<T>::kE, U = NB == 1 && !GATHER ? 8 / RB : NB <= 2 ? 4 / RB : 2;  // steps whose loads are in flight together
    const int g = (threadIdx.x & 63) >> 4;
    auto load = [&](int c, int have, Operand<T>(&oa)[RB], Operand<T>(&ob)[NB]) {
#pragma unroll
        for (int i = 0; i < RB; ++i) oa[i] = load_operand(row[i] + c, have);
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            ob[j] = Operand<T>{};
            if (col[j]) ob[j] = GATHER ? gather_operand(col[j] + c * col_step, col_step, have) : load_operand(col[j] + c, have);
        }
    };
    auto multiply = [&](const Operand<T>(&oa)[RB], const Operand<T>(&ob)[NB]) {
#pragma unroll
        for (int i = 0; i < RB; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j) acc[i][j] = block_product(oa[i], ob[j], acc[i][j]);
    };
    int c = c0 + g * E, at = c0;
    for (; at + U * kStep<T> <= c1; at += U * kStep<T>, c += U * kStep<T>) {
        Operand<T> oa[U][RB], ob[U][NB];
#pragma unroll
        for (int u = 0; u < U; ++u) load(c + u * kStep<T>, E, oa[u], ob[u]);
#pragma unroll
        for (int u = 0; u < U; ++u) multiply(oa[u], ob[u]);
    }
    for (; at < c1; at += kStep<T>, c += kStep<T>) {
        Operand<T> oa[RB], ob[NB];
        load(c, c1 - c, oa, ob);
        multiply(oa, ob);
    }
}

// The rows of one adapter among 1024: their offsets from the first, in order, in
// `list`; returns how many.  All threads of the workgroup take part (NW waves);
// `each` is called with every row's adapter once: each(row, adapter).
template <int NW, typename Id, typename Each>
__device__ __forceinline__ int list_rows(const Id *ids, int64_t at, int64_t end, int adapter, int *list, int *count,
                                         Each each)
{
    constexpr int G = 16 / NW > 0 ? 16 / NW : 1;  // groups of 64 ids a wave looks at
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint64_t who[G];
    __syncthreads();  // the list before has been read
#pragma unroll
    for (int k = 0; k < G; ++k) {
        const int64_t row = at + (wave * G + k) * 64 + lane;
        const int id = row < end ? ids[row] : -1;
        if (row < end) each(row, id);
        who[k] = __ballot(row < end && id == adapter);
        if (lane == 0) count[wave * G + k] = __popcll(who[k]);
    }
    __syncthreads();
    int total = 0, before = 0;
#pragma unroll
    for (int k = 0; k < 16; ++k) {
        if (k < wave * G) before += count[k];
        total += count[k];
    }
#pragma unroll
    for (int k = 0; k < G; ++k) {
        if (who[k] >> lane & 1) list[before + __popcll(who[k] & ((1ull << lane) - 1))] = (wave * G + k) * 64 + lane;
        before += __popcll(who[k]);
    }
    __syncthreads();
    return total;
}

// Rows times their adapter's factor, t[row][j] = s_i sum_c v[row][c] f_i[j][c]:
// f [n][r][C] (TRANS false: A) or [n][C][r] (true: B).  A workgroup takes one
// adapter's rows among 1024, 16 to a product, so that mixed rows cost no more
// products than sorted ones; workgroups with different `slot` take different
// sixteens.  W waves share the summed axis of a product.
template <typename T>
struct RankArgs {
    const T *v, *f;
    int64_t vs, rows;
    int C, n, r, slots;
    const float *scale;
    const int *ids;
    float *t;
};

template <typename T, int NB, int W, bool TRANS>
__global__ __launch_bounds__(W > 4 ? 64 * W : 256) void rank_rows(RankArgs<T> a)
{
    constexpr int NW = W > 4 ? W : 4, PER = NW / W, RB = W == 1 ? 2 : 1;  // RB sixteens of rows to a product
    __shared__ float part[W > 1 ? W * 256 : 1];
    __shared__ int list[1024], count[16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, q = lane & 15, g = lane >> 4;
    const int n = a.n, r = a.r;
    const int64_t units = (a.rows + 1023) / 1024 * n;
    for (int64_t unit = blockIdx.y; unit < units; unit += gridDim.y) {
        const int64_t chunk = unit / n, at = chunk * 1024;
        const int i = (int)(unit - chunk * n);
        const bool others = i == 0 && blockIdx.x == 0;  // this workgroup also writes the rows without an adapter
        const int total = list_rows<NW>(a.ids, at, a.rows, i, list, count, [&](int64_t row, int id) {
            if (others && (id < 0 || id >= n))
                for (int j = 0; j < r; ++j) a.t[row * r + j] = id < 0 ? 0.f : NAN;
        });
        const float sc = a.scale ? a.scale[i] : 1.f;
        constexpr int S = kStep<T>;
        const int run = W == 1 ? a.C : (a.C + W * S - 1) / (W * S) * S;
        const int c0 = std::min(a.C, wave % W * run), c1 = std::min(a.C, c0 + run);
        for (int tile = blockIdx.x * PER + wave / W; tile * 16 * RB < total; tile += a.slots * PER) {
            const T *row[RB];
            const T *col[NB];
            f4 acc[RB][NB];
#pragma unroll
            for (int b = 0; b < RB; ++b) row[b] = a.v + (at + list[std::min((tile * RB + b) * 16 + q, total - 1)]) * a.vs;
#pragma unroll
            for (int j = 0; j < NB; ++j) {
                const int c = j * 16 + q;
                col[j] = c >= r ? nullptr : TRANS ? a.f + (int64_t)i * r * a.C + c : a.f + ((int64_t)i * r + c) * a.C;
#pragma unroll
                for (int b = 0; b < RB; ++b) acc[b][j] = f4{0.f, 0.f, 0.f, 0.f};
            }
            row_products<TRANS, T, RB, NB>(row, col, r, c0, c1, acc);
#pragma unroll
            for (int j = 0; j < NB; ++j) {
                if constexpr (W > 1) {
                    __syncthreads();
#pragma unroll
                    for (int e = 0; e < 4; ++e) part[wave * 256 + e * 64 + lane] = acc[0][j][e];
                    __syncthreads();
                    if (wave == 0) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            float s = 0.f;
#pragma unroll
                            for (int k = 0; k < W; ++k) s += part[k * 256 + e * 64 + lane];
                            acc[0][j][e] = s;
                        }
                    }
                }
                if (wave % W == 0) {
#pragma unroll
                    for (int b = 0; b < RB; ++b)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int k = (tile * RB + b) * 16 + g * 4 + e;
                            if (k < total && j * 16 + q < r) a.t[(at + list[k]) * r + j * 16 + q] = acc[b][j][e] * sc;
                        }
                }
            }
        }
    }
}

// Few outputs: columns 0 .. M - 1 of the product are W's rows, the next ones
// the rows of as many of the tile's adapters' A as fit (the others in further
// passes over the tile's rows); the products go through
// LDS, where each row's outputs take up their hidden values.  A wave takes 16 RB
// rows (W = 1), or 16 shared by W waves.
template <typename T, int RB, int NB, int W>
__global__ __launch_bounds__(W > 4 ? 64 * W : 256) void project_narrow(ProjArgs a, T *y, int64_t ys, float *hidden)
{
    constexpr int P = NB * 16 + 1, NW = W > 4 ? W : 4;
    __shared__ float part[NW][16 * RB][P];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, q = lane & 15, g = lane >> 4;
    const int64_t tiles = (a.rows + 16 * RB - 1) / (16 * RB);
    constexpr int PER = NW / W;
    const T *x = (const T *)a.x, *w = (const T *)a.w, *fa = (const T *)a.a, *fb = (const T *)a.b;
    const int M = a.M, r = a.r, n = a.n;
    const int fit = n ? (NB * 16 - M) / r : 0;  // adapters a pass has columns for
    for (int64_t tile0 = (int64_t)blockIdx.x * PER; tile0 < tiles; tile0 += (int64_t)gridDim.x * PER) {
        const int64_t row0 = (tile0 + wave / W) * 16 * RB;
        int id = -1;  // of row `lane` of the wave's
        if (n && lane < 16 * RB && row0 + lane < a.rows) id = a.ids[row0 + lane];
        const bool bad = id >= n;
        int state = lane < 16 * RB && row0 + lane < a.rows ? 0 : 3;  // 0: to do, 1: this pass, 2: done, 3: no row
        int slot = -1;  // the row's adapter among the pass's
        const T *row[RB];
#pragma unroll
        for (int i = 0; i < RB; ++i) row[i] = x + clamp_row(row0 + i * 16 + q, a.rows) * a.xs;
        constexpr int S = kStep<T>;
        const int run = W == 1 ? a.K : (a.K + W * S - 1) / (W * S) * S;
        const int c0 = std::min(a.K, wave % W * run), c1 = std::min(a.K, c0 + run);
        for (int last = -1;;) {
            // the next adapters that fit beside W's columns, and the rows they serve;
            // rows without an adapter go with the first pass
            const T *col[NB];
            f4 acc[RB][NB];
            int colslot[NB];
#pragma unroll
            for (int j = 0; j < NB; ++j) {
                const int c = j * 16 + q;
                colslot[j] = c < M || !n ? -1 : (c - M) / r;
                col[j] = c < M ? w + c * a.ws : nullptr;
#pragma unroll
                for (int i = 0; i < RB; ++i) acc[i][j] = f4{0.f, 0.f, 0.f, 0.f};
            }
            if (state == 0 && (id < 0 || bad)) state = 1;
            for (int s = 0; s < fit; ++s) {
                const int cur = next_adapter(bad ? -1 : id, last);
                if (cur >= n) break;
                last = cur;
                if (state == 0 && id == cur) {
                    state = 1;
                    slot = s;
                }
#pragma unroll
                for (int j = 0; j < NB; ++j)
                    if (colslot[j] == s) col[j] = fa + ((int64_t)cur * r + (j * 16 + q - M - s * r)) * a.K;
            }
            if (!__any(state == 1)) break;
            row_products<false, T, RB, NB>(row, col, 1, c0, c1, acc);
            if (W > 1) __syncthreads();
#pragma unroll
            for (int i = 0; i < RB; ++i)
#pragma unroll
                for (int j = 0; j < NB; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) part[wave][i * 16 + g * 4 + e][j * 16 + q] = acc[i][j][e];
            if (W > 1) {
                __syncthreads();
                for (int k = threadIdx.x; k < 16 * RB * NB * 16; k += 64 * NW) {
                    const int rr = k / (NB * 16), c = k % (NB * 16);
                    float s = part[0][rr][c];
#pragma unroll
                    for (int o = 1; o < W; ++o) s += part[o][rr][c];
                    part[0][rr][c] = s;
                }
                __syncthreads();
            } else {
                __builtin_amdgcn_wave_barrier();
            }
            const float(*sum)[P] = part[W > 1 ? 0 : wave];
            if (wave % W == 0) {
                for (int k = lane; k < (16 * RB * M + 63) / 64 * 64; k += 64) {
                    const int rr = k / M, m = k - rr * M;
                    const bool mine = __shfl(state, rr & 63) == 1 && rr < 16 * RB;
                    const int i = __shfl(id, rr & 63), at = M + __shfl(slot, rr & 63) * r;
                    if (!mine) continue;
                    float v = sum[rr][m];
                    if (i >= 0 && i < n) {
                        const T *bi = fb + ((int64_t)i * M + m) * r;
                        float z = 0.f;
                        for (int j = 0; j < r; ++j) z = fmaf(sum[rr][at + j], to_f32(bi[j]), z);
                        v = fmaf(z, a.scale ? a.scale[i] : 1.f, v);
                    }
                    if (a.bias) v += a.bias[m];
                    store_as(y + (row0 + rr) * ys + m, i >= n && n ? NAN : v);
                }
                if (hidden) {
                    for (int k = lane; k < (16 * RB * r + 63) / 64 * 64; k += 64) {
                        const int rr = k / r, j = k - rr * r;
                        const bool mine = __shfl(state, rr & 63) == 1 && rr < 16 * RB;
                        const int i = __shfl(id, rr & 63), at = M + __shfl(slot, rr & 63) * r;
                        if (mine) hidden[(row0 + rr) * r + j] = i >= n ? NAN : i < 0 ? 0.f : sum[rr][at + j];
                    }
                }
            }
            if (state == 1) state = 2;
            if (!__any(state == 0)) break;
            if (W == 1) __builtin_amdgcn_wave_barrier();
        }
        if (W > 1) __syncthreads();
    }
}

// One of the two factors' gradients: out_i[j][c] = s_i? sum over rows of i of
// t[row][j] v[row][c], stored [n][r][C] (by_rank) or [n][C][r].
template <typename T>
struct FactorJob {
    const float *t;
    const T *v;
    int64_t vs;
    int C, by_rank, ctiles;
    const float *scale;
    T *out;
    float *parts;  // [n][runs][r][C]
};

template <typename T>
struct FactorArgs {
    FactorJob<T> job[2];
    int64_t rows, run_rows;
    int runs, n, r;
    const int *ids;
    uint8_t *used;  // [n][runs]: the run holds rows of the adapter
    const T *b;     // both in one pass: [n][M][r]
};

// Four adjacent values of a row from column c on, 0 past its C columns.  Rows of
// four or more (LOAD 0: a multiple of four; 1: any): always one load, from
// inside the row, moved into place, without a branch that would keep the next
// row's load waiting.  LOAD 2: shorter rows.
template <int LOAD, typename T>
__device__ __forceinline__ void four(const T *v, int c, int C, bool have, float (&vv)[4])
{
    if constexpr (LOAD == 2) {
#pragma unroll
        for (int e = 0; e < 4; ++e) vv[e] = c + e < C ? to_f32(v[c + e]) : 0.f;
    } else {
        float w[4];
        const int from = min(c, C - 4), move = c - from;
        unpack<T, 4>(load_words<4 * sizeof(T)>(v + from), w);
        if constexpr (LOAD == 1) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float x = w[e];
#pragma unroll
                for (int k = 1; k < 4; ++k) x = move == k ? (e + k < 4 ? w[(e + k) & 3] : 0.f) : x;
                w[e] = x;  // later e only look at later w
            }
        }
        have &= c < C;
#pragma unroll
        for (int e = 0; e < 4; ++e) vv[e] = w[e];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) vv[e] = have ? vv[e] : 0.f;
}

// Where sums go: the part of a run, or the gradient itself when there is one
// run (times the adapter's scale, unless it is the sum of no rows, 0 at any
// scale); four adjacent columns of rank j.
template <typename T>
__device__ __forceinline__ void store_sums(const FactorArgs<T> &a, const FactorJob<T> &job, int64_t unit, int i, int j, int c,
                                           f4 s, bool seen)
{
    if (j >= a.r) return;
    if (a.runs > 1 && c + 4 <= job.C) {
        store_words<16>(job.parts + (unit * a.r + j) * job.C + c, __builtin_bit_cast(Words<16>::type, s));
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (c + e >= job.C) return;
        if (a.runs > 1) job.parts[(unit * a.r + j) * job.C + c + e] = s[e];
        else
            store_as(job.out + (job.by_rank ? ((int64_t)i * a.r + j) * job.C + c + e : ((int64_t)i * job.C + c + e) * a.r + j),
                     job.scale && seen ? s[e] * job.scale[i] : s[e]);
    }
}

// Workgroup: one adapter, one run of rows, 64 WC columns.  The run's rows that
// name the adapter are listed in LDS, 1024 ids at a time, and are the summed
// axis of float32 products (bf16 values are exact in them), four at a time, a
// wave's loads of 4 kGroups rows in flight together.  WC waves take 64 columns
// each, so that no sum crosses waves; where there are fewer columns, 4 / WC
// waves share the rows and their sums are joined in LDS.  Two jobs (both
// factors) by blockIdx.x; FUSED (M and r up to 16; MB: M's bound) makes both in
// one pass over the rows: lane q holds column q of its adapter's B and makes
// B^T g of its row from the row's 16 lanes, so it never goes through memory;
// both sums take the scale at the end.
template <int NB>
constexpr int kGroups = NB == 1 ? 8 : NB == 2 ? 4 : 2;

template <typename T, int NB, int WC, int LOAD, int MB>
__global__ __launch_bounds__(256) void factor_grad(FactorArgs<T> a)
{
    constexpr bool FUSED = MB > 0;
    constexpr int G = kGroups<NB>, WR = 4 / WC;
    __shared__ int list[1024], count[16];
    __shared__ float sums[WR > 1 ? 4 : 1][WR > 1 ? (4 * NB + 1) * 4 : 1][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, q = lane & 15, g = lane >> 4;
    const int which = !FUSED && blockIdx.x >= (unsigned)a.job[0].ctiles;
    const FactorJob<T> &job = a.job[which], &jb = a.job[1];
    const int c0 = ((int)blockIdx.x - (which ? a.job[0].ctiles : 0)) * 64 * WC + wave % WC * 64, wr = wave / WC;
    const int r = a.r, M = jb.C, C = job.C;
    const bool second = FUSED && blockIdx.x == 0 && wave % WC == 0;  // this wave also makes the other factor's
    for (int64_t unit = blockIdx.y; unit < (int64_t)a.n * a.runs; unit += gridDim.y) {
        const int i = (int)(unit / a.runs), run = (int)(unit - (int64_t)i * a.runs);
        const int64_t begin = run * a.run_rows, end = std::min(a.rows, begin + a.run_rows);
        float bi[FUSED ? MB : 1];
        if constexpr (FUSED) {
#pragma unroll
            for (int m = 0; m < MB; ++m) bi[m] = m < M && q < r ? to_f32(a.b[((int64_t)i * M + m) * r + q]) : 0.f;
        }
        f4 acc[4][NB], gb = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int p = 0; p < 4; ++p)
#pragma unroll
            for (int j = 0; j < NB; ++j) acc[p][j] = f4{0.f, 0.f, 0.f, 0.f};
        bool seen = false;
        for (int64_t at = begin; at < end; at += 1024) {
            const int total = list_rows<4>(a.ids, at, end, i, list, count, [](int64_t, int) {});
            seen |= total > 0;
            if (c0 >= C && !second) continue;
            for (int l = wr * 4 * G; l < total; l += WR * 4 * G) {
                float tv[G][NB], vv[G][4], gv[FUSED ? G : 1];
#pragma unroll
                for (int k = 0; k < G; ++k) {
                    const bool have = l + k * 4 + g < total;
                    const int64_t row = at + list[have ? l + k * 4 + g : l];
#pragma unroll
                    for (int j = 0; j < NB; ++j) {
                        const float *t = FUSED ? jb.t : job.t;
                        tv[k][j] = t[row * r + std::min(j * 16 + q, r - 1)];
                        tv[k][j] = have && j * 16 + q < r ? tv[k][j] : 0.f;
                    }
                    if constexpr (FUSED) {
                        gv[k] = to_f32(jb.v[row * jb.vs + std::min(q, M - 1)]);
                        gv[k] = have && q < M ? gv[k] : 0.f;
                    }
                    four<LOAD>(job.v + row * job.vs, c0 + q * 4, C, have, vv[k]);
                }
#pragma unroll
                for (int k = 0; k < G; ++k) {
                    if constexpr (FUSED) {
                        if (second) gb = __builtin_amdgcn_mfma_f32_16x16x4f32(tv[k][0], gv[k], gb, 0, 0, 0);
                        float u = 0.f;
#pragma unroll
                        for (int m = 0; m < MB; ++m) u = fmaf(__shfl(gv[k], (lane & 48) + m), bi[m], u);
                        // no row, no term: 0 times an infinite factor would be NaN
                        tv[k][0] = l + k * 4 + g < total ? u : 0.f;
                    }
#pragma unroll
                    for (int p = 0; p < 4; ++p)
#pragma unroll
                        for (int j = 0; j < NB; ++j)
                            acc[p][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(tv[k][j], vv[k][p], acc[p][j], 0, 0, 0);
                }
            }
        }
        if (threadIdx.x == 0 && blockIdx.x == 0 && a.used) a.used[unit] = seen;
        if (!seen && a.runs > 1) continue;
        if constexpr (WR > 1) {
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 4; ++e) {
#pragma unroll
                for (int j = 0; j < NB; ++j)
#pragma unroll
                    for (int p = 0; p < 4; ++p) sums[wave][(j * 4 + p) * 4 + e][lane] = acc[p][j][e];
                sums[wave][NB * 16 + e][lane] = gb[e];
            }
            __syncthreads();
            if (wr == 0) {
#pragma unroll
                for (int o = 1; o < WR; ++o)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
#pragma unroll
                        for (int j = 0; j < NB; ++j)
#pragma unroll
                            for (int p = 0; p < 4; ++p) acc[p][j][e] += sums[o * WC + wave][(j * 4 + p) * 4 + e][lane];
                        gb[e] += sums[o * WC + wave][NB * 16 + e][lane];
                    }
            }
            if (wr != 0) continue;
        }
        // element e of lane l: rank 16 j + 4 g + e; block p: column c0 + 4 q + p
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                store_sums(a, job, unit, i, j * 16 + g * 4 + e, c0 + q * 4,
                           f4{acc[0][j][e], acc[1][j][e], acc[2][j][e], acc[3][j][e]}, seen);
        if (second && q < M) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int j = g * 4 + e;
                if (j >= r) continue;
                if (a.runs > 1) jb.parts[(unit * r + j) * M + q] = gb[e];
                else store_as(jb.out + ((int64_t)i * M + q) * r + j, jb.scale && seen ? gb[e] * jb.scale[i] : gb[e]);
            }
        }
    }
}

// Sums the parts of the runs that hold rows of the adapter: 64 values to a
// workgroup, each wave a quarter of these runs in their order, the quarters
// joined in order.
template <typename T>
__global__ __launch_bounds__(256) void factor_join(FactorArgs<T> a)
{
    __shared__ float sums[4][64];
    __shared__ int list[1024], count[16];
    const FactorJob<T> &job = a.job[blockIdx.y];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int per_adapter = a.r * job.C, blocks = (per_adapter + 63) / 64;
    for (int64_t unit = blockIdx.x; unit < (int64_t)a.n * blocks; unit += gridDim.x) {
        const int i = (int)(unit / blocks), k = (int)(unit - (int64_t)i * blocks) * 64 + lane;
        const float *parts = job.parts + (int64_t)i * a.runs * per_adapter + std::min(k, per_adapter - 1);
        float s = 0.f;
        bool seen = false;
        for (int at = 0; at < a.runs; at += 1024) {
            const int total = list_rows<4>(a.used + (int64_t)i * a.runs, at, a.runs, 1, list, count, [](int64_t, int) {});
            seen |= total > 0;
            const int quarter = (total + 3) / 4, to = std::min(total, (wave + 1) * quarter);
            for (int l = wave * quarter; l < to; l += 8) {
                float v[8];  // in flight together
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = parts[(int64_t)(at + list[std::min(l + k, to - 1)]) * per_adapter];
#pragma unroll
                for (int k = 0; k < 8; ++k) s += l + k < to ? v[k] : 0.f;
            }
        }
        __syncthreads();
        sums[wave][lane] = s;
        __syncthreads();
        if (wave == 0 && k < per_adapter) {
            s = (sums[0][lane] + sums[1][lane]) + (sums[2][lane] + sums[3][lane]);
            if (job.scale && seen) s *= job.scale[i];  // 0 at any scale where no row names the adapter
            const int j = k / job.C, c = k - j * job.C;
            store_as(job.out + (int64_t)i * per_adapter + (job.by_rank ? k : c * a.r + j), s);
        }
    }
}

// -- choices and workspace ---------------------------------------------------------
size_t up256(size_t v) { return (v + 255) & ~(size_t)255; }
size_t rank_bytes(const ProjArgs &a) { return up256((size_t)a.rows * a.r * sizeof(float)); }

// W's and A's rows as columns of one product.  Adapters in runs: 1M x 200 -> 20
// float32, rank 8: 498 us (its bytes at a copy's rate: 186), rows times A first
// and tiles of 64 columns then 817; 300,000 x 200 -> 2, rank 16, 64 adapters: 97
// and 359; a long axis of few rows, 4093 x 4096 -> 40 bf16, rank 16: 59 and 47.
// In any order the columns are multiplied again for every few adapters that 16 or
// 32 rows name, and this way loses where these are many: the same 300,000 rows
// 1882 and 625, with 8 adapters 576 and 358, at rank 4 141 and 351; 4093 x 4096 ->
// 40 175 and 60.  The order of the ids is not known here.
bool narrow(const ProjArgs &a) { return a.M + a.r <= 64; }

// Waves that share the summed axis of a product: the fewer rows and the longer
// the axis, the more (bf16, 20 outputs, rank 8: 2048 x 4096 with eight 19 us, with
// four 40, with one 65; 20,000 x 4096 with four 63, with one 103; 40,000 x 1024
// with four 48, with one 43).  The same rule wherever rows meet A: the hidden
// rows then have the same bits from every kernel.
template <typename T>
int axis_waves(int64_t rows, int C)
{
    const int steps = C / kStep<T>;
    if (rows <= 8192 && steps >= 32) return rows <= 256 ? 16 : 8;
    return steps >= 8 && rows <= (steps >= 64 ? 65536 : 16384) ? 4 : 1;
}

// Both factors' gradients in one pass: 1M x 200 -> 2 float32, rank 4: 237 us, with
// the ranks' rows through memory and two passes 548.
bool both(const ProjArgs &a) { return a.M <= 16 && a.r <= 16; }

struct RunPlan {
    int64_t run_rows;
    int runs;
    size_t parts[2], used;  // bytes
};

// Runs of rows: enough workgroups for the card where the rows of an adapter lie
// together (then one in n of them works), parts of at most 256 MB.
RunPlan run_plan(const ProjArgs &a)
{
    const int64_t ctiles = both(a) ? (a.K + 255) / 256 : (a.K + 255) / 256 + (a.M + 255) / 256;
    const double part = (double)a.n * a.r * (a.K + a.M) * sizeof(float);
    // below 512 rows a launch to join them costs more than the runs save
    int64_t runs = a.rows < 512 ? 1 : std::max<int64_t>(1, std::min<int64_t>(2048 / ctiles, a.rows / 128));
    runs = std::max<int64_t>(1, std::min<int64_t>(runs, (int64_t)(268435456.0 / part)));
    RunPlan p;
    p.run_rows = std::max<int64_t>(64, ((a.rows + runs - 1) / runs + 63) / 64 * 64);
    p.runs = (int)std::max<int64_t>(1, (a.rows + p.run_rows - 1) / p.run_rows);
    p.parts[0] = p.runs > 1 ? up256((size_t)a.n * p.runs * a.r * a.K * sizeof(float)) : 0;
    p.parts[1] = p.runs > 1 ? up256((size_t)a.n * p.runs * a.r * a.M * sizeof(float)) : 0;
    p.used = p.runs > 1 ? up256((size_t)a.n * p.runs) : 0;
    return p;
}

template <typename T, int NB, bool TRANS>
hipError_t go_rank(const T *v, int64_t vs, int64_t rows, int C, const T *f, int n, int r, const float *scale,
                   const int *ids, float *t, hipStream_t s)
{
    const int waves = axis_waves<T>(rows, C);
    // The 64 sixteens of 1024 rows over several workgroups of an adapter where
    // there are too few otherwise; a workgroup without rows costs the look at
    // their ids (550,000 mixed rows of 13 adapters, eight each: 779 us).
    const int64_t units = (rows + 1023) / 1024 * n;
    const int64_t most = waves == 1 ? 8 : std::min<int64_t>(64, (rows + 15) / 16);
    const int slots = (int)std::max<int64_t>(1, std::min<int64_t>(most, 4096 / units));
    const RankArgs<T> a{v, f, vs, rows, C, n, r, slots, scale, ids, t};
    const dim3 grid(slots, (unsigned)std::min<int64_t>(units, 65535));
    if (waves == 16) hipLaunchKernelGGL((rank_rows<T, NB, 16, TRANS>), grid, dim3(1024), 0, s, a);
    else if (waves == 8) hipLaunchKernelGGL((rank_rows<T, NB, 8, TRANS>), grid, dim3(512), 0, s, a);
    else if (waves == 4) hipLaunchKernelGGL((rank_rows<T, NB, 4, TRANS>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((rank_rows<T, NB, 1, TRANS>), grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

template <typename T, bool TRANS>
hipError_t rank_product(const T *v, int64_t vs, int64_t rows, int C, const T *f, int n, int r, const float *scale,
                        const int *ids, float *t, hipStream_t s)
{
    if (r <= 16) return go_rank<T, 1, TRANS>(v, vs, rows, C, f, n, r, scale, ids, t, s);
    if (r <= 32) return go_rank<T, 2, TRANS>(v, vs, rows, C, f, n, r, scale, ids, t, s);
    if (r <= 64) return go_rank<T, 4, TRANS>(v, vs, rows, C, f, n, r, scale, ids, t, s);
    return go_rank<T, 8, TRANS>(v, vs, rows, C, f, n, r, scale, ids, t, s);
}

template <typename T, int NB>
hipError_t go_narrow(const ProjArgs &a, T *y, int64_t ys, float *hidden, hipStream_t s)
{
    const int64_t tiles = (a.rows + 15) / 16;
    const int waves = axis_waves<T>(a.rows, a.K);
    if (waves == 16)
        hipLaunchKernelGGL((project_narrow<T, 1, NB, 16>), dim3(grid_of(tiles)), dim3(1024), 0, s, a, y, ys, hidden);
    else if (waves == 8)
        hipLaunchKernelGGL((project_narrow<T, 1, NB, 8>), dim3(grid_of(tiles)), dim3(512), 0, s, a, y, ys, hidden);
    else if (waves == 4)
        hipLaunchKernelGGL((project_narrow<T, 1, NB, 4>), dim3(grid_of(tiles)), dim3(256), 0, s, a, y, ys, hidden);
    else
        hipLaunchKernelGGL((project_narrow<T, 2, NB, 1>), dim3(grid_of((tiles + 7) / 8)), dim3(256), 0, s, a, y, ys, hidden);
    return hipGetLastError();
}

template <typename T>
hipError_t project(const ProjArgs &a, int dtype, T *y, int64_t ys, float *hidden, float *h, float *parts, hipStream_t s)
{
    if (narrow(a)) {
        // columns for four adapters, as rows in any order name them, but for no
        // more than 32 where one needs no more
        const int cols = std::max(a.M + a.r, std::min(32, a.M + a.r * std::min(a.n, 4)));
        if (cols <= 16) return go_narrow<T, 1>(a, y, ys, hidden, s);
        if (cols <= 32) return go_narrow<T, 2>(a, y, ys, hidden, s);
        return go_narrow<T, 4>(a, y, ys, hidden, s);
    }
    if (a.n) {
        hipError_t e = rank_product<T, false>((const T *)a.x, a.xs, a.rows, a.K, (const T *)a.a, a.n, a.r, nullptr, a.ids, h, s);
        if (e != hipSuccess) return e;
    }
    const WideArgs w{a.x, a.w, a.b, y, a.rows, a.xs, a.ws, ys, a.K, a.M, a.n, a.r, a.bias, a.scale, h, a.ids, parts};
    return launch_wide(w, dtype, false, s);
}

template <typename T>
hipError_t join_factors(const FactorArgs<T> &a, hipStream_t s)
{
    const int most = a.r * std::max(a.job[0].C, a.job[1].C);
    hipLaunchKernelGGL(factor_join<T>, dim3(grid_of((int64_t)a.n * ((most + 63) / 64)), 2), dim3(256), 0, s, a);
    return hipGetLastError();
}

template <typename T, int NB, int WC, int MB>
hipError_t go_factor(FactorArgs<T> &a, hipStream_t s)
{
    for (FactorJob<T> &j : a.job) j.ctiles = (j.C + 64 * WC - 1) / (64 * WC);
    const dim3 grid(a.job[0].ctiles + (MB ? 0 : a.job[1].ctiles), (unsigned)std::min<int64_t>((int64_t)a.n * a.runs, 65535));
    const int c0 = a.job[0].C, c1 = MB ? c0 : a.job[1].C;
    if (std::min(c0, c1) < 4) hipLaunchKernelGGL((factor_grad<T, NB, WC, 2, MB>), grid, dim3(256), 0, s, a);
    else if (c0 % 4 || c1 % 4) hipLaunchKernelGGL((factor_grad<T, NB, WC, 1, MB>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((factor_grad<T, NB, WC, 0, MB>), grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

template <typename T, int NB, int MB>
hipError_t go_factor(FactorArgs<T> &a, hipStream_t s)
{
    const int C = MB ? a.job[0].C : std::max(a.job[0].C, a.job[1].C);
    return C <= 64 ? go_factor<T, NB, 1, MB>(a, s) : C <= 128 ? go_factor<T, NB, 2, MB>(a, s) : go_factor<T, NB, 4, MB>(a, s);
}

template <typename T>
hipError_t project_grad(const ProjArgs &a, int dtype, const T *g, int64_t gs, const float *h, T *gx, int64_t gxs, T *ga,
                        T *gb, char *ws, hipStream_t s)
{
    hipError_t e;
    float *u = (float *)ws;
    ws += rank_bytes(a);
    float *own = (float *)ws;
    ws += rank_bytes(a);
    float *parts = (float *)ws;  // the rows' gradient and the factors' one after the other
    const bool fused = both(a);
    if (a.n && a.rows) {
        if (!fused || gx) {
            e = rank_product<T, true>(g, gs, a.rows, a.M, (const T *)a.b, a.n, a.r, a.scale, a.ids, u, s);
            if (e != hipSuccess) return e;
        }
        if (!h && ga) {
            e = rank_product<T, false>((const T *)a.x, a.xs, a.rows, a.K, (const T *)a.a, a.n, a.r, nullptr, a.ids, own, s);
            if (e != hipSuccess) return e;
            h = own;
        }
    }
    if (ga) {
        const RunPlan p = run_plan(a);
        FactorArgs<T> f{};
        // u has the scale already where it goes through memory
        f.job[0] = FactorJob<T>{u, (const T *)a.x, a.xs, a.K, 1, 0, fused ? a.scale : nullptr, ga, (float *)ws};
        f.job[1] = FactorJob<T>{h, g, gs, a.M, 0, 0, a.scale, gb, (float *)(ws + p.parts[0])};
        f.rows = a.rows;
        f.run_rows = p.run_rows;
        f.runs = p.runs;
        f.n = a.n;
        f.r = a.r;
        f.ids = a.ids;
        f.used = p.runs > 1 ? (uint8_t *)(ws + p.parts[0] + p.parts[1]) : nullptr;
        f.b = (const T *)a.b;
        if (fused) e = a.M <= 4 ? go_factor<T, 1, 4>(f, s) : go_factor<T, 1, 16>(f, s);
        else if (a.r <= 16) e = go_factor<T, 1, 0>(f, s);
        else if (a.r <= 32) e = go_factor<T, 2, 0>(f, s);
        else if (a.r <= 64) e = go_factor<T, 4, 0>(f, s);
        else e = go_factor<T, 8, 0>(f, s);
        if (e == hipSuccess && p.runs > 1) e = join_factors(f, s);
        if (e != hipSuccess) return e;
    }
    if (gx && a.rows) {
        const WideArgs w{g, a.w, a.a, gx, a.rows, gs, a.ws, gxs, a.M, a.K, a.n, a.r, nullptr, nullptr, u, a.ids, parts};
        return launch_wide(w, dtype, true, s);
    }
    return hipSuccess;
}

}  // namespace

size_t project_workspace(const ProjArgs &a, int dtype)
{
    if (!a.rows || narrow(a)) return 0;
    return rank_bytes(a) + wide_parts(a.rows, a.M, a.K, dtype);
}

hipError_t launch_project(const ProjArgs &a, int dtype, void *y, int64_t ys, float *hidden, void *ws, hipStream_t s)
{
    float *h = hidden ? hidden : (float *)ws, *parts = (float *)((char *)ws + rank_bytes(a));
    return dtype == DT_BF16 ? project(a, dtype, (uint16_t *)y, ys, hidden, h, parts, s)
                            : project(a, dtype, (float *)y, ys, hidden, h, parts, s);
}

size_t project_grad_workspace(const ProjArgs &a, int dtype)
{
    const size_t rows = a.rows ? wide_parts(a.rows, a.K, a.M, dtype) : 0;
    if (!a.n) return rows;
    const RunPlan p = run_plan(a);
    return 2 * rank_bytes(a) + std::max(rows, p.parts[0] + p.parts[1] + p.used);
}

hipError_t launch_project_grad(const ProjArgs &a, int dtype, const void *g, int64_t gs, const float *hidden, void *gx,
                               int64_t gxs, void *ga, void *gb, void *ws, hipStream_t s)
{
    if (dtype == DT_BF16)
        return project_grad(a, dtype, (const uint16_t *)g, gs, hidden, (uint16_t *)gx, gxs, (uint16_t *)ga, (uint16_t *)gb,
                            (char *)ws, s);
    return project_grad(a, dtype, (const float *)g, gs, hidden, (float *)gx, gxs, (float *)ga, (float *)gb, (char *)ws, s);
}

}  // namespace fs
