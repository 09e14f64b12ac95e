// The shared projection's matrix product with the adapters' part added to its
// accumulators: out = v W + t F_i, i the adapter of the row.
//
// A workgroup computes a BM x BN tile, its four waves a quarter each.  The
// summed axis is walked 128 bytes of each row at a time: global loads of the
// next step are in flight while the present one's products run from LDS, where
// a row's 16-byte pieces are stored in an order turned by the row (piece p of
// row q at p ^ (q % 8)), so that the 16 rows an operand load touches fall on
// different banks.  For the gradient of the rows W lies the other way round;
// its tile keeps the order of memory, and bf16 operands are transposed by the
// LDS read itself.
//
// The adapters' part: for every adapter that a row of the tile names, the
// product of t with its factor, blocks of 16 x 16, added only to the rows that
// name it (an infinity in one adapter stays out of the others' rows).  bf16: t
// goes in as three bf16 values, each the rounding of what the ones before
// leave, which keep its 24 bits.
#include <algorithm>
#include <type_traits>

#include "project.h"

namespace fs {
namespace {

typedef short s4 __attribute__((ext_vector_type(4)));

// Tile steps: 128 bytes of the summed axis.
template <typename T>
constexpr int kDepth = 128 / sizeof(T);

// Float values as one operand (float32), or three (bf16: what each rounding leaves).
__device__ __forceinline__ void split_operand(const float *v, Operand<float> *o)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) o[0].v[e] = v[e];
}
__device__ __forceinline__ void split_operand(const float *v, Operand<uint16_t> *o)
{
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        float rest = v[e];
#pragma unroll
        for (int p = 0; p < 3; ++p) {
            o[p].v[e] = to_bf16(rest);
            rest -= to_f32(o[p].v[e]);
        }
    }
}

template <typename T, bool TRANS, int BM, int BN>
__global__ __launch_bounds__(256) void project_wide(WideArgs a, int tiles_m, int tiles_n)
{
    constexpr int D = kDepth<T>, E = Operand<T>::kE, S = D / kStep<T>;  // depth, lane values, block products a step
    constexpr int WM = BM / 32, WN = BN / 32;                            // 16 x 16 blocks of a wave
    constexpr int PA = BM * 8 / 256, PB = BN * 8 / 256;                  // 16-byte pieces a thread stages
    constexpr int BP = TRANS ? BN + (sizeof(T) == 2 ? 16 : 4) : 0;       // pitch of W's tile as in memory
    constexpr int BBYTES = TRANS ? D * BP * (int)sizeof(T) : BN * 128;
    __shared__ __align__(16) char lds_a[2][BM * 128];
    __shared__ __align__(16) char lds_b[2][BBYTES];

    // Tiles in the order of the XCDs (workgroup i runs on XCD i % 8): each takes
    // a run of them, eight tile rows deep, so that its L2 holds their operands.
    const int tiles = tiles_m * tiles_n;
    int tile = blockIdx.x;
    {
        const int per = tiles / 8, more = tiles % 8, xcd = tile % 8;
        tile = xcd * per + min(xcd, more) + tile / 8;
        const int group = 8 * tiles_n, g0 = tile / group * 8, high = min(8, tiles_m - g0);
        const int in = tile % group;
        tile = (g0 + in % high) * tiles_n + in / high;
    }
    const int64_t m0 = (int64_t)(tile / tiles_n) * BM;
    const int n0 = tile % tiles_n * BN;

    const T *v = reinterpret_cast<const T *>(a.v), *w = reinterpret_cast<const T *>(a.w);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, q = lane & 15, g = lane >> 4;
    const int wm = (wave >> 1) * (BM / 2), wn = (wave & 1) * (BN / 2);

    Lane16<T> ra[PA], rb[PB];
    auto take = [&](const T *p, int have) {
        Lane16<T> r;
        if (have >= E) r = *reinterpret_cast<const Lane16<T> *>(p);
        else {
#pragma unroll
            for (int e = 0; e < E; ++e) r.v[e] = e < have ? p[e] : (T)0;
        }
        return r;
    };
    auto fetch = [&](int c0) {
#pragma unroll
        for (int i = 0; i < PA; ++i) {
            const int piece = i * 256 + threadIdx.x, c = c0 + (piece & 7) * E;
            ra[i] = take(v + clamp_row(m0 + (piece >> 3), a.rows) * a.vs + c, a.C - c);
        }
#pragma unroll
        for (int i = 0; i < PB; ++i) {
            const int piece = i * 256 + threadIdx.x;
            if constexpr (TRANS) {
                const int row = c0 + piece / (BN / E), col = n0 + piece % (BN / E) * E;
                rb[i] = take(w + (int64_t)row * a.ws + col, row < a.C ? a.cols - col : 0);
            } else {
                const int c = c0 + (piece & 7) * E;
                rb[i] = take(w + (int64_t)min(n0 + (piece >> 3), a.cols - 1) * a.ws + c, a.C - c);
            }
        }
    };
    auto turned = [](int row, int piece) { return row * 128 + ((piece ^ (row & 7)) << 4); };
    auto put = [&](int at) {
#pragma unroll
        for (int i = 0; i < PA; ++i) {
            const int piece = i * 256 + threadIdx.x;
            *reinterpret_cast<Lane16<T> *>(__builtin_assume_aligned(lds_a[at] + turned(piece >> 3, piece & 7), 16)) = ra[i];
        }
#pragma unroll
        for (int i = 0; i < PB; ++i) {
            const int piece = i * 256 + threadIdx.x;
            char *to = TRANS ? lds_b[at] + (piece / (BN / E) * BP + piece % (BN / E) * E) * (int)sizeof(T)
                             : lds_b[at] + turned(piece >> 3, piece & 7);
            *reinterpret_cast<Lane16<T> *>(__builtin_assume_aligned(to, 16)) = rb[i];
        }
    };
    f4 acc[WM][WN];
#pragma unroll
    for (int i = 0; i < WM; ++i)
#pragma unroll
        for (int j = 0; j < WN; ++j) acc[i][j] = f4{0.f, 0.f, 0.f, 0.f};

    auto products = [&](int at) {
#pragma unroll
        for (int s = 0; s < S; ++s) {
            Operand<T> oa[WM], ob[WN];
#pragma unroll
            for (int i = 0; i < WM; ++i)
                oa[i] = *reinterpret_cast<const Operand<T> *>(lds_a[at] + turned(wm + i * 16 + q, s * 4 + g));
#pragma unroll
            for (int j = 0; j < WN; ++j) {
                if constexpr (!TRANS) {
                    ob[j] = *reinterpret_cast<const Operand<T> *>(lds_b[at] + turned(wn + j * 16 + q, s * 4 + g));
                } else if constexpr (sizeof(T) == 4) {
                    const float *b = reinterpret_cast<const float *>(lds_b[at]) + (s * 16 + g * 4) * BP + wn + j * 16 + q;
#pragma unroll
                    for (int e = 0; e < 4; ++e) ob[j].v[e] = b[e * BP];
                } else {
                    // 16 lanes read four rows of 16 columns, four columns a lane, and get a column each
                    const uint16_t *b = reinterpret_cast<const uint16_t *>(lds_b[at]) +
                                        (s * 32 + g * 8 + (q >> 2)) * BP + wn + j * 16 + (q & 3) * 4;
                    const s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                        (__attribute__((address_space(3))) s4 *)(b));
                    const s4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                        (__attribute__((address_space(3))) s4 *)(b + 4 * BP));
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        ob[j].v[e] = (uint16_t)lo[e];
                        ob[j].v[e + 4] = (uint16_t)hi[e];
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < WM; ++i)
#pragma unroll
                for (int j = 0; j < WN; ++j) acc[i][j] = block_product(oa[i], ob[j], acc[i][j]);
        }
    };

    const int steps = (a.C + D - 1) / D;
    fetch(0);
    put(0);
    __syncthreads();
    for (int s = 0; s < steps; ++s) {
        if (s + 1 < steps) fetch((s + 1) * D);
        products(s & 1);
        if (s + 1 < steps) put((s + 1) & 1);
        __syncthreads();
    }

    // the adapters' part: lane l looks after the ids of rows l, l + 64 of the tile
    int mine[BM / 64];
    const int64_t wave_row = m0 + wm;
    if (a.n) {
#pragma unroll
        for (int i = 0; i < BM / 64; ++i) {
            const int64_t row = m0 + i * 64 + lane;
            mine[i] = row < a.rows ? a.ids[row] : -1;
        }
        for (int last = -1;;) {
            int cur = 0x7fffffff;
#pragma unroll
            for (int i = 0; i < BM / 64; ++i) cur = min(cur, next_adapter(mine[i], last));
            if (cur >= a.n) break;
            last = cur;
            // which of the wave's rows: row 16 i + 4 g + e
            bool hit[WM][4];
            bool any = false;
#pragma unroll
            for (int i = 0; i < WM; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int r = wm + i * 16 + g * 4 + e;
                    int id = __shfl(mine[0], r & 63);
                    if constexpr (BM == 128) {
                        const int up = __shfl(mine[BM / 64 - 1], r & 63);
                        id = r >= 64 ? up : id;
                    }
                    hit[i][e] = id == cur;
                    any |= hit[i][e];
                }
            if (!__any(any)) continue;
            const float sc = !TRANS && a.scale ? a.scale[cur] : 1.f;
            const T *f = reinterpret_cast<const T *>(a.f) + (int64_t)cur * a.cols * a.r;
            constexpr int Q = sizeof(T) == 2 ? 3 : 1;
#pragma unroll
            for (int i = 0; i < WM; ++i) {
                bool in = false;
#pragma unroll
                for (int e = 0; e < 4; ++e) in |= hit[i][e];
                if (!__any(in)) continue;
                f4 z[WN];
#pragma unroll
                for (int j = 0; j < WN; ++j) z[j] = f4{0.f, 0.f, 0.f, 0.f};
                const float *t = a.t + clamp_row(wave_row + i * 16 + q, a.rows) * a.r;
                for (int k0 = 0; k0 < a.r; k0 += kStep<T>) {
                    const int k = k0 + g * E;
                    float tv[E];
#pragma unroll
                    for (int e = 0; e < E; ++e) tv[e] = k + e < a.r ? t[k + e] * sc : 0.f;
                    Operand<T> ot[Q];
                    split_operand(tv, ot);
#pragma unroll
                    for (int j = 0; j < WN; ++j) {
                        const int col = min(n0 + wn + j * 16 + q, a.cols - 1);
                        const Operand<T> of = TRANS ? gather_operand(f + (int64_t)k * a.cols + col, a.cols, a.r - k)
                                                    : load_operand(f + (int64_t)col * a.r + k, a.r - k);
#pragma unroll
                        for (int p = 0; p < Q; ++p) z[j] = block_product(ot[p], of, z[j]);
                    }
                }
#pragma unroll
                for (int j = 0; j < WN; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[i][j][e] += hit[i][e] ? z[j][e] : 0.f;
            }
        }
    }

#pragma unroll
    for (int i = 0; i < WM; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int64_t row = wave_row + i * 16 + g * 4 + e;
            bool bad = false;
            if (a.n) {
                const int r = wm + i * 16 + g * 4 + e;
                int id = __shfl(mine[0], r & 63);
                if constexpr (BM == 128) {
                    const int up = __shfl(mine[BM / 64 - 1], r & 63);
                    id = r >= 64 ? up : id;
                }
                bad = id >= a.n;
            }
#pragma unroll
            for (int j = 0; j < WN; ++j) {
                const int col = n0 + wn + j * 16 + q;
                if (row < a.rows && col < a.cols) {
                    const float y = acc[i][j][e] + (a.bias ? a.bias[col] : 0.f);
                    store_as(reinterpret_cast<T *>(a.out) + row * a.os + col, bad ? NAN : y);
                }
            }
        }
}

template <typename T, bool TRANS, int BM, int BN>
hipError_t go(const WideArgs &a, hipStream_t s)
{
    const int64_t tm = (a.rows + BM - 1) / BM;
    const int tn = (a.cols + BN - 1) / BN;
    // a launch holds fewer than 2^24 workgroups: more rows in several
    const int64_t most = std::max<int64_t>(1, (1 << 22) / tn);
    for (int64_t at = 0; at < tm; at += most) {
        WideArgs p = a;
        const int64_t m = std::min(most, tm - at), row = at * BM;
        p.v = (const T *)a.v + row * a.vs;
        p.out = (T *)a.out + row * a.os;
        p.rows = a.rows - row;
        if (at + m < tm) p.rows = std::min<int64_t>(p.rows, m * BM);
        if (a.n) {
            p.t = a.t + row * a.r;
            p.ids = a.ids + row;
        }
        hipLaunchKernelGGL((project_wide<T, TRANS, BM, BN>), dim3((unsigned)(m * tn)), dim3(256), 0, s, p, (int)m, tn);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename T, bool TRANS>
hipError_t choose(const WideArgs &a, hipStream_t s)
{
    const int64_t big = ((a.rows + 127) / 128) * ((a.cols + 127) / 128);
    if (big >= 256) return go<T, TRANS, 128, 128>(a, s);
    return go<T, TRANS, 64, 64>(a, s);
}

}  // namespace

hipError_t launch_wide(const WideArgs &a, int dtype, bool trans, hipStream_t s)
{
    if (dtype == DT_BF16) return trans ? choose<uint16_t, true>(a, s) : choose<uint16_t, false>(a, s);
    return trans ? choose<float, true>(a, s) : choose<float, false>(a, s);
}

}  // namespace fs
