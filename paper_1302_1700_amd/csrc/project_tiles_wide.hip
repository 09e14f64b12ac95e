// The shared projection's matrix product with the adapters' part added to its
// accumulators: out = v W + t F_i, i the adapter of the row.
//
// A workgroup of WR x WC waves computes a BM x BN tile, a part of BM / WR x BN /
// WC each wave: four waves for tiles of 64 and 128, eight for 256.  The summed
// axis is walked 128 bytes of each row at a time through two LDS buffers: while
// a step's products run, the next one is written to LDS from registers and the
// one after that is on its way from memory; one barrier a step.  A step is two
// halves.  In the smaller tiles each half's operands are read while the other
// half's products run, and no product waits for LDS.  The 256 x 256 tile has no
// registers for a second set of operands: it reads a half, waits, multiplies.
//
// LDS keeps a row's 16-byte pieces in an order turned by the row (piece p of
// row q at p ^ (q % 8)), so that the 16 rows an operand load touches fall on
// different banks.  For the gradient of the rows W lies the other way round;
// its tile keeps the order of memory, and bf16 operands are transposed by the
// LDS read itself.
//
// Blocks are computed as (columns) x (rows): a lane ends up with four adjacent
// columns of one row, stored together, and has one row's adapter to look at.
//
// The adapters' part: for every adapter that a row of the wave names, the
// product of t with its factor, added only to the rows that name it (an
// infinity in one adapter stays out of the others' rows).  bf16: t goes in as
// three bf16 values, each the rounding of what the ones before leave, which
// keep its 24 bits.
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

// The adapter's part of four columns of a row, added to y term by term.  Seldom
// taken: its addresses are kept from being computed ahead and held in registers.
template <typename T, bool TRANS>
__device__ __forceinline__ void add_adapter(const WideArgs &a, int64_t row, int col, float (&y)[4])
{
    asm volatile("" : "+v"(row), "+v"(col));
    const int id = a.ids[row];
    if (id < 0 || id >= a.n) return;
    const T *f = reinterpret_cast<const T *>(a.f) + (int64_t)id * a.cols * a.r;
    const float *t = a.t + row * a.r, sc = !TRANS && a.scale ? a.scale[id] : 1.f;
    float z[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
    for (int j = 0; j < a.r; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int c = min(col + e, a.cols - 1);
            z[e] = fmaf(t[j], to_f32(TRANS ? f[(int64_t)j * a.cols + c] : f[(int64_t)c * a.r + j]), z[e]);
        }
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = fmaf(z[e], sc, y[e]);
}

// WR x WC waves; two of them to a SIMD, 256 registers each.
template <typename T, bool TRANS, int BM, int BN, int WR, int WC>
__global__ __launch_bounds__(64 * WR * WC, 2) void project_tiles(WideArgs a, int tiles_m, int tiles_n, int per_split)
{
    constexpr int D = kDepth<T>, E = Operand<T>::kE;
    static_assert(D == 2 * kStep<T>, "two block products a step");
    constexpr int NT = 64 * WR * WC, RT = NT / 8;            // threads, rows staged at once
    constexpr int WM = BM / 16 / WR, WN = BN / 16 / WC;      // 16 x 16 blocks of a wave
    constexpr int PA = BM / RT, PB = BN / RT;                // 16-byte pieces a thread stages
    constexpr bool AHEAD = WM * WN <= 16;                    // registers for both halves' operands
    constexpr int BP = TRANS ? BN + (sizeof(T) == 2 ? 16 : 4) : 0;  // pitch of W's tile in the order of memory
    constexpr int A_BYTES = BM * 128, B_BYTES = TRANS ? D * BP * (int)sizeof(T) : BN * 128;
    __shared__ __align__(16) char lds[2 * (A_BYTES + B_BYTES)];

    // Tiles in the order of the XCDs (workgroup i runs on XCD i % 8): each takes
    // a run of them, eight tile rows deep, so that its L2 holds their operands.
    int tile;
    {
        const int tiles = tiles_m * tiles_n, per = tiles / 8, more = tiles % 8, xcd = blockIdx.x % 8;
        tile = xcd * per + min(xcd, more) + blockIdx.x / 8;
        const int group = 8 * tiles_n, g0 = tile / group * 8, high = min(8, tiles_m - g0), in = tile % group;
        tile = (g0 + in % high) * tiles_n + in / high;
    }
    // blockIdx.y's stretch of the summed axis (per_split: the whole of it)
    const int c_begin = (int)blockIdx.y * per_split, C = min(a.C - c_begin, per_split);
    const int64_t m0 = (int64_t)(tile / tiles_n) * BM;
    const int n0 = tile % tiles_n * BN;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, q = lane & 15, g = lane >> 4;
    const int wm = wave / WC * (BM / WR), wn = wave % WC * (BN / WC);

    // What the thread stages: pieces of rows (a row's eight pieces by eight
    // threads), or of W's rows of BN columns; a row or column past the end is
    // the last one, its products are not stored.
    constexpr int RPB = BN / E;  // pieces of a row of W as in memory
    const T *va = reinterpret_cast<const T *>(a.v) + m0 * a.vs + c_begin;
    const T *wb = reinterpret_cast<const T *>(a.w) + (TRANS ? (int64_t)c_begin * a.ws + n0 : (int64_t)n0 * a.ws + c_begin);
    // Large tiles: buffer loads, whose addresses are one register a piece and a
    // scalar that moves along (as pointers they took two each and spilled).
    // The host sends only 16-byte aligned rows of less than 2^31 bytes a tile, and
    // whole steps.  Smaller tiles: any row stride.
    constexpr bool BUFFER = !AHEAD;
    using Place = typename std::conditional<BUFFER, uint32_t, int64_t>::type;
    Place pa[PA], pb[PB];  // a thread's places from there, in bytes
#pragma unroll
    for (int i = 0; i < PA; ++i)
        pa[i] = (Place)(((clamp_row(m0 + i * RT + (threadIdx.x >> 3), a.rows) - m0) * a.vs + (threadIdx.x & 7) * E) * sizeof(T));
#pragma unroll
    for (int i = 0; i < PB; ++i) {
        const int piece = i * NT + threadIdx.x;
        if constexpr (TRANS) {
            int col = piece % RPB * E;
            if (a.cols % E == 0) col = min(n0 + col, a.cols - E) - n0;  // whole pieces lie inside or outside
            pb[i] = (Place)((piece / RPB * a.ws + col) * sizeof(T));
        } else {
            pb[i] = (Place)(((min(n0 + i * RT + (int)(threadIdx.x >> 3), a.cols - 1) - n0) * a.ws + (threadIdx.x & 7) * E) *
                               sizeof(T));
        }
    }
    const auto place = [](const T *base, Place bytes) {
        return reinterpret_cast<const T *>(reinterpret_cast<const char *>(base) + bytes);
    };
    // steps are fetched in their order: the bases move along
    typedef decltype(Operand<T>::v) Piece;  // 16 bytes
    Piece ra[PA], rb[PB];
    auto advance = [&]() {
        va += D;
        wb += TRANS ? D * a.ws : D;
    };
    const __amdgpu_buffer_rsrc_t buf_a = __builtin_amdgcn_make_buffer_rsrc((void *)va, 0, 0x7fffffff, 0x00020000);
    const __amdgpu_buffer_rsrc_t buf_b = __builtin_amdgcn_make_buffer_rsrc((void *)wb, 0, 0x7fffffff, 0x00020000);
    int move_a = 0, move_b = 0;
    auto fetch = [&]() {
        if constexpr (BUFFER) {
#pragma unroll
            for (int i = 0; i < PA; ++i)
                ra[i] = __builtin_bit_cast(Piece, __builtin_amdgcn_raw_buffer_load_b128(buf_a, pa[i], move_a, 0));
#pragma unroll
            for (int i = 0; i < PB; ++i)
                rb[i] = __builtin_bit_cast(Piece, __builtin_amdgcn_raw_buffer_load_b128(buf_b, pb[i], move_b, 0));
            // past the last step the last one again: nobody reads it
            const bool more = move_a + 128 < C * (int)sizeof(T);
            move_a += more ? 128 : 0;
            move_b += more ? (TRANS ? D * (int)a.ws * (int)sizeof(T) : 128) : 0;
        } else {
#pragma unroll
            for (int i = 0; i < PA; ++i) ra[i] = __builtin_bit_cast(Piece, load_words<16>(place(va, pa[i])));
#pragma unroll
            for (int i = 0; i < PB; ++i) rb[i] = __builtin_bit_cast(Piece, load_words<16>(place(wb, pb[i])));
            advance();
        }
    };
    // the last step's terms past the end are 0, and W's columns past the end stay unread
    auto fetch_checked = [&](int step) {
        const int c0 = step * D;
#pragma unroll
        for (int i = 0; i < PA; ++i) ra[i] = load_operand(place(va, pa[i]), C - c0 - (int)(threadIdx.x & 7) * E).v;
#pragma unroll
        for (int i = 0; i < PB; ++i) {
            if constexpr (TRANS) {
                const int piece = i * NT + threadIdx.x;
                const int have = a.cols % E == 0 ? E : a.cols - (n0 + piece % RPB * E);
                rb[i] = load_operand(place(wb, pb[i]), c0 + piece / RPB < C ? have : 0).v;
            } else {
                rb[i] = load_operand(place(wb, pb[i]), C - c0 - (int)(threadIdx.x & 7) * E).v;
            }
        }
        advance();
    };
    auto put = [&](int at) {
        char *la = lds + at * (A_BYTES + B_BYTES), *lb = la + A_BYTES;
        const int turned = (threadIdx.x >> 3) * 128 + (((threadIdx.x & 7) ^ (threadIdx.x >> 3 & 7)) << 4);
#pragma unroll
        for (int i = 0; i < PA; ++i)
            *reinterpret_cast<Piece *>(la + i * RT * 128 + turned) = ra[i];
#pragma unroll
        for (int i = 0; i < PB; ++i) {
            const int piece = i * NT + threadIdx.x;
            char *to = TRANS ? lb + (piece / RPB * BP + piece % RPB * E) * (int)sizeof(T) : lb + i * RT * 128 + turned;
            *reinterpret_cast<Piece *>(to) = rb[i];
        }
    };
    f4 acc[WM][WN];
#pragma unroll
    for (int i = 0; i < WM; ++i)
#pragma unroll
        for (int j = 0; j < WN; ++j) acc[i][j] = f4{0.f, 0.f, 0.f, 0.f};

    // The adapters' part first, while the accumulators are all that is held.
    int id[WM];
#pragma unroll
    for (int i = 0; i < WM; ++i) {
        const int64_t row = m0 + wm + i * 16 + q;
        id[i] = a.n && row < a.rows ? a.ids[row] : -1;
    }
    bool bad = false;  // one of the lane's rows names an adapter that is not there
#pragma unroll
    for (int i = 0; i < WM; ++i) bad |= a.n && id[i] >= a.n;
    int again = 0;  // the lane's rows (bit i) whose adapter's part is added at the end
    if (a.n && per_split >= a.C) {
        for (int last = -1;;) {
            int low = 0x7fffffff;
#pragma unroll
            for (int i = 0; i < WM; ++i) low = id[i] > last ? min(low, id[i]) : low;
            const int cur = next_adapter(low, last);
            if (cur >= a.n) break;
            last = cur;
            const float sc = !TRANS && a.scale ? a.scale[cur] : 1.f;
            const T *f = reinterpret_cast<const T *>(a.f) + (int64_t)cur * a.cols * a.r;
            constexpr int Q = sizeof(T) == 2 ? 3 : 1, H = WM < 4 ? WM : 4;
            for (int k0 = 0; k0 < a.r; k0 += kStep<T>) {
                const int k = k0 + g * E;
                // Whole operands lie inside or outside the rank: loads without
                // branches, all in flight together.
                const bool even = a.r % E == 0;
                const int at = even ? min(k, a.r - E) : k, have = even ? E : a.r - k;
                Operand<T> of[WN];
#pragma unroll
                for (int j = 0; j < WN; ++j) {
                    const int col = min(n0 + wn + j * 16 + q, a.cols - 1);
                    of[j] = TRANS ? gather_operand(f + (int64_t)at * a.cols + col, a.cols, have)
                                  : load_operand(f + (int64_t)col * a.r + at, have);
                }
#pragma unroll
                for (int h = 0; h < WM; h += H) {
                    float tv[H][E];
#pragma unroll
                    for (int i = 0; i < H; ++i) {
                        const float *t = a.t + clamp_row(m0 + wm + (h + i) * 16 + q, a.rows) * a.r + at;
                        if (even) {
#pragma unroll
                            for (int e = 0; e < E; e += 4) unpack<float, 4>(load_words<16>(t + e), tv[i] + e);
                        } else {
#pragma unroll
                            for (int e = 0; e < E; ++e) tv[i][e] = e < have ? t[e] : 0.f;
                        }
                    }
#pragma unroll
                    for (int i = 0; i < H; ++i) {
                        const bool hit = id[h + i] == cur;
                        if (!__any(hit)) continue;
                        Operand<T> ot[Q];
#pragma unroll
                        for (int e = 0; e < E; ++e) tv[i][e] = k < a.r ? tv[i][e] : 0.f;
                        split_operand(tv[i], ot);
#pragma unroll
                        for (int j = 0; j < WN; ++j) {
                            f4 z = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                            for (int p = 0; p < Q; ++p) z = block_product(of[j], ot[p], z);
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const float y = acc[h + i][j][e];
                                acc[h + i][j][e] = TRANS ? y + (hit ? z[e] : 0.f) : hit ? fmaf(z[e], sc, y) : y;
                            }
                        }
                    }
                }
            }
        }
    }

    // A row where that is not finite gets it at the end instead, term by term:
    // these products also have terms that the definition does not, 0 in exact
    // arithmetic but NaN beside an infinity.  They are the lanes past the rank (the
    // factor's last values once more, times 0) and, of a bf16 product, the second
    // and third parts of a value (which an infinity does not have, nor a float32
    // value that rounds to one).  Finite rows pay a look at the accumulators for
    // it (without adapters too: inside the condition above the 256 x 256 tile
    // spills 480 bytes a thread); masks on every operand instead: 550,000 x 242 ->
    // 15, 13 mixed adapters, the gradients: 1173 us, without them 1063.
#pragma unroll
    for (int i = 0; i < WM; ++i) {
        f4 zero = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < WN; ++j) zero = __builtin_elementwise_fma(acc[i][j], f4{0.f, 0.f, 0.f, 0.f}, zero);
        const bool off = zero[0] + zero[1] + zero[2] + zero[3] != 0.f;
        again |= off ? 1 << i : 0;
    }
    if (BUFFER || __any(again)) {  // (as a branch the largest tile spills)
#pragma unroll
        for (int i = 0; i < WM; ++i)
#pragma unroll
            for (int j = 0; j < WN; ++j) acc[i][j] = again & 1 << i ? f4{0.f, 0.f, 0.f, 0.f} : acc[i][j];
    }

    auto read = [&](int at, int half, Operand<T>(&oa)[WM], Operand<T>(&ob)[WN]) {
        const char *la = lds + at * (A_BYTES + B_BYTES), *lb = la + A_BYTES;
        const int turned = q * 128 + (((half * 4 + g) ^ (q & 7)) << 4);
#pragma unroll
        for (int i = 0; i < WM; ++i)
            oa[i] = *reinterpret_cast<const Operand<T> *>(la + (wm + i * 16) * 128 + turned);
#pragma unroll
        for (int j = 0; j < WN; ++j) {
            if constexpr (!TRANS) {
                ob[j] = *reinterpret_cast<const Operand<T> *>(lb + (wn + j * 16) * 128 + turned);
            } else if constexpr (sizeof(T) == 4) {
                const float *b = reinterpret_cast<const float *>(lb) + (half * 16 + g * 4) * BP + wn + j * 16 + q;
#pragma unroll
                for (int e = 0; e < 4; ++e) ob[j].v[e] = b[e * BP];
            } else {
                // 16 lanes read four rows of 16 columns, four columns a lane, and get a column each
                const uint16_t *b = reinterpret_cast<const uint16_t *>(lb) + (half * 32 + g * 8 + (q >> 2)) * BP + wn +
                                    j * 16 + (q & 3) * 4;
                const s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4 *)(b));
                const s4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4 *)(b + 4 * BP));
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    ob[j].v[e] = (uint16_t)lo[e];
                    ob[j].v[e + 4] = (uint16_t)hi[e];
                }
            }
        }
    };
    auto products = [&](const Operand<T>(&oa)[WM], const Operand<T>(&ob)[WN]) {
#pragma unroll
        for (int i = 0; i < WM; ++i)
#pragma unroll
            for (int j = 0; j < WN; ++j) acc[i][j] = block_product(ob[j], oa[i], acc[i][j]);
    };

    const int steps = (C + D - 1) / D;
    // steps that are read without checks
    const int whole = TRANS && a.cols % E != 0 && n0 + BN > a.cols ? 0 : C / D;
    auto get = [&](int step) {
        if (BUFFER || step < whole) fetch();
        else if (step < steps) fetch_checked(step);
    };
    get(0);
    put(0);
    get(1);
    __syncthreads();
    int s = 0;
    if constexpr (AHEAD) {
        Operand<T> oa[2][WM], ob[2][WN];
        read(0, 0, oa[0], ob[0]);
        for (; s + 2 < whole; ++s) {
            put((s + 1) & 1);
            fetch();
            read(s & 1, 1, oa[1], ob[1]);
            products(oa[0], ob[0]);
            __syncthreads();
            read((s + 1) & 1, 0, oa[0], ob[0]);
            products(oa[1], ob[1]);
        }
        for (; s < steps; ++s) {
            if (s + 1 < steps) put((s + 1) & 1);
            get(s + 2);
            read(s & 1, 1, oa[1], ob[1]);
            products(oa[0], ob[0]);
            __syncthreads();
            if (s + 1 < steps) read((s + 1) & 1, 0, oa[0], ob[0]);
            products(oa[1], ob[1]);
        }
    } else {
        Operand<T> oa[WM], ob[WN];
        for (; s < steps; ++s) {
            put((s + 1) & 1);
            fetch();
            read(s & 1, 0, oa, ob);
            __builtin_amdgcn_s_setprio(1);
            products(oa, ob);
            __builtin_amdgcn_s_setprio(0);
            read(s & 1, 1, oa, ob);
            __builtin_amdgcn_s_setprio(1);
            products(oa, ob);
            __builtin_amdgcn_s_setprio(0);
            __syncthreads();
        }
    }

    if (per_split < a.C) {
        float *part = a.parts + (int64_t)blockIdx.y * a.rows * a.cols;
#pragma unroll
        for (int i = 0; i < WM; ++i) {
            const int64_t row = m0 + wm + i * 16 + q;
            if (row >= a.rows) continue;
#pragma unroll
            for (int j = 0; j < WN; ++j) {
                const int col = n0 + wn + j * 16 + g * 4;
                float *to = part + row * a.cols + col;
                if (col + 4 <= a.cols) store_words<16>(to, __builtin_bit_cast(Words<16>::type, acc[i][j]));
                else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (col + e < a.cols) to[e] = acc[i][j][e];
                }
            }
        }
        return;
    }

#pragma unroll
    for (int j = 0; j < WN; ++j) {
        const int col = n0 + wn + j * 16 + g * 4;
        float bias[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) bias[e] = a.bias && col + e < a.cols ? a.bias[col + e] : 0.f;
#pragma unroll
        for (int i = 0; i < WM; ++i) {
            const int64_t row = m0 + wm + i * 16 + q;
            if (row >= a.rows) continue;
            const bool wrong = bad && a.ids[row] >= a.n;
            float out[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) out[e] = wrong ? NAN : acc[i][j][e] + bias[e];
            if (again & 1 << i) add_adapter<T, TRANS>(a, row, col, out);
            T *to = reinterpret_cast<T *>(a.out) + row * a.os + col;
            if (col + 4 <= a.cols) store_words<4 * sizeof(T)>(to, pack<T, 4>(out));
            else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (col + e < a.cols) store_as(to + e, out[e]);
            }
        }
    }
}

// Joins the stretches of the summed axis in their order and adds the adapters'
// part: a thread to four columns of a row.
template <typename T, bool TRANS>
__global__ __launch_bounds__(256) void project_join(WideArgs a, int splits)
{
    constexpr int E = Operand<T>::kE;
    const int quads = (a.cols + 3) / 4;
    const int64_t total = a.rows * quads;
    for (int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x; k < total; k += (int64_t)gridDim.x * 256) {
        const int64_t row = k / quads;
        const int col = (int)(k - row * quads) * 4, have = min(4, a.cols - col);
        const int id = a.n ? a.ids[row] : -1;
        float y[4] = {0.f, 0.f, 0.f, 0.f}, z[4] = {0.f, 0.f, 0.f, 0.f};
        // four columns from inside the row, moved into place where the row ends
        const int from = min(col, max(a.cols - 4, 0)), move = col - from;
        for (int s0 = 0; s0 < splits; s0 += 8) {
            float v[8][4];  // in flight together
#pragma unroll
            for (int s = 0; s < 8; ++s) {
                const float *p = a.parts + ((int64_t)min(s0 + s, splits - 1) * a.rows + row) * a.cols;
                if (a.cols >= 4) unpack<float, 4>(load_words<16>(p + from), v[s]);
                else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[s][e] = e < have ? p[col + e] : 0.f;
                }
            }
#pragma unroll
            for (int s = 0; s < 8; ++s)
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] += s0 + s < splits ? v[s][e] : 0.f;
        }
        if (move) {
#pragma unroll
            for (int e = 0; e < 3; ++e) y[e] = move == 1 ? y[e + 1] : move == 2 ? y[(e + 2) & 3] : y[3];
        }
        if (id >= 0 && id < a.n) {
            const T *f = reinterpret_cast<const T *>(a.f) + (int64_t)id * a.cols * a.r;
            const float *t = a.t + row * a.r;
            if constexpr (TRANS) {
#pragma unroll 4
                for (int j = 0; j < a.r; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        z[e] = fmaf(t[j], to_f32(f[(int64_t)j * a.cols + min(col + e, a.cols - 1)]), z[e]);
            } else {
                const bool whole = a.r % E == 0;
                for (int j = 0; j < a.r; j += E) {
                    Operand<T> o[4];  // of the four columns, in flight together
                    float tv[E];
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        o[e] = load_operand(f + (int64_t)min(col + e, a.cols - 1) * a.r + j, whole ? E : a.r - j);
#pragma unroll
                    for (int p = 0; p < E; ++p) tv[p] = t[min(j + p, a.r - 1)];
#pragma unroll
                    for (int p = 0; p < E; ++p)
                        if (whole || j + p < a.r) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) z[e] = fmaf(tv[p], to_f32((T)o[e].v[p]), z[e]);
                        }
                }
            }
            const float sc = !TRANS && a.scale ? a.scale[id] : 1.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = fmaf(z[e], sc, y[e]);
        }
        T *to = reinterpret_cast<T *>(a.out) + row * a.os + col;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < have) store_as(to + e, a.n && id >= a.n ? NAN : y[e] + (a.bias ? a.bias[col + e] : 0.f));
    }
}

template <typename T, bool TRANS, int BM, int BN, int WR, int WC>
hipError_t go(const WideArgs &a, int splits, int per_split, hipStream_t s)
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
        hipLaunchKernelGGL((project_tiles<T, TRANS, BM, BN, WR, WC>), dim3((unsigned)(m * tn), splits), dim3(64 * WR * WC), 0, s,
                           p, (int)m, tn, per_split);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

struct WidePlan {
    int tile, splits, per_split;
};

// 256 x 256 tiles where three CUs in four get one (4096^3 bf16 with adapters: 157
// us, in tiles of 128 183, of 64 267), 128 x 128 ones where each does (2048^3: 40,
// in tiles of 64 58), else 64 x 64 ones.  Where these are few and the summed axis
// long, it is split in stretches of four steps or more, joined by a second launch
// (32 x 4096 x 4096: 24 us, whole 65; 300 x 2048 x 2048, 160 tiles of 32 steps:
// 27, whole 22; 1500 x 1024 x 1000 float32, 384 tiles: 55, whole 53).
WidePlan wide_plan(int64_t rows, int cols, int C, int dtype, bool large)
{
    const auto tiles = [&](int b) { return ((rows + b - 1) / b) * ((cols + b - 1) / b); };
    WidePlan p{64, 1, C};
    if (large && dtype == DT_BF16 && tiles(256) >= 192) p.tile = 256;
    else if (tiles(128) >= 256) p.tile = 128;
    else if (tiles(64) < 512) {
        const int depth = dtype == DT_BF16 ? 64 : 32, steps = (C + depth - 1) / depth;
        const int splits = (int)std::min<int64_t>((511 + tiles(64)) / tiles(64), steps / 4);
        if (splits > 1 && steps >= (tiles(64) < 96 ? 16 : 40)) {
            p.per_split = (steps + splits - 1) / splits * depth;
            p.splits = (C + p.per_split - 1) / p.per_split;
        }
    }
    return p;
}

template <typename T, bool TRANS>
hipError_t run(const WideArgs &a, int dtype, hipStream_t s)
{
    const auto apart = [](const void *p, int64_t stride, int64_t rows) {
        return ((uintptr_t)p & 15) == 0 && stride * sizeof(T) % 16 == 0 && stride * (int64_t)sizeof(T) * rows < (1ll << 31);
    };
    const bool large = apart(a.v, a.vs, 256) && a.C % 64 == 0 && (!TRANS || a.cols % 8 == 0) && apart(a.w, a.ws, TRANS ? a.C + 64 : 256);
    const WidePlan p = wide_plan(a.rows, a.cols, a.C, dtype, large);
    if constexpr (sizeof(T) == 2)
        if (p.tile == 256) return go<T, TRANS, 256, 256, 2, 4>(a, 1, a.C, s);
    if (p.tile == 128) return go<T, TRANS, 128, 128, 2, 2>(a, 1, a.C, s);
    hipError_t e = go<T, TRANS, 64, 64, 2, 2>(a, p.splits, p.per_split, s);
    if (e != hipSuccess || p.splits == 1) return e;
    hipLaunchKernelGGL((project_join<T, TRANS>), dim3(grid_of((a.rows * ((a.cols + 3) / 4) + 255) / 256)), dim3(256), 0, s, a,
                       p.splits);
    return hipGetLastError();
}

}  // namespace

size_t wide_parts(int64_t rows, int cols, int C, int dtype)
{
    const WidePlan p = wide_plan(rows, cols, C, dtype, false);
    return p.splits > 1 ? (size_t)p.splits * rows * cols * sizeof(float) : 0;
}

hipError_t launch_wide(const WideArgs &a, int dtype, bool trans, hipStream_t s)
{
    if (dtype == DT_BF16) return trans ? run<uint16_t, true>(a, dtype, s) : run<uint16_t, false>(a, dtype, s);
    return trans ? run<float, true>(a, dtype, s) : run<float, false>(a, dtype, s);
}

}  // namespace fs
