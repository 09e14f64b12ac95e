// What the kernels of the projection with adapters share: loads of a lane's
// matrix-core operands, and the walk over the adapters that a tile's rows name.
//
// Matrix-core operands.  A 16 x 16 block of products takes, per lane l, kE
// adjacent values along the summed axis of row (or column) l % 16, starting at
// kE * (l / 16): float32 as kE = 4 products of 4 terms each, the terms dealt
// out so that a lane's four lie side by side in memory (both operands agree,
// and a sum has no order), bf16 as one of 32 terms, kE = 8.  The block's value
// [4 * (l / 16) + e][l % 16] ends in element e of lane l.
#pragma once

#include "rows.h"

namespace fs {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef uint16_t h8 __attribute__((ext_vector_type(8)));

template <typename T>
struct Operand;
template <>
struct Operand<float> {
    static constexpr int kE = 4;
    f4 v;
};
template <>
struct Operand<uint16_t> {
    static constexpr int kE = 8;
    h8 v;
};

template <typename T>
constexpr int kStep = 4 * Operand<T>::kE;  // terms of the summed axis a block product takes

__device__ __forceinline__ f4 block_product(const Operand<float> &a, const Operand<float> &b, f4 c)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[e], b.v[e], c, 0, 0, 0);
    return c;
}
__device__ __forceinline__ f4 block_product(const Operand<uint16_t> &a, const Operand<uint16_t> &b, f4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8, a.v), __builtin_bit_cast(bf8, b.v), c, 0, 0, 0);
}

// kE adjacent values at p (any alignment of the element); `have` of them exist,
// the rest are 0.
template <typename T>
__device__ __forceinline__ Operand<T> load_operand(const T *p, int have)
{
    Operand<T> o;
    if (have >= Operand<T>::kE) {
        o.v = __builtin_bit_cast(decltype(o.v), load_words<16>(p));
    } else {
#pragma unroll
        for (int e = 0; e < Operand<T>::kE; ++e) o.v[e] = e < have ? p[e] : (T)0;
    }
    return o;
}

// The same from values `step` elements apart.
template <typename T>
__device__ __forceinline__ Operand<T> gather_operand(const T *p, int64_t step, int have)
{
    Operand<T> o;
#pragma unroll
    for (int e = 0; e < Operand<T>::kE; ++e) o.v[e] = e < have ? p[e * step] : (T)0;
    return o;
}

// The smallest adapter above `last` that one of the wave's lanes names (its
// `id`, -1: none); INT_MAX when there is no more.
__device__ __forceinline__ int next_adapter(int id, int last)
{
    int v = id > last ? id : 0x7fffffff;
#pragma unroll
    for (int d = 32; d; d >>= 1) v = min(v, __shfl_xor(v, d));
    return __builtin_amdgcn_readfirstlane(v);
}

__device__ __forceinline__ int64_t clamp_row(int64_t row, int64_t rows) { return row < rows ? row : rows - 1; }

inline int grid_of(int64_t blocks) { return (int)(blocks < 1 ? 1 : blocks > (1 << 22) ? (1 << 22) : blocks); }

// out[rows][cols] = v[rows][C] times the shared matrix w (kernels of
// project_tiles_wide.hip): TRANS false: w [cols][C] (rows' outputs), true: w
// [C][cols] (rows' gradients); plus t [rows][r] (float32, already scaled for
// the gradient, times scale[i] otherwise) times the adapter's factor f:
// [n][cols][r] (TRANS false) or [n][r][cols] (true).
struct WideArgs {
    const void *v, *w, *f;
    void *out;
    int64_t rows, vs, ws, os;
    int C, cols, n, r;
    const float *bias, *scale, *t;
    const int *ids;
    float *parts;  // wide_parts() bytes: where the summed axis is split
};
size_t wide_parts(int64_t rows, int cols, int C, int dtype);
hipError_t launch_wide(const WideArgs &a, int dtype, bool trans, hipStream_t s);

}  // namespace fs
