// Internal declarations of the row operators (fs_logprobs, fs_project and
// their gradients): launch arguments, and the conversions their kernels share.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fs_internal.h"

namespace fs {

// The thread-local message behind fs_last_error (api.hip); returns `status`.
int row_error(int status, const char *msg);

struct LogprobArgs {
    const void *x;          // [rows][V], stride elements apart
    int64_t rows, stride;
    int V;
    float inv_t;            // 1 / temperature
    const int *labels;      // [rows] or null
    int n_top;
    float *logp, *entropy;  // [rows] or null
    float *norm;            // [rows][2] or null
    int *top_id;            // [rows][n_top] or null
    float *top_logp;        // [rows][n_top] or null
};

struct LogprobGradArgs {
    const void *x;
    int64_t rows, stride;
    int V;
    float inv_t;
    const int *labels;
    const float *norm, *entropy, *g_logp, *g_entropy;
    void *g;                // [rows][V], g_stride apart
    int64_t g_stride;
};

struct ProjArgs {
    int64_t rows;
    int K, M, n, r;         // inputs, outputs, adapters, rank
    const void *x, *w;
    int64_t xs, ws;         // row strides
    const float *bias;      // or null
    const void *a, *b;      // [n][r][K], [n][M][r]
    const float *scale;     // [n] or null
    const int *ids;         // [rows], null when n == 0
};

size_t logprobs_workspace(int64_t rows, int V, int dtype, int n_top);
hipError_t launch_logprobs(const LogprobArgs &a, int dtype, void *ws, hipStream_t s);
hipError_t launch_logprobs_grad(const LogprobGradArgs &a, int dtype, hipStream_t s);
size_t project_workspace(const ProjArgs &a, int dtype);
hipError_t launch_project(const ProjArgs &a, int dtype, void *y, int64_t ys, float *hidden, void *ws, hipStream_t s);
size_t project_grad_workspace(const ProjArgs &a, int dtype);
hipError_t launch_project_grad(const ProjArgs &a, int dtype, const void *g, int64_t gs, const float *hidden, void *gx,
                               int64_t gxs, void *ga, void *gb, void *ws, hipStream_t s);

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
// bf16, round to nearest even (the hardware's conversion)
__device__ __forceinline__ uint16_t to_bf16(float f) { return __builtin_bit_cast(uint16_t, (__bf16)f); }
__device__ __forceinline__ void store_as(float *p, float v) { *p = v; }
__device__ __forceinline__ void store_as(uint16_t *p, float v) { *p = to_bf16(v); }

// 4, 8 or 16 adjacent bytes at an address of any alignment its elements may
// have: one load or store (as an array of 16-bit elements the compiler takes
// it apart).
template <int BYTES>
struct Words {
    typedef uint32_t type __attribute__((ext_vector_type(BYTES / 4)));
    typedef uint32_t at2 __attribute__((ext_vector_type(BYTES / 4), aligned(2)));
    typedef uint32_t at4 __attribute__((ext_vector_type(BYTES / 4), aligned(4)));
};
template <int BYTES, typename T>
__device__ __forceinline__ typename Words<BYTES>::type load_words(const T *p)
{
    if constexpr (sizeof(T) == 2) return *reinterpret_cast<const typename Words<BYTES>::at2 *>(p);
    else return *reinterpret_cast<const typename Words<BYTES>::at4 *>(p);
}
template <int BYTES, typename T>
__device__ __forceinline__ void store_words(T *p, typename Words<BYTES>::type v)
{
    if constexpr (sizeof(T) == 2) *reinterpret_cast<typename Words<BYTES>::at2 *>(p) = v;
    else *reinterpret_cast<typename Words<BYTES>::at4 *>(p) = v;
}
// The N elements of such words as float32, and back.
template <typename T, int N, typename W>
__device__ __forceinline__ void unpack(W w, float *v)
{
#pragma unroll
    for (int e = 0; e < N; ++e) {
        if constexpr (sizeof(T) == 4) v[e] = __uint_as_float(w[e]);
        else v[e] = __uint_as_float(e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
    }
}
template <typename T, int N>
__device__ __forceinline__ typename Words<N * sizeof(T)>::type pack(const float *v)
{
    typename Words<N * sizeof(T)>::type w;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < N; ++e) w[e] = __float_as_uint(v[e]);
    } else {
#pragma unroll
        for (int e = 0; e < N / 2; ++e) w[e] = (uint32_t)to_bf16(v[2 * e]) | (uint32_t)to_bf16(v[2 * e + 1]) << 16;
    }
    return w;
}

}  // namespace fs
