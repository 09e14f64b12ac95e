// A fully connected layer on rows with a low-rank adapter of each row's own
// choice, and its gradient:  y = W x + bias + s_i B_i (A_i x), i = ids[row].
// One thread per output value, one wave per row's product with a factor.
#include <algorithm>

#include "rows.h"

namespace fs {
namespace {

__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

// out[row][j] = s * sum_c v[row][c] f[i][...]: f [n][r][C] (by_rank) or [n][C][r]
template <typename T>
__global__ __launch_bounds__(256) void factor_rows(const T *v, int64_t vs, int64_t rows, int C, const T *f, int by_rank,
                                                   int n, int r, const float *scale, const int *ids, float *out)
{
    const int lane = threadIdx.x & 63;
    for (int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); row < rows; row += (int64_t)gridDim.x * 4) {
        const int i = ids[row];
        for (int j = 0; j < r; ++j) {
            float t = 0.f;
            if (i >= 0 && i < n) {
                const T *fi = f + (int64_t)i * r * C;
                for (int c = lane; c < C; c += 64)
                    t = fmaf(to_f32(v[row * vs + c]), to_f32(by_rank ? fi[(int64_t)j * C + c] : fi[(int64_t)c * r + j]), t);
                t = wave_sum(t);
                if (scale) t *= scale[i];
            }
            if (lane == 0) out[row * r + j] = i >= n ? NAN : t;
        }
    }
}

template <typename T>
__global__ __launch_bounds__(256) void project_each(ProjArgs a, T *y, int64_t ys, const float *h)
{
    const T *x = (const T *)a.x, *w = (const T *)a.w, *b = (const T *)a.b;
    const int64_t total = a.rows * a.M;
    for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < total; t += (int64_t)gridDim.x * 256) {
        const int64_t row = t / a.M;
        const int m = (int)(t - row * a.M);
        float v = 0.f;
        for (int c = 0; c < a.K; ++c) v = fmaf(to_f32(x[row * a.xs + c]), to_f32(w[m * a.ws + c]), v);
        const int i = a.n ? a.ids[row] : -1;
        if (i >= a.n) v = NAN;
        else if (i >= 0) {
            float z = 0.f;
            for (int j = 0; j < a.r; ++j) z = fmaf(h[row * a.r + j], to_f32(b[((int64_t)i * a.M + m) * a.r + j]), z);
            v += a.scale ? z * a.scale[i] : z;
        }
        store_as(y + row * ys + m, a.bias ? v + a.bias[m] : v);
    }
}

template <typename T>
__global__ __launch_bounds__(256) void grad_rows_each(ProjArgs a, const T *g, int64_t gs, const float *u, T *gx, int64_t gxs)
{
    const T *w = (const T *)a.w, *fa = (const T *)a.a;
    const int64_t total = a.rows * a.K;
    for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < total; t += (int64_t)gridDim.x * 256) {
        const int64_t row = t / a.K;
        const int k = (int)(t - row * a.K);
        float v = 0.f;
        for (int m = 0; m < a.M; ++m) v = fmaf(to_f32(g[row * gs + m]), to_f32(w[m * a.ws + k]), v);
        const int i = a.n ? a.ids[row] : -1;
        if (i >= a.n) v = NAN;
        else if (i >= 0)
            for (int j = 0; j < a.r; ++j) v = fmaf(u[row * a.r + j], to_f32(fa[((int64_t)i * a.r + j) * a.K + k]), v);
        store_as(gx + row * gxs + k, v);
    }
}

// out[i][j][c] (or [i][c][j]) = sum over rows of adapter i of s_i? * t[row][j] v[row][c]
template <typename T>
__global__ __launch_bounds__(256) void factor_grad_each(const float *t, const T *v, int64_t vs, int64_t rows, int C, int n,
                                                        int r, const float *scale, const int *ids, T *out, int by_rank)
{
    const int64_t total = (int64_t)n * r * C;
    for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < total; q += (int64_t)gridDim.x * 256) {
        const int c = (int)(q % C), j = (int)(q / C % r), i = (int)(q / C / r);
        double s = 0;
        for (int64_t row = 0; row < rows; ++row)
            if (ids[row] == i) s += (double)(t[row * r + j] * to_f32(v[row * vs + c]));
        if (scale) s *= scale[i];
        store_as(out + (by_rank ? q : ((int64_t)i * C + c) * r + j), (float)s);
    }
}

int grid_for(int64_t n, int per) { return (int)std::max<int64_t>(1, std::min<int64_t>((n + per - 1) / per, 1 << 20)); }

size_t rank_rows(const ProjArgs &a) { return ((size_t)a.rows * a.r * sizeof(float) + 255) & ~(size_t)255; }

template <typename T>
hipError_t project(const ProjArgs &a, T *y, int64_t ys, float *h, hipStream_t s)
{
    if (a.n)
        hipLaunchKernelGGL(factor_rows<T>, dim3(grid_for(a.rows, 4)), dim3(256), 0, s, (const T *)a.x, a.xs, a.rows, a.K,
                           (const T *)a.a, 1, a.n, a.r, nullptr, a.ids, h);
    hipLaunchKernelGGL(project_each<T>, dim3(grid_for(a.rows * a.M, 256)), dim3(256), 0, s, a, y, ys, h);
    return hipGetLastError();
}

template <typename T>
hipError_t project_grad(const ProjArgs &a, const T *g, int64_t gs, const float *h, T *gx, int64_t gxs, T *ga, T *gb,
                        float *hw, float *u, hipStream_t s)
{
    if (a.n && a.rows) {
        hipLaunchKernelGGL(factor_rows<T>, dim3(grid_for(a.rows, 4)), dim3(256), 0, s, g, gs, a.rows, a.M, (const T *)a.b,
                           0, a.n, a.r, a.scale, a.ids, u);
        if (!h && ga) {
            hipLaunchKernelGGL(factor_rows<T>, dim3(grid_for(a.rows, 4)), dim3(256), 0, s, (const T *)a.x, a.xs, a.rows,
                               a.K, (const T *)a.a, 1, a.n, a.r, nullptr, a.ids, hw);
            h = hw;
        }
    }
    if (gx && a.rows)
        hipLaunchKernelGGL(grad_rows_each<T>, dim3(grid_for(a.rows * a.K, 256)), dim3(256), 0, s, a, g, gs, u, gx, gxs);
    if (ga) {
        hipLaunchKernelGGL(factor_grad_each<T>, dim3(grid_for((int64_t)a.n * a.r * a.K, 256)), dim3(256), 0, s, u,
                           (const T *)a.x, a.xs, a.rows, a.K, a.n, a.r, nullptr, a.ids, ga, 1);
        hipLaunchKernelGGL(factor_grad_each<T>, dim3(grid_for((int64_t)a.n * a.r * a.M, 256)), dim3(256), 0, s, h, g, gs,
                           a.rows, a.M, a.n, a.r, a.scale, a.ids, gb, 0);
    }
    return hipGetLastError();
}

}  // namespace

size_t project_workspace(const ProjArgs &a, int) { return rank_rows(a); }

hipError_t launch_project(const ProjArgs &a, int dtype, void *y, int64_t ys, float *hidden, void *ws, hipStream_t s)
{
    float *h = hidden ? hidden : (float *)ws;
    return dtype == DT_BF16 ? project(a, (uint16_t *)y, ys, h, s) : project(a, (float *)y, ys, h, s);
}

size_t project_grad_workspace(const ProjArgs &a, int) { return 2 * rank_rows(a); }

hipError_t launch_project_grad(const ProjArgs &a, int dtype, const void *g, int64_t gs, const float *hidden, void *gx,
                               int64_t gxs, void *ga, void *gb, void *ws, hipStream_t s)
{
    float *u = (float *)ws, *hw = (float *)((char *)ws + rank_rows(a));
    if (dtype == DT_BF16)
        return project_grad(a, (const uint16_t *)g, gs, hidden, (uint16_t *)gx, gxs, (uint16_t *)ga, (uint16_t *)gb, hw, u, s);
    return project_grad(a, (const float *)g, gs, hidden, (float *)gx, gxs, (float *)ga, (float *)gb, hw, u, s);
}

}  // namespace fs
