// Log probabilities of labels, entropy and best classes of rows of scores, and
// their gradient.
//
// With m the row's maximum, d_j = (x_j - m) / T <= 0, S = sum exp(d_j) and
// D = sum exp(d_j) d_j: log p_j = d_j - ln S and the entropy is ln S - D / S,
// two terms >= 0, so nothing cancels where the scores are far from 0.
// One wave per row, lanes striding over the classes.
#include <algorithm>

#include "rows.h"

namespace fs {
namespace {

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

template <typename T>
__device__ __forceinline__ T wave_max(T v)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) {
        const T o = __shfl_xor(v, d);
        v = o > v ? o : v;
    }
    return v;
}
__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

template <typename T>
__global__ __launch_bounds__(256) void logprobs_row(LogprobArgs a)
{
    const int lane = threadIdx.x & 63;
    for (int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); row < a.rows; row += (int64_t)gridDim.x * 4) {
        const T *x = reinterpret_cast<const T *>(a.x) + row * a.stride;
        float m = -INFINITY;
        bool bad = false;  // NaN or +inf
        for (int j = lane; j < a.V; j += 64) {
            const float v = to_f32(x[j]);
            bad |= !(v < INFINITY);
            m = fmaxf(m, v);
        }
        m = wave_max(m);
        bad = __any(bad);
        const bool empty = m == -INFINITY;
        float s = 0.f, d = 0.f;
        for (int j = lane; j < a.V; j += 64) {
            const float t = empty ? -INFINITY : (to_f32(x[j]) - m) * a.inv_t;
            const float e = expf(t);
            s += e;
            d += e * fmaxf(t, -1e30f);  // a class ruled out: 0, not 0 * inf
        }
        s = wave_sum(s);
        d = wave_sum(d);
        float log_s = empty ? 0.f : logf(s), ent = empty ? 0.f : log_s - d / s;
        if (bad) m = log_s = ent = NAN;
        if (lane == 0) {
            if (a.norm) {
                a.norm[2 * row] = m;
                a.norm[2 * row + 1] = log_s;
            }
            if (a.entropy) a.entropy[row] = ent;
            if (a.logp) {
                const int y = a.labels[row];
                float lp = 0.f;
                if (y >= a.V) lp = NAN;
                else if (y >= 0) lp = bad ? NAN : empty ? -INFINITY : (to_f32(x[y]) - m) * a.inv_t - log_s;
                a.logp[row] = lp;
            }
        }
        uint64_t last = ~0ull;  // the class listed before
        for (int t = 0; t < a.n_top; ++t) {
            uint64_t best = 0;
            if (!bad && last) {
                for (int j = lane; j < a.V; j += 64) {
                    const float v = to_f32(x[j]);
                    const uint64_t k = v == -INFINITY ? 0 : score_key(v, (uint32_t)j);
                    if (k < last && k > best) best = k;
                }
                best = wave_max(best);
            }
            last = best;
            if (lane == 0) {
                if (a.top_id) a.top_id[row * a.n_top + t] = best ? key_id(best) : -1;
                if (a.top_logp)
                    a.top_logp[row * a.n_top + t] =
                        bad ? NAN : best ? (key_score(best) - m) * a.inv_t - log_s : -INFINITY;
            }
        }
    }
}

template <typename T>
__global__ __launch_bounds__(256) void logprobs_grad_row(LogprobGradArgs a)
{
    const int lane = threadIdx.x & 63;
    for (int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); row < a.rows; row += (int64_t)gridDim.x * 4) {
        const T *x = reinterpret_cast<const T *>(a.x) + row * a.stride;
        T *g = reinterpret_cast<T *>(a.g) + row * a.g_stride;
        float m = a.norm[2 * row], log_s = a.norm[2 * row + 1];
        const bool empty = m == -INFINITY;
        const int y = a.labels ? a.labels[row] : -1;
        float gl = y >= 0 ? a.g_logp[row] : 0.f;
        if (y >= a.V) m = NAN;
        const float ge = a.g_entropy ? a.g_entropy[row] : 0.f, ent = a.g_entropy ? a.entropy[row] : 0.f;
        for (int j = lane; j < a.V; j += 64) {
            const float lp = (to_f32(x[j]) - m) * a.inv_t - log_s;
            const float p = expf(lp);
            float v = gl * ((j == y ? 1.f : 0.f) - p) - ge * p * (fmaxf(lp, -1e30f) + ent);
            v = empty && y < a.V ? 0.f : v * a.inv_t;
            store_as(g + j, v);
        }
    }
}

int row_grid(int64_t rows, int per_block) { return (int)std::min<int64_t>((rows + per_block - 1) / per_block, 1 << 20); }

}  // namespace

size_t logprobs_workspace(int64_t, int, int, int) { return 0; }

hipError_t launch_logprobs(const LogprobArgs &a, int dtype, void *, hipStream_t s)
{
    const dim3 grid(row_grid(a.rows, 4));
    if (dtype == DT_BF16) hipLaunchKernelGGL(logprobs_row<uint16_t>, grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL(logprobs_row<float>, grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_logprobs_grad(const LogprobGradArgs &a, int dtype, hipStream_t s)
{
    const dim3 grid(row_grid(a.rows, 4));
    if (dtype == DT_BF16) hipLaunchKernelGGL(logprobs_grad_row<uint16_t>, grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL(logprobs_grad_row<float>, grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace fs
