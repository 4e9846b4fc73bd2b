// cyc_window_grad.hip -- the gradient of attention with a sliding window and sinks.
//
// With P_ij = exp(S_ij - lse_i) over the keys that i sees, D_i = dO_i.O_i and dS_ij = P_ij (dO_i.V_j - D_i):
//     dQ_i = sum_j dS_ij K_j / sqrt(d),   dK_j = sum_i dS_ij Q_i / sqrt(d),   dV_j = sum_i P_ij dO_i,
// the last two also over the heads that share key j.  One wave per query for dQ and one per key for dK and dV, lanes along d.
#include "cyc_window.h"

namespace cyc {
namespace {

__device__ __forceinline__ float wave_sum(float x)
{
#pragma unroll
    for (int m = 32; m; m >>= 1) x += __shfl_xor(x, m);
    return x;
}

template <int E> __device__ __forceinline__ void load(float (&x)[E], const char *row)
{
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = (float)((const __bf16 *)row)[(threadIdx.x & 63) * E + e];
}
template <int E> __device__ __forceinline__ float dot(const float (&x)[E], const float (&y)[E])
{
    float s = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) s = __builtin_fmaf(x[e], y[e], s);
    return wave_sum(s);
}
template <int E> __device__ __forceinline__ void store(char *row, const float (&x)[E], float scale)
{
#pragma unroll
    for (int e = 0; e < E; ++e) ((__bf16 *)row)[(threadIdx.x & 63) * E + e] = (__bf16)(x[e] * scale);
}
__device__ __forceinline__ const char *row_of(const Strided &x, int64_t b, int h, int i) { return x.base + b * x.batch + h * x.head + i * x.row; }

template <int D> __global__ __launch_bounds__(256) void grad_q_kernel(WindowProblem p, float *Ds)
{
    constexpr int E = D / 64;
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= (int64_t)p.batch * p.heads * p.N) return;
    const int i = (int)(row % p.N), h = (int)(row / p.N % p.heads), position = i + p.M - p.N, g = h / p.group;
    const int64_t b = row / p.N / p.heads;
    const float scale = 1.0f / __builtin_sqrtf((float)D);
    float q[E], o[E], dO[E], k[E], v[E], dq[E] = {};
    load(q, row_of(p.Q, b, h, i));
    load(o, row_of(p.O, b, h, i));
    load(dO, row_of(p.dO, b, h, i));
    const float Di = dot(o, dO), lse = p.lse[row];
    if ((threadIdx.x & 63) == 0) Ds[row] = Di;
    for (int j = 0; j <= position; ++j) {
        if (!sees(position, j, p.window, p.sinks)) continue;
        load(k, row_of(p.K, b, g, j));
        load(v, row_of(p.V, b, g, j));
        const float w = expf(dot(q, k) * scale - lse) * (dot(dO, v) - Di);
#pragma unroll
        for (int e = 0; e < E; ++e) dq[e] = __builtin_fmaf(w, k[e], dq[e]);
    }
    store((char *)row_of(p.dQ, b, h, i), dq, scale);
}

template <int D> __global__ __launch_bounds__(256) void grad_kv_kernel(WindowProblem p, const float *Ds)
{
    constexpr int E = D / 64;
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= (int64_t)p.batch * p.kv_heads * p.M) return;
    const int j = (int)(row % p.M), g = (int)(row / p.M % p.kv_heads);
    const int64_t b = row / p.M / p.kv_heads;
    const float scale = 1.0f / __builtin_sqrtf((float)D);
    float q[E], dO[E], k[E], v[E], dk[E] = {}, dv[E] = {};
    load(k, row_of(p.K, b, g, j));
    load(v, row_of(p.V, b, g, j));
    for (int h = g * p.group; h < (g + 1) * p.group; ++h)
        for (int i = 0; i < p.N; ++i) {
            if (!sees(i + p.M - p.N, j, p.window, p.sinks)) continue;
            const int64_t at = (b * p.heads + h) * p.N + i;
            load(q, row_of(p.Q, b, h, i));
            load(dO, row_of(p.dO, b, h, i));
            const float w = expf(dot(q, k) * scale - p.lse[at]), ds = w * (dot(dO, v) - Ds[at]);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                dk[e] = __builtin_fmaf(ds, q[e], dk[e]);
                dv[e] = __builtin_fmaf(w, dO[e], dv[e]);
            }
        }
    store((char *)row_of(p.dK, b, g, j), dk, scale);
    store((char *)row_of(p.dV, b, g, j), dv, 1.0f);
}

}  // namespace

int64_t window_grad_workspace_bytes(const WindowProblem &p) { return ((int64_t)p.batch * p.heads * p.N * 4 + 15) / 16 * 16; }

hipError_t launch_window_grad(const WindowProblem &p, void *workspace, int64_t, hipStream_t s)
{
    const int64_t rows = (int64_t)p.batch * p.heads * p.N, keys = (int64_t)p.batch * p.kv_heads * p.M;
    const dim3 grid((unsigned)((rows + 3) / 4)), kgrid((unsigned)((keys + 3) / 4)), block(256);
    float *Ds = (float *)workspace;
    hipError_t e = hipSuccess;
    if (rows) e = p.d == 128 ? launch_kernel(grad_q_kernel<128>, grid, block, s, p, Ds) : launch_kernel(grad_q_kernel<64>, grid, block, s, p, Ds);
    if (e != hipSuccess || keys == 0) return e;
    return p.d == 128 ? launch_kernel(grad_kv_kernel<128>, kgrid, block, s, p, (const float *)Ds)
                      : launch_kernel(grad_kv_kernel<64>, kgrid, block, s, p, (const float *)Ds);
}

}  // namespace cyc
