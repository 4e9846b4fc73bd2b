// cyc_window.hip -- attention with a sliding window and sinks, over dense keys and over a paged cache.
//
//     O_i = sum_j exp(S_ij - lse_i) V_j,   S_ij = Q_i.K_j / sqrt(d),   lse_i = log sum_j exp S_ij   over the keys j that i sees.
//
// One wave per query and head: it walks the visible keys with a running maximum m, sum l and output o,
//     mh = max(m, S),  l <- exp(m - mh) l + exp(S - mh),  o <- exp(m - mh) o + exp(S - mh) V_j,
// its lanes sharing the d elements of a row.
#include "cyc_window.h"

#include <climits>

namespace cyc {
namespace {

__device__ __forceinline__ float wave_sum(float x)
{
#pragma unroll
    for (int m = 32; m; m >>= 1) x += __shfl_xor(x, m);
    return x;
}

// fetch(j, &k, &v): the addresses of key j's rows, or false where there is none that may be read
template <int D, class Fetch>
__device__ __forceinline__ void walk(const char *q, char *o, float *lse, int position, int window, int sinks, bool bad, Fetch &&fetch)
{
    constexpr int E = D / 64;
    const int l = threadIdx.x & 63;
    float qv[E], acc[E], m = -__builtin_inff(), sum = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        qv[e] = (float)((const __bf16 *)q)[l * E + e] * (1.0f / __builtin_sqrtf((float)D));
        acc[e] = 0;
    }
    const int lo = position - window + 1;                      // (window INT_MAX: below zero)
    for (int j = 0; j <= position && !bad; ++j) {
        if (j >= sinks && j < lo) {
            j = lo - 1;
            continue;
        }
        const char *k, *v;
        if (!fetch(j, &k, &v)) {
            bad = true;
            break;
        }
        float s = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) s = __builtin_fmaf(qv[e], (float)((const __bf16 *)k)[l * E + e], s);
        s = wave_sum(s);
        const float mh = __builtin_fmaxf(m, s), keep = m == mh ? 1.0f : expf(m - mh), w = expf(s - mh);
        sum = sum * keep + w;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = acc[e] * keep + w * (float)((const __bf16 *)v)[l * E + e];
        m = mh;
    }
    const bool empty = position < 0;
#pragma unroll
    for (int e = 0; e < E; ++e) ((__bf16 *)o)[l * E + e] = (__bf16)(bad ? __builtin_nanf("") : empty ? 0.0f : acc[e] / sum);
    if (lse && l == 0) *lse = empty ? -__builtin_inff() : m + logf(sum);
}

template <int D> __global__ __launch_bounds__(256) void window_kernel(WindowProblem p)
{
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= (int64_t)p.batch * p.heads * p.N) return;
    const int i = (int)(row % p.N), h = (int)(row / p.N % p.heads);
    const int64_t b = row / p.N / p.heads;
    const char *K = p.K.base + b * p.K.batch + h / p.group * p.K.head, *V = p.V.base + b * p.V.batch + h / p.group * p.V.head;
    walk<D>(p.Q.base + b * p.Q.batch + h * p.Q.head + i * p.Q.row, (char *)p.O.base + b * p.O.batch + h * p.O.head + i * p.O.row,
            p.lse ? p.lse + row : nullptr, i + p.M - p.N, p.window, p.sinks, false, [&](int j, const char **k, const char **v) {
                *k = K + j * p.K.row;
                *v = V + j * p.V.row;
                return true;
            });
}

template <int D> __global__ __launch_bounds__(256) void paged_kernel(PagedProblem p)
{
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= (int64_t)p.tokens * p.heads) return;
    const int t = (int)(row / p.heads), h = (int)(row % p.heads), b = sequence_of(p.starts, p.seqs, t);
    const int first = p.starts[b], end = p.starts[b + 1], n = p.lengths[b];
    if (t < first || t >= end) return;
    const bool bad = first < 0 || end > p.tokens || end - first > p.max_new || n < 0 || n > ((int64_t)p.max_pages << p.page_shift);
    const int *table = p.table + b * p.table_stride;
    walk<D>(p.Q + t * p.q_token + h * p.q_head, p.O + t * p.o_token + h * p.o_head, nullptr, n - end + t, p.window, p.sinks, bad,
            [&](int j, const char **k, const char **v) {
                const int at = table[j >> p.page_shift];
                if ((unsigned)at >= (unsigned)p.pages) return false;
                const int64_t off = at * p.page_bytes + h / p.group * p.head_bytes + (j & ((1 << p.page_shift) - 1)) * p.row_bytes;
                *k = p.K + off;
                *v = p.V + off;
                return true;
            });
}

}  // namespace

int64_t window_workspace_bytes(const WindowProblem &) { return 0; }

hipError_t launch_window(const WindowProblem &p, void *, int64_t, hipStream_t s)
{
    const int64_t rows = (int64_t)p.batch * p.heads * p.N;
    const dim3 grid((unsigned)((rows + 3) / 4)), block(256);
    return p.d == 128 ? launch_kernel(window_kernel<128>, grid, block, s, p) : launch_kernel(window_kernel<64>, grid, block, s, p);
}

int64_t paged_workspace_bytes(const PagedProblem &) { return 0; }

hipError_t launch_paged(const PagedProblem &p, void *, int64_t, hipStream_t s)
{
    const int64_t rows = (int64_t)p.tokens * p.heads;
    const dim3 grid((unsigned)((rows + 3) / 4)), block(256);
    return p.d == 128 ? launch_kernel(paged_kernel<128>, grid, block, s, p) : launch_kernel(paged_kernel<64>, grid, block, s, p);
}

}  // namespace cyc
