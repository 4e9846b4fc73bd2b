// cyc_window.h -- what the kernels of attention with a window share: arguments, and which keys a position sees.
#pragma once
#include "cyc_internal.h"

namespace cyc {

// Key j is visible to position p: the sinks and the last `window` positions up to p itself (window INT_MAX: all of them).
__host__ __device__ inline bool sees(int p, int j, int window, int sinks) { return j <= p && (p - j < window || j < sinks); }

// How long `all` equal workgroups take, of which a compute unit holds two: `two` (any unit) a round of 512, `one` where there are 256 or fewer.
__host__ __device__ inline int64_t rounds_time(unsigned all, int64_t two, int64_t one)
{
    const unsigned rest = all % 512;
    return all / 512 * two + (rest == 0 ? 0 : rest <= 256 ? one : two);
}
// Tiles of kt keys that `rows` rows, of `group` heads at `queries` positions or fewer, see at most among `keys`.
int64_t most_tiles(int64_t keys, int window, int sinks, int64_t rows, int64_t group, int64_t queries, int64_t kt);

// batch x heads x rows, row by row of d bfloat16; strides in bytes
struct Strided {
    const char *base;
    int64_t batch, head, row;
};

// One call of cyc_recurrence_attention_window or of its gradient.  Query i stands at position i + M - N; head h reads key head h / group.
struct WindowProblem {
    Strided Q, K, V, O;
    float *lse;                          // batch x heads x N, dense; may be null going forward
    int batch, heads, kv_heads, group, N, M, d;
    int window, sinks;
    Strided dO, dQ, dK, dV;              // gradient only
};

// One call of cyc_recurrence_attention_paged.  Sequence b's new tokens are rows starts[b] .. starts[b+1] - 1 of Q and O; they are the
// last ones of its lengths[b] keys, key j of which is row j % page of page table[b][j / page].
struct PagedProblem {
    const char *Q, *K, *V;
    char *O;
    int64_t q_token, q_head, o_token, o_head;              // bytes
    int64_t page_bytes, head_bytes, row_bytes;             // strides within the cache, K and V alike
    const int *table, *lengths, *starts;
    int64_t table_stride;                                  // entries
    int tokens, seqs, heads, kv_heads, group, d;
    int pages, page_shift, max_pages, max_new;
    int window, sinks;
};

// One call of cyc_cache_append.
struct AppendProblem {
    const char *K, *V;
    char *K_cache, *V_cache;
    int64_t k_token, k_head, v_token, v_head, page_bytes, head_bytes, row_bytes, table_stride;
    const int *table, *lengths, *starts;
    int tokens, seqs, kv_heads, d, pages, page_shift, max_pages;
};

int64_t window_workspace_bytes(const WindowProblem &p);
hipError_t launch_window(const WindowProblem &p, void *workspace, int64_t workspace_bytes, hipStream_t s);
int64_t window_grad_workspace_bytes(const WindowProblem &p);
hipError_t launch_window_grad(const WindowProblem &p, void *workspace, int64_t workspace_bytes, hipStream_t s);
int64_t paged_workspace_bytes(const PagedProblem &p);
hipError_t launch_paged(const PagedProblem &p, void *workspace, int64_t workspace_bytes, hipStream_t s);
hipError_t launch_append(const AppendProblem &p, hipStream_t s);

// The sequence that row t of Q belongs to: the last b with starts[b] <= t (starts ascends; whatever it holds, 0 <= b < seqs).
__device__ __forceinline__ int sequence_of(const int *starts, int seqs, int t)
{
    int lo = 0, hi = seqs - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (starts[mid] <= t) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

}  // namespace cyc
