// cyc_cache.hip -- new keys and values into the pages of a cache.
//
// Row t of K and V belongs to sequence b, starts[b] <= t < starts[b+1], and is its key lengths[b] - starts[b+1] + t.  A thread
// moves 16 bytes of K and of V, neighbours along a row; bound by memory for many tokens (16000 tokens x 8 heads x 128:
// 13 us, 4.9 TB/s read and written) and by the launch for few.
#include "cyc_window.h"

namespace cyc {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

__global__ __launch_bounds__(256) void append_kernel(AppendProblem p, int chunks)
{
    const int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (x >= (int64_t)p.tokens * chunks) return;
    const int t = (int)(x / chunks), part = (int)(x % chunks), per = p.d / 8, h = part / per, c = part % per;
    const int b = sequence_of(p.starts, p.seqs, t), first = p.starts[b], end = p.starts[b + 1], n = p.lengths[b];
    if (t < first || t >= end || first < 0 || end > p.tokens) return;
    const int64_t j = (int64_t)n - end + t;
    if (j < 0 || j >= (int64_t)p.max_pages << p.page_shift) return;
    const int at = p.table[b * p.table_stride + (j >> p.page_shift)];
    if ((unsigned)at >= (unsigned)p.pages) return;
    const int64_t off = at * p.page_bytes + h * p.head_bytes + (j & ((1 << p.page_shift) - 1)) * p.row_bytes + c * 16;
    *(i32x4 *)(p.K_cache + off) = *(const i32x4 *)(p.K + t * p.k_token + h * p.k_head + c * 16);
    *(i32x4 *)(p.V_cache + off) = *(const i32x4 *)(p.V + t * p.v_token + h * p.v_head + c * 16);
}

}  // namespace

hipError_t launch_append(const AppendProblem &p, hipStream_t s)
{
    const int chunks = p.kv_heads * (p.d / 8);
    const int64_t total = (int64_t)p.tokens * chunks;
    return launch_kernel(append_kernel, dim3((unsigned)((total + 255) / 256)), dim3(256), s, p, chunks);
}

}  // namespace cyc
