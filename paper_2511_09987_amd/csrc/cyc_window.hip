// cyc_window.hip -- attention with a sliding window and sinks, over dense keys and over a paged cache.
//
//     O_i = sum_j exp(S_ij - lse_i) V_j,   S_ij = Q_i.K_j / sqrt(d),   lse_i = log sum_j exp S_ij   over the keys j that i sees.
//
// A row is a (query, head) pair of one key head, row r = query r / group, head r % group of the group: heads that share keys
// share their tiles too, and one new token fills a wave as far as its group goes.  A workgroup takes a tile of rows and walks the
// tiles of keys that any of them sees, first those of the sinks, then those of the window, with a running maximum, sum and output per
// row (cyc_attn.hip has the recurrence and the operand layouts, which are the same here: S^T = K Q^T with the rows stationary in registers,
// O^T = V^T P^T).  A wave skips the tiles that none of its rows sees and masks only those that some row sees in part.
// Rows see different keys, so what must not reach a row is kept out twice: a masked score becomes -inf, its weight 0; and since 0 times
// an infinity or NaN in V would still spoil the sum, a masked tile whose values are not all finite is multiplied without those,
// which then go to the rows that see them.  Keys that no row of the workgroup sees are not read at all: rows
// of a tile outside [0, sinks) and the window's span are copied from a key inside.
//
// Many rows are bounded by vector work and by what one phase of a wave waits for from another: the matrix units are busy 35 % of the time (32/8
// heads x 8192 x 128, window 1024: 164 us, 790 TFLOP/s; a tile that all rows see 1100; with constant inputs, which draw less power, 6 % less
// time).  Few rows are bounded by memory (64 sequences of 1000 to 8000 keys, 32/8 heads x 128: 218 us and 6 for the join, 5.4 TB/s).
#include "cyc_window.h"
#include "cyc_tile.h"

#include <algorithm>
#include <climits>

namespace cyc {
namespace {

struct TileProblem {
    const char *Q, *K, *V;
    char *O;
    float *lse;
    int64_t q_batch, q_head, q_row, o_batch, o_head, o_row;         // bytes
    int64_t k_batch, k_head, k_row, v_batch, v_head, v_row;
    int64_t page_bytes, table_stride;
    const int *table, *lengths, *starts;
    int batch, kv_heads, group, N, M;                                // paged: batch = sequences, N and M by sequence
    int tiles;                                                       // tiles of rows (paged, long sequences: of all of them together)
    int tokens, pages, page_shift, max_pages, max_new, short_rows;
    int window, sinks, splits, run_tiles;                            // runs of keys: how many, and, few rows of sequences in pages, tiles in each at most
    float scale_log2e;
    // what a run leaves: part[run][row][d], refs[run][row][2].  Rows are those of O, (token or query, head) pairs, or, in launches for few rows,
    // SHORT_ROWS for each (problem, key head)
    float *part, *refs;
    int64_t part_rows, rows;                                         // rows of a run there; rows of O
    // paged, long sequences: splits is the most runs there may be, *chosen receives how many there are; most_tiles: of any list
    int *chosen;
    int most_tiles;
};
constexpr int LONG_ROWS = 128, SHORT_ROWS = 16;
constexpr int LEAST_TILES = 8;           // of a run of few rows: what pays for its start

enum Addressing { DENSE, PAGED_SHORT, PAGED_LONG };

// Sequence b's new tokens, those that lie within the call's whatever starts and lengths hold, and its keys: none where `bad`, and the rows are
// NaN.  What a workgroup writes and what joins it go by these numbers alone.
struct Sequence {
    int first, N, M;
    bool bad;
    __device__ __forceinline__ Sequence(const TileProblem &p, int b)
    {
        const int start = p.starts[b], end = p.starts[b + 1];
        M = p.lengths[b];
        bad = start < 0 || end > p.tokens || end < start || M < 0 || M > ((int64_t)p.max_pages << p.page_shift);
        first = start < 0 ? 0 : start > p.tokens ? p.tokens : start;
        N = (end < first ? first : end > p.tokens ? p.tokens : end) - first;
        bad |= N > p.max_new;
        if (bad) M = 0;
    }
};

// What a workgroup finds out about the sequences of its call, 64 at a time, a lane for each.
__device__ __forceinline__ int wave_most(int x)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) {
        const int y = __shfl_xor(x, d);
        x = x > y ? x : y;
    }
    return __builtin_amdgcn_readfirstlane(x);
}
// the most keys of any
__device__ __forceinline__ int most_keys(const int *lengths, int seqs)
{
    int most = 0;
    for (int b = threadIdx.x & 63; b < seqs; b += 64) most = lengths[b] > most ? lengths[b] : most;
    return wave_most(most);
}
// The tiles of `per` rows of the sequences with more than `less` rows, one sequence after the other: how many there are, the most keys of such a
// sequence and, for one tile, which sequence it belongs to and which of its tiles it is.
struct Tiles {
    int total = 0, keys = 0, seq = -1, tile = 0;
    int upto = 0, own = 0;                                 // of the last 64: tiles up to this lane's sequence, and its own
    // all: look at all sequences (total and keys are right then), not only up to the tile's
    __device__ __forceinline__ void find(const TileProblem &p, int per, int slot, bool all)
    {
        const int l = threadIdx.x & 63;
        int most = 0;
        for (int b0 = 0; b0 < p.batch && (all || seq < 0); b0 += 64) {
            const int b = b0 + l;
            int first = b < p.batch ? p.starts[b] : 0, end = b < p.batch ? p.starts[b + 1] : 0;
            const int length = all && b < p.batch ? p.lengths[b] : 0;
            first = first < 0 ? 0 : first > p.tokens ? p.tokens : first;
            end = end < first ? first : end > p.tokens ? p.tokens : end;
            const int rows = (end - first) * p.group, tiles = rows > p.short_rows ? (rows + per - 1) / per : 0;
            most = tiles > 0 && length > most ? length : most;
            own = upto = tiles;
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const int below = __shfl_up(upto, d);
                upto += l >= d ? below : 0;
            }
            pick(b0, slot);
            total += __builtin_amdgcn_readlane(upto, 63);
        }
        if (all) keys = wave_most(most);
    }
    // the slot's tile, if it is one of the last 64 sequences, the first of which is b0
    __device__ __forceinline__ void pick(int b0, int slot)
    {
        const uint64_t past = __builtin_amdgcn_ballot_w64(total + upto > slot);
        if (past == 0 || seq >= 0) return;
        const int at = __builtin_ctzll(past);
        seq = b0 + at;
        tile = slot - total - __builtin_amdgcn_readlane(upto - own, at);
    }
};

// Many rows: the time in nanoseconds of `groups` workgroups, each walking up to `tiles` tiles of keys, that are cut into `runs` runs each.  The chip
// holds 512, two on a compute unit, which take 1900 ns a tile of 64 keys x 128 rows x d 128 together (128 keys x d 64: 3100, twice the
// weights), or 1650 (2600) where there is one; to start takes 4 us.  Runs add a launch and the partial outputs, which are written and read
// at 3 TB/s.  (1024 + 7 x 1 tokens behind 6800 keys, 8 key heads, 256 workgroups: one run 209 us, two 147.)
__host__ __device__ inline int64_t part_time(int64_t rows, int64_t d) { return rows * (d + 2) * 4 / 3000; }      // of a run
__host__ __device__ inline int64_t long_cost(int groups, int tiles, int runs, int64_t part, int d)
{
    // (32-bit divisions: every workgroup of a paged call does this)
    const unsigned length = (unsigned)(tiles + runs - 1) / runs;
    const int64_t two = (int64_t)(d == 128 ? 1900 : 3100) * length + 4000, one = (int64_t)(d == 128 ? 1650 : 2600) * length + 4000;
    return rounds_time((unsigned)groups * runs, two, one) + (runs > 1 ? 6000 + part * runs : 0);
}

// D: head dimension; KT: keys per tile; NWAVE waves of QB * 16 rows.
template <int D, int KT, int NWAVE, int QB, Addressing A>
__global__ __launch_bounds__(NWAVE * 64, 2) void tile_kernel(const TileProblem p)
{
    constexpr int QW = QB * 16, ROWS = NWAVE * QW;
    constexpr int ROW = D * 2;            // bytes per row
    constexpr int CPR = ROW / 16;         // 16-byte chunks per row: 16 (D = 128) or 8 (D = 64)
    constexpr int DS = D / 32;            // MFMA k-steps over d
    constexpr int DT = D / 16;            // 16-wide d tiles of the output
    constexpr int TILE_BYTES = KT * ROW;
    constexpr bool PAGED = A != DENSE;
    // LDS: two stages of the K tile, then two of the V tile; chunk c of row r sits in slot c ^ swzK(r) resp. c ^ swzV(r), so that
    // the rows that one operand read touches fall on distinct banks
    __shared__ __attribute__((aligned(1024))) char lds_raw[4 * TILE_BYTES];
    CYC_LDS char *lds = (CYC_LDS char *)lds_raw;
    const uint32_t lds_base = (uint32_t)(uintptr_t)lds;
    auto swzK = [](int r) { return CPR == 16 ? (r & 15) : ((r >> 1) & 7); };
    auto swzV = [](int r) { return CPR == 16 ? ((r & 7) << 1) : (((r >> 1) & 3) << 1); };

    const int l = threadIdx.x & 63, lq = l & 15, g = l >> 4;
    const int w = NWAVE == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int splits = p.splits, run_tiles = p.run_tiles;       // runs of keys and tiles in each
    int b, head, tile, run, N = p.N, M = p.M, first = 0; // problem, key head, tile of rows, run of keys; queries, keys, first token
    bool bad = false;
    if constexpr (A == DENSE) {
        // tiles with the most keys first, the shortest last, when few workgroups are left to run beside them
        const Place at(blockIdx.x, p.batch * p.kv_heads, p.tiles * splits);
        const int t = at.unit / splits;
        run = at.unit - t * splits;
        tile = p.tiles - 1 - t;
        b = at.pair / p.kv_heads;
        head = at.pair - b * p.kv_heads;
    } else {
        if constexpr (A == PAGED_SHORT) {
            // first runs first: what the longest sequences have more than the others comes last, and on all XCDs
            const int pairs = p.batch * p.kv_heads;
            run = blockIdx.x / pairs;
            const int pair = blockIdx.x - run * pairs;
            b = pair / p.kv_heads;
            head = pair - b * p.kv_heads;
            tile = 0;
            // the host knows how wide the table is, not how long the sequences are: runs as long as the longest one needs
            if (splits > 1) {
                const int most = (most_keys(p.lengths, p.batch) + KT - 1) / KT, length = (most + splits - 1) / splits;
                run_tiles = length < LEAST_TILES ? LEAST_TILES : length < run_tiles ? length : run_tiles;
            }
        } else {
            // Likewise, and how many runs is decided here too, where the number of tiles of rows is known.  All workgroups that have work come
            // first: 504 of them fill the chip's 512 places as long as none is held by one that only finds nothing to do.
            Tiles rows;
            const int work = blockIdx.x / p.kv_heads, splits_most = splits;
            if (splits > 1) {
                rows.find(p, ROWS, INT_MAX, true);
                const int most = (rows.keys + KT - 1) / KT, tiles = most < p.most_tiles ? most : p.most_tiles;
                const int64_t part = part_time(p.rows, D);
                int64_t best = long_cost(rows.total * p.kv_heads, tiles, 1, part, D);
                int runs = 1;
                for (int r = 2; r <= splits && r * 4 <= tiles; ++r) {
                    const int64_t cost = long_cost(rows.total * p.kv_heads, tiles, r, part, D);
                    runs = cost < best ? r : runs;
                    best = cost < best ? cost : best;
                }
                splits = __builtin_amdgcn_readfirstlane(runs);
                if (blockIdx.x == 0 && threadIdx.x == 0) *p.chosen = splits;
            }
            // (eight neighbours, whose key heads are different or whose tiles follow one another, run on the eight XCDs)
            head = blockIdx.x - work * p.kv_heads;
            const int slot = work / splits;
            run = work - slot * splits;
            if (splits_most > 1 && p.batch <= 64) {
                rows.total = 0;                            // (one look at the sequences was enough)
                rows.pick(0, slot);
            } else {
                rows = Tiles();
                rows.find(p, ROWS, slot, false);
            }
            if (rows.seq < 0) return;
            b = rows.seq;
            tile = rows.tile;
        }
        const Sequence of(p, b);
        first = of.first;
        N = of.N;
        M = of.M;
        bad = of.bad;
        if (N == 0) return;
        if constexpr (A == PAGED_SHORT) {
            // longer sequences have a launch of their own, unless the caller had announced that there are none
            if ((int64_t)N * p.group > ROWS) {
                if (N <= p.max_new || run > 0) return;
                for (int64_t x = l; x < (int64_t)N * p.group * (D / 8); x += 64) {
                    const int64_t r = x / (D / 8);
                    char *o = p.O + (first + r / p.group) * p.o_row + (head * p.group + r % p.group) * p.o_head;
                    *(i32x4 *)(o + x % (D / 8) * 16) = (i32x4){0x7fc07fc0, 0x7fc07fc0, 0x7fc07fc0, 0x7fc07fc0};
                }
                return;
            }
        }
    }
    const int group = p.group, R = N * group, window = p.window, sinks = p.sinks, pages = p.pages, page_shift = p.page_shift;
    const int64_t k_row = p.k_row, v_row = p.v_row, page_bytes = p.page_bytes;
    const int *table = p.table + b * p.table_stride;
    const float scale_log2e = p.scale_log2e;
    const char *Q = p.Q + b * (PAGED ? 0 : p.q_batch) + (int64_t)head * group * p.q_head + (int64_t)first * p.q_row;
    char *O = p.O + b * (PAGED ? 0 : p.o_batch) + (int64_t)head * group * p.o_head + (int64_t)first * p.o_row;
    const char *K = p.K + (PAGED ? 0 : b * p.k_batch) + (int64_t)head * p.k_head, *V = p.V + (PAGED ? 0 : b * p.v_batch) + (int64_t)head * p.v_head;

    // ---- the keys that the rows of the workgroup see, and this run's share of their tiles (none, if the list ends before)
    const int row_first = tile * ROWS, row_last = (R - row_first < ROWS ? R : row_first + ROWS) - 1;
    const KeyList<KT> list(row_first, row_last, group, N, M, window, sinks);
    if (A != PAGED_SHORT && splits > 1) {
        // equal runs of what these rows see, which need not be what others see
        run_tiles = (int)((unsigned)(list.count + splits - 1) / (unsigned)splits);
        run_tiles = run_tiles < 4 ? 4 : run_tiles;
    }
    const int u_first = run * run_tiles, left = list.count - u_first;
    const int ntiles = left < run_tiles || run == splits - 1 ? left : run_tiles;
    auto tile_key = [&](int u) __attribute__((always_inline)) { return list.tile_key(u + u_first); };

    // ---- this wave's rows: first and last position, and per lane what its rows (one per 16-row block) see
    const int r0 = row_first + w * QW;
    const bool idle = r0 > row_last;                      // uniform: a wave without rows helps to copy
    const int p_lo = idle ? 0 : __builtin_amdgcn_readfirstlane(r0 / group + M - N);
    const int r_last = r0 + QW - 1 < row_last ? r0 + QW - 1 : row_last;
    const int p_hi = idle ? -1 : __builtin_amdgcn_readfirstlane(r_last / group + M - N);
    int row_hi[QB], row_lo[QB];
    i32x4 qf[QB][DS];
#pragma unroll
    for (int jq = 0; jq < QB; ++jq) {
        int r = r0 + jq * 16 + lq;
        r = r < row_last ? r : row_last;                  // rows past the last repeat it and are not stored
        const int i = r / group, h = r - i * group;
        row_hi[jq] = i + M - N;
        row_lo[jq] = (row_hi[jq] < 0 ? 0 : row_hi[jq]) - window + 1;
        const char *q = Q + i * p.q_row + h * p.q_head + g * 16;
#pragma unroll
        for (int ks = 0; ks < DS; ++ks) qf[jq][ks] = *(const i32x4 *)(q + ks * 64);
    }
    // ---- copies of a tile of K and V into a stage.  Paged: lane j looks up the page of the tile's key j a tile ahead and makes it the key's
    // offset in the cache; a copy starts at that of its first row, whose neighbours lie on the same page, or, at the ends of the list and
    // in pages of a few rows, every lane at that of its own row.
    typedef TileCopies<KT, ROW, NWAVE> Copies;
    constexpr int ENTRIES = (KT + 63) / 64;
    int entry[ENTRIES];
    const bool small_strides = k_row < MOST_STRIDE && v_row < MOST_STRIDE && (!PAGED || (1 << page_shift) >= Copies::RPC);
    auto look_up = [&](int u) __attribute__((always_inline)) {
        const int k0 = tile_key(u) + l;
#pragma unroll
        for (int x = 0; x < ENTRIES; ++x) entry[x] = table[list.seen_key(k0 + x * 64) >> page_shift];
    };
    auto issue = [&](int u) __attribute__((always_inline)) {
        const int k0 = tile_key(u);
        const uint32_t dst = lds_base + (u & 1) * TILE_BYTES;
        int64_t at[ENTRIES];
        if constexpr (PAGED) {
#pragma unroll
            for (int x = 0; x < ENTRIES; ++x) {
                const bool outside = (unsigned)entry[x] >= (unsigned)pages;
                bad |= outside;
                at[x] = (outside ? 0 : entry[x]) * page_bytes + (list.seen_key(k0 + x * 64 + l) & ((1 << page_shift) - 1)) * k_row;
            }
        }
        if (small_strides && list.inside(k0)) {
            if constexpr (!PAGED) {
                Copies::whole(K + k0 * k_row, k_row, dst, w, l, swzK);
                Copies::whole(V + k0 * v_row, v_row, dst + 2 * TILE_BYTES, w, l, swzV);
            } else {
                const int row0 = w * Copies::RPC + l / CPR;
                const uint32_t row_off = l / CPR * (uint32_t)k_row, chunk_k = (l % CPR) ^ swzK(row0), chunk_v = (l % CPR) ^ swzV(row0);
#pragma unroll
                for (int x = 0; x < Copies::COUNT; ++x) {
                    const int r = (x * Copies::STEP + w * Copies::RPC) % 64;        // uniform
                    const int64_t from = at[x * Copies::STEP / 64];
                    const int64_t off = (int64_t)__builtin_amdgcn_readlane((int)(from >> 32), r) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)from, r);
                    copy16_from(K + off, row_off + ((chunk_k ^ swzK(x * Copies::STEP)) << 4), dst + (w + x * NWAVE) * 1024);
                    copy16_from(V + off, row_off + ((chunk_v ^ swzV(x * Copies::STEP)) << 4), dst + 2 * TILE_BYTES + (w + x * NWAVE) * 1024);
                }
            }
        } else {
            auto offset = [&](int r, int64_t stride) __attribute__((always_inline)) {
                if constexpr (!PAGED) return list.seen_key(k0 + r) * stride;
                return (int64_t)__shfl((int)(at[r / 64 % ENTRIES] >> 32), r % 64) << 32 | (uint32_t)__shfl((int)at[r / 64 % ENTRIES], r % 64);
            };
            Copies::any(dst, w, l, [&](int r) { return K + offset(r, k_row); }, swzK);
            Copies::any(dst + 2 * TILE_BYTES, w, l, [&](int r) { return V + offset(r, v_row); }, swzV);
        }
    };

    // ---- running state of this lane's rows: reference in the log2 domain, this lane's share of the sum, O^T accumulators
    float m2[QB], sum[QB], part_sum[QB];
    f32x4 acc_o[DT][QB];
#pragma unroll
    for (int jq = 0; jq < QB; ++jq) {
        m2[jq] = -__builtin_inff();
        sum[jq] = 0;
#pragma unroll
        for (int id = 0; id < DT; ++id) acc_o[id][jq] = (f32x4){0, 0, 0, 0};
    }
    // A tile is worked off in parts of 32 keys.
    constexpr int PARTS = KT / 32, SF = DS * 2, VF = DT;  // of a part: fragments of K (16 keys x 32 d) and of V (32 keys x 16 d)
    f32x4 s[2][2][QB];                                    // S^T of two parts: [part % 2][16-key block][row block]
    i32x4 pf[2][QB];                                      // P^T as B operand: [part % 2][row block]
    // this lane's addresses: K by rows; V transposed, k-slots 0..3 = keys 4 (l/16) .. +3 of the part, k-slots 4..7 = those 16 further on (the
    // order P^T is packed in).  They change stage from tile to tile.
    // 32-d step ks of K lies at kaddr ^ ks << 6, 16-d tile id of V at vaddr ^ id << 5.
    uint32_t kaddr = lds_base + lq * ROW + ((g ^ swzK(lq)) << 4);
    const int v_row0 = 4 * g + (lq >> 2);
    uint32_t vaddr = lds_base + 2 * TILE_BYTES + v_row0 * ROW + ((((lq & 3) >> 1) ^ swzV(v_row0)) << 4) + (lq & 1) * 8;

    // ---- weights against the reference m2 (which follows the running maximum lazily, as in cyc_attn.hip), their sum, and P^T packed
    // pair X of a part: row block X / 4, 16-key block X / 2 % 2, elements X % 2 * 2 and the next
    auto weigh_pair = [&](auto part_c, auto x_c) __attribute__((always_inline)) {
        constexpr int P = decltype(part_c)::value, X = decltype(x_c)::value, jq = X / 4, ik = X / 2 % 2, r = X % 2 * 2;
        const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[P][ik][jq][r], scale_log2e, -m2[jq]));
        const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[P][ik][jq][r + 1], scale_log2e, -m2[jq]));
        part_sum[jq] = (X % 4 == 0 ? 0.0f : part_sum[jq]) + (p0 + p1);
        const bf16x2 pair = __builtin_convertvector((f32x2){p0, p1}, bf16x2);
        pf[P][jq][ik * 2 + (r >> 1)] = __builtin_bit_cast(int, pair);
    };
    constexpr unsigned short LAG_BITS = 0x4380;           // 2^8 as bfloat16
    // the part's weights are all at most 2^8, after moving the reference where they were not; then they count
    auto settle = [&](auto part_c) __attribute__((always_inline)) {
        constexpr int P = decltype(part_c)::value;
        u16x2 most = {0, 0};
#pragma unroll
        for (int jq = 0; jq < QB; ++jq)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int word = pf[P][jq][r];
                most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, word));
            }
        const unsigned short t0 = most[0], t1 = most[1];
        if (__builtin_expect(__builtin_amdgcn_ballot_w64((t0 > t1 ? t0 : t1) > LAG_BITS) != 0, 0)) {
#pragma unroll
            for (int jq = 0; jq < QB; ++jq) {
                float top = s[P][0][jq][0];
#pragma unroll
                for (int ik = 0; ik < 2; ++ik)
#pragma unroll
                    for (int r = 0; r < 4; ++r) top = __builtin_fmaxf(top, s[P][ik][jq][r]);
                // (a row that has seen nothing yet keeps a finite reference: weights 0 against it, and any score lifts it)
                const float mh = __builtin_fmaxf(__builtin_fmaxf(m2[jq], query_max(top) * scale_log2e), -3.0e38f);
                const float keep = __builtin_amdgcn_exp2f(m2[jq] - mh);
                m2[jq] = mh;
                sum[jq] *= keep;
#pragma unroll
                for (int id = 0; id < DT; ++id) acc_o[id][jq] *= keep;
            }
            static_for<4 * QB>([&](auto x_c) __attribute__((always_inline)) { weigh_pair(part_c, x_c); });
        }
#pragma unroll
        for (int jq = 0; jq < QB; ++jq) sum[jq] += part_sum[jq];
    };

    // ---- a tile that every row of the wave sees whole.  Phase j multiplies K for part j and V for part j - 2 and takes the weights of part
    // j - 1 in between, so that matrix and vector instructions of one wave have each other to wait for.  All fragments of the tile are one
    // stream, whose reads run WIN fragments ahead: those of phase j are S(j) and then V(j - 2).
    constexpr int WIN = 4, FRAGS = PARTS * (SF + VF);
    constexpr auto phase_start = [](int j) { return (j < PARTS ? j : PARTS) * SF + (j > 2 ? j - 2 : 0) * VF; };
    constexpr auto phase_of = [=](int f) { int j = 0; while (phase_start(j + 1) <= f) ++j; return j; };
    constexpr auto is_k = [=](int f) { const int j = phase_of(f); return j < PARTS && f - phase_start(j) < SF; };
    constexpr auto reads_of = [=](int first, int last) { int n = 0; for (int f = first; f <= last; ++f) n += is_k(f) ? 1 : 2; return n; };
    i32x4 kf[WIN];
    i32x2 va[WIN], vb[WIN];
    auto request = [&](uint32_t k_at, uint32_t v_at, auto f_c) __attribute__((always_inline)) {
        constexpr int f = decltype(f_c)::value;
        if constexpr (f < FRAGS) {
            constexpr int j = phase_of(f), i = f - phase_start(j);
            if constexpr (is_k(f)) lds_read128<(j * 32 + i % 2 * 16) * ROW>(kf[f % WIN], k_at ^ (i / 2 << 6));
            else {
                constexpr int id = i - (j < PARTS ? SF : 0), off = (j - 2) * 32 * ROW;
                lds_read_tr64<off>(va[f % WIN], v_at ^ (id << 5));
                lds_read_tr64<off + 16 * ROW>(vb[f % WIN], v_at ^ (id << 5));
            }
        }
    };
    auto whole_tile = [&]() __attribute__((always_inline)) {
        const uint32_t k_at = fresh(kaddr), v_at = fresh(vaddr);
        static_for<WIN>([&](auto f_c) __attribute__((always_inline)) { request(k_at, v_at, f_c); });
        static_for<PARTS + 2>([&](auto j_c) __attribute__((always_inline)) {
            constexpr int j = decltype(j_c)::value, f0 = phase_start(j), n = phase_start(j + 1) - f0;
            if constexpr (j < PARTS) {
#pragma unroll
                for (int ik = 0; ik < 2; ++ik)
#pragma unroll
                    for (int jq = 0; jq < QB; ++jq) s[j & 1][ik][jq] = (f32x4){0, 0, 0, 0};
            }
            static_for<n>([&](auto i_c) __attribute__((always_inline)) {
                constexpr int i = decltype(i_c)::value, f = f0 + i, ahead = f + WIN - 1 < FRAGS - 1 ? f + WIN - 1 : FRAGS - 1;
                if constexpr (is_k(f)) {
                    lds_wait<reads_of(f + 1, ahead)>(kf[f % WIN]);
#pragma unroll
                    for (int jq = 0; jq < QB; ++jq) s[j & 1][i % 2][jq] = mfma16(kf[f % WIN], qf[jq][i / 2], s[j & 1][i % 2][jq]);
                } else {
                    constexpr int id = i - (j < PARTS ? SF : 0);
                    lds_wait2<reads_of(f + 1, ahead)>(va[f % WIN], vb[f % WIN]);
                    const i32x4 vf = mfma_frag(va[f % WIN], vb[f % WIN]);
#pragma unroll
                    for (int jq = 0; jq < QB; ++jq) acc_o[id][jq] = mfma16(vf, pf[j & 1][jq], acc_o[id][jq]);
                }
                request(k_at, v_at, std::integral_constant<int, f + WIN>{});
                if constexpr (j >= 1 && j <= PARTS) {
                    constexpr int x0 = i * 4 * QB / n, x1 = (i + 1) * 4 * QB / n;
                    static_for<x1 - x0>([&](auto x_c) __attribute__((always_inline)) {
                        weigh_pair(std::integral_constant<int, (j - 1) & 1>{}, std::integral_constant<int, x0 + decltype(x_c)::value>{});
                    });
                }
            });
            if constexpr (j >= 1 && j <= PARTS) {
                // (a tile of one part has nothing to put beside its weights)
                if constexpr (n == 0) static_for<4 * QB>([&](auto x_c) __attribute__((always_inline)) { weigh_pair(std::integral_constant<int, (j - 1) & 1>{}, x_c); });
                settle(std::integral_constant<int, (j - 1) & 1>{});
            }
        });
    };

    // ---- any other tile, part by part
    auto visible = [&](int key, int jq) __attribute__((always_inline)) { return (key <= row_hi[jq]) & ((key >= row_lo[jq]) | (key < sinks)); };
    const std::integral_constant<int, 0> only;
    auto some_of_tile = [&](int k0, int stage) __attribute__((always_inline)) {
        const int l = fresh(threadIdx.x & 63), g = l >> 4;
        const uint32_t k_at = fresh(kaddr), v_at = fresh(vaddr);
#pragma unroll 1
        for (int part = 0; part < PARTS; ++part) {
            const int key0 = k0 + part * 32, key1 = key0 + 31, off = part * 32 * ROW;
            if (key0 > p_hi || (key0 >= sinks && p_lo >= 0 && key1 < p_lo - window + 1)) continue;
            const bool all = key1 <= p_lo && (key0 >= p_hi - window + 1 || key1 < sinks);
#pragma unroll
            for (int ik = 0; ik < 2; ++ik) {
#pragma unroll
                for (int jq = 0; jq < QB; ++jq) s[0][ik][jq] = (f32x4){0, 0, 0, 0};
#pragma unroll
                for (int ks = 0; ks < DS; ++ks) {
                    const i32x4 k = *(const CYC_LDS i32x4 *)(uintptr_t)((k_at ^ ks << 6) + off + ik * 16 * ROW);
#pragma unroll
                    for (int jq = 0; jq < QB; ++jq) s[0][ik][jq] = mfma16(k, qf[jq][ks], s[0][ik][jq]);
                }
            }
            i32x2 a[DT], c[DT];                                       // V, on its way while the weights are taken
            static_for<DT>([&](auto id_c) __attribute__((always_inline)) {
                constexpr int id = decltype(id_c)::value;
                lds_read_tr64<0>(a[id], (v_at ^ id << 5) + off);
                lds_read_tr64<16 * ROW>(c[id], (v_at ^ id << 5) + off);
            });
            if (!all) {
#pragma unroll
                for (int jq = 0; jq < QB; ++jq)
#pragma unroll
                    for (int ik = 0; ik < 2; ++ik)
#pragma unroll
                        for (int r = 0; r < 4; ++r) s[0][ik][jq][r] = visible(key0 + 4 * g + ik * 16 + r, jq) ? s[0][ik][jq][r] : -__builtin_inff();
            }
            static_for<4 * QB>([&](auto x_c) __attribute__((always_inline)) { weigh_pair(only, x_c); });
            settle(only);
            static_for<DT>([&](auto id_c) __attribute__((always_inline)) {
                constexpr int id = decltype(id_c)::value;
                lds_wait2<2 * (DT - 1 - id)>(a[id], c[id]);
            });
            const bool careful = !all && any_infinite<DT>([&](auto id_c) __attribute__((always_inline)) { return mfma_frag(a[decltype(id_c)::value], c[decltype(id_c)::value]); });
            // with finite values alone where some are not; those go, key by key, to the rows that see them
            if (__builtin_expect(careful, 0)) {
#pragma unroll
                for (int id = 0; id < DT; ++id) {
                    a[id] = (i32x2){finite_pair(a[id][0]), finite_pair(a[id][1])};
                    c[id] = (i32x2){finite_pair(c[id][0]), finite_pair(c[id][1])};
                }
            }
#pragma unroll
            for (int id = 0; id < DT; ++id)
#pragma unroll
                for (int jq = 0; jq < QB; ++jq) acc_o[id][jq] = mfma16(mfma_frag(a[id], c[id]), pf[0][jq], acc_o[id][jq]);
            if (__builtin_expect(careful, 0)) {
                for (int key = 0; key < 32; ++key) {
                    const CYC_LDS char *row = lds + (2 + stage) * TILE_BYTES + off + key * ROW;
                    const int word = ((const CYC_LDS int *)row)[l % (ROW / 4)];
                    if (__builtin_amdgcn_ballot_w64(finite_pair(word) != word) == 0) continue;
#pragma unroll
                    for (int id = 0; id < DT; ++id) {
                        const int chunk = (id * 16 + 4 * g) >> 3, within = ((id * 16 + 4 * g) & 7) * 2;
                        const bf16x4 v = *(const CYC_LDS bf16x4 *)(row + ((chunk ^ swzV(key)) << 4) + within);
#pragma unroll
                        for (int jq = 0; jq < QB; ++jq)
#pragma unroll
                            for (int r = 0; r < 4; ++r) acc_o[id][jq][r] += (visible(key0 + key, jq) & !__builtin_isfinite((float)v[r])) ? (float)v[r] : 0.0f;
                    }
                }
            }
        }
    };

    // ---- One barrier per tile: tile u has landed and every wave is done with tile u-1, whose stage tile u+1 is then requested into.  The
    // tiles that all rows see whole come first, in a loop of their own: with both kinds in one, the compiler keeps a second set of
    // accumulators.
    if (ntiles > 0) {
        if constexpr (PAGED) look_up(0);
        issue(0);
        if constexpr (PAGED) {
            if (ntiles > 1) look_up(1);
        }
    }
    int u = 0;
    auto arrive = [&]() __attribute__((always_inline)) {
        landed_barrier();
        if (u + 1 < ntiles) {
            issue(u + 1);
            if constexpr (PAGED) {
                if (u + 2 < ntiles) look_up(u + 2);
            }
        }
    };
    auto leave = [&]() __attribute__((always_inline)) {
        const int turn = u & 1 ? -TILE_BYTES : TILE_BYTES;
        kaddr += turn;
        vaddr += turn;
        ++u;
    };
    while (u < ntiles && u + u_first < list.whole) {
        arrive();
        if (!idle) whole_tile();
        leave();
    }
    while (u < ntiles) {
        arrive();
        some_of_tile(tile_key(u), u & 1);
        leave();
    }

    if constexpr (PAGED) {
        // a lane of any wave may have met a table entry that is none: the whole tile of rows is in doubt
        bool any = __builtin_amdgcn_ballot_w64(bad) != 0;
        if constexpr (NWAVE > 1) {
            landed_barrier();
            if (l == 0) ((CYC_LDS int *)lds)[w] = any;
            landed_barrier();
#pragma unroll
            for (int x = 0; x < NWAVE; ++x) any |= ((CYC_LDS int *)lds)[x] != 0;
        }
        bad = any;
    }
    // ---- O = o / sum.  Accumulator register r of lane l: d = 16 id + 4 (l/16) + r, row 16 jq + l%16.
#pragma unroll
    for (int jq = 0; jq < QB; ++jq) {
        const int r = r0 + jq * 16 + lq;
        const float tot = bad ? __builtin_nanf("") : query_sum(sum[jq]);
        if (r > row_last) continue;
        const int i = r / group, h = head * group + r - i * group;
        if (splits > 1) {
            const int64_t slot = run * p.part_rows + (QB == 1 ? ((int64_t)b * p.kv_heads + head) * ROWS + r : PAGED ? (int64_t)(first + i) * (p.kv_heads * group) + h : ((int64_t)b * (p.kv_heads * group) + h) * N + i);
            if (ntiles > 0)
#pragma unroll
                for (int id = 0; id < DT; ++id) *(f32x4 *)(p.part + slot * D + id * 16 + 4 * g) = acc_o[id][jq];
            if (g == 0) *(f32x2 *)(p.refs + slot * 2) = (f32x2){m2[jq], tot};
        } else {
            const bool empty = row_hi[jq] < 0 && !bad;
#pragma unroll
            for (int id = 0; id < DT; ++id) {
                bf16x4 o;
#pragma unroll
                for (int x = 0; x < 4; ++x) o[x] = (__bf16)(empty ? 0.0f : acc_o[id][jq][x] / tot);
                *(bf16x4 *)(O + i * p.o_row + (r - i * group) * p.o_head + (id * 16 + 4 * g) * 2) = o;
            }
            if (!PAGED && p.lse && g == 0)
                p.lse[((int64_t)b * (p.kv_heads * group) + h) * N + i] = empty ? -__builtin_inff() : (m2[jq] + __builtin_amdgcn_logf(tot)) * 0.69314718055994531f;
        }
    }
}

// Joins the runs of a row in ascending order: O = sum_x exp(m_x - m) o_x / sum_x exp(m_x - m) l_x, m the largest m_x.  One thread per four
// d; bound by a launch and the reads of part.  A run without tiles has m_x = -inf and l_x = 0, and no o_x.  The lanes of a row look at all
// runs at once (1024 + 7 x 1 tokens, two runs and 28: 21 us one run after the other, now 14).
struct Parts {
    const float *part, *refs;
    int64_t rows;
    int splits;
};
template <int D, bool PAGED> __global__ __launch_bounds__(256) void join_kernel(const TileProblem p, const Parts shorts, const Parts longs, bool by_slot)
{
    constexpr int PER = 1024 / D;                                     // rows of a workgroup
    const int c = threadIdx.x % (D / 4) * 4, heads = p.kv_heads * p.group;
    int h, i, position;
    int64_t b = 0, row, at;                                           // problem; row of O; row among the parts
    bool few;
    if constexpr (PAGED) {
        auto position_in = [&](const Sequence &of) { return of.bad ? 0 : of.M - of.N + i - of.first; };
        if (by_slot) {
            at = (int64_t)blockIdx.x * PER + threadIdx.x / (D / 4);
            if (at >= shorts.rows) return;
            const int unit = (int)(at / SHORT_ROWS), r = (int)(at % SHORT_ROWS), seq = unit / p.kv_heads;
            const Sequence of(p, seq);
            if (r >= of.N * p.group || (int64_t)of.N * p.group > p.short_rows) return;
            i = of.first + r / p.group;
            h = (unit - seq * p.kv_heads) * p.group + r % p.group;
            row = (int64_t)i * heads + h;
            few = true;
            position = position_in(of);
        } else {
            // a workgroup's rows are of one token, whose sequence it looks up once
            const int chunks = (heads + PER - 1) / PER;
            i = blockIdx.x / chunks;
            h = (blockIdx.x - i * chunks) * PER + threadIdx.x / (D / 4);
            if (h >= heads) return;
            const int seq = sequence_of(p.starts, p.batch, i);
            const Sequence of(p, seq);
            if (i < of.first || i >= of.first + of.N) return;
            few = (int64_t)of.N * p.group <= p.short_rows;
            if (!few && longs.splits == 0) return;                    // (no launch for it: its rows are NaN already)
            at = row = (int64_t)i * heads + h;
            if (few) at = ((int64_t)seq * p.kv_heads + h / p.group) * SHORT_ROWS + (i - of.first) * p.group + h % p.group;
            position = position_in(of);
        }
    } else {
        at = row = (int64_t)blockIdx.x * PER + threadIdx.x / (D / 4);
        if (row >= p.rows) return;
        i = (int)(row % p.N);
        h = (int)(row / p.N % heads);
        b = row / p.N / heads;
        position = i + p.M - p.N;
        few = shorts.splits > 0;
        if (few) at = (b * p.kv_heads + h / p.group) * SHORT_ROWS + i * p.group + h % p.group;
    }
    Parts from = few ? shorts : longs;
    if (PAGED && !few && from.splits > 1) from.splits = *p.chosen;
    if (from.splits <= 1) return;
    const float *ref = from.refs + at * 2, *part = from.part + at * D + c;
    constexpr int LANES = D / 4, BATCH = 8;                           // lanes of a row, one for a run; runs on their way together
    const int l = threadIdx.x % LANES, at_lane = (threadIdx.x & 63) - l;
    const f32x2 none = {-__builtin_inff(), 0};
    float m = -__builtin_inff();
    for (int x = l; x < from.splits; x += LANES) m = __builtin_fmaxf(m, ref[x * from.rows * 2]);
#pragma unroll
    for (int d = LANES / 2; d; d >>= 1) m = __builtin_fmaxf(m, __shfl_xor(m, d));
    f32x4 o = {0, 0, 0, 0};
    float tot = 0;
    for (int base = 0; base < from.splits; base += LANES) {
        const int x = base + l;
        const f32x2 mt = x < from.splits ? *(const f32x2 *)(ref + x * from.rows * 2) : none;
        const float keep = mt[0] == m ? 1.0f : __builtin_amdgcn_exp2f(mt[0] - m), sum = mt[1];
        // (only the last runs have no tiles)
        const uint64_t some = __builtin_amdgcn_ballot_w64(!(mt[0] == none[0] && mt[1] == 0)) >> at_lane & (((uint64_t)1 << LANES) - 1);
        const int n = some ? 64 - __builtin_clzll(some) : 0;
        for (int y0 = 0; y0 < n; y0 += BATCH) {
            f32x4 v[BATCH];
#pragma unroll
            for (int i = 0; i < BATCH; ++i) v[i] = *(const f32x4 *)(part + (base + (y0 + i < n ? y0 + i : n - 1)) * from.rows * D);
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                const float k = __shfl(keep, at_lane + y0 + i), t = __shfl(sum, at_lane + y0 + i);
                if (y0 + i >= n) break;
                tot = __builtin_fmaf(k, t, tot);
#pragma unroll
                for (int z = 0; z < 4; ++z) o[z] = __builtin_fmaf(k, v[i][z], o[z]);
            }
        }
    }
    const bool empty = position < 0;
    bf16x4 out;
#pragma unroll
    for (int y = 0; y < 4; ++y) out[y] = (__bf16)(empty ? 0.0f : o[y] / tot);
    *(bf16x4 *)(p.O + b * p.o_batch + h * p.o_head + i * p.o_row + c * 2) = out;
    if (!PAGED && p.lse && c == 0) p.lse[row] = empty ? -__builtin_inff() : (m + __builtin_amdgcn_logf(tot)) * 0.69314718055994531f;
}

template <int D> constexpr int LONG_KEYS = 8192 / D;
template <int D> constexpr int SHORT_KEYS = 4096 / D;

// Runs of `tiles` tiles that workgroups are cut into, each `length` of them (the last one less).
struct Runs {
    int count = 0, length = 0;           // count 0: no launch
};
Runs runs_of(int64_t tiles, int64_t want)
{
    tiles = std::max<int64_t>(tiles, 1);
    const int64_t length = (tiles + want - 1) / want;
    return {(int)((tiles + length - 1) / length), (int)length};
}

struct Mapping {
    Runs shorts, longs;                  // of sequences with up to SHORT_ROWS rows and of the others
    int64_t short_rows = 0, long_rows = 0;   // rows that a run leaves of them
};

int64_t part_bytes(int64_t rows, int64_t d, int splits) { return splits > 1 ? (rows * splits * (d + 2) * 4 + 15) / 16 * 16 : 0; }
// (and 16 bytes for what the device chooses)
int64_t workspace_bytes_of(const Mapping &m, int64_t d)
{
    const int64_t parts = part_bytes(m.short_rows, d, m.shorts.count) + part_bytes(m.long_rows, d, m.longs.count);
    return parts > 0 ? parts + 16 : 0;
}
constexpr int64_t MOST_PART = 128 << 20;

// Few rows: memory is the bound.  Keys of equal lists stream best through two workgroups on a compute unit (16 x 8 key heads x 8192 keys of
// d 128: one run 290 us, four 97, ten 118, 32 132); sequences in pages have lengths that differ and that the host does not know, so that
// more and shorter runs even out what the compute units get (64 x 8 key heads, 1000 to 8000 keys: two runs 247 us, six 224, twenty
// 247).  A run has at least eight tiles, which pays for its start.
Runs choose_short(int64_t pairs, int64_t tiles, int64_t rows, int64_t d, int64_t groups)
{
    return runs_of(tiles, std::max<int64_t>(std::min<int64_t>({MOST_PART / (rows * (d + 2) * 4), tiles / LEAST_TILES, groups / pairs, 64}), 1));
}

// Many rows: the runs that long_cost says, of `most` at most.
constexpr int MOST_RUNS = 16;
Runs choose_long(int64_t groups, int64_t tiles, int64_t rows, int64_t d)
{
    int64_t best = 1;
    const int64_t part = part_time(rows, d);
    auto cost = [&](int64_t r) { return long_cost((int)groups, (int)tiles, (int)r, part, (int)d); };
    if (groups * MOST_RUNS < (1 << 30))
        for (int64_t r = 2; r <= MOST_RUNS && r * 4 <= tiles && rows * (d + 2) * 4 * r <= MOST_PART; ++r)
            if (cost(r) < cost(best)) best = r;
    return runs_of(tiles, best);
}
// Sequences in pages: the device decides (tile_kernel) and needs a grid and memory for what it may choose.  Runs come into question below four
// rounds of workgroups, and where one run leaves no compute unit free only for lists that pay for it: to count the sequences takes each workgroup
// more than 1 us, and a chip full of workgroups with 19 tiles each takes 60 us without and 65 with.
Runs most_long(int64_t groups, int64_t tiles, int64_t rows, int64_t d)
{
    if (groups > 256 && tiles < 32) return {1, (int)tiles};
    const int64_t most = std::min<int64_t>({MOST_RUNS / 2, tiles / 4, MOST_PART / (rows * (d + 2) * 4), 2048 / std::max<int64_t>(groups, 1)});
    return {(int)std::max<int64_t>(most, 1), (int)tiles};
}

Mapping window_mapping(const WindowProblem &p)
{
    const int64_t R = (int64_t)p.N * p.group, pairs = (int64_t)p.batch * p.kv_heads, rows = R * pairs;
    const bool shorts = R <= SHORT_ROWS;
    Mapping m;
    m.short_rows = pairs * SHORT_ROWS;
    m.long_rows = rows;
    if (shorts) m.shorts = choose_short(pairs, most_tiles(p.M, p.window, p.sinks, SHORT_ROWS, p.group, p.N, 4096 / p.d), m.short_rows, p.d, 512);
    else m.longs = choose_long(pairs * ((R + LONG_ROWS - 1) / LONG_ROWS), most_tiles(p.M, p.window, p.sinks, LONG_ROWS, p.group, p.N, 8192 / p.d), rows, p.d);
    return m;
}

Mapping paged_mapping(const PagedProblem &p)
{
    const int64_t all = (int64_t)p.max_pages << p.page_shift, rows = (int64_t)p.tokens * p.heads;
    auto tiles = [&](int64_t tile_rows, int64_t kt) { return most_tiles(all, p.window, p.sinks, tile_rows, p.group, p.max_new, kt); };
    Mapping m;
    m.short_rows = (int64_t)p.seqs * p.kv_heads * SHORT_ROWS;
    m.long_rows = rows;
    const bool longs = (int64_t)p.max_new * p.group > SHORT_ROWS;
    if (!longs || (p.seqs > 1 && p.group <= SHORT_ROWS)) m.shorts = choose_short((int64_t)p.seqs * p.kv_heads, tiles(SHORT_ROWS, 4096 / p.d), m.short_rows, p.d, 3200);
    if (longs) m.longs = most_long((int64_t)p.tokens * p.group / LONG_ROWS * p.kv_heads, tiles(LONG_ROWS, 8192 / p.d), rows, p.d);
    return m;
}

template <int D, bool PAGED> hipError_t launch_tiles(TileProblem t, Mapping m, void *workspace, int64_t workspace_bytes, hipStream_t s)
{
    if (workspace_bytes_of(m, D) > workspace_bytes)
        for (Runs *r : {&m.shorts, &m.longs})
            if (r->count) *r = {1, INT_MAX};
    t.chosen = (int *)((char *)workspace + workspace_bytes_of(m, D) - 16);
    t.most_tiles = m.longs.length;
    t.scale_log2e = (float)(1.4426950408889634 / __builtin_sqrt((double)D));
    char *free = (char *)workspace;
    auto launch = [&](auto kernel, int threads, int64_t groups, const Runs &runs, int64_t rows, Parts *parts) {
        t.splits = runs.count;
        t.run_tiles = runs.length;
        t.part = (float *)free;
        t.refs = t.part + rows * D * runs.count;
        t.part_rows = rows;
        free += part_bytes(rows, D, runs.count);
        *parts = {t.part, t.refs, rows, runs.count};
        if (groups * runs.count >= ((int64_t)1 << 31)) return hipErrorInvalidValue;
        return launch_kernel(kernel, dim3((unsigned)(groups * runs.count)), dim3(threads), s, t);
    };
    hipError_t e = hipSuccess;
    Parts shorts{}, longs{};
    const int64_t pairs = (int64_t)t.batch * t.kv_heads;
    if (m.shorts.count) e = launch(tile_kernel<D, SHORT_KEYS<D>, 1, 1, PAGED ? PAGED_SHORT : DENSE>, 64, pairs, m.shorts, m.short_rows, &shorts);
    if (e == hipSuccess && m.longs.count)
        e = launch(tile_kernel<D, LONG_KEYS<D>, 4, 2, PAGED ? PAGED_LONG : DENSE>, 256, t.tiles * (PAGED ? t.kv_heads : pairs), m.longs, m.long_rows, &longs);
    if (e != hipSuccess || std::max(shorts.splits, longs.splits) <= 1) return e;
    // (paged: by tokens, or by the rows that runs of few rows leave, where only those have runs and are fewer: 24 sequences with 3500 tokens, 16 heads, 6 us -> 4)
    const int64_t per = 1024 / D, heads = (int64_t)t.kv_heads * t.group, of_tokens = t.tokens * ((heads + per - 1) / per), of_slots = (m.short_rows + per - 1) / per;
    const bool by_slot = PAGED && longs.splits <= 1 && of_slots < of_tokens;
    const int64_t groups = !PAGED ? (t.rows + per - 1) / per : by_slot ? of_slots : of_tokens;
    return launch_kernel(join_kernel<D, PAGED>, dim3((unsigned)groups), dim3(256), s, t, shorts, longs, by_slot);
}

}  // namespace

int64_t most_tiles(int64_t keys, int window, int sinks, int64_t rows, int64_t group, int64_t queries, int64_t kt)
{
    const int64_t span = window + std::min(queries, (rows - 1) / group + 2);
    return std::min((keys + kt - 1) / kt, (std::min<int64_t>(span, keys) + kt - 1) / kt + 1 + (std::min<int64_t>(sinks, keys) + kt - 1) / kt);
}

int64_t window_workspace_bytes(const WindowProblem &p) { return workspace_bytes_of(window_mapping(p), p.d); }

hipError_t launch_window(const WindowProblem &p, void *workspace, int64_t workspace_bytes, hipStream_t s)
{
    TileProblem t{};
    t.Q = p.Q.base, t.K = p.K.base, t.V = p.V.base, t.O = (char *)p.O.base, t.lse = p.lse;
    t.q_batch = p.Q.batch, t.q_head = p.Q.head, t.q_row = p.Q.row, t.o_batch = p.O.batch, t.o_head = p.O.head, t.o_row = p.O.row;
    t.k_batch = p.K.batch, t.k_head = p.K.head, t.k_row = p.K.row, t.v_batch = p.V.batch, t.v_head = p.V.head, t.v_row = p.V.row;
    t.batch = p.batch, t.kv_heads = p.kv_heads, t.group = p.group, t.N = p.N, t.M = p.M;
    t.window = p.window, t.sinks = p.sinks;
    t.rows = (int64_t)p.batch * p.heads * p.N;
    const Mapping m = window_mapping(p);
    t.tiles = m.shorts.count ? 1 : (int)(((int64_t)p.N * p.group + LONG_ROWS - 1) / LONG_ROWS);
    return p.d == 128 ? launch_tiles<128, false>(t, m, workspace, workspace_bytes, s) : launch_tiles<64, false>(t, m, workspace, workspace_bytes, s);
}

int64_t paged_workspace_bytes(const PagedProblem &p) { return workspace_bytes_of(paged_mapping(p), p.d); }

hipError_t launch_paged(const PagedProblem &p, void *workspace, int64_t workspace_bytes, hipStream_t s)
{
    TileProblem t{};
    t.Q = p.Q, t.K = p.K, t.V = p.V, t.O = p.O;
    t.q_head = p.q_head, t.q_row = p.q_token, t.o_head = p.o_head, t.o_row = p.o_token;
    t.k_head = t.v_head = p.head_bytes, t.k_row = t.v_row = p.row_bytes, t.page_bytes = p.page_bytes, t.table_stride = p.table_stride;
    t.table = p.table, t.lengths = p.lengths, t.starts = p.starts;
    t.batch = p.seqs, t.kv_heads = p.kv_heads, t.group = p.group, t.tokens = p.tokens, t.pages = p.pages, t.page_shift = p.page_shift;
    t.max_pages = p.max_pages, t.max_new = p.max_new, t.window = p.window, t.sinks = p.sinks;
    t.rows = (int64_t)p.tokens * p.heads;
    const Mapping m = paged_mapping(p);
    t.short_rows = m.shorts.count ? SHORT_ROWS : 0;
    t.tiles = m.longs.count ? (int)((int64_t)p.tokens * p.group / LONG_ROWS + p.seqs) : 0;
    return p.d == 128 ? launch_tiles<128, true>(t, m, workspace, workspace_bytes, s) : launch_tiles<64, true>(t, m, workspace, workspace_bytes, s);
}

}  // namespace cyc
