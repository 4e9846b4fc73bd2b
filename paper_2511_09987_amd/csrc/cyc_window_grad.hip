// cyc_window_grad.hip -- the gradient of attention with a sliding window and sinks.
//
// With P_ij = exp(S_ij - lse_i) over the keys that i sees, D_i = dO_i.O_i and dS_ij = P_ij (dO_i.V_j - D_i):
//     dQ_i = sum_j dS_ij K_j / sqrt(d),   dK_j = sum_i dS_ij Q_i / sqrt(d),   dV_j = sum_i P_ij dO_i,
// the last two also over the heads that share key j.  Two kernels, so that every sum stays with one owner and no atomic adds are needed:
// one keeps rows (query, head) and walks their keys for dQ (three products a pair), the other keeps keys and walks the rows that
// see them for dK and dV (four); P is taken again in the second.  Seven products for the five of the formulas, against the
// 4 d bytes per pair that P and dS would cost in memory.
//
// Rows (resp. keys) stay in MFMA operand registers, as in cyc_window.hip, and the other side streams through LDS in tiles that are read
// in two ways: row by row (16 bytes of a row per lane) for the products along d, transposed for those along rows or keys.  The
// accumulators of the first kind, rounded, are operands of the second kind as they are.
// What a row does not see is kept out as in cyc_window.hip: P and dS are 0 there by selection, and a masked tile that is not all finite
// is multiplied without what is not, which then goes to those that see it.
#include "cyc_window.h"
#include "cyc_tile.h"

#include <algorithm>
#include <climits>

namespace cyc {
namespace {

// In a tile of rows of ROW bytes chunk c of row r sits in slot c ^ swizzle(r).  Sixteen lanes read 16 bytes each of a row-wise operand at
// a time, rows 0-3 and 12-15 at one chunk and 4-11 at its neighbour (or the other way round), and eight rows of 32 bytes of a transposed
// one: with this map both fall on all 64 banks.  Linear in the bits of r.
template <int CPR> __device__ __forceinline__ constexpr int swizzle(int r)
{
    const int high = r >> 3 & 1;
    return CPR == 16 ? ((r & 7) ^ high << 2) << 1 | high : ((r >> 1 & 3) ^ high << 1) << 1 | high;
}

constexpr int TILE = 32;                 // rows of a tile of queries, keys of a step

// What both kernels do with a tile of 32 rows in LDS.  D: head dimension.
template <int D> struct Tile {
    static constexpr int ROW = D * 2, CPR = ROW / 16, DS = D / 32, DT = D / 16, WIN = 4;
    // this lane's addresses within a tile: row l % 16 (chunk l / 16 of 64 bytes) and, transposed, row 4 (l / 16) + (l % 16) / 4
    static __device__ __forceinline__ uint32_t row_address(uint32_t base, int l)
    {
        const int lq = l & 15, g = l >> 4;
        return base + lq * ROW + ((g ^ swizzle<CPR>(lq)) << 4);
    }
    static __device__ __forceinline__ uint32_t column_address(uint32_t base, int l)
    {
        const int lq = l & 15, g = l >> 4, row = 4 * g + (lq >> 2);
        return base + row * ROW + ((((lq & 3) >> 1) ^ swizzle<CPR>(row)) << 4) + (lq & 1) * 8;
    }
    // first[n] and second[n] = rows 16 H .. 16 H + 15 of the tile (A operand) that lies A bytes, resp. B bytes, behind `address`, times the NB
    // stationary operands x[n][ks], resp. y[n][ks]
    template <int H, int A, int B, int NB>
    static __device__ __forceinline__ void products(f32x4 (&first)[NB], f32x4 (&second)[NB], uint32_t address, const i32x4 (&x)[NB][DS], const i32x4 (&y)[NB][DS])
    {
        constexpr int N = DS * 2;
        i32x4 f[WIN];
        static_for<WIN>([&](auto ic) __attribute__((always_inline)) {
            constexpr int i = decltype(ic)::value;
            lds_read128<(i < DS ? A : B) + H * 16 * ROW>(f[i], address ^ (i % DS << 6));
        });
#pragma unroll
        for (int n = 0; n < NB; ++n) first[n] = second[n] = (f32x4){0, 0, 0, 0};
        static_for<N>([&](auto ic) __attribute__((always_inline)) {
            constexpr int i = decltype(ic)::value, ks = i % DS, next = i + WIN;
            constexpr int later = N - 1 - i < WIN - 1 ? N - 1 - i : WIN - 1;
            lds_wait<later>(f[i % WIN]);
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                if constexpr (i < DS) first[n] = mfma16(f[i % WIN], x[n][ks], first[n]);
                else second[n] = mfma16(f[i % WIN], y[n][ks], second[n]);
            }
            if constexpr (next < N) lds_read128<(next < DS ? A : B) + H * 16 * ROW>(f[i % WIN], address ^ (next % DS << 6));
        });
    }
    // acc[id][n] += (tile)^T y[n]: A operand d 16 id + l % 16, k-slots 0..3 the rows 4 (l / 16) .. +3, k-slots 4..7 those 16 further down
    template <int OFF, int NB> static __device__ __forceinline__ void accumulate(f32x4 (&acc)[DT][NB], uint32_t address, const i32x4 (&y)[NB])
    {
        i32x2 a[WIN], c[WIN];
        static_for<WIN>([&](auto ic) __attribute__((always_inline)) {
            constexpr int i = decltype(ic)::value;
            lds_read_tr64<OFF>(a[i], address ^ (i << 5));
            lds_read_tr64<OFF + 16 * ROW>(c[i], address ^ (i << 5));
        });
        static_for<DT>([&](auto ic) __attribute__((always_inline)) {
            constexpr int i = decltype(ic)::value;
            constexpr int later = DT - 1 - i < WIN - 1 ? DT - 1 - i : WIN - 1;
            lds_wait2<2 * later>(a[i % WIN], c[i % WIN]);
            const i32x4 f = mfma_frag(a[i % WIN], c[i % WIN]);
#pragma unroll
            for (int n = 0; n < NB; ++n) acc[i][n] = mfma16(f, y[n], acc[i][n]);
            if constexpr (i + WIN < DT) {
                lds_read_tr64<OFF>(a[i % WIN], address ^ ((i + WIN) << 5));
                lds_read_tr64<OFF + 16 * ROW>(c[i % WIN], address ^ ((i + WIN) << 5));
            }
        });
    }
    static __device__ __forceinline__ bool infinite(const CYC_LDS char *tile, int l)
    {
        return any_infinite<TILE * ROW / 1024>([&](auto ic) __attribute__((always_inline)) { return ((const CYC_LDS i32x4 *)tile)[decltype(ic)::value * 64 + l]; });
    }
    // accumulate() with the finite values alone; then add(n, value) of every other value, row by row, where seen(row, n)
    template <int NB, class Seen, class Add>
    static __device__ __forceinline__ void accumulate_carefully(f32x4 (&acc)[DT][NB], uint32_t address, const CYC_LDS char *tile, int l, const i32x4 (&y)[NB], Seen &&seen, Add &&add)
    {
#pragma unroll
        for (int id = 0; id < DT; ++id) {
            i32x2 a, c;
            asm volatile("ds_read_b64_tr_b16 %0, %2\n\tds_read_b64_tr_b16 %1, %2 offset:%3\n\ts_waitcnt lgkmcnt(0)"
                         : "=&v"(a), "=&v"(c) : "v"(address ^ (id << 5)), "n"(16 * ROW));
            const i32x4 clean = {finite_pair(a[0]), finite_pair(a[1]), finite_pair(c[0]), finite_pair(c[1])};
#pragma unroll
            for (int n = 0; n < NB; ++n) acc[id][n] = mfma16(clean, y[n], acc[id][n]);
        }
        const int g = l >> 4;
        for (int r = 0; r < TILE; ++r) {
            const CYC_LDS char *row = tile + r * ROW;
            const int word = ((const CYC_LDS int *)row)[l % (ROW / 4)];
            if (__builtin_amdgcn_ballot_w64(finite_pair(word) != word) == 0) continue;
#pragma unroll
            for (int id = 0; id < DT; ++id) {
                const int chunk = (id * 16 + 4 * g) >> 3, within = ((id * 16 + 4 * g) & 7) * 2;
                const bf16x4 v = *(const CYC_LDS bf16x4 *)(row + ((chunk ^ swizzle<CPR>(r)) << 4) + within);
#pragma unroll
                for (int n = 0; n < NB; ++n)
#pragma unroll
                    for (int x = 0; x < 4; ++x) acc[id][n][x] += seen(r, n) & !__builtin_isfinite((float)v[x]) ? add((float)v[x]) : 0.0f;
            }
        }
    }
};

// x rounded to bfloat16 as half H of an operand of the second products
template <int H, int NB> __device__ __forceinline__ void pack(i32x4 (&y)[NB], const f32x4 (&x)[NB])
{
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int r = 0; r < 4; r += 2) {
            const bf16x2 pair = __builtin_convertvector((f32x2){x[n][r], x[n][r + 1]}, bf16x2);
            y[n][H * 2 + (r >> 1)] = __builtin_bit_cast(int, pair);
        }
}

__device__ __forceinline__ float not_a_number(float) { return __builtin_nanf(""); }
__device__ __forceinline__ float itself(float x) { return x; }

// lse and D of every row by head, lse in the log2 domain, heads padded to whole tiles
__host__ __device__ inline int64_t padded_rows(int N) { return ((int64_t)N + TILE - 1) / TILE * TILE; }

// ---- dQ.  A workgroup of four waves keeps 128 rows r (query r / group, head r % group of a key head) and walks the keys that any of them
// sees in tiles of 64, two steps of 32 to a barrier.  Also writes lse and D of its rows for the other kernel.
constexpr int KEY_TILE = 64;

template <int D> __global__ __launch_bounds__(256, 2) void grad_q_kernel(const WindowProblem p, int tiles, float scale, float *lse2, float *Ds)
{
    typedef Tile<D> T;
    constexpr int ROW = T::ROW, CPR = T::CPR, DS = T::DS, DT = T::DT, QB = 2, QW = 32, ROWS = 128;
    constexpr int TILE_BYTES = KEY_TILE * ROW;
    __shared__ __attribute__((aligned(1024))) char lds_raw[4 * TILE_BYTES];        // two stages of K, then two of V
    CYC_LDS char *lds = (CYC_LDS char *)lds_raw;
    const uint32_t lds_base = (uint32_t)(uintptr_t)lds;
    const int l = threadIdx.x & 63, lq = l & 15, g = l >> 4, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Place at(blockIdx.x, p.batch * p.kv_heads, tiles);
    const int tile = tiles - 1 - at.unit;                                           // (the most keys first)
    const int64_t b = at.pair / p.kv_heads;
    const int head = at.pair - (int)b * p.kv_heads;
    const int group = p.group, N = p.N, M = p.M, R = N * group, window = p.window, sinks = p.sinks;
    const char *K = p.K.base + b * p.K.batch + head * p.K.head, *V = p.V.base + b * p.V.batch + head * p.V.head;
    const int64_t k_row = p.K.row, v_row = p.V.row;

    const int row_first = tile * ROWS, row_last = (R - row_first < ROWS ? R : row_first + ROWS) - 1;
    const KeyList<KEY_TILE> list(row_first, row_last, group, N, M, window, sinks);
    const int ntiles = list.count;

    const int r0 = row_first + w * QW;
    const bool idle = r0 > row_last;
    const int p_lo = idle ? 0 : __builtin_amdgcn_readfirstlane(r0 / group + M - N);
    const int r_last = r0 + QW - 1 < row_last ? r0 + QW - 1 : row_last;
    const int p_hi = idle ? -1 : __builtin_amdgcn_readfirstlane(r_last / group + M - N);
    int row_hi[QB], row_lo[QB];
    float lse[QB], Di[QB];
    i32x4 qf[QB][DS], of[QB][DS];
#pragma unroll
    for (int jq = 0; jq < QB; ++jq) {
        int r = r0 + jq * 16 + lq;
        const bool mine = r <= row_last;
        r = mine ? r : row_last;
        const int i = r / group, h = head * group + r - i * group;
        row_hi[jq] = i + M - N;
        row_lo[jq] = (row_hi[jq] < 0 ? 0 : row_hi[jq]) - window + 1;
        const char *q = p.Q.base + b * p.Q.batch + h * p.Q.head + i * p.Q.row + g * 16, *o = p.O.base + b * p.O.batch + h * p.O.head + i * p.O.row + g * 16;
        const char *dO = p.dO.base + b * p.dO.batch + h * p.dO.head + i * p.dO.row + g * 16;
        float dot = 0;
#pragma unroll
        for (int ks = 0; ks < DS; ++ks) {
            qf[jq][ks] = *(const i32x4 *)(q + ks * 64);
            of[jq][ks] = *(const i32x4 *)(dO + ks * 64);
            const bf16x8 x = *(const bf16x8 *)(o + ks * 64), y = __builtin_bit_cast(bf16x8, of[jq][ks]);
#pragma unroll
            for (int e = 0; e < 8; ++e) dot = __builtin_fmaf((float)x[e], (float)y[e], dot);
        }
        Di[jq] = query_sum(dot);
        const int64_t row = b * p.heads + h;
        lse[jq] = p.lse[row * N + i] * 1.4426950408889634f;
        if (mine && g == 0) {
            lse2[row * padded_rows(N) + i] = lse[jq];
            Ds[row * padded_rows(N) + i] = Di[jq];
        }
    }

    typedef TileCopies<KEY_TILE, ROW, 4> Copies;
    const bool small_strides = k_row < MOST_STRIDE && v_row < MOST_STRIDE;
    auto issue = [&](int u) __attribute__((always_inline)) {
        const int k0 = list.tile_key(u);
        const uint32_t dst = lds_base + (u & 1) * TILE_BYTES;
        if (small_strides && list.inside(k0)) {
            Copies::whole(K + k0 * k_row, k_row, dst, w, l, swizzle<CPR>);
            Copies::whole(V + k0 * v_row, v_row, dst + 2 * TILE_BYTES, w, l, swizzle<CPR>);
        } else {
            Copies::any(dst, w, l, [&](int r) { return K + list.seen_key(k0 + r) * k_row; }, swizzle<CPR>);
            Copies::any(dst + 2 * TILE_BYTES, w, l, [&](int r) { return V + list.seen_key(k0 + r) * v_row; }, swizzle<CPR>);
        }
    };

    f32x4 acc[DT][QB];
#pragma unroll
    for (int id = 0; id < DT; ++id)
#pragma unroll
        for (int jq = 0; jq < QB; ++jq) acc[id][jq] = (f32x4){0, 0, 0, 0};
    uint32_t by_row = T::row_address(lds_base, l), by_column = T::column_address(lds_base, l);
    if (ntiles > 0) issue(0);
    for (int u = 0; u < ntiles; ++u) {
        landed_barrier();
        if (u + 1 < ntiles) issue(u + 1);
#pragma unroll 1
        for (int half = 0; half < KEY_TILE / TILE; ++half) {
            const int k0 = list.tile_key(u) + half * TILE, k1 = k0 + TILE - 1;
            const bool none = k0 > p_hi || (k0 >= sinks && p_lo >= 0 && k1 < p_lo - window + 1);
            if (!none) {
                const bool all = k1 <= p_lo && (k0 >= p_hi - window + 1 || k1 < sinks);
                auto visible = [&](int key, int jq) __attribute__((always_inline)) { return (key <= row_hi[jq]) & ((key >= row_lo[jq]) | (key < sinks)); };
                i32x4 y[QB];                                     // dS^T as B operand
                static_for<2>([&](auto cc) __attribute__((always_inline)) {
                    constexpr int c = decltype(cc)::value;
                    f32x4 s[QB], dp[QB];                         // S^T and dP^T: 16 keys x [16 rows]
                    T::template products<c, 0, 2 * TILE_BYTES>(s, dp, by_row, qf, of);
#pragma unroll
                    for (int jq = 0; jq < QB; ++jq)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const float P = __builtin_amdgcn_exp2f(__builtin_fmaf(s[jq][r], scale, -lse[jq]));
                            s[jq][r] = P * (dp[jq][r] - Di[jq]);
                        }
                    if (!all) {
#pragma unroll
                        for (int jq = 0; jq < QB; ++jq)
#pragma unroll
                            for (int r = 0; r < 4; ++r) s[jq][r] = visible(k0 + c * 16 + 4 * g + r, jq) ? s[jq][r] : 0.0f;
                    }
                    pack<c>(y, s);
                });
                const CYC_LDS char *here = lds + (u & 1) * TILE_BYTES + half * TILE * ROW;
                const bool careful = !all && T::infinite(here, l);
                if (__builtin_expect(careful, 0)) T::accumulate_carefully(acc, by_column, here, l, y, [&](int r, int jq) { return visible(k0 + r, jq); }, not_a_number);
                else T::template accumulate<0>(acc, by_column, y);
            }
            by_row += TILE * ROW;
            by_column += TILE * ROW;
        }
        const int turn = u & 1 ? -2 * TILE_BYTES : 0;                                // both halves done: the other stage follows, or the first
        by_row += turn;
        by_column += turn;
    }

    const float back = 1.0f / __builtin_sqrtf((float)D);
#pragma unroll
    for (int jq = 0; jq < QB; ++jq) {
        const int r = r0 + jq * 16 + lq;
        if (r > row_last) continue;
        const int i = r / group, h = head * group + r - i * group;
        char *dq = (char *)p.dQ.base + b * p.dQ.batch + h * p.dQ.head + i * p.dQ.row;
#pragma unroll
        for (int id = 0; id < DT; ++id) {
            bf16x4 o;
#pragma unroll
            for (int x = 0; x < 4; ++x) o[x] = (__bf16)(acc[id][jq][x] * back);
            *(bf16x4 *)(dq + (id * 16 + 4 * g) * 2) = o;
        }
    }
}

// ---- dK and dV.  A workgroup of four waves keeps 64 * KB keys of one key head and walks the rows that see any of them, head after head in
// tiles of 32 queries.  Keys that many rows see, the sinks before all, and keys of calls with few of them have their rows cut into runs,
// which different workgroups take and a second kernel adds up in ascending order.
struct Runs {
    int tiles;                           // tiles of keys
    int first, first_runs, runs;         // tiles below `first` have first_runs runs, the others `runs`
    __host__ __device__ int per_pair() const { return first * first_runs + (tiles - first) * runs; }
    // partial sums kept: those of the first tiles, and of the others where they have more than one run
    __host__ __device__ int kept_tiles() const { return runs > 1 ? tiles : first_runs > 1 ? first : 0; }
    __host__ __device__ int kept_per_pair() const { return runs > 1 ? per_pair() : first_runs > 1 ? first * first_runs : 0; }
    __host__ __device__ int slot(int tile) const { return tile < first ? tile * first_runs : first * first_runs + (tile - first) * runs; }
    __host__ __device__ int runs_of(int tile) const { return tile < first ? first_runs : runs; }
};

constexpr int KEY_BLOCKS = 2;            // 16-key blocks of a wave: what the registers hold at d = 128
constexpr int KEYS = 64 * KEY_BLOCKS;

// The code for tiles that are not all finite takes registers that the usual case does not have to spare (96 of them spilled, and
// half the speed), so it has a launch of its own: CAREFUL false does without and leaves a mark where it met such a masked tile, CAREFUL true
// does the marked workgroups again.
template <int D, bool CAREFUL>
__global__ __launch_bounds__(256, 2) void grad_kv_kernel(const WindowProblem p, const Runs runs, float scale, const float *lse2, const float *Ds, float *part, int *marks)
{
    typedef Tile<D> T;
    constexpr int ROW = T::ROW, CPR = T::CPR, DS = T::DS, DT = T::DT, KB = KEY_BLOCKS, KW = 16 * KB;
    constexpr int TILE_BYTES = TILE * ROW, STAGE = 2 * TILE_BYTES + 1024;
    // a stage: the tile of Q, that of dO, lse and D of its rows
    __shared__ __attribute__((aligned(1024))) char lds_raw[2 * STAGE];
    CYC_LDS char *lds = (CYC_LDS char *)lds_raw;
    const uint32_t lds_base = (uint32_t)(uintptr_t)lds;
    const int l = threadIdx.x & 63, lq = l & 15, g = l >> 4, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int mark = blockIdx.x * 4;
    if (CAREFUL && marks[mark] + marks[mark + 1] + marks[mark + 2] + marks[mark + 3] == 0) return;
    bool marked = false;
    const Place at(blockIdx.x, p.batch * p.kv_heads, runs.per_pair());
    const int pair = at.pair, slot = at.unit;
    const int in_first = runs.first * runs.first_runs;
    const int tile = __builtin_amdgcn_readfirstlane(slot < in_first ? slot / runs.first_runs : runs.first + (slot - in_first) / runs.runs);
    const int run = slot - runs.slot(tile), nruns = runs.runs_of(tile);
    const int64_t b = __builtin_amdgcn_readfirstlane(pair / p.kv_heads);
    const int head = pair - (int)b * p.kv_heads;
    const int group = p.group, N = p.N, M = p.M, window = p.window, sinks = p.sinks;

    // ---- the queries that see any of the keys k_first .. k_last, and this run's share of the tiles (head, 32 queries)
    const int k_first = tile * KEYS, k_last = (M - k_first < KEYS ? M : k_first + KEYS) - 1;
    const int i_first = k_first - (M - N) > 0 ? k_first - (M - N) : 0;
    const int64_t reach = (int64_t)k_last + window - 1 - (M - N);
    const int i_last = k_first < sinks || reach > N - 1 ? N - 1 : (int)reach;
    const int t_first = i_first / TILE, per_head = i_last >= i_first ? i_last / TILE - t_first + 1 : 0;
    const int all_tiles = per_head * group;
    const int u_first = __builtin_amdgcn_readfirstlane((int)((int64_t)all_tiles * run / nruns));
    const int u_last = __builtin_amdgcn_readfirstlane((int)((int64_t)all_tiles * (run + 1) / nruns));

    // ---- this wave's keys as B operands
    const int kw = k_first + w * KW, kw_last = kw + KW - 1;
    i32x4 kf[KB][DS], vf[KB][DS];
#pragma unroll
    for (int n = 0; n < KB; ++n) {
        int key = kw + n * 16 + lq;
        key = key < M ? key : M - 1;
        const char *k = p.K.base + b * p.K.batch + head * p.K.head + key * p.K.row + g * 16, *v = p.V.base + b * p.V.batch + head * p.V.head + key * p.V.row + g * 16;
#pragma unroll
        for (int ks = 0; ks < DS; ++ks) {
            kf[n][ks] = *(const i32x4 *)(k + ks * 64);
            vf[n][ks] = *(const i32x4 *)(v + ks * 64);
        }
    }

    const int64_t q_row = p.Q.row, q_head = p.Q.head, o_row = p.dO.row, o_head = p.dO.head, padded = padded_rows(N);
    const char *Q = p.Q.base + b * p.Q.batch + head * group * q_head, *dO = p.dO.base + b * p.dO.batch + head * group * o_head;
    const float *stats = (l < 32 ? lse2 : Ds) + (b * p.heads + head * group) * padded + (l & 31);
    typedef TileCopies<TILE, ROW, 4> Copies;
    const bool small_strides = q_row < MOST_STRIDE && o_row < MOST_STRIDE;
    auto issue = [&](int u) __attribute__((always_inline)) {
        const int h = __builtin_amdgcn_readfirstlane(u / per_head), i0 = __builtin_amdgcn_readfirstlane((t_first + u - h * per_head) * TILE);
        const uint32_t dst = lds_base + ((u - u_first) & 1) * STAGE;
        const char *q = Q + h * q_head, *o = dO + h * o_head;
        if (small_strides && i0 + TILE <= N) {
            Copies::whole(q + i0 * q_row, q_row, dst, w, l, swizzle<CPR>);
            Copies::whole(o + i0 * o_row, o_row, dst + TILE_BYTES, w, l, swizzle<CPR>);
        } else {
            Copies::any(dst, w, l, [&](int r) { return q + (i0 + r < N ? i0 + r : N - 1) * q_row; }, swizzle<CPR>);
            Copies::any(dst + TILE_BYTES, w, l, [&](int r) { return o + (i0 + r < N ? i0 + r : N - 1) * o_row; }, swizzle<CPR>);
        }
        if (w == 0)
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" : : "s"(dst + 2 * TILE_BYTES), "v"(stats + h * padded + i0) : "memory", "m0");
    };

    f32x4 dk[DT][KB], dv[DT][KB];
#pragma unroll
    for (int id = 0; id < DT; ++id)
#pragma unroll
        for (int n = 0; n < KB; ++n) dk[id][n] = dv[id][n] = (f32x4){0, 0, 0, 0};
    uint32_t by_row = T::row_address(lds_base, l), by_column = T::column_address(lds_base, l);
    if (u_first < u_last) issue(u_first);
    for (int u = u_first; u < u_last; ++u) {
        landed_barrier();
        if (u + 1 < u_last) issue(u + 1);
        const int stage = (u - u_first) & 1, i0 = (t_first + u % per_head) * TILE;
        const int p0 = i0 + M - N, p1 = (i0 + TILE < N ? i0 + TILE : N) - 1 + M - N;
        const bool none = kw >= M || p1 < kw || (kw >= sinks && (int64_t)p0 - kw_last >= window);
        if (!none) {
            const bool all = kw_last <= p0 && kw_last < M && i0 + TILE <= N && (p1 - kw < window || kw_last < sinks);
            const CYC_LDS char *here = lds + stage * STAGE;
            uint32_t row_address = by_row, column_address = by_column;
            asm("" : "+v"(row_address), "+v"(column_address));       // (the addresses that derive from them are cheaper taken than kept)
            auto visible = [&](int r, int n) __attribute__((always_inline)) {
                const int position = p0 + r, key = kw + n * 16 + lq;
                return (i0 + r < N) & (key <= position) & ((position - key < window) | (key < sinks));
            };
            i32x4 py[KB], dsy[KB];                                   // P and dS as B operands
            static_for<2>([&](auto cc) __attribute__((always_inline)) {
                constexpr int c = decltype(cc)::value;
                f32x4 s[KB], dp[KB];                                 // S and dP: 16 queries x [16 keys]
                T::template products<c, 0, TILE_BYTES>(s, dp, row_address, kf, vf);
                const f32x4 lse = *(const CYC_LDS f32x4 *)(here + 2 * TILE_BYTES + (c * 16 + 4 * g) * 4);
                const f32x4 Di = *(const CYC_LDS f32x4 *)(here + 2 * TILE_BYTES + 128 + (c * 16 + 4 * g) * 4);
#pragma unroll
                for (int n = 0; n < KB; ++n)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float P = __builtin_amdgcn_exp2f(__builtin_fmaf(s[n][r], scale, -lse[r]));
                        s[n][r] = P;
                        dp[n][r] = P * (dp[n][r] - Di[r]);
                    }
                if (!all) {
#pragma unroll
                    for (int n = 0; n < KB; ++n)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const bool seen = visible(c * 16 + 4 * g + r, n);
                            s[n][r] = seen ? s[n][r] : 0.0f;
                            dp[n][r] = seen ? dp[n][r] : 0.0f;
                        }
                }
                pack<c>(py, s);
                pack<c>(dsy, dp);
            });
            const bool careful = !all && (T::infinite(here, l) || T::infinite(here + TILE_BYTES, l));
            if (CAREFUL && careful) {
                T::accumulate_carefully(dv, column_address + TILE_BYTES, here + TILE_BYTES, l, py, visible, itself);
                T::accumulate_carefully(dk, column_address, here, l, dsy, visible, not_a_number);
            } else {
                marked |= careful;
                T::template accumulate<TILE_BYTES>(dv, column_address, py);
                T::template accumulate<0>(dk, column_address, dsy);
            }
        }
        const int turn = stage ? -STAGE : STAGE;
        by_row += turn;
        by_column += turn;
    }

    if (!CAREFUL && l == 0) marks[mark + w] = marked;
    // accumulator register r of lane l: d = 16 id + 4 (l/16) + r, key kw + 16 n + l%16
    const float back = 1.0f / __builtin_sqrtf((float)D);
#pragma unroll
    for (int n = 0; n < KB; ++n) {
        const int key = kw + n * 16 + lq;
        if (nruns > 1) {
            float *to = part + (((int64_t)pair * runs.kept_per_pair() + slot) * 2 * KEYS + w * KW + n * 16 + lq) * D;
#pragma unroll
            for (int id = 0; id < DT; ++id) {
                *(f32x4 *)(to + id * 16 + 4 * g) = dk[id][n];
                *(f32x4 *)(to + (int64_t)KEYS * D + id * 16 + 4 * g) = dv[id][n];
            }
            continue;
        }
        if (key >= M) continue;
        char *to_k = (char *)p.dK.base + b * p.dK.batch + head * p.dK.head + key * p.dK.row, *to_v = (char *)p.dV.base + b * p.dV.batch + head * p.dV.head + key * p.dV.row;
#pragma unroll
        for (int id = 0; id < DT; ++id) {
            bf16x4 x, y;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                x[r] = (__bf16)(dk[id][n][r] * back);
                y[r] = (__bf16)dv[id][n][r];
            }
            *(bf16x4 *)(to_k + (id * 16 + 4 * g) * 2) = x;
            *(bf16x4 *)(to_v + (id * 16 + 4 * g) * 2) = y;
        }
    }
}

// Adds the runs of a tile of keys in ascending order; a thread takes four d of a key's dK and dV.
template <int D> __global__ __launch_bounds__(256) void grad_join_kernel(const WindowProblem p, const Runs runs, const float *part)
{
    const int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int c = (int)(x % (D / 4)) * 4, in_tile = (int)(x / (D / 4) % KEYS);
    const int64_t rest = x / (D / 4) / KEYS;
    const int tile = (int)(rest % runs.kept_tiles());
    const int64_t pair = rest / runs.kept_tiles(), b = pair / p.kv_heads;
    const int head = (int)(pair % p.kv_heads), key = tile * KEYS + in_tile;
    if (b >= p.batch || key >= p.M || runs.runs_of(tile) <= 1) return;
    const float *from = part + ((pair * runs.kept_per_pair() + runs.slot(tile)) * 2 * KEYS + in_tile) * D + c;
    f32x4 dk = {0, 0, 0, 0}, dv = {0, 0, 0, 0};
    for (int run = 0; run < runs.runs_of(tile); ++run, from += 2 * KEYS * D) {
        dk += *(const f32x4 *)from;
        dv += *(const f32x4 *)(from + KEYS * D);
    }
    const float back = 1.0f / __builtin_sqrtf((float)D);
    bf16x4 u, v;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        u[r] = (__bf16)(dk[r] * back);
        v[r] = (__bf16)dv[r];
    }
    *(bf16x4 *)((char *)p.dK.base + b * p.dK.batch + head * p.dK.head + key * p.dK.row + c * 2) = u;
    *(bf16x4 *)((char *)p.dV.base + b * p.dV.batch + head * p.dV.head + key * p.dV.row + c * 2) = v;
}

// The chip takes 512 workgroups at a time.  With fewer tiles of keys than that their rows are cut into runs of at least eight steps; the
// tiles of sinks, which every later row sees, into runs as long as the other tiles' work.
Runs choose_runs(const WindowProblem &p)
{
    const int keys = KEYS;
    Runs r = {(p.M + keys - 1) / keys, 0, 1, 1};
    const int64_t pairs = (int64_t)p.batch * p.kv_heads;
    const int64_t usual = std::min<int64_t>(p.N, (int64_t)p.window + keys), steps = (usual + TILE - 1) / TILE * p.group;
    const int64_t all_steps = ((int64_t)p.N + TILE - 1) / TILE * p.group;
    r.runs = (int)std::max<int64_t>(1, std::min({512 / std::max<int64_t>(1, pairs * r.tiles), steps / 8, (int64_t)64}));
    r.first = (int)std::min<int64_t>(r.tiles, ((int64_t)std::min(p.sinks, p.M) + keys - 1) / keys);
    if (p.window == INT_MAX) r.first = 0;
    const int64_t run_steps = std::max<int64_t>(1, (steps + r.runs - 1) / r.runs);
    r.first_runs = (int)std::max<int64_t>(r.runs, std::min<int64_t>((all_steps + run_steps - 1) / run_steps, 256));
    if (r.first == 0) r.first_runs = r.runs;
    return r;
}

int64_t stats_bytes(const WindowProblem &p) { return ((int64_t)p.batch * p.heads * padded_rows(p.N) * 8 + 255) / 256 * 256; }

int64_t marks_bytes(const WindowProblem &p) { return (int64_t)p.batch * p.kv_heads * choose_runs(p).per_pair() * 16; }

template <int D> hipError_t launch_grad(const WindowProblem &p, void *workspace, hipStream_t s)
{
    float *lse2 = (float *)workspace, *Ds = lse2 + (int64_t)p.batch * p.heads * padded_rows(p.N), *part = (float *)((char *)workspace + stats_bytes(p) + (p.M > 0 ? marks_bytes(p) : 0));
    int *marks = (int *)((char *)workspace + stats_bytes(p));
    const float scale = (float)(1.4426950408889634 / __builtin_sqrt((double)D));
    const int tiles = (int)(((int64_t)p.N * p.group + 127) / 128);
    const int64_t pairs = (int64_t)p.batch * p.kv_heads;
    const Runs runs = choose_runs(p);
    if (tiles * pairs >= ((int64_t)1 << 31) || runs.per_pair() * pairs >= ((int64_t)1 << 31)) return hipErrorInvalidValue;
    hipError_t e = hipSuccess;
    if (p.N > 0) e = launch_kernel(grad_q_kernel<D>, dim3((unsigned)(tiles * pairs)), dim3(256), s, p, tiles, scale, lse2, Ds);
    if (e != hipSuccess || p.M == 0) return e;
    auto keys_of = [&](auto kernel) {
        return launch_kernel(kernel, dim3((unsigned)(runs.per_pair() * pairs)), dim3(256), s, p, runs, scale, (const float *)lse2, (const float *)Ds, part, marks);
    };
    e = keys_of(grad_kv_kernel<D, false>);
    if (e == hipSuccess) e = keys_of(grad_kv_kernel<D, true>);
    if (e != hipSuccess || runs.kept_tiles() == 0) return e;
    const int64_t threads = pairs * runs.kept_tiles() * KEYS * (D / 4);
    return launch_kernel(grad_join_kernel<D>, dim3((unsigned)((threads + 255) / 256)), dim3(256), s, p, runs, (const float *)part);
}

}  // namespace

int64_t window_grad_workspace_bytes(const WindowProblem &p)
{
    const int64_t keys = KEYS;
    return stats_bytes(p) + (p.M > 0 ? marks_bytes(p) + (int64_t)p.batch * p.kv_heads * choose_runs(p).kept_per_pair() * 2 * keys * p.d * 4 : 0);
}

hipError_t launch_window_grad(const WindowProblem &p, void *workspace, int64_t, hipStream_t s)
{
    return p.d == 128 ? launch_grad<128>(p, workspace, s) : launch_grad<64>(p, workspace, s);
}

}  // namespace cyc
