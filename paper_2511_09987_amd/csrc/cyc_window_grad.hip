// cyc_window_grad.hip -- the gradient of attention with a sliding window and sinks.
//
// With P_ij = exp(S_ij - lse_i) over the keys that i sees, D_i = dO_i.O_i and dS_ij = P_ij (dO_i.V_j - D_i):
//     dQ_i = sum_j dS_ij K_j / sqrt(d),   dK_j = sum_i dS_ij Q_i / sqrt(d),   dV_j = sum_i P_ij dO_i,
// the last two also over the heads that share key j.  Two kernels, so that every sum stays with one owner and no atomic adds are needed:
// one keeps rows (query, head) and walks their keys for dQ (three products a pair), the other keeps keys and walks the rows that
// see them for dK and dV (four); P is taken again in the second.  Seven products for the five of the formulas, against the 4 bytes per
// pair that P and dS would cost in memory, written and read: about the time of the two products, and room that grows with N M.
// Bounded by vector work and waits beside the products, which keep the matrix units busy 38 to 53 % of the time: 4 x 16 heads x 4096 x 128, causal,
// 850 to 900 us in all, traced one by one dQ 363 us and dK and dV 519 at least, 1.1 PFLOP/s of products (with constant inputs, which draw less power, 12 %
// less time); 2 x 32/8 heads, window 1024, 196 and 283.
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

// Both kernels multiply in groups of four LDS reads, the reads of the next group on their way meanwhile: four fragments of rows
// (16 bytes a lane each) or the halves of two transposed ones.
struct Group {
    i32x4 rows[4];
    i32x2 columns[4];
};
template <int PENDING, bool COLUMNS> __device__ __forceinline__ void arrived(Group &x)
{
    if constexpr (COLUMNS) asm volatile("s_waitcnt lgkmcnt(%4)" : "+v"(x.columns[0]), "+v"(x.columns[1]), "+v"(x.columns[2]), "+v"(x.columns[3]) : "n"(PENDING));
    else asm volatile("s_waitcnt lgkmcnt(%4)" : "+v"(x.rows[0]), "+v"(x.rows[1]), "+v"(x.rows[2]), "+v"(x.rows[3]) : "n"(PENDING));
}

// what is left beside products: nothing, or the elements M * COUNT / MS .. of COUNT beside product M of MS
template <int N> constexpr std::integral_constant<int, N> number{};
constexpr auto nothing = [](auto) __attribute__((always_inline)) {};
template <int COUNT, int MS, int M, class F> __device__ __forceinline__ void share(F &&f)
{
    constexpr int from = M * COUNT / MS, to = (M + 1) * COUNT / MS;
    static_for<to - from>([&](auto i_c) __attribute__((always_inline)) { f(std::integral_constant<int, from + decltype(i_c)::value>{}); });
}

// A tile of rows of D elements in LDS.
template <int D> struct Tile {
    static constexpr int ROW = D * 2, CPR = ROW / 16, DS = D / 32, DT = D / 16;
    // this lane's addresses within a tile: row l % 16 (chunk l / 16 of 64 bytes; 32-element step ks is at ^ ks << 6) and, transposed, row
    // 4 (l / 16) + (l % 16) / 4 (16-element tile id is at ^ id << 5)
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
    // Rows: steps 2 J and 2 J + 1 of rows 0-15 and 16-31 (x.rows: step, half).  A operand of the products along d.
    template <int J, int OFF> static __device__ __forceinline__ void request_rows(Group &x, uint32_t address)
    {
        static_for<4>([&](auto i_c) __attribute__((always_inline)) {
            constexpr int i = decltype(i_c)::value;
            lds_read128<OFF + i % 2 * 16 * ROW>(x.rows[i], address ^ (2 * J + i / 2) << 6);
        });
    }
    // Columns: 16-element tiles 2 J and 2 J + 1 of 32 rows.  A operand, d 16 id + l % 16; k-slots 0..3 are the rows 4 (l / 16) .. +3, k-slots 4..7
    // those 16 further down: the order in which accumulators of the products along d, rounded, make a B operand.
    template <int J, int OFF> static __device__ __forceinline__ void request_columns(Group &x, uint32_t address)
    {
        static_for<4>([&](auto i_c) __attribute__((always_inline)) {
            constexpr int i = decltype(i_c)::value;
            lds_read_tr64<OFF + i % 2 * 16 * ROW>(x.columns[i], address ^ (2 * J + i / 2) << 5);
        });
    }
    // The products of a group, beside(m) after the m-th: vector instructions that the matrix cores hide.
    // out[half][n] = (rows) x[n], from zero at J = 0
    template <int J, int NB, class Beside>
    static __device__ __forceinline__ void multiply_rows(f32x4 (&out)[2][NB], const Group &f, const i32x4 (&x)[NB][DS], Beside &&beside)
    {
        static_for<4 * NB>([&](auto m_c) __attribute__((always_inline)) {
            constexpr int m = decltype(m_c)::value, i = m / NB, n = m % NB;
            out[i % 2][n] = mfma16(f.rows[i], x[n][2 * J + i / 2], J == 0 && i < 2 ? (f32x4){0, 0, 0, 0} : out[i % 2][n]);
            beside(m_c);
        });
    }
    // acc[id][n] += (columns) y[n]
    template <int J, int NB, class Beside>
    static __device__ __forceinline__ void multiply_columns(f32x4 (&acc)[DT][NB], const Group &x, const i32x4 (&y)[NB], Beside &&beside)
    {
        static_for<2 * NB>([&](auto m_c) __attribute__((always_inline)) {
            constexpr int m = decltype(m_c)::value, i = m / NB, n = m % NB;
            acc[2 * J + i][n] = mfma16(mfma_frag(x.columns[2 * i], x.columns[2 * i + 1]), y[n], acc[2 * J + i][n]);
            beside(m_c);
        });
    }
    // acc[id][n] += (tile)^T y[n] on its own
    template <int OFF, int NB> static __device__ __forceinline__ void accumulate(f32x4 (&acc)[DT][NB], uint32_t address, const i32x4 (&y)[NB])
    {
        Group x[2];
        request_columns<0, OFF>(x[0], address);
        static_for<DT / 2>([&](auto j_c) __attribute__((always_inline)) {
            constexpr int j = decltype(j_c)::value;
            if constexpr (j + 1 < DT / 2) request_columns<j + 1, OFF>(x[(j + 1) % 2], address);
            arrived<(j + 1 < DT / 2 ? 4 : 0), true>(x[j % 2]);
            multiply_columns<j>(acc, x[j % 2], y, nothing);
        });
    }
    static __device__ __forceinline__ bool infinite(const CYC_LDS char *tile, int l)
    {
        return any_infinite<TILE * ROW / 1024>([&](auto ic) __attribute__((always_inline)) { return ((const CYC_LDS i32x4 *)tile)[decltype(ic)::value * 64 + l]; });
    }
    // accumulate() with the finite values alone; then add(value) of every other value, row by row, where seen(row, n)
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
                    for (int x = 0; x < 4; ++x) acc[id][n][x] += (seen(r, n) & !__builtin_isfinite((float)v[x])) ? add((float)v[x]) : 0.0f;
            }
        }
    }
};

// two values, rounded, as one word of a B operand
__device__ __forceinline__ int pack(float x, float y)
{
    const bf16x2 pair = __builtin_convertvector((f32x2){x, y}, bf16x2);
    return __builtin_bit_cast(int, pair);
}

__device__ __forceinline__ float not_a_number(float) { return __builtin_nanf(""); }
__device__ __forceinline__ float itself(float x) { return x; }

// Is any of the wave's N sums `sum(i)` no finite number?  (0 times an infinity or NaN is NaN, and stays.)
template <int N, class Sum> __device__ __forceinline__ bool not_finite(Sum &&sum)
{
    float zero = 0;
    static_for<N>([&](auto i_c) __attribute__((always_inline)) {
        const f32x4 x = sum(i_c);
#pragma unroll
        for (int r = 0; r < 4; ++r) zero = __builtin_fmaf(x[r], 0.0f, zero);
    });
    return __builtin_amdgcn_ballot_w64(zero != 0) != 0;
}

// lse and D of every row by head, lse in the log2 domain, heads padded to whole tiles
__host__ __device__ inline int64_t padded_rows(int N) { return ((int64_t)N + TILE - 1) / TILE * TILE; }

// ---- dQ.  A workgroup of four waves keeps 128 rows r (query r / group, head r % group of a key head) and walks the keys that any of them
// sees in tiles of 64, two steps of 32 to a barrier.  Also writes lse and D of its rows for the other kernel.  Where there are few workgroups, each
// list of keys is cut into runs, which different workgroups take and the last kernel adds up.
constexpr int KEY_TILE = 64, LEAST_TILES = 4;   // of a run

template <int D> __global__ __launch_bounds__(256, 2) void grad_q_kernel(const WindowProblem p, int tiles, int runs, float scale, float *lse2, float *Ds, float *part)
{
    typedef Tile<D> T;
    constexpr int ROW = T::ROW, CPR = T::CPR, DS = T::DS, DT = T::DT, QB = 2, QW = 32, ROWS = 128;
    constexpr int TILE_BYTES = KEY_TILE * ROW;
    __shared__ __attribute__((aligned(1024))) char lds_raw[4 * TILE_BYTES];        // two stages of K, then two of V
    CYC_LDS char *lds = (CYC_LDS char *)lds_raw;
    const uint32_t lds_base = (uint32_t)(uintptr_t)lds;
    const int l = threadIdx.x & 63, lq = l & 15, g = l >> 4, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Place at(blockIdx.x, p.batch * p.kv_heads, tiles * runs);
    const int run = at.unit % runs, tile = tiles - 1 - at.unit / runs;              // (the most keys first)
    const int64_t b = at.pair / p.kv_heads;
    const int head = at.pair - (int)b * p.kv_heads;
    const int group = p.group, N = p.N, M = p.M, R = N * group, window = p.window, sinks = p.sinks;
    const char *K = p.K.base + b * p.K.batch + head * p.K.head, *V = p.V.base + b * p.V.batch + head * p.V.head;
    const int64_t k_row = p.K.row, v_row = p.V.row;

    const int row_first = tile * ROWS, row_last = (R - row_first < ROWS ? R : row_first + ROWS) - 1;
    const KeyList<KEY_TILE> list(row_first, row_last, group, N, M, window, sinks);
    const int per = runs == 1 ? list.count : max((list.count + runs - 1) / runs, LEAST_TILES);
    const int u_first = run * per, u_last = run == runs - 1 || u_first + per > list.count ? list.count : u_first + per;

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
        if (mine && g == 0 && run == 0) {
            lse2[row * padded_rows(N) + i] = lse[jq];
            Ds[row * padded_rows(N) + i] = Di[jq];
        }
    }

    typedef TileCopies<KEY_TILE, ROW, 4> Copies;
    const bool small_strides = k_row < MOST_STRIDE && v_row < MOST_STRIDE;
    auto issue = [&](int u) __attribute__((always_inline)) {
        const int k0 = list.tile_key(u);
        const uint32_t dst = lds_base + ((u - u_first) & 1) * TILE_BYTES;
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
    f32x4 s[2][2][QB], dp[2][QB];                                    // S^T of two parts of 32 keys, dP^T of one: [16 keys][16 rows]
    i32x4 y[2][QB];                                                  // dS^T as B operand, of two parts
    Group x[2];
    // 16 (key, row) pairs a lane; number e: [row block][16-key block][element]
    auto weigh = [&](auto part_c, auto e_c) __attribute__((always_inline)) {
        constexpr int P = decltype(part_c)::value, e = decltype(e_c)::value, jq = e / 8, ik = e / 4 % 2, r = e % 4;
        s[P][ik][jq][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[P][ik][jq][r], scale, -lse[jq]));
    };
    auto slope = [&](auto part_c, auto e_c) __attribute__((always_inline)) {     // elements 2 e and 2 e + 1
        constexpr int P = decltype(part_c)::value, e = 2 * decltype(e_c)::value, jq = e / 8, ik = e / 4 % 2, r = e % 4;
        y[P][jq][ik * 2 + r / 2] = pack(s[P][ik][jq][r] * (dp[ik][jq][r] - Di[jq]), s[P][ik][jq][r + 1] * (dp[ik][jq][r + 1] - Di[jq]));
    };
    // A tile that all rows see whole, two parts of 32 keys, as one stream of groups: S(0), dP(0), S(1), dP(1), dQ(0), dQ(1).  P of a part is taken
    // beside its dP, dS(0) beside S(1), dS(1) beside dQ(0).
    auto whole_tile = [&]() __attribute__((always_inline)) {
        constexpr int NS = DS / 2, NQ = DT / 2, GROUPS = 4 * NS + 2 * NQ;
        const std::integral_constant<int, 0> one;
        const std::integral_constant<int, 1> two;
        const uint32_t row_at = fresh(by_row), column_at = fresh(by_column);
        auto request = [&](auto n_c) __attribute__((always_inline)) {
            constexpr int n = decltype(n_c)::value;
            if constexpr (n < 4 * NS) T::template request_rows<n % NS, n / NS % 2 * 2 * TILE_BYTES + n / (2 * NS) * TILE * ROW>(x[n % 2], row_at);
            else if constexpr (n < GROUPS) T::template request_columns<(n - 4 * NS) % NQ, (n - 4 * NS) / NQ * TILE * ROW>(x[n % 2], column_at);
        };
        request(one);
        static_for<GROUPS>([&](auto n_c) __attribute__((always_inline)) {
            constexpr int n = decltype(n_c)::value;
            request(std::integral_constant<int, n + 1>{});
            arrived<(n + 1 < GROUPS ? 4 : 0), (n >= 4 * NS)>(x[n % 2]);
            if constexpr (n < 4 * NS) {
                constexpr int phase = n / NS, j = n % NS, MS = NS * 4 * QB, part = phase / 2;
                auto beside = [&](auto m_c) __attribute__((always_inline)) {
                    constexpr int m = j * 4 * QB + decltype(m_c)::value;
                    if constexpr (phase == 1 || phase == 3) share<16, MS, m>([&](auto e_c) __attribute__((always_inline)) { weigh(std::integral_constant<int, part>{}, e_c); });
                    if constexpr (phase == 2) share<8, MS, m>([&](auto e_c) __attribute__((always_inline)) { slope(one, e_c); });
                };
                if constexpr (phase % 2 == 0) T::template multiply_rows<j>(s[part], x[n % 2], qf, beside);
                else T::template multiply_rows<j>(dp, x[n % 2], of, beside);
            } else {
                constexpr int part = (n - 4 * NS) / NQ, j = (n - 4 * NS) % NQ, MS = NQ * 2 * QB;
                T::template multiply_columns<j>(acc, x[n % 2], y[part], [&](auto m_c) __attribute__((always_inline)) {
                    if constexpr (part == 0) share<8, MS, j * 2 * QB + decltype(m_c)::value>([&](auto e_c) __attribute__((always_inline)) { slope(two, e_c); });
                });
            }
        });
    };
    auto some_of_tile = [&](int k_tile, int stage) __attribute__((always_inline)) {
        const int l = fresh(threadIdx.x & 63), g = l >> 4;
#pragma unroll 1
        for (int half = 0; half < KEY_TILE / TILE; ++half) {
            const int k0 = k_tile + half * TILE, k1 = k0 + TILE - 1;
            if (k0 > p_hi || (k0 >= sinks && p_lo >= 0 && k1 < p_lo - window + 1)) continue;
            const bool all = k1 <= p_lo && (k0 >= p_hi - window + 1 || k1 < sinks);
            const uint32_t row_at = fresh(by_row) + half * TILE * ROW, column_at = fresh(by_column) + half * TILE * ROW;
            T::template request_rows<0, 0>(x[0], row_at);
            static_for<DS>([&](auto n_c) __attribute__((always_inline)) {
                constexpr int n = decltype(n_c)::value, j = n % (DS / 2);
                if constexpr (n + 1 < DS) T::template request_rows<(n + 1) % (DS / 2), (n + 1) / (DS / 2) * 2 * TILE_BYTES>(x[(n + 1) % 2], row_at);
                arrived<(n + 1 < DS ? 4 : 0), false>(x[n % 2]);
                if constexpr (n < DS / 2) T::template multiply_rows<j>(s[0], x[n % 2], qf, nothing);
                else T::template multiply_rows<j>(dp, x[n % 2], of, nothing);
            });
            auto visible = [&](int key, int jq) __attribute__((always_inline)) { return (key <= row_hi[jq]) & ((key >= row_lo[jq]) | (key < sinks)); };
            static_for<16>([&](auto e_c) __attribute__((always_inline)) {
                constexpr int e = decltype(e_c)::value, jq = e / 8, ik = e / 4 % 2, r = e % 4;
                weigh(std::integral_constant<int, 0>{}, e_c);
                const float ds = s[0][ik][jq][r] * (dp[ik][jq][r] - Di[jq]);
                s[0][ik][jq][r] = all | visible(k0 + ik * 16 + 4 * g + r, jq) ? ds : 0.0f;
            });
#pragma unroll
            for (int jq = 0; jq < QB; ++jq)
#pragma unroll
                for (int i = 0; i < 4; ++i) y[0][jq][i] = pack(s[0][i / 2][jq][i % 2 * 2], s[0][i / 2][jq][i % 2 * 2 + 1]);
            const CYC_LDS char *here = lds + stage * TILE_BYTES + half * TILE * ROW;
            if (__builtin_expect(!all && T::infinite(here, l), 0)) T::accumulate_carefully(acc, column_at, here, l, y[0], [&](int r, int jq) __attribute__((always_inline)) { return visible(k0 + r, jq); }, not_a_number);
            else T::template accumulate<0>(acc, column_at, y[0]);
        }
    };
    if (u_first < u_last) issue(u_first);
    int u = u_first;
    auto arrive = [&]() __attribute__((always_inline)) {
        landed_barrier();
        if (u + 1 < u_last) issue(u + 1);
    };
    auto leave = [&]() __attribute__((always_inline)) {
        const int turn = (u - u_first) & 1 ? -TILE_BYTES : TILE_BYTES;
        by_row += turn;
        by_column += turn;
        ++u;
    };
    while (u < u_last && u < list.whole) {                                         // (see tile_kernel: a loop for each kind of tile)
        arrive();
        if (!idle) whole_tile();
        leave();
    }
    while (u < u_last) {
        arrive();
        some_of_tile(list.tile_key(u), (u - u_first) & 1);
        leave();
    }

    const float back = 1.0f / __builtin_sqrtf((float)D);
#pragma unroll
    for (int jq = 0; jq < QB; ++jq) {
        const int r = r0 + jq * 16 + lq;
        if (r > row_last) continue;
        const int i = r / group, h = head * group + r - i * group;
        if (runs > 1) {
            float *to = part + (((int64_t)run * p.batch * p.heads + b * p.heads + h) * N + i) * D + 4 * g;
#pragma unroll
            for (int id = 0; id < DT; ++id) *(f32x4 *)(to + id * 16) = acc[id][jq];
            continue;
        }
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

// Masked tiles go through the same stream of groups as whole ones, P and dS set to 0 where a query does not see a key (3 x 12 heads x 1777 x
// d 64, window 333: 51 us with code of their own, one phase after the other, 40 so).  That 0 times an infinity or NaN in Q or dO is NaN shows
// in the sums at the end, and the code that keeps those out takes registers that the usual case does not have to spare (96 of them
// spilled, and half the speed).  So it has a launch of its own: CAREFUL false does without and leaves a mark where its sums are not all
// finite, CAREFUL true does the marked workgroups again.

// What a workgroup does, with its two stages and the values of its keys in `lds`.
template <int D> constexpr int STAGE_BYTES = 2 * TILE * D * 2 + 1024;             // the tile of Q, that of dO, lse and D of its rows
template <int D> constexpr int KEYS_LDS = 2 * STAGE_BYTES<D> + KEYS * D * 2;
template <int D, bool CAREFUL>
__device__ __forceinline__ void keys_of_block(const WindowProblem &p, const Runs &runs, float scale, const float *lse2, const float *Ds, float *part, int *used, int *marks, int block, CYC_LDS char *lds)
{
    typedef Tile<D> T;
    constexpr int ROW = T::ROW, CPR = T::CPR, DS = T::DS, DT = T::DT, KB = KEY_BLOCKS, KW = 16 * KB, TILE_BYTES = TILE * ROW, STAGE = STAGE_BYTES<D>;
    const uint32_t lds_base = (uint32_t)(uintptr_t)lds;
    const int l = threadIdx.x & 63, lq = l & 15, g = l >> 4, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int mark = block * 4;
    // the short runs of the first tiles after all others, beside the last of which they find places
    const int pairs = p.batch * p.kv_heads, in_first = runs.first * runs.first_runs, of_others = pairs * (runs.per_pair() - in_first);
    const bool is_first = block >= of_others;
    const Place at(is_first ? block - of_others : block, pairs, is_first ? in_first : runs.per_pair() - in_first);
    const int pair = at.pair, slot = at.unit + (is_first ? 0 : in_first);
    const int tile = __builtin_amdgcn_readfirstlane(slot < in_first ? slot / runs.first_runs : runs.first + (slot - in_first) / runs.runs);
    const int run = slot - runs.slot(tile), nruns = runs.runs_of(tile);
    const int64_t b = __builtin_amdgcn_readfirstlane(pair / p.kv_heads);
    const int head = pair - (int)b * p.kv_heads;
    const int group = p.group, N = p.N, M = p.M, window = p.window, sinks = p.sinks;

    // ---- the queries that see any of the keys k_first .. k_last, as tiles (head, 32 queries): first those whose queries all see all keys of the
    // workgroup, head by head, then the others; this run's share of them.  (The same share with CAREFUL, which repeats single runs beside others.)
    const int shift = M - N, k_first = tile * KEYS, k_last = (M - k_first < KEYS ? M : k_first + KEYS) - 1;
    const int i_first = k_first > shift ? k_first - shift : 0;
    const int64_t reach = (int64_t)k_last + window - 1 - shift;
    const int i_last = k_first < sinks || reach > N - 1 ? N - 1 : (int)reach;
    const int t_first = i_first / TILE, t_last = i_last >= i_first ? i_last / TILE : t_first - 1, per_head = t_last - t_first + 1;
    const int all_from = k_first + KEYS - 1 - shift > 0 ? (k_first + KEYS - 1 - shift + TILE - 1) / TILE : 0;
    const int64_t all_reach = (int64_t)k_first + window - TILE - shift;                              // the last tile's first query
    const int all_to = k_first + KEYS <= sinks || all_reach >= N ? N / TILE : all_reach < 0 ? 0 : min((int)(all_reach / TILE) + 1, N / TILE);
    const int w_first = all_from > t_first ? all_from : t_first;
    const int whole = k_first + KEYS > M || all_to <= w_first ? 0 : all_to - w_first;     // of a head
    const int others = per_head - whole, all_tiles = per_head * group, whole_tiles = whole * group;
    const int o_first = whole > 0 && w_first == t_first ? w_first + whole : t_first;
    const int u_first = __builtin_amdgcn_readfirstlane((int)((int64_t)all_tiles * run / nruns));
    const int u_last = __builtin_amdgcn_readfirstlane((int)((int64_t)all_tiles * (run + 1) / nruns));
    int next_head, next_tile;                                        // of the tile to be requested next
    if (u_first < whole_tiles) {
        next_head = u_first / max(whole, 1);
        next_tile = w_first + u_first - next_head * whole;
    } else {
        const int v = u_first - whole_tiles;
        next_head = others > 0 ? v / others : 0;
        next_tile = t_first + v - next_head * others;
        if (whole > 0 && next_tile >= w_first) next_tile += whole;
    }
    next_head = __builtin_amdgcn_readfirstlane(next_head);
    next_tile = __builtin_amdgcn_readfirstlane(next_tile);
    auto advance = [&](int u) __attribute__((always_inline)) {        // from tile u to u + 1
        ++next_tile;
        if (u < whole_tiles) {
            if (next_tile == w_first + whole) {
                ++next_head;
                next_tile = w_first;
                if (u + 1 == whole_tiles) {
                    next_head = 0;
                    next_tile = o_first;
                }
            }
        } else {
            if (whole > 0 && next_tile == w_first) next_tile += whole;
            if (next_tile > t_last) {
                ++next_head;
                next_tile = o_first;
            }
        }
    };

    // ---- this wave's keys: K as B operands in registers, V, for which those do not suffice at d = 128, in LDS behind the two stages
    const int kw = k_first + w * KW, kw_last = kw + KW - 1;
    i32x4 kf[KB][DS];
#pragma unroll
    for (int n = 0; n < KB; ++n) {
        int key = kw + n * 16 + lq;
        key = key < M ? key : M - 1;
        const char *k = p.K.base + b * p.K.batch + head * p.K.head + key * p.K.row + g * 16;
#pragma unroll
        for (int ks = 0; ks < DS; ++ks) kf[n][ks] = *(const i32x4 *)(k + ks * 64);
    }
    {
        const char *V = p.V.base + b * p.V.batch + head * p.V.head;
        TileCopies<KW, ROW, 1>::any(lds_base + 2 * STAGE + w * KW * ROW, 0, l, [&](int r) { return V + (kw + r < M ? kw + r : M - 1) * p.V.row; }, swizzle<CPR>);
    }

    const int64_t q_row = p.Q.row, q_head = p.Q.head, o_row = p.dO.row, o_head = p.dO.head, padded = padded_rows(N);
    const char *Q = p.Q.base + b * p.Q.batch + head * group * q_head, *dO = p.dO.base + b * p.dO.batch + head * group * o_head;
    const float *stats = (l < 32 ? lse2 : Ds) + (b * p.heads + head * group) * padded + (l & 31);
    typedef TileCopies<TILE, ROW, 4> Copies;
    const bool small_strides = q_row < MOST_STRIDE && o_row < MOST_STRIDE;
    auto issue = [&](int u) __attribute__((always_inline)) {
        const int i0 = next_tile * TILE;
        const uint32_t dst = lds_base + ((u - u_first) & 1) * STAGE;
        const char *q = Q + next_head * q_head, *o = dO + next_head * o_head;
        if (small_strides && i0 + TILE <= N) {
            Copies::whole(q + i0 * q_row, q_row, dst, w, l, swizzle<CPR>);
            Copies::whole(o + i0 * o_row, o_row, dst + TILE_BYTES, w, l, swizzle<CPR>);
        } else {
            Copies::any(dst, w, l, [&](int r) { return q + (i0 + r < N ? i0 + r : N - 1) * q_row; }, swizzle<CPR>);
            Copies::any(dst + TILE_BYTES, w, l, [&](int r) { return o + (i0 + r < N ? i0 + r : N - 1) * o_row; }, swizzle<CPR>);
        }
        if (w == 0)
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off"
                         : : "s"(__builtin_amdgcn_readfirstlane(dst + 2 * TILE_BYTES)), "v"(stats + next_head * padded + i0) : "memory", "m0");
    };

    f32x4 dk[DT][KB], dv[DT][KB];
#pragma unroll
    for (int id = 0; id < DT; ++id)
#pragma unroll
        for (int n = 0; n < KB; ++n) dk[id][n] = dv[id][n] = (f32x4){0, 0, 0, 0};
    uint32_t by_row = T::row_address(lds_base, l), by_column = T::column_address(lds_base, l);
    f32x4 s[2][KB], dp[2][KB];                                       // S and dP: [16 queries][16 keys]
    f32x4 lse[2], Di[2];
    i32x4 py[KB], dsy[KB];                                           // P and dS as B operands
    Group x[2];
    // 16 (query, key) pairs a lane; number e: [16-query block][key block][element]
    // What a lane's two keys see, as distances in positions: query row r of a tile sees key n if 0 <= p0 + r - key < limit[n], the sinks' limit being
    // that of the call's last position.  (Rows behind the last query repeat it and see nothing.)
    int limit[KB], ahead;                                            // ahead: p0 + 4 (l/16) - the first key
    auto seen = [&](auto c_c, auto n_c, auto r_c) __attribute__((always_inline)) {
        constexpr int n = decltype(n_c)::value;
        return (unsigned)(ahead + (decltype(c_c)::value * 16 + decltype(r_c)::value - n * 16)) < (unsigned)limit[n];
    };
    auto weigh = [&](auto masked, auto e_c) __attribute__((always_inline)) {
        constexpr int e = decltype(e_c)::value, c = e / 8, n = e / 4 % 2, r = e % 4;
        s[c][n][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[c][n][r], scale, -lse[c][r]));
        if constexpr (decltype(masked)::value) s[c][n][r] = seen(number<c>, number<n>, number<r>) ? s[c][n][r] : 0.0f;
        if constexpr (r % 2 == 1) py[n][c * 2 + r / 2] = pack(s[c][n][r - 1], s[c][n][r]);
    };
    auto slope = [&](auto masked, auto e_c) __attribute__((always_inline)) {       // elements 2 e and 2 e + 1
        constexpr int e = 2 * decltype(e_c)::value, c = e / 8, n = e / 4 % 2, r = e % 4;
        float x = s[c][n][r] * (dp[c][n][r] - Di[c][r]), y = s[c][n][r + 1] * (dp[c][n][r + 1] - Di[c][r + 1]);
        if constexpr (decltype(masked)::value) {
            x = seen(number<c>, number<n>, number<r>) ? x : 0.0f;
            y = seen(number<c>, number<n>, number<r + 1>) ? y : 0.0f;
        }
        dsy[n][c * 2 + r / 2] = pack(x, y);
    };
    auto read_stats = [&](f32x4(&to)[2], const CYC_LDS char *from) __attribute__((always_inline)) {
#pragma unroll
        for (int c = 0; c < 2; ++c) to[c] = *(const CYC_LDS f32x4 *)(from + (c * 16 + 4 * g) * 4);
    };
    // step ks of dO's two halves and of V's two key blocks, and their four products
    auto request_values = [&](auto ks_c, Group &to, uint32_t row_at, uint32_t v_at) __attribute__((always_inline)) {
        constexpr int ks = decltype(ks_c)::value;
        lds_read128<TILE_BYTES>(to.rows[0], row_at ^ ks << 6);
        lds_read128<TILE_BYTES + 16 * ROW>(to.rows[1], row_at ^ ks << 6);
        lds_read128<0>(to.rows[2], v_at ^ ks << 6);
        lds_read128<16 * ROW>(to.rows[3], v_at ^ ks << 6);
    };
    auto multiply_values = [&](auto ks_c, const Group &f, auto &&beside) __attribute__((always_inline)) {
        constexpr int ks = decltype(ks_c)::value;
        static_for<4>([&](auto m_c) __attribute__((always_inline)) {
            constexpr int m = decltype(m_c)::value, c = m / 2, n = m % 2;
            dp[c][n] = mfma16(f.rows[c], f.rows[2 + n], ks == 0 ? (f32x4){0, 0, 0, 0} : dp[c][n]);
            beside(m_c);
        });
    };
    const uint32_t values = T::row_address(lds_base + 2 * STAGE + w * KW * ROW, l);
    // A tile as one stream of groups: S, dP beside which P is taken, dV beside which dS is, dK.  masked: not all queries see all keys.
    auto stream_tile = [&](auto masked, const CYC_LDS char *here) __attribute__((always_inline)) {
        constexpr int NS = DS / 2, NQ = DT / 2, GROUPS = NS + DS + 2 * NQ;
        const uint32_t row_at = fresh(by_row), column_at = fresh(by_column), v_at = fresh(values);
        auto request = [&](auto n_c) __attribute__((always_inline)) {
            constexpr int n = decltype(n_c)::value;
            if constexpr (n < NS) T::template request_rows<n, 0>(x[n % 2], row_at);
            else if constexpr (n < NS + DS) request_values(std::integral_constant<int, n - NS>{}, x[n % 2], row_at, v_at);
            else if constexpr (n < GROUPS) T::template request_columns<(n - NS - DS) % NQ, n - NS - DS < NQ ? TILE_BYTES : 0>(x[n % 2], column_at);
        };
        request(std::integral_constant<int, 0>{});
        static_for<GROUPS>([&](auto n_c) __attribute__((always_inline)) {
            constexpr int n = decltype(n_c)::value;
            if constexpr (n == NS - 1) read_stats(lse, here + 2 * TILE_BYTES);
            if constexpr (n == NS + DS - 1) read_stats(Di, here + 2 * TILE_BYTES + 128);
            request(std::integral_constant<int, n + 1>{});
            arrived<(n + 1 < GROUPS ? 4 : 0), (n >= NS + DS)>(x[n % 2]);
            if constexpr (n < NS) T::template multiply_rows<n>(s, x[n % 2], kf, nothing);
            else if constexpr (n < NS + DS) {
                multiply_values(std::integral_constant<int, n - NS>{}, x[n % 2], [&](auto m_c) __attribute__((always_inline)) {
                    share<16, 4 * DS, (n - NS) * 4 + decltype(m_c)::value>([&](auto e_c) __attribute__((always_inline)) { weigh(masked, e_c); });
                });
            } else if constexpr (n < NS + DS + NQ) {
                T::template multiply_columns<n - NS - DS>(dv, x[n % 2], py, [&](auto m_c) __attribute__((always_inline)) {
                    share<8, 2 * KB * NQ, (n - NS - DS) * 2 * KB + decltype(m_c)::value>([&](auto e_c) __attribute__((always_inline)) { slope(masked, e_c); });
                });
            } else T::template multiply_columns<n - NS - DS - NQ>(dk, x[n % 2], dsy, nothing);
        });
    };
    bool touched = false;                                            // has this wave met a tile whose queries see any of its keys?
    auto some_of_tile = [&](int i0, const CYC_LDS char *here) __attribute__((always_inline)) {
        const int p0 = i0 + shift, p1 = (i0 + TILE < N ? i0 + TILE : N) - 1 + shift;
        if (kw >= M || p1 < kw || (kw >= sinks && (int64_t)p0 - kw_last >= window)) return;
        touched = true;
        if constexpr (!CAREFUL) {
            const int l = fresh(threadIdx.x & 63);
            const int key = kw + (l & 15), left = M - key;
            ahead = p0 + 4 * (l >> 4) - key;
#pragma unroll
            for (int n = 0; n < KB; ++n) limit[n] = max(min(left - n * 16, key + n * 16 < sinks ? INT_MAX : window), 0);
            stream_tile(std::true_type{}, here);
            return;
        }
        const bool all = kw_last <= p0 && kw_last < M && i0 + TILE <= N && (p1 - kw < window || kw_last < sinks);
        const int l = fresh(threadIdx.x & 63), g = l >> 4, lq = l & 15;
        const uint32_t row_at = fresh(by_row), column_at = fresh(by_column), v_at = fresh(values);
        constexpr int NS = DS / 2;
        auto request = [&](auto n_c) __attribute__((always_inline)) {
            constexpr int n = decltype(n_c)::value;
            if constexpr (n < NS) T::template request_rows<n, 0>(x[n % 2], row_at);
            else if constexpr (n < NS + DS) request_values(std::integral_constant<int, n - NS>{}, x[n % 2], row_at, v_at);
        };
        request(std::integral_constant<int, 0>{});
        static_for<NS + DS>([&](auto n_c) __attribute__((always_inline)) {
            constexpr int n = decltype(n_c)::value;
            request(std::integral_constant<int, n + 1>{});
            arrived<(n + 1 < NS + DS ? 4 : 0), false>(x[n % 2]);
            if constexpr (n < NS) T::template multiply_rows<n>(s, x[n % 2], kf, nothing);
            else multiply_values(std::integral_constant<int, n - NS>{}, x[n % 2], nothing);
        });
        read_stats(lse, here + 2 * TILE_BYTES);
        read_stats(Di, here + 2 * TILE_BYTES + 128);
        auto visible = [&](int r, int n) __attribute__((always_inline)) {
            const int position = p0 + r, key = kw + n * 16 + lq;
            return (i0 + r < N) & (key <= position) & ((position - key < window) | (key < sinks));
        };
        static_for<16>([&](auto e_c) __attribute__((always_inline)) {
            constexpr int e = decltype(e_c)::value, c = e / 8, n = e / 4 % 2, r = e % 4;
            const bool seen = all | visible(c * 16 + 4 * g + r, n);
            const float P = __builtin_amdgcn_exp2f(__builtin_fmaf(s[c][n][r], scale, -lse[c][r])), dS = P * (dp[c][n][r] - Di[c][r]);
            s[c][n][r] = seen ? P : 0.0f;
            dp[c][n][r] = seen ? dS : 0.0f;
        });
#pragma unroll
        for (int n = 0; n < KB; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                py[n][i] = pack(s[i / 2][n][i % 2 * 2], s[i / 2][n][i % 2 * 2 + 1]);
                dsy[n][i] = pack(dp[i / 2][n][i % 2 * 2], dp[i / 2][n][i % 2 * 2 + 1]);
            }
        const bool careful = !all && (T::infinite(here, l) || T::infinite(here + TILE_BYTES, l));
        if (careful) {
            T::accumulate_carefully(dv, column_at + TILE_BYTES, here + TILE_BYTES, l, py, visible, itself);
            T::accumulate_carefully(dk, column_at, here, l, dsy, visible, not_a_number);
        } else {
            T::template accumulate<TILE_BYTES>(dv, column_at, py);
            T::template accumulate<0>(dk, column_at, dsy);
        }
    };
    int u = u_first, i0 = 0;
    auto arrive = [&]() __attribute__((always_inline)) {
        landed_barrier();
        i0 = next_tile * TILE;
        advance(u);
        if (u + 1 < u_last) issue(u + 1);
    };
    auto leave = [&]() __attribute__((always_inline)) {
        const int turn = (u - u_first) & 1 ? -STAGE : STAGE;
        by_row += turn;
        by_column += turn;
        ++u;
    };
    if (u_first < u_last) issue(u_first);
    while (!CAREFUL && u < u_last && u < whole_tiles) {
        arrive();
        touched = true;
        stream_tile(std::false_type{}, lds + ((u - u_first) & 1) * STAGE);
        leave();
    }
    while (u < u_last) {
        arrive();
        some_of_tile(i0, lds + ((u - u_first) & 1) * STAGE);
        leave();
    }

    if constexpr (!CAREFUL) {
        const bool marked = not_finite<2 * DT * KB>([&](auto i_c) __attribute__((always_inline)) {
            constexpr int i = decltype(i_c)::value;
            return i % 2 ? dk[i / 2 / KB][i / 2 % KB] : dv[i / 2 / KB][i / 2 % KB];
        });
        if (l == 0) marks[mark + w] = marked;
    }
    // accumulator register r of lane l: d = 16 id + 4 (l/16) + r, key kw + 16 n + l%16
    const float back = 1.0f / __builtin_sqrtf((float)D);
#pragma unroll
    for (int n = 0; n < KB; ++n) {
        const int key = kw + n * 16 + lq;
        if (nruns > 1) {
            // (most keys of a tile with sinks see nothing more after a while: nothing is kept of those)
            const int64_t kept = (int64_t)pair * runs.kept_per_pair() + slot;
            if (n == 0 && l == 0) used[kept * 4 + w] = touched;
            if (!touched) continue;
            float *to = part + (kept * 2 * KEYS + w * KW + n * 16 + lq) * D;
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

template <int D>
__global__ __launch_bounds__(256, 2) void grad_kv_kernel(const WindowProblem p, const Runs runs, float scale, const float *lse2, const float *Ds, float *part, int *used, int *marks)
{
    __shared__ __attribute__((aligned(1024))) char lds[KEYS_LDS<D>];
    keys_of_block<D, false>(p, runs, scale, lse2, Ds, part, used, marks, blockIdx.x, (CYC_LDS char *)lds);
}
// a few workgroups look through all marks, a lane at one
template <int D>
__global__ __launch_bounds__(256, 2) void grad_kv_careful_kernel(const WindowProblem p, const Runs runs, float scale, const float *lse2, const float *Ds, float *part, int *used, int *marks)
{
    __shared__ __attribute__((aligned(1024))) char lds[KEYS_LDS<D>];
    const int64_t blocks = (int64_t)p.batch * p.kv_heads * runs.per_pair(), step = gridDim.x;
    for (int64_t first = blockIdx.x; first < blocks; first += 64 * step) {
        const int64_t mine = first + (threadIdx.x & 63) * step;
        i32x4 m = {0, 0, 0, 0};
        if (mine < blocks) m = ((const i32x4 *)marks)[mine];
        for (uint64_t todo = __builtin_amdgcn_ballot_w64((m[0] | m[1] | m[2] | m[3]) != 0); todo; todo &= todo - 1) {
            const int block = (int)(first + __builtin_ctzll(todo) * step);
            keys_of_block<D, true>(p, runs, scale, lse2, Ds, part, used, marks, block, (CYC_LDS char *)lds);
            landed_barrier();                                         // (LDS is free again)
        }
    }
}

// Adds the runs in ascending order, a thread four d of a row.  The first workgroups: of a tile of keys, dK and dV, those runs in which the keys' wave did
// anything; the others: of dQ.
constexpr int MOST_RUNS = 256;
template <int D>
__global__ __launch_bounds__(256) void grad_join_kernel(const WindowProblem p, const Runs runs, int q_runs, const float *part, const int *used, const float *q_part)
{
    constexpr int PER = 1024 / D;                                     // keys of a workgroup, all of one wave of the other kernel; rows of dQ
    const float back = 1.0f / __builtin_sqrtf((float)D);
    const int of_keys = p.batch * p.kv_heads * runs.kept_tiles() * (KEYS / PER);
    if ((int)blockIdx.x >= of_keys) {
        const int64_t rows = (int64_t)p.batch * p.heads * p.N, row = (int64_t)(blockIdx.x - of_keys) * PER + threadIdx.x / (D / 4);
        const int d = threadIdx.x % (D / 4) * 4;
        if (row >= rows) return;
        f32x4 dq = {0, 0, 0, 0};
#pragma unroll 8
        for (int x = 0; x < q_runs; ++x) dq += *(const f32x4 *)(q_part + (x * rows + row) * D + d);
        const int64_t pair = row / p.N;
        bf16x4 o;
#pragma unroll
        for (int r = 0; r < 4; ++r) o[r] = (__bf16)(dq[r] * back);
        *(bf16x4 *)((char *)p.dQ.base + pair / p.heads * p.dQ.batch + pair % p.heads * p.dQ.head + row % p.N * p.dQ.row + d * 2) = o;
        return;
    }
    __shared__ int list[MOST_RUNS], counts[4];
    const int l = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int64_t block = blockIdx.x / (KEYS / PER);                   // (pair, tile)
    const int in_tile = (int)(blockIdx.x % (KEYS / PER)) * PER + threadIdx.x / (D / 4), c = threadIdx.x % (D / 4) * 4;
    const int tile = (int)(block % runs.kept_tiles()), n = runs.runs_of(tile);
    const int64_t pair = block / runs.kept_tiles(), b = pair / p.kv_heads;
    const int head = (int)(pair % p.kv_heads), key = tile * KEYS + in_tile;
    const int64_t kept = pair * runs.kept_per_pair() + runs.slot(tile);
    const bool mine = threadIdx.x < n && used[(kept + threadIdx.x) * 4 + in_tile / (16 * KEY_BLOCKS)];
    const uint64_t votes = __builtin_amdgcn_ballot_w64(mine);
    if (l == 0) counts[w] = __builtin_popcountll(votes);
    __syncthreads();
    int before = __builtin_popcountll(votes & (((uint64_t)1 << l) - 1)), count = 0;
    for (int x = 0; x < 4; ++x) {
        before += x < w ? counts[x] : 0;
        count += counts[x];
    }
    if (mine) list[before] = threadIdx.x;
    __syncthreads();
    if (key >= p.M) return;
    const float *from = part + (kept * 2 * KEYS + in_tile) * D + c;
    f32x4 dk = {0, 0, 0, 0}, dv = {0, 0, 0, 0};
#pragma unroll 4
    for (int x = 0; x < count; ++x) {
        const float *run = from + (int64_t)list[x] * 2 * KEYS * D;
        dk += *(const f32x4 *)run;
        dv += *(const f32x4 *)(run + KEYS * D);
    }
    bf16x4 u, v;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        u[r] = (__bf16)(dk[r] * back);
        v[r] = (__bf16)dv[r];
    }
    *(bf16x4 *)((char *)p.dK.base + b * p.dK.batch + head * p.dK.head + key * p.dK.row + c * 2) = u;
    *(bf16x4 *)((char *)p.dV.base + b * p.dV.batch + head * p.dV.head + key * p.dV.row + c * 2) = v;
}

// How the rows of a tile of keys are cut.  The chip takes 512 workgroups at a time, which count in rounds: 496 and 64 of the same length last
// twice as long as 496 (2 x 8 key heads x 4096 x 128, window 1024, sinks 4: 378 us so).  The tiles of sinks, whose rows are all that
// follow, go last in many short runs, which fill what the others leave over (the whole gradient 511 us with them first, 481 so); the others are cut where
// that makes fewer or shorter rounds, at a cost: three steps of 32 rows to start a run, the partial sums, written and read, and a launch.
// The partial sums of the sinks' tiles, and those of the others, take 64 MB at most.
constexpr int64_t MOST_PART = 128 << 20;

Runs choose_runs(const WindowProblem &p)
{
    Runs best = {(p.M + KEYS - 1) / KEYS, 0, 1, 1};
    const int64_t pairs = (int64_t)p.batch * p.kv_heads, part = pairs * KEYS * p.d * 8;              // bytes of a run of a tile of each pair
    const int64_t all_steps = ((int64_t)p.N + TILE - 1) / TILE * p.group, steps = std::min<int64_t>(all_steps, ((int64_t)p.window + KEYS + TILE - 1) / TILE * p.group);
    const int64_t step = p.d == 128 ? 1500 : 900;                     // nanoseconds, two workgroups on a compute unit
    const bool cut = steps < all_steps;                               // else every tile's rows are those that follow
    int64_t early = 0, early_length = 0;                              // runs of sinks
    if (cut && p.sinks > 0 && best.tiles > 0) {
        best.first = (int)std::min<int64_t>(best.tiles, ((int64_t)std::min(p.sinks, p.M) + KEYS - 1) / KEYS);
        best.first_runs = (int)std::max<int64_t>(1, std::min<int64_t>({(all_steps + 15) / 16, 1024 / (pairs * best.first), MOST_PART / 2 / (part * best.first), MOST_RUNS}));
        early = pairs * best.first * best.first_runs;
        early_length = all_steps / best.first_runs + 3;
    }
    const int64_t others = pairs * (best.tiles - best.first), mean = cut ? steps : (steps + 1) / 2;
    int64_t best_cost = INT64_MAX;
    // (tiles of sinks have at least as many runs as the others: grad_join_kernel goes through all tiles or those alone)
    auto runs_of_first = [&](int64_t r) { return best.first == 0 ? 0 : std::max<int64_t>(best.first_runs, r); };
    auto fits = [&](int64_t r) { return part * (best.tiles - best.first) * r <= MOST_PART / 2 && part * best.first * runs_of_first(r) <= MOST_PART / 2; };
    for (int64_t r = 1; r == 1 || (r <= 32 && others > 0 && steps / r >= 8 && fits(r)); ++r) {
        const int64_t n = others * r, length = (mean + r - 1) / r + 3, longest = (steps + r - 1) / r + 3, work = (early * early_length + n * length) / 512;
        int64_t time;                                                 // in steps
        if (!cut) time = std::max(work, longest);                     // (rows of very different numbers even out)
        else if (early + n <= 512) time = std::max(early_length, length);
        else if (n <= 512) time = early_length + length;
        else time = std::max(early_length + 2 * length, work + length / 2);
        int64_t cost = time * step;
        if (r > 1) cost += 6000 + part * ((best.tiles - best.first) * r + best.first * (runs_of_first(r) - runs_of_first(1))) / 2000;
        if (cost < best_cost) {
            best_cost = cost;
            best.runs = (int)r;
        }
    }
    best.first_runs = best.first == 0 ? best.runs : (int)runs_of_first(best.runs);
    return best;
}

// How the keys of a tile of rows are cut.  A tile of 64 keys x 128 rows x d 128 takes two workgroups on a compute unit 2800 ns, a lone one 1600
// (d 64: 1800, 1200); each run brings partial sums, and all together the join (8 heads x 100 x 8192 x 128: one run 204 us, 26
// 17 and the join 4; one head x 8192 x 8192 x 128 199, and 55 and 9).
int row_runs(const WindowProblem &p)
{
    const int64_t groups = (int64_t)p.batch * p.kv_heads * (((int64_t)p.N * p.group + 127) / 128), rows = (int64_t)p.batch * p.heads * p.N;
    const int64_t tiles = most_tiles(p.M, p.window, p.sinks, 128, p.group, p.N, KEY_TILE);
    auto cost = [&](int64_t r) {
        const int64_t length = (tiles + r - 1) / r, two = (p.d == 128 ? 2800 : 1800) * length + 4000, one = (p.d == 128 ? 1600 : 1200) * length + 4000;
        return rounds_time((unsigned)(groups * r), two, one) + (r > 1 ? 4000 + rows * p.d * 8 * r / 3000 : 0);
    };
    int64_t best = 1;
    if (groups < (1 << 20))
        for (int64_t r = 2; r <= 32 && r * LEAST_TILES <= tiles && rows * p.d * 4 * r <= MOST_PART / 2; ++r)
            if (cost(r) < cost(best)) best = r;
    return (int)best;
}

int64_t stats_bytes(const WindowProblem &p) { return ((int64_t)p.batch * p.heads * padded_rows(p.N) * 8 + 255) / 256 * 256; }

// Where a call keeps what in its workspace, in bytes.
struct Layout {
    int64_t marks, used, part, q_part, end;
    Layout(const WindowProblem &p, const Runs &runs, int q_runs)
    {
        const int64_t pairs = p.M > 0 ? (int64_t)p.batch * p.kv_heads : 0;
        marks = stats_bytes(p);
        used = marks + pairs * runs.per_pair() * 16;
        part = used + pairs * runs.kept_per_pair() * 16;
        q_part = part + pairs * runs.kept_per_pair() * 2 * KEYS * p.d * 4;
        end = q_part + (q_runs > 1 ? (int64_t)p.batch * p.heads * p.N * p.d * 4 * q_runs : 0);
    }
};

template <int D> hipError_t launch_grad(const WindowProblem &p, void *workspace, hipStream_t s)
{
    const Runs runs = choose_runs(p);
    const int q_runs = row_runs(p);
    const Layout at(p, runs, q_runs);
    char *mem = (char *)workspace;
    float *lse2 = (float *)mem, *Ds = lse2 + (int64_t)p.batch * p.heads * padded_rows(p.N), *part = (float *)(mem + at.part), *q_part = (float *)(mem + at.q_part);
    int *marks = (int *)(mem + at.marks), *used = (int *)(mem + at.used);
    const float scale = (float)(1.4426950408889634 / __builtin_sqrt((double)D));
    const int tiles = (int)(((int64_t)p.N * p.group + 127) / 128);
    const int64_t pairs = (int64_t)p.batch * p.kv_heads, blocks = runs.per_pair() * pairs;
    if (tiles * pairs * q_runs >= ((int64_t)1 << 31) || blocks >= ((int64_t)1 << 31)) return hipErrorInvalidValue;
    hipError_t e = hipSuccess;
    if (p.N > 0) e = launch_kernel(grad_q_kernel<D>, dim3((unsigned)(tiles * pairs * q_runs)), dim3(256), s, p, tiles, q_runs, scale, lse2, Ds, q_part);
    if (e != hipSuccess || p.M == 0) return e;
    auto keys_of = [&](auto kernel, int64_t grid) {
        return launch_kernel(kernel, dim3((unsigned)grid), dim3(256), s, p, runs, scale, (const float *)lse2, (const float *)Ds, part, used, marks);
    };
    e = keys_of(grad_kv_kernel<D>, blocks);
    if (e == hipSuccess) e = keys_of(grad_kv_careful_kernel<D>, std::min<int64_t>(blocks, 256));
    const int64_t of_keys = pairs * runs.kept_tiles() * (KEYS * D / 1024), of_rows = q_runs > 1 ? ((int64_t)p.batch * p.heads * p.N * D + 1023) / 1024 : 0;
    if (e != hipSuccess || of_keys + of_rows == 0) return e;
    return launch_kernel(grad_join_kernel<D>, dim3((unsigned)(of_keys + of_rows)), dim3(256), s, p, runs, q_runs, (const float *)part, (const int *)used, (const float *)q_part);
}

}  // namespace

int64_t window_grad_workspace_bytes(const WindowProblem &p) { return Layout(p, choose_runs(p), row_runs(p)).end; }

hipError_t launch_window_grad(const WindowProblem &p, void *workspace, int64_t, hipStream_t s)
{
    return p.d == 128 ? launch_grad<128>(p, workspace, s) : launch_grad<64>(p, workspace, s);
}

}  // namespace cyc
