// cyc_tile.h -- device helpers shared by the kernels of attention with a window and its gradient: copies into LDS, reads from it that are waited for one by one,
// reductions over the four lanes of a query, and the layout of a tile of rows.
#pragma once
#include "cyc_internal.h"

namespace cyc {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

#define CYC_LDS __attribute__((address_space(3)))

// x, taken anew: what derives from it in a rare branch is not computed ahead of the loop and kept in registers for it
__device__ __forceinline__ int fresh(int x)
{
    asm volatile("" : "+v"(x));
    return x;
}

// 64 lanes x 16 bytes from global memory, an address per lane, into LDS at lds_addr + lane * 16
__device__ __forceinline__ void copy16_from(const char *src, uint32_t lds_addr)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" : : "s"(__builtin_amdgcn_readfirstlane(lds_addr)), "v"(src) : "memory", "m0");
}

// the same from a wave-uniform base and an offset per lane
__device__ __forceinline__ void copy16_from(const char *base, uint32_t lane_off, uint32_t lds_addr)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(__builtin_amdgcn_readfirstlane(lds_addr)), "v"(lane_off), "s"(base) : "memory", "m0");
}

__device__ __forceinline__ i32x4 mfma_frag(i32x2 lo, i32x2 hi) { return (i32x4){lo[0], lo[1], hi[0], hi[1]}; }
__device__ __forceinline__ f32x4 mfma16(i32x4 a, i32x4 b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

template <int... I, class F> __device__ __forceinline__ void static_for_each(std::integer_sequence<int, I...>, F &&f)
{
    (f(std::integral_constant<int, I>{}), ...);
}
// f(integral_constant<int, 0>) .. f(integral_constant<int, N-1>): a loop whose index is a constant expression
template <int N, class F> __device__ __forceinline__ void static_for(F &&f) { static_for_each(std::make_integer_sequence<int, N>{}, f); }

// 16 bytes per lane from LDS address addr + OFF, with no wait: dst is valid only after lds_wait
template <int OFF> __device__ __forceinline__ void lds_read128(i32x4 &dst, uint32_t addr)
{
    static_assert(OFF >= 0 && OFF < 65536, "the offset field of an LDS instruction has 16 bits");
    asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(dst) : "v"(addr), "n"(OFF));
}
// wait until at most PENDING LDS operations issued after the read of x are outstanding; x is valid from here on
template <int PENDING> __device__ __forceinline__ void lds_wait(i32x4 &x) { asm volatile("s_waitcnt lgkmcnt(%1)" : "+v"(x) : "n"(PENDING)); }
// the transposing read of four 16-bit elements per lane, likewise without a wait
template <int OFF> __device__ __forceinline__ void lds_read_tr64(i32x2 &dst, uint32_t addr)
{
    static_assert(OFF >= 0 && OFF < 65536, "the offset field of an LDS instruction has 16 bits");
    asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(dst) : "v"(addr), "n"(OFF));
}
template <int PENDING> __device__ __forceinline__ void lds_wait2(i32x2 &x, i32x2 &y) { asm volatile("s_waitcnt lgkmcnt(%2)" : "+v"(x), "+v"(y) : "n"(PENDING)); }

// this wave's copies have landed and its LDS reads have returned (the stages it read are about to be requested into
// again by other waves); then meet the other waves
__device__ __forceinline__ void landed_barrier() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// f over the values of lanes l, l^16, l^32, l^48.  The swaps exchange halves (rows 2,3 of the first operand with rows 0,1 of the
// second) resp. odd rows of the first with even rows of the second; fed the same value twice, the two results together
// hold the value of both partners.  (Elements are copied to scalars before the bit cast: a bit cast applied to a
// vector element directly reads element 0 whatever the index.)
template <class F> __device__ __forceinline__ float over_query(float x, F &&f)
{
    const unsigned u = __builtin_bit_cast(unsigned, x);
    const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const unsigned a0 = a[0], a1 = a[1];
    const unsigned v = __builtin_bit_cast(unsigned, f(__builtin_bit_cast(float, a0), __builtin_bit_cast(float, a1)));
    const auto b = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    const unsigned b0 = b[0], b1 = b[1];
    return f(__builtin_bit_cast(float, b0), __builtin_bit_cast(float, b1));
}
__device__ __forceinline__ float query_max(float x) { return over_query(x, [](float a, float b) { return __builtin_fmaxf(a, b); }); }
__device__ __forceinline__ float query_sum(float x) { return over_query(x, [](float a, float b) { return a + b; }); }

// a packed pair of bfloat16 with 0 in place of infinities and NaNs
__device__ __forceinline__ int finite_pair(int pair)
{
    const unsigned u = (unsigned)pair, low = (u & 0x7f80u) == 0x7f80u ? 0 : u & 0xffffu, high = (u & 0x7f800000u) == 0x7f800000u ? 0 : u & 0xffff0000u;
    return (int)(low | high);
}

// Which of `pairs` (batch element, key head) and which of its `units` a workgroup takes.  Workgroups go to the eight XCDs round robin by their
// index and each XCD has its own L2: a pair stays on one XCD, whose 64 places (32 compute units x 2) go through the units of one
// pair after the other, or of as many side by side as fill them, unit after unit: with the longest units first, those of the last pair
// would otherwise begin when there is nothing left to run beside them (64 pairs x 32 units of a causal mask, gradient: 955 us, and
// 892 two by two).  (Fewer than eight pairs share the XCDs, with neighbouring units on different ones, so that the long ones are spread over all.)
struct Place {
    int pair, unit;
    __device__ __forceinline__ Place(int at, int pairs, int units)
    {
        // pairs in groups of `together`, then as many eights of them as are left, then the rest
        const int together = 8 * ((63 + units) / units), full = pairs / together * together, eights = pairs / 8 * 8;
        const int start = at / units;                                // (of the pairs before: a group's workgroups follow one another)
        const int base = start < full ? start / together * together : start < eights ? full : eights;
        const int side = start < full ? together : start < eights ? eights - full : pairs - eights, local = at - base * units;
        unit = local / side;
        pair = base + local - unit * side;
    }
};

// The keys that the rows r_first .. r_last of a call see, [0, sink_end) and [lo, hi], as a list of tiles of KT keys: first the tiles that all
// rows see whole, then the others.  Row r stands at position r / group + M - N.
template <int KT> struct KeyList {
    int lo, hi, sink_end;
    int whole_sinks, first_whole, whole;         // whole tiles: 0 .. whole_sinks - 1, then first_whole on; `whole` of them
    int sink_tiles, window_tile, count;          // tiles 0 .. sink_tiles - 1 and from window_tile on, whole or not
    __device__ __forceinline__ KeyList(int r_first, int r_last, int group, int N, int M, int window, int sinks)
    {
        const int p_first = r_first / group + M - N;
        hi = r_last / group + M - N;
        lo = p_first >= window ? p_first - window + 1 : 0;
        sink_end = sinks < lo ? sinks : lo;
        sink_tiles = (sink_end + KT - 1) / KT;
        window_tile = lo / KT > sink_tiles ? lo / KT : sink_tiles;
        const int window_tiles = hi / KT - window_tile + 1 > 0 ? hi / KT - window_tile + 1 : 0;
        count = hi < 0 ? 0 : sink_tiles + window_tiles;
        // whole: up to the first row's position, and from the last row's window on or among the sinks
        const int past = p_first < 0 ? 0 : (p_first + 1) / KT, last_lo = hi >= window ? hi - window + 1 : 0;
        whole_sinks = sink_end / KT;
        first_whole = (last_lo + KT - 1) / KT;
        if (first_whole < window_tile) first_whole = window_tile;
        whole = count == 0 ? 0 : whole_sinks + (past > first_whole ? past - first_whole : 0);
    }
    __device__ __forceinline__ int tile_key(int u) const
    {
        if (u < whole) return (u < whole_sinks ? u : first_whole - whole_sinks + u) * KT;
        u -= whole - whole_sinks;                // 0 .. sink_tiles - 1 less the whole ones, then the window's tiles less the whole ones
        if (u < sink_tiles) return u * KT;
        u += window_tile - sink_tiles;
        return (u < first_whole ? u : u + whole - whole_sinks) * KT;
    }
    // a key of the list in place of one that no row sees
    __device__ __forceinline__ int seen_key(int key) const
    {
        key = key < hi ? key : hi;
        return key >= sink_end && key < lo ? lo : key;
    }
    __device__ __forceinline__ bool inside(int k0) const { return k0 + KT - 1 <= hi && (k0 >= lo || k0 + KT <= sink_end); }
};

// Copies of tiles of KT rows of ROW bytes into LDS by NWAVE waves: copy x of wave w moves the rows x * STEP + w * RPC .. of the tile, a lane 16
// bytes of one of them.  swizzle(r) gives the slots of row r's chunks.
template <int KT, int ROW, int NWAVE> struct TileCopies {
    static constexpr int CPR = ROW / 16, RPC = 64 / CPR, STEP = NWAVE * RPC, COUNT = KT / STEP;
    // A whole tile of dense rows: a base for all lanes and an offset each, which costs no vector instructions.  Strides below 2^25.
    template <class Swizzle>
    static __device__ __forceinline__ void whole(const char *rows, int64_t stride, uint32_t lds_addr, int w, int l, Swizzle &&swizzle)
    {
        const int row0 = w * RPC + l / CPR;
        const uint32_t row_off = row0 * (uint32_t)stride, chunk = (l % CPR) ^ swizzle(row0);
#pragma unroll
        for (int x = 0; x < COUNT; ++x) copy16_from(rows + x * STEP * stride, row_off + ((chunk ^ swizzle(x * STEP)) << 4), lds_addr + (w + x * NWAVE) * 1024);
    }
    // row(r): the address of row r's bytes
    template <class Row, class Swizzle>
    static __device__ __forceinline__ void any(uint32_t lds_addr, int w, int l, Row &&row, Swizzle &&swizzle)
    {
        l = fresh(l);
#pragma unroll
        for (int x = 0; x < COUNT; ++x) {
            const int r = x * STEP + w * RPC + l / CPR;
            copy16_from(row(r) + (((l % CPR) ^ swizzle(r)) << 4), lds_addr + (w + x * NWAVE) * 1024);
        }
    }
};
constexpr int64_t MOST_STRIDE = (int64_t)1 << 25;

// Is there an infinity or NaN among the values that `read(i)`, i < N, yields?  0 times them is NaN, a sum that has met one stays NaN:
// N products with zeros on matrix cores that are waiting anyway.
template <int N, class Read> __device__ __forceinline__ bool any_infinite(Read &&read)
{
    f32x4 zero = {0, 0, 0, 0};
    static_for<N>([&](auto ic) __attribute__((always_inline)) { zero = mfma16(read(ic), (i32x4){0, 0, 0, 0}, zero); });
    return __builtin_amdgcn_ballot_w64(!(zero[0] == 0 && zero[1] == 0 && zero[2] == 0 && zero[3] == 0)) != 0;
}

}  // namespace cyc
