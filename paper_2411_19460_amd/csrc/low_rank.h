// The low-rank term of a product on the matrix cores: what the rows' adapters add to a tile of x w^T, straight from memory to operands.
#pragma once
#include "mfma_common.h"

namespace ssdk {

// Where (column, r) of the other factor lies packed: 16 bytes a column and eight ranks, the sixteen columns of a tile side by side.
static __device__ __forceinline__ int64_t packed_up(int64_t col, int r, int rank) { return col / 16 * 16 * rank + (r >> 3) * 128 + col % 16 * 8 + (r & 7); }
// Where part 0 or 1 (split_low) of (row, r) of a narrow product lies for the wide one: the same, a tile's second parts behind its first ones.
static __device__ __forceinline__ int64_t packed_low(int64_t row, int r, int rank, int part) {
    return (row / 16 * 2 + part) * 16 * rank + (r >> 3) * 128 + row % 16 * 8 + (r & 7);
}

// The next bf16 part of v, which keeps the rest.  Parts are cut off, not rounded, so that they have one sign, and where nothing is left the
// rest is 2^-30 of v instead of zero: times an infinity of the other operand all parts are the infinity that v would be (a zero, or a part
// of the other sign, would make a NaN of it).  An infinity's rest is itself, a NaN's a NaN.
static __device__ __forceinline__ __bf16 cut(float& v) {
    const float top = __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, v) & 0xffff0000u);
    v = top == v ? v * 0x1p-30f : v - top;
    return (__bf16)top;
}
static __device__ __forceinline__ void split_low(float v, __bf16& hi, __bf16& lo) {  // 16 bits of v or more
    hi = cut(v);
    lo = (__bf16)v;
}

// acc[i][j] += low[t, :] up_a^T for the rows t = m0 + 16 i + lane % 16 and the columns n0 + 16 j + 4 (lane / 16) + 0..3, a the adapter
// of row t: the accumulator layout of 16 x 16 x 32 MFMAs that are issued with the columns' operand first.  The rows lie in one tile of
// the plan (LOW_TILE).  Nothing goes through LDS: a lane's eight values are one piece of memory in both operands.  `low` comes in the
// order in which lanes ask for it (packed_low), in two bf16 parts, an MFMA each: in one alone it would bring a rounding of its own, as large
// as the result's where the term is all that the result has; in two it is off by 2^-16 of its products (8192 rows 2560 -> 10576, rank 64:
// 391 us a call with one part, 397 with two).  A row keeps the products with its own
// adapter alone, by a selection and not by zeros in `low`: an infinity in one adapter stays with the rows that have it.  Of the
// tile's adapters this call takes numbers u0, u0 + ustep, ..., UB of them at a time: with more than one all of their operands are asked
// for before the first is used, and none is left out for having no row here.
template <int MT, int NT, int UB = 1>
static __device__ __forceinline__ void add_low_rank(mf::f32x4 (&acc)[MT][NT], const LowRankTerm& lr, int m0, int M, int n0, int N, int lane, int u0, int ustep) {
    using namespace mf;
    const int tile = m0 / LOW_TILE, nu = lr.tile_n[tile], q = lane >> 4, l16 = lane & 15;
    const int* list = lr.tile_a + (int64_t)tile * LOW_TILE;
    const int listed = list[lane];  // the first 64, a lane each
    auto number = [&](int u) { return u < 64 ? __builtin_amdgcn_readlane(listed, u) : list[u]; };
    int of_row[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int m = m0 + 16 * i + l16;
        of_row[i] = m < M ? lr.ids[m] : -1;
    }
    if (u0 >= nu) return;
    // What does not exist is fetched from beyond a descriptor's end: zeros.
    constexpr uint32_t OUT = 0x80000000u;
    const int tiles = M <= m0 ? 0 : (M - m0 + 15) / 16 < MT ? (M - m0 + 15) / 16 : MT;
    const rsrc_t rl = make_rows(lr.low + (int64_t)m0 * 2 * lr.rank, tiles, lr.rank * 64);
    auto k_of = [&](int k0) { return k0 + 8 * q < lr.rank ? (uint32_t)(k0 / 8 + q) : OUT; };  // this lane's eight ranks from k0 on
    struct Low {
        bf16x8 part[2][MT];
    };
    auto low_of = [&](int k0, Low& a) {  // (rows without an adapter have zeros; nothing here waits for the rows' adapters)
        const uint32_t kb = k_of(k0);
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int i = 0; i < MT; ++i) a.part[p][i] = rows_load(rl, kb == OUT ? OUT : (2 * i + p) * lr.rank * 32 + kb * 256 + l16 * 16);
    };
    // the operands of adapter number u of the tile (none beyond its last)
    auto fetch = [&](int k0, int u, int& ad, bf16x8 (&b)[NT]) {
        const uint32_t kb = k_of(k0);
        ad = u >= nu ? -2 : number(u);
        const int own = ad < 0 || N < n0 ? 0 : N - n0 < 16 * NT ? N - n0 : 16 * NT;  // columns that exist
        const rsrc_t ru = make_rows(lr.up + ((int64_t)(ad < 0 ? 0 : ad) * lr.width + n0) * lr.rank, lr.packed ? (own + 15) & ~15 : own, lr.rank * 2);
        const uint32_t at = lr.packed ? kb * 256 + l16 * 16 : (l16 * lr.rank + kb * 8) * 2;
#pragma unroll
        for (int j = 0; j < NT; ++j) b[j] = rows_load(ru, kb == OUT ? OUT : at + j * lr.rank * 32);
    };
    auto add = [&](int ad, const Low& a, const bf16x8 (&b)[NT]) {
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            f32x4 t[MT];
#pragma unroll
            for (int i = 0; i < MT; ++i) t[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[j], a.part[0][i], acc[i][j], 0, 0, 0);
#pragma unroll
            for (int i = 0; i < MT; ++i) t[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[j], a.part[1][i], t[i], 0, 0, 0);
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][j][e] = of_row[i] == ad ? t[i][e] : acc[i][j][e];
        }
    };
    auto here = [&](int ad) {  // a row of this wave has it
        bool any = false;
#pragma unroll
        for (int i = 0; i < MT; ++i) any = any || of_row[i] == ad;
        return __any(any);
    };
    Low a;
    if constexpr (UB == 1 && MT * NT <= 8) {
        // Registers to spare: while an adapter's operands are multiplied those of the next (of the next ranks behind the last) are under way.
        Low r;
        low_of(0, r);
        int k0 = 0, u = u0, k1, u1, ad, ad1;
        auto after = [&](int k, int v, int& kn, int& un) { kn = v + ustep < nu ? k : k + 32, un = v + ustep < nu ? v + ustep : u0; };
        auto work = [&](int k, int v, int which, const bf16x8 (&b)[NT]) {
            if (v == u0) {
                a = r;
                if (k + 32 < lr.rank) low_of(k + 32, r);
            }
            if (here(which)) add(which, a, b);
        };
        bf16x8 b[NT], c[NT];
        fetch(k0, u, ad, b);
        for (;;) {
            after(k0, u, k1, u1);
            if (k1 < lr.rank) fetch(k1, u1, ad1, c);
            work(k0, u, ad, b);
            if (k1 >= lr.rank) break;
            after(k1, u1, k0, u);
            if (k0 < lr.rank) fetch(k0, u, ad, b);
            work(k1, u1, ad1, c);
            if (k0 >= lr.rank) break;
        }
        return;
    }
    for (int k0 = 0; k0 < lr.rank; k0 += 32) {
        low_of(k0, a);
        for (int u = u0; u < nu; u += UB * ustep) {
            int ad[UB];
            if (UB == 1) {
                ad[0] = number(u);
                if (!here(ad[0])) continue;
            }
            bf16x8 b[UB][NT];
#pragma unroll
            for (int v = 0; v < UB; ++v) fetch(k0, u + v * ustep, ad[v], b[v]);
#pragma unroll
            for (int v = 0; v < UB; ++v) add(ad[v], a, b[v]);
        }
    }
}

}  // namespace ssdk
