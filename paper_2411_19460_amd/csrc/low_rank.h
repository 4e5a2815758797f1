// The low-rank term of a product on the matrix cores: what the rows' adapters add to a tile of x w^T, straight from memory to operands.
#pragma once
#include "mfma_common.h"

namespace ssdk {

// acc[i][j] += low[t, :] up_a^T for the rows t = m0 + 16 i + lane % 16 and the columns n0 + 16 j + 4 (lane / 16) + 0..3, a the adapter
// of row t: the accumulator layout of 16 x 16 x 32 MFMAs that are issued with the columns' operand first.  The rows lie in one tile of
// the plan (LOW_TILE).  Both operands have the rank contiguous, so a lane's eight values are one piece of memory and nothing goes
// through LDS.  `low` is rounded to bf16: the result is, and the term is the smaller part of it.  A row keeps the products with its own
// adapter alone, by a selection and not by zeros in `low`: an infinity in one adapter stays with the rows that have it.  Of the
// tile's adapters this call takes numbers u0, u0 + ustep, ..., UB of them at a time: with more than one all of their operands are asked
// for before the first is used, and none is left out for having no row here.
template <int MT, int NT, int UB = 1>
static __device__ __forceinline__ void add_low_rank(mf::f32x4 (&acc)[MT][NT], const LowRankTerm& lr, int m0, int M, int n0, int N, int lane, int u0, int ustep) {
    using namespace mf;
    const int tile = m0 / LOW_TILE, nu = lr.tile_n[2 * tile], a0 = lr.tile_n[2 * tile + 1], q = lane >> 4, l16 = lane & 15;
    const int* list = lr.tile_a + (int64_t)tile * LOW_TILE;
    int of_row[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int m = m0 + 16 * i + l16;
        of_row[i] = m < M ? lr.ids[m] : -1;
    }
    if (u0 >= nu) return;
    // What does not exist is fetched from beyond a descriptor's end: zeros.
    constexpr uint32_t OUT = 0x80000000u;
    const int rows = M - m0 < 16 * MT ? M - m0 : 16 * MT;
    const rsrc_t rl = make_rows(lr.low + (int64_t)m0 * lr.rank, rows < 0 ? 0 : rows, lr.rank * 4);
    for (int k0 = 0; k0 < lr.rank; k0 += 32) {
        const int k = k0 + 8 * q;
        const uint32_t kb = k < lr.rank ? (uint32_t)k : OUT;
        bf16x8 a[MT];
#pragma unroll
        for (int i = 0; i < MT; ++i) {  // (rows without an adapter have zeros; nothing here waits for the rows' adapters)
            const uint32_t at = ((16 * i + l16) * lr.rank + kb) * 4;
            const f32x4 p0 = __builtin_bit_cast(f32x4, rows_load(rl, kb == OUT ? OUT : at)), p1 = __builtin_bit_cast(f32x4, rows_load(rl, kb == OUT ? OUT : at + 16));
#pragma unroll
            for (int e = 0; e < 4; ++e) a[i][e] = (__bf16)p0[e], a[i][4 + e] = (__bf16)p1[e];
        }
        for (int u = u0; u < nu; u += UB * ustep) {
            int ad[UB];
#pragma unroll
            for (int v = 0; v < UB; ++v) ad[v] = u + v * ustep < nu ? u + v * ustep ? list[u + v * ustep] : a0 : -2;
            if (UB == 1) {
                bool any = false;
#pragma unroll
                for (int i = 0; i < MT; ++i) any = any || of_row[i] == ad[0];
                if (!__any(any)) continue;
            }
            bf16x8 b[UB][NT];
#pragma unroll
            for (int v = 0; v < UB; ++v) {
                const int own = UB == 1 || ad[v] >= 0 ? N - n0 < 16 * NT ? N - n0 : 16 * NT : 0;  // columns that exist
                const rsrc_t ru = make_rows(lr.up + ((int64_t)(ad[v] < 0 ? 0 : ad[v]) * lr.width + n0) * lr.rank, own < 0 ? 0 : own, lr.rank * 2);
#pragma unroll
                for (int j = 0; j < NT; ++j) b[v][j] = rows_load(ru, kb == OUT ? OUT : ((16 * j + l16) * lr.rank + kb) * 2);
            }
#pragma unroll
            for (int v = 0; v < UB; ++v)
#pragma unroll
                for (int j = 0; j < NT; ++j)
#pragma unroll
                    for (int i = 0; i < MT; ++i) {
                        const f32x4 t = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[v][j], a[i], (f32x4)(0.f), 0, 0, 0);
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[i][j][e] += of_row[i] == ad[v] ? t[e] : 0.f;
                    }
        }
    }
}

}  // namespace ssdk
