// Low-rank adapters beside a shared projection: every row t of a call belongs to a request that has an adapter a(t), or none,
//     h[t, :] = s_a x[t, :] A_a^T            out[t, :] = x[t, :] W^T + h[t, :] B_a^T
//     g[t, :] = s_a dout[t, :] B_a           dx[t, :]  = dout[t, :] W + g[t, :] A_a
//     dA_a = sum_{t of a} g[t, :]^T x[t, :]  dB_a = sum_{t of a} dout[t, :]^T h[t, :]
// with the projection W frozen.  The products with W and the low-rank terms that join them are tiles of linear.hip; here are the plan
// of a batch (which rows share an adapter), the narrow products h and g, and the adapters' gradients.
// h and g are fp32, and so is everything that is summed: the gradients leave in fp32, and would lose 16 of its bits with either in bf16.  For the
// wide products, whose results are bf16, they come in two bf16 parts.
#include <string.h>

#include <type_traits>

#include "low_rank.h"
#include "low_steps.h"
#include "mfma_common.h"

namespace ssdk {
namespace {

using namespace mf;

// ---- the plan of a batch ----
// Rows in the order of their adapters (stable; rows without one last), cut into units of rows that share one: short units for the
// narrow products, long ones for the gradients, where a unit is what is summed before anything leaves for memory.  And for every tile
// of the wide product the adapters that its rows have.  Words of 32 bits; host and device derive the places from (rows, adapters).
constexpr int MAX_RANK = 256;

// A unit: rows perm[first .. first + count - 1] of an adapter (a == n: rows without one).  row0 >= 0: they are row0, row0 + 1, ...  One load
// tells a workgroup all that it needs; units that a batch does not have are there with no rows.
struct Unit {
    int a, first, count, row0;
};
struct Plan {
    int rows, n, long_unit, max_short, max_long, tiles;
    __host__ __device__ int max_several() const { return rows / long_unit < n ? rows / long_unit : n; }  // adapters of several long units, at most
    int64_t ids, perm, start, first_long, first_slot, several, short_u, long_u, tile_n, tile_a, counts, words;
};

int long_unit_of(int64_t rows) {  // about sixteen units where all rows share an adapter, one where rows are few
    const int64_t u = (rows / 16 + 63) / 64 * 64;
    return (int)(rows <= 1024 ? 1024 : u < 512 ? 512 : u);
}

Plan plan_of(int64_t rows, int32_t n) {
    Plan p;
    p.rows = (int)rows;
    p.n = n;
    p.long_unit = long_unit_of(rows);
    auto least = [](int64_t a, int64_t b) { return (int)(a < b ? a : b); };
    p.max_short = least(rows, rows / SHORT_UNIT + n + 1);
    p.max_long = (int)(rows / p.long_unit + n);
    p.tiles = (int)((rows + LOW_TILE - 1) / LOW_TILE);
    int64_t at = 0;
    auto take = [&](int64_t words) {
        const int64_t here = at;
        at += (words + 3) / 4 * 4;
        return here;
    };
    p.ids = take(rows);
    p.perm = take(rows);
    p.start = take(n + 2);        // of adapter a in perm; [n]: of the rows without one
    p.first_long = take(n + 1);
    p.first_slot = take(n + 1);   // partial sums of the gradients: adapters of several long units
    p.several = take(p.max_several());  // those adapters, -1 behind the last
    p.short_u = take(4 * (int64_t)p.max_short);
    p.long_u = take(4 * (int64_t)p.max_long);
    p.tile_n = take(p.tiles);
    p.tile_a = take((int64_t)p.tiles * LOW_TILE);
    p.counts = take(n + 1);
    p.words = at;
    return p;
}
// Adapters of several long units have at most two units for each long_unit of their rows.
int64_t most_slots(const Plan& p) {
    return p.rows <= p.long_unit ? 0 : 2 * ((int64_t)p.rows / p.long_unit);
}

constexpr int PTHR = 256;

__device__ __forceinline__ int block_sum(int v, int* lds) {  // every thread gets the sum over the workgroup
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    return lds[0] + lds[1] + lds[2] + lds[3];
}

__device__ __forceinline__ int clean(int a, int n) { return a >= 0 && a < n ? a : -1; }

// Workgroups 0 .. tiles - 1: the rows' adapters (anything outside 0 .. n - 1 is none) and the list of a tile; the others count the rows
// of an adapter each (the last: of none).
__global__ __launch_bounds__(PTHR) void k_plan_count(Plan p, const int* row_adapter, int* plan) {
    __shared__ int lds[LOW_TILE];
    const int tid = threadIdx.x;
    if ((int)blockIdx.x < p.tiles) {
        const int64_t row = (int64_t)blockIdx.x * LOW_TILE + tid;
        const int a = row < p.rows ? clean(row_adapter[row], p.n) : -2;
        if (row < p.rows) plan[p.ids + row] = a;
        lds[tid] = a;
        __syncthreads();
        bool first = a >= 0;
        for (int j = 0; j < tid; ++j) first = first && lds[j] != a;
        __syncthreads();
        lds[tid] = first ? a : 0x7fffffff;
        __syncthreads();
        int place = 0;
        for (int j = 0; j < LOW_TILE; ++j) place += lds[j] < a;
        if (first) plan[p.tile_a + (int64_t)blockIdx.x * LOW_TILE + place] = a;
        const int listed = block_sum(first, lds);
        if (tid == 0) plan[p.tile_n + blockIdx.x] = listed;
        return;
    }
    const int mine = blockIdx.x - p.tiles;
    int c = 0;
    for (int64_t r = tid; r < p.rows; r += PTHR) {
        const int a = clean(row_adapter[r], p.n);
        c += (a < 0 ? p.n : a) == mine;
    }
    c = block_sum(c, lds);
    if (tid == 0) plan[p.counts + mine] = c;
}

// Workgroup a: where the rows and units of adapter a begin, its rows in order, its units.
__global__ __launch_bounds__(PTHR) void k_plan_rows(Plan p, int* plan) {
    __shared__ int lds[4];
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, a = blockIdx.x;
    auto shorts = [](int c) { return (c + SHORT_UNIT - 1) / SHORT_UNIT; };
    auto longs = [&](int c) { return c ? (c + p.long_unit - 1) / p.long_unit : 1; };  // (an adapter without rows has one unit without any: its gradients are zeros)
    int start = 0, fs = 0, fl = 0, fp = 0, fm = 0;
    for (int b = tid; b < a; b += PTHR) {
        const int c = plan[p.counts + b], l = longs(c);
        start += c;
        fs += shorts(c);
        fl += l;
        fp += l > 1 ? l : 0;
        fm += l > 1;
    }
    start = block_sum(start, lds);
    fs = block_sum(fs, lds);
    fl = block_sum(fl, lds);
    fp = block_sum(fp, lds);
    fm = block_sum(fm, lds);
    const int mine = plan[p.counts + a], ns = shorts(mine), nl = a < p.n ? longs(mine) : 0;
    if (tid == 0) {
        plan[p.start + a] = start;
        plan[p.first_long + a] = fl;
        plan[p.first_slot + a] = fp;
        if (nl > 1) plan[p.several + fm] = a;
        if (a == p.n) plan[p.start + a + 1] = start + mine;
    }
    Unit *su = (Unit*)(plan + p.short_u), *lu = (Unit*)(plan + p.long_u);
    if (a == p.n) {
        for (int u = fs + ns + tid; u < p.max_short; u += PTHR) su[u] = Unit{0, 0, 0, 0};
        for (int u = fl + tid; u < p.max_long; u += PTHR) lu[u] = Unit{-1, 0, 0, 0};
        for (int u = fm + tid; u < p.max_several(); u += PTHR) plan[p.several + u] = -1;
    }
    int at = start;
    const int wanted = a < p.n ? a : -1;
    for (int64_t r0 = 0; r0 < p.rows && at < start + mine; r0 += PTHR) {
        const int64_t r = r0 + tid;
        const bool is = r < p.rows && plan[p.ids + r] == wanted;
        const uint64_t m = __ballot(is);
        __syncthreads();
        if (lane == 0) lds[wv] = __popcll(m);
        __syncthreads();
        int before = 0;
        for (int q = 0; q < 4; ++q) before += q < wv ? lds[q] : 0;
        if (is) plan[p.perm + at + before + __popcll(m & ((1ull << lane) - 1))] = (int)r;
        at += lds[0] + lds[1] + lds[2] + lds[3];
    }
    __syncthreads();  // the rows are in place (for this workgroup), the units can say whether theirs follow one another
    const int* rows = plan + p.perm + start;
    auto unit = [&](int u, int len) {
        Unit t = {a, start + u * len, mine - u * len < len ? mine - u * len : len, 0};
        if (t.count == 0) return t;
        t.row0 = rows[u * len];
        if (rows[u * len + t.count - 1] != t.row0 + t.count - 1) t.row0 = -1;  // (they ascend)
        return t;
    };
    for (int u = tid; u < ns; u += PTHR) su[fs + u] = unit(u, SHORT_UNIT);
    if (a < p.n)
        for (int u = tid; u < nl; u += PTHR) lu[fl + u] = unit(u, p.long_unit);
}

// ---- the narrow products ----
// low[t, r] = s_a sum_k X[t, k] U_a[r, k].  A workgroup takes a short unit and 16 RT of the ranks; its eight waves share out k in steps
// of 64 and their sums meet in LDS.  A step's rows come in as 128 contiguous bytes a row (eight rows an access) and are turned into
// operands through LDS of the wave's own, without a barrier; fetched straight as operands (sixteen rows an access) the same loads took
// 8192 x 2560 at rank 64 39 us instead of 24.  KROW: U is stored with k as the row index ([K, rank], the output side of an adapter) and is
// read transposed.  Bound by the rows' reading where rows are many (4096 x 10576, rank 16: 24 us, 3.6 TB/s; 16384 x 2560, rank 32: 30 us,
// 2.8 TB/s, the packing of the other factor included), by a unit's way through k where they are few (1 row of 2560 4.3 us, 64 of 5120 7.0, 600 of 4384 7.8).
struct LowParams {
    const __bf16* x;
    int64_t ldx;
    const __bf16* u;
    const float* scale;
    float* low;      // [rows, rank], or null
    __bf16* packed;  // the same in two parts for the wide product (packed_low), or null
    int K, rank;
    bool halves;     // a workgroup for each half of a unit
};
constexpr int STEP_PITCH = 144;  // bytes of a row of a step in LDS: 64 k, and sixteen rows fall into distinct banks
template <int RT>
constexpr int low_pitch() { return 32 * RT + 16; }
template <int RT, bool KROW>
constexpr int low_tiles() { return SHORT_UNIT * STEP_PITCH + (KROW ? 64 * low_pitch<RT>() : 16 * RT * STEP_PITCH); }  // of a wave
template <int RT, bool KROW>
constexpr int low_lds() {
    constexpr int tiles = LWAVES * low_tiles<RT, KROW>(), sums = LWAVES * SHORT_UNIT * 16 * RT * 4;
    return tiles > sums ? tiles : sums;
}

template <int RT, bool KROW, int MT>
__device__ __forceinline__ void low_unit(const LowParams& lp, const int* perm, const Unit un, int r0, char* lds) {
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), q = lane >> 4, l16 = lane & 15;
    const int nr = lp.rank - r0 < 16 * RT ? lp.rank - r0 : 16 * RT;  // ranks of this workgroup
    const int cnt = un.count, a = un.a, r8 = lane >> 3, c8 = (lane & 7) * 8;  // fetching lanes: eight rows of 64 k
    const __bf16* xr[2 * MT];
#pragma unroll
    for (int i = 0; i < 2 * MT; ++i) {
        const int r = i * 8 + r8 < cnt ? i * 8 + r8 : cnt - 1;
        int64_t row = un.row0 + r;
        if (un.row0 < 0) row = perm[un.first + r];
        xr[i] = lp.x + row * lp.ldx + c8;
    }
    const __bf16* ua = lp.u + (int64_t)a * lp.rank * lp.K;
    const __bf16* ur[2 * RT];  // KROW: not used
#pragma unroll
    for (int t = 0; t < 2 * RT; ++t) {
        const int r = r0 + 8 * t + r8;
        ur[t] = ua + (int64_t)(r < lp.rank ? r : lp.rank - 1) * lp.K + c8;
    }
    char *mx = lds + w * low_tiles<RT, KROW>(), *mu = mx + SHORT_UNIT * STEP_PITCH;
    const float s = lp.scale[a];
    const int vpr = nr / 8;  // KROW: 16-byte pieces of a row of U; (row, piece) of this lane's
    int kp[2 * RT], cp[2 * RT];
#pragma unroll
    for (int i = 0; i < 2 * RT; ++i) {
        kp[i] = low_piece_row(i * 64 + lane, vpr);
        cp[i] = (i * 64 + lane) - kp[i] * vpr;
    }
    f32x4 acc[RT][MT];
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int i = 0; i < MT; ++i) acc[t][i] = (f32x4)(0.f);
    // U steps at a time: all that they need is asked for before the first is used.  WHOLE: all of their k exist; else what lies beyond K
    // comes from k = 0 and is put to zero (in both operands: an infinity there would be a NaN).
    constexpr int U = low_group(RT, MT);
    const bf16x8 zero = (bf16x8)((__bf16)0.f);
    auto steps = [&](int k0, auto whole) {
        constexpr bool WHOLE = decltype(whole)::value;
        bf16x8 xv[U][2 * MT], uv[U][2 * RT];
#pragma unroll
        for (int s = 0; s < U; ++s) {
            const int ks = k0 + 64 * LWAVES * s, kc = WHOLE || ks + c8 < lp.K ? ks : -c8;
#pragma unroll
            for (int i = 0; i < 2 * MT; ++i) xv[s][i] = *(const bf16x8*)(xr[i] + kc);
#pragma unroll
            for (int i = 0; i < 2 * RT; ++i) {
                if (KROW) {
                    uv[s][i] = *(const bf16x8*)(ua + (int64_t)low_row_asked(ks, low_piece_asked(kp[i]), WHOLE, lp.K) * lp.rank + r0 + 8 * cp[i]);
                } else {
                    uv[s][i] = *(const bf16x8*)(ur[i] + kc);
                }
            }
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int s = 0; s < U; ++s) {
            const int ks = k0 + 64 * LWAVES * s;
            if (!WHOLE && ks >= lp.K) break;
            const bool in = WHOLE || ks + c8 < lp.K;
#pragma unroll
            for (int i = 0; i < 2 * MT; ++i) *(bf16x8*)(mx + (i * 8 + r8) * STEP_PITCH + 2 * c8) = in ? xv[s][i] : zero;
#pragma unroll
            for (int i = 0; i < 2 * RT; ++i) {
                if (!KROW) *(bf16x8*)(mu + (i * 8 + r8) * STEP_PITCH + 2 * c8) = in ? uv[s][i] : zero;
                else if (low_piece_there(kp[i])) *(bf16x8*)(mu + kp[i] * low_pitch<RT>() + 16 * cp[i]) = WHOLE || ks + kp[i] < lp.K ? uv[s][i] : zero;
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the wave's own rows: its LDS operations are done in order
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                bf16x8 xo[MT], uo[RT];
#pragma unroll
                for (int i = 0; i < MT; ++i) xo[i] = *(const bf16x8*)(mx + (i * 16 + l16) * STEP_PITCH + 64 * h + 16 * q);
#pragma unroll
                for (int t = 0; t < RT; ++t) {
                    if (KROW) {
                        const char* p = mu + (32 * h + 8 * q + (l16 >> 2)) * low_pitch<RT>() + 32 * t + 8 * (l16 & 3);
                        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p);
                        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 4 * low_pitch<RT>()));
                        uo[t] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
                    } else {
                        uo[t] = *(const bf16x8*)(mu + (t * 16 + l16) * STEP_PITCH + 64 * h + 16 * q);
                    }
                }
#pragma unroll
                for (int t = 0; t < RT; ++t)
#pragma unroll
                    for (int i = 0; i < MT; ++i) acc[t][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(uo[t], xo[i], acc[t][i], 0, 0, 0);
            }
            asm volatile("" ::: "memory");  // the next step's rows come in behind these reads
        }
    };
    int k0 = 64 * w;
    for (; low_whole(k0, U, lp.K); k0 += low_advance(U)) steps(k0, std::true_type{});
    if (k0 < lp.K) steps(k0, std::false_type{});
    __syncthreads();
    // lane -> row l16 of the unit's tile i, four consecutive ranks
    float* sums = (float*)lds;
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int i = 0; i < MT; ++i) *(f32x4*)(sums + (w * SHORT_UNIT + i * 16 + l16) * 16 * RT + 16 * t + 4 * q) = acc[t][i];
    __syncthreads();
    for (int v = tid; v < MT * 16 * 4 * RT; v += 64 * LWAVES) {
        const int r = v / (4 * RT), c = 4 * (v - r * 4 * RT);
        if (r >= cnt || c >= nr) continue;
        f32x4 o = (f32x4)(0.f);
#pragma unroll
        for (int u = 0; u < LWAVES; ++u) o += *(const f32x4*)(sums + (u * SHORT_UNIT + r) * 16 * RT + c);
        const int64_t at = un.row0 < 0 ? perm[un.first + r] : un.row0 + r;
        o *= s;
        if (lp.low) *(f32x4*)(lp.low + at * lp.rank + r0 + c) = o;
        if (lp.packed) {
            bf16x4 hi, lo;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                __bf16 h, l;
                split_low(o[e], h, l);
                hi[e] = h, lo[e] = l;
            }
            *(bf16x4*)(lp.packed + packed_low(at, r0 + c, lp.rank, 0)) = hi;
            *(bf16x4*)(lp.packed + packed_low(at, r0 + c, lp.rank, 1)) = lo;
        }
    }
}

// The adapters' other factor packed for the wide product (see LowRankTerm): pieces of 64 columns of an adapter, eight ranks at a time.  A
// workgroup takes one such piece of `group` adapters, of those that have rows.
struct PackJob {
    const __bf16* from;  // [adapters][width][rank], or (KROW) [adapters][rank][width]
    __bf16* to;
    int width, rank, blocks, group;  // blocks: of 64 columns, times groups of adapters; 0: no such job
};
template <bool KROW>
__device__ __forceinline__ void pack_piece(const PackJob& pj, const Plan& p, const int* plan, int id) {
    const int per = (pj.width + 63) / 64, g = id / per, c = (id - g * per) * 64 + (KROW ? threadIdx.x & 63 : threadIdx.x >> 3);
    const int end = p.n - g * pj.group < pj.group ? p.n : (g + 1) * pj.group;
    for (int a0 = g * pj.group; a0 < end; a0 += 64) {
        const int mine = a0 + (threadIdx.x & 63);
        uint64_t left = __ballot(mine < end && plan[p.start + mine] != plan[p.start + mine + 1]);
        for (; left; left &= left - 1) {
            const int a = a0 + __builtin_ctzll(left);
            if (c >= pj.width) continue;
            __bf16* to = pj.to + (int64_t)a * ((pj.width + 15) & ~15) * pj.rank;
            for (int r = 8 * (KROW ? threadIdx.x >> 6 : threadIdx.x & 7); r < pj.rank; r += 64) {
                bf16x8 v;
                if (KROW)
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = pj.from[((int64_t)a * pj.rank + r + e) * pj.width + c];
                else v = *(const bf16x8*)(pj.from + ((int64_t)a * pj.width + c) * pj.rank + r);
                *(bf16x8*)(to + packed_up(c, r, pj.rank)) = v;
            }
        }
    }
}

template <int RT, bool KROW>
__global__ __launch_bounds__(64 * LWAVES, 2) void k_low(LowParams lp, Plan p, const int* plan, PackJob pj) {
    extern __shared__ __attribute__((aligned(16))) char low_lds_mem[];
    const int u = blockIdx.x, units = gridDim.x - pj.blocks;
    if (u >= units) {  // behind the units, which take longer
        if (blockIdx.y == 0) pack_piece<KROW>(pj, p, plan, u - units);
        return;
    }
    Unit un = ((const Unit*)(plan + p.short_u))[lp.halves ? u >> 1 : u];
    if (lp.halves) {
        const int skip = u & 1 ? SHORT_UNIT / 2 : 0, left = un.count - skip;
        un.count = left < 0 ? 0 : left < SHORT_UNIT / 2 ? left : SHORT_UNIT / 2;
        un.first += skip;
        if (un.row0 >= 0) un.row0 += skip;
    }
    const int r0 = blockIdx.y * 16 * RT;
    const int* perm = plan + p.perm;
    if (un.count == 0) return;
    if (un.a == p.n) {  // rows without an adapter
        const int nr = lp.rank - r0 < 16 * RT ? lp.rank - r0 : 16 * RT;
        for (int v = threadIdx.x; v < un.count * nr; v += 64 * LWAVES) {
            const int64_t row = un.row0 < 0 ? perm[un.first + v / nr] : un.row0 + v / nr;
            if (lp.low) lp.low[row * lp.rank + r0 + v % nr] = 0.f;
            if (lp.packed) lp.packed[packed_low(row, r0 + v % nr, lp.rank, 0)] = lp.packed[packed_low(row, r0 + v % nr, lp.rank, 1)] = (__bf16)0.f;
        }
        return;
    }
    if (un.count <= 16) low_unit<RT, KROW, 1>(lp, perm, un, r0, low_lds_mem);
    else low_unit<RT, KROW, 2>(lp, perm, un, r0, low_lds_mem);
}

template <int RT, bool KROW>
hipError_t launch_low_rt(LowParams lp, const Plan& p, const int* plan, const PackJob& pj, hipStream_t st) {
    constexpr int LDS = low_lds<RT, KROW>();
    // where units leave half of the 256 compute units idle: 1905 rows of 5120, rank 8, 10.2 -> 7.6 us; 600 rows of 4384 9.8 -> 7.8; with 133
    // units (4096 rows of 2560), whose halves no longer run all at once, 8.4 -> 9.9
    lp.halves = p.max_short * ((lp.rank + 16 * RT - 1) / (16 * RT)) <= 128;
    static bool raised[64];
    if (LDS > 65536) {
        int dev = 0;
        if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return hipErrorInvalidDevice;
        if (!raised[dev]) {
            const hipError_t e = hipFuncSetAttribute((const void*)k_low<RT, KROW>, hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
            if (e != hipSuccess) return e;
            raised[dev] = true;
        }
    }
    hipLaunchKernelGGL((k_low<RT, KROW>), dim3((lp.halves ? 2 : 1) * p.max_short + pj.blocks, (lp.rank + 16 * RT - 1) / (16 * RT)), dim3(64 * LWAVES), LDS, st, lp, p, plan, pj);
    return hipGetLastError();
}

template <bool KROW>
hipError_t launch_low_products(const LowParams& lp, const Plan& p, const int* plan, const PackJob& pj, hipStream_t st) {
    // Few units: a workgroup for every sixteen ranks, x fetched again for the others (64 rows 5120 -> 2560 rank 32: 9.7 -> 6.7 us with
    // sixteen instead of all thirty-two).  Where ranks are what lies side by side (KROW) thirty-two, half a cache line: 73 rows
    // 10576 -> rank 128 34 us with sixteen.
    if (lp.rank <= 16 || (!KROW && p.max_short * ((lp.rank + 15) / 16) <= 256)) return launch_low_rt<1, KROW>(lp, p, plan, pj, st);
    if (KROW && p.max_short * ((lp.rank + 31) / 32) <= 256) return launch_low_rt<2, KROW>(lp, p, plan, pj, st);
    if (lp.rank <= 32) return launch_low_rt<2, KROW>(lp, p, plan, pj, st);
    return launch_low_rt<4, KROW>(lp, p, plan, pj, st);
}

// ---- the adapters' gradients ----
// G[r, c] = sum over the rows t of a long unit of S[t, r] X[t, c], X = x (dA, with S = g) or dout (dB, with S = h).  The contraction runs
// over the rows of both operands, which therefore go through LDS to be read transposed.  S is fp32: three bf16 parts of one sign (cut)
// hold its 24 bits, and each takes an MFMA (the arithmetic stays far below the reading of X).  A workgroup takes 128 columns and up to 64 ranks of a unit,
// 64 rows a step, the next two steps' rows under way; in PARTS 2 halves of a larger workgroup take the steps in turn.  4096 rows of 2560 and 10576, rank 16: 27 us, 3.9 TB/s; 16384 rows of 5120 and 2560,
// rank 32: 85 us, 3.0 TB/s (S comes again for every block of columns, and its parts are worked out again).
// Rows beyond the unit's end are zero in both operands.
struct GradJob {
    const __bf16* x;
    int64_t ldx;
    const float* s;
    float* out;   // [adapters][rank][cols], or transposed [adapters][cols][rank]
    float* part;  // the same, by slots
    int cols;
    int blocks;   // of columns
};
struct GradParams {
    GradJob job[2];  // 0: dA, 1: dB (transposed)
    int rank, accumulate;
};
// In LDS a row of X is 256 bytes, eight blocks of sixteen columns; a row of S holds its three parts in blocks of sixteen ranks, eight or
// (RT 4) sixteen.  Half a wave's transposing read takes one block of each of the rows 0 .. 3 and 8 .. 11 of a step's sixteen: block b of
// row k lies at place b ^ (k % 4 + 4 (k / 8 % 2)), which spreads them over all banks.
constexpr int GCOLS = 128;
constexpr int s_row(int rt) { return rt == 4 ? 512 : 256; }
__device__ __forceinline__ int block_at(int k, int block) { return 32 * (block ^ ((k & 3) + ((k >> 1) & 4))); }

template <int RT, bool TRANS, int PARTS>
__device__ __forceinline__ void grad_unit(const GradJob& jb, const GradParams& gp, const Plan& p, const int* plan, const Unit un, int u, int cb, int r0, char* lds) {
    const int tid = threadIdx.x & 255, part_of = PARTS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 8), lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6), q = lane >> 4, l16 = lane & 15;
    const int a = un.a, cnt = un.count, fl = plan[p.first_long + a], nl = plan[p.first_long + a + 1] - fl;
    const int* perm = plan + p.perm + un.first;
    auto row = [&](int t) -> int64_t { return un.row0 < 0 ? perm[t] : un.row0 + t; };
    const int c0 = cb * GCOLS;
    char *lx = lds + part_of * 64 * (256 + s_row(RT)), *ls = lx + 64 * 256;
    // Even and odd steps are summed apart where two parts could have them, so that a result's bits do not depend on how many other adapters there are.
    constexpr int SETS = RT <= 2 && PARTS == 1 ? 2 : 1;
    f32x4 sets[SETS][RT][2];
#pragma unroll
    for (int t = 0; t < SETS * RT * 2; ++t) sets[t / (2 * RT)][t / 2 % RT][t & 1] = (f32x4)(0.f);
    auto& acc = sets[0];
    struct Rows {
        bf16x8 x[4];
        f32x4 s[RT];
    };
    auto load = [&](Rows& w, int t0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {  // 64 rows of 16 pieces
            const int v = i * 256 + tid, t = v >> 4, c = (v & 15) * 8;
            w.x[i] = (bf16x8)((__bf16)0.f);
            if (t0 + t < cnt && c0 + c < jb.cols) w.x[i] = *(const bf16x8*)(jb.x + row(t0 + t) * jb.ldx + c0 + c);
        }
#pragma unroll
        for (int i = 0; i < RT; ++i) {  // 64 rows of 4 RT pieces of four ranks
            const int v = i * 256 + tid, t = v / (4 * RT), r = 4 * (v % (4 * RT));
            w.s[i] = (f32x4)(0.f);
            if (t0 + t < cnt && r0 + r < gp.rank) w.s[i] = *(const f32x4*)(jb.s + row(t0 + t) * gp.rank + r0 + r);
        }
    };
    auto use = [&](Rows& w, int next, f32x4 (&acc)[RT][2]) {
        __syncthreads();  // the operands before these have been read
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int v = i * 256 + tid;
            *(bf16x8*)(lx + (v >> 4) * 256 + block_at(v >> 4, (v & 15) >> 1) + (v & 1) * 16) = w.x[i];
        }
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            const int v = i * 256 + tid, t = v / (4 * RT), r = 4 * (v % (4 * RT));
#pragma unroll
            for (int part = 0; part < 3; ++part) {
                bf16x4 b;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float v = w.s[i][e];
                    b[e] = cut(v);
                    w.s[i][e] = v;
                }
                *(bf16x4*)(ls + t * s_row(RT) + block_at(t, part * RT + (r >> 4)) + 2 * (r & 15)) = b;
            }
        }
        __syncthreads();
        load(w, next);  // two steps ahead
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int k = 32 * h + 8 * q + (l16 >> 2);
            bf16x8 xo[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const char* at = lx + k * 256 + block_at(k, 2 * wv + j) + 8 * (l16 & 3);
                const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at);
                const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + 4 * 256));  // (the same place: k + 4)
                xo[j] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
            }
#pragma unroll
            for (int part = 0; part < 3; ++part)
#pragma unroll
                for (int t = 0; t < RT; ++t) {
                    const char* at = ls + k * s_row(RT) + block_at(k, part * RT + t) + 8 * (l16 & 3);
                    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at);
                    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + 4 * s_row(RT)));
                    const bf16x8 so = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
                    for (int j = 0; j < 2; ++j)
                        acc[t][j] = TRANS ? __builtin_amdgcn_mfma_f32_16x16x32_bf16(so, xo[j], acc[t][j], 0, 0, 0)
                                          : __builtin_amdgcn_mfma_f32_16x16x32_bf16(xo[j], so, acc[t][j], 0, 0, 0);
                }
        }
    };
    Rows ra, rb;
    const int mine = 64 * part_of;  // the parts take steps in turn
    load(ra, mine);
    load(rb, mine + 64 * PARTS);
    for (int t0 = 0; t0 < cnt; t0 += 128 * PARTS) {
        use(ra, t0 + mine + 128 * PARTS, acc);
        if (t0 + 64 * PARTS < cnt) use(rb, t0 + mine + 192 * PARTS, sets[SETS - 1]);
    }
    if (SETS == 2)
#pragma unroll
        for (int t = 0; t < 2 * RT; ++t) acc[t >> 1][t & 1] += sets[SETS - 1][t >> 1][t & 1];
    if (PARTS == 2) {  // their sums meet
        f32x4* sums = (f32x4*)lds;
        __syncthreads();
        if (part_of == 1)
#pragma unroll
            for (int t = 0; t < 2 * RT; ++t) sums[t * 256 + tid] = acc[t >> 1][t & 1];
        __syncthreads();
        if (part_of == 1) return;
#pragma unroll
        for (int t = 0; t < 2 * RT; ++t) acc[t >> 1][t & 1] += sums[t * 256 + tid];
    }
    // TRANS: lane -> column l16, four consecutive ranks; else lane -> rank l16, four consecutive columns
    const bool direct = nl == 1;
    const int64_t size = (int64_t)gp.rank * jb.cols;
    float* org = direct ? jb.out + a * size : jb.part + (plan[p.first_slot + a] + (u - fl)) * size;
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int r = r0 + 16 * t + (TRANS ? 4 * q : l16), c = c0 + wv * 32 + j * 16 + (TRANS ? l16 : 4 * q);
            if (r >= gp.rank || c >= jb.cols) continue;
            f32x4* at = (f32x4*)(org + (TRANS ? (int64_t)c * gp.rank + r : (int64_t)r * jb.cols + c));
            *at = direct && gp.accumulate ? *at + acc[t][j] : acc[t][j];
        }
}

template <int RT, int PARTS>
__global__ __launch_bounds__(256 * PARTS) void k_adapter_grads(GradParams gp, Plan p, const int* plan) {
    __shared__ __attribute__((aligned(16))) char lds[PARTS * 64 * (256 + s_row(RT))];
    const int u = blockIdx.y;
    const Unit un = ((const Unit*)(plan + p.long_u))[u];
    if (un.a < 0) return;
    const int b = blockIdx.x, r0 = blockIdx.z * 16 * RT;
    if (b < gp.job[0].blocks) grad_unit<RT, false, PARTS>(gp.job[0], gp, p, plan, un, u, b, r0, lds);
    else grad_unit<RT, true, PARTS>(gp.job[1], gp, p, plan, un, u, b - gp.job[0].blocks, r0, lds);
}

// Adapters of several units: their sums in order.
__global__ __launch_bounds__(256) void k_adapter_grads_sum(GradParams gp, Plan p, const int* plan, int blocks0) {
    const int a = plan[p.several + blockIdx.y];
    if (a < 0) return;
    const int nl = plan[p.first_long + a + 1] - plan[p.first_long + a];
    const GradJob& jb = gp.job[(int)blockIdx.x < blocks0 ? 0 : 1];
    const int64_t size = (int64_t)gp.rank * jb.cols;
    const int64_t i = ((int64_t)(blockIdx.x - ((int)blockIdx.x < blocks0 ? 0 : blocks0)) * 256 + threadIdx.x) * 4;
    if (i >= size) return;
    f32x4 s = (f32x4)(0.f);
    const float* part = jb.part + plan[p.first_slot + a] * size + i;
    for (int u = 0; u < nl; ++u) s += *(const f32x4*)(part + u * size);
    f32x4* at = (f32x4*)(jb.out + a * size + i);
    *at = gp.accumulate ? *at + s : s;
}

bool al(const void* p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

int check_shape(const ssd_adapter_shape_t* s) {
    if (!s) return SSD_ERR_NULL;
    const int rc = linear_check(s->rows, s->in_dim, s->out_dim, s->x_row_stride, s->out_row_stride);
    if (rc != SSD_OK) return rc;
    if (s->dx_row_stride && (s->dx_row_stride < s->in_dim || (s->dx_row_stride & 7))) return SSD_ERR_SHAPE;
    if (s->rank <= 0 || s->rank > MAX_RANK || s->nadapters <= 0 || s->nadapters > SSD_MAX_ADAPTERS) return SSD_ERR_SHAPE;
    if (s->rank & 7) return SSD_ERR_DIVISIBILITY;
    return SSD_OK;
}

size_t pad(size_t b) { return (b + 255) / 256 * 256; }
size_t low_bytes(const ssd_adapter_shape_t* s) { return pad((size_t)s->rows * s->rank * sizeof(float)); }
size_t packed_bytes(const ssd_adapter_shape_t* s) { return pad((size_t)(s->rows + 15) / 16 * 16 * s->rank * 2 * 2); }  // two parts
size_t factor_bytes(const ssd_adapter_shape_t* s, int width) { return pad((size_t)s->nadapters * s->rank * ((width + 15) & ~15) * 2); }
// Whether the forward product takes b packed, which costs the narrow one a pass over it.  8192 rows 2560 -> 10576 rank 64: the call 384 ->
// 378 us; 7116 rows 1024 -> 4384 rank 16: the narrow product 6.0 -> 8.7, the wide one the same.
bool packs_b(const ssd_adapter_shape_t* s) { return s->rows >= 2048 && s->rank > 32; }
PackJob pack_of(const ssd_adapter_shape_t* s, const void* from, void* to, int width) {
    // workgroups by the thousand, not by the number of adapters: of a large set few have rows
    const int64_t per = (width + 63) / 64, group = (s->nadapters * per + 2047) / 2048;
    return {(const __bf16*)from, (__bf16*)to, width, s->rank, (int)((s->nadapters + group - 1) / group * per), (int)group};
}
LowRankTerm term_of(const Plan& p, const int* plan, const void* low, const void* up, bool packed, const ssd_adapter_shape_t* s, int width) {
    return {plan + p.ids, plan + p.tile_n, plan + p.tile_a, (const bf16_t*)low, (const bf16_t*)up, s->rank, packed ? (width + 15) & ~15 : width, packed};
}
size_t part_bytes(const Plan& p, const ssd_adapter_shape_t* s, int cols) { return pad((size_t)most_slots(p) * s->rank * cols * sizeof(float)); }

LowProduct product_of(const ssd_adapter_shape_t* s, bool input_grad, const void* x, const void* w, void* out) {
    const int64_t ldx = s->x_row_stride ? s->x_row_stride : s->in_dim, ldo = s->out_row_stride ? s->out_row_stride : s->out_dim;
    if (input_grad) return {true, s->rows, s->in_dim, s->out_dim, x, ldo, w, out, s->dx_row_stride ? s->dx_row_stride : s->in_dim};
    return {false, s->rows, s->in_dim, s->out_dim, x, ldx, w, out, ldo};
}
size_t slice_bytes(const ssd_adapter_shape_t* s, bool input_grad) {
    if (!s->rows) return 0;
    return pad(linear_low_bytes(product_of(s, input_grad, (const void*)256, (const void*)256, (void*)256)));
}

template <int RT>
hipError_t launch_grads_rt(const GradParams& gp, const Plan& p, const int* plan, hipStream_t st) {
    const dim3 grid(gp.job[0].blocks + gp.job[1].blocks, p.max_long, (gp.rank + 16 * RT - 1) / (16 * RT));
    // Up to some two workgroups a compute unit (units without rows among them) the steps of a unit one after another are the time: two parts.
    // 600 rows of 1024 and 4384, 129 workgroups, 14.1 -> 10.2 us; 1000 rows of one adapter, 43, 31 -> 19; 4096 rows of four, 516, 19.4 -> 14.8;
    // 1500 rows of 2560 and 10576 at rank 32, 618, 24.5 -> 25.2; 4096 rows of these at rank 16, 1236, 28.7 -> 32.  (Ranks beyond 32: LDS.)
    if constexpr (RT <= 2)
        if ((int64_t)grid.x * grid.y <= 576) {
            hipLaunchKernelGGL((k_adapter_grads<RT, 2>), grid, dim3(512), 0, st, gp, p, plan);
            return hipGetLastError();
        }
    hipLaunchKernelGGL((k_adapter_grads<RT, 1>), grid, dim3(256), 0, st, gp, p, plan);
    return hipGetLastError();
}

}  // namespace
}  // namespace ssdk

using namespace ssdk;

extern "C" size_t ssd_adapter_plan_bytes(int64_t rows, int32_t nadapters) {
    if (rows < 0 || rows > SSD_MAX_ADAPTER_ROWS || nadapters <= 0 || nadapters > SSD_MAX_ADAPTERS) return 0;
    return pad((size_t)plan_of(rows, nadapters).words * sizeof(int));
}

extern "C" int ssd_adapter_plan(int64_t rows, int32_t nadapters, const int32_t* row_adapter, void* plan, size_t plan_bytes, void* hip_stream) {
    const size_t need = ssd_adapter_plan_bytes(rows, nadapters);
    if (!need) return SSD_ERR_SHAPE;
    if (!plan || (rows && !row_adapter)) return SSD_ERR_NULL;
    if (!al(row_adapter, 4)) return SSD_ERR_ARG;
    if (!al(plan, 256) || plan_bytes < need) return SSD_ERR_WORKSPACE;
    const Plan p = plan_of(rows, nadapters);
    hipStream_t st = (hipStream_t)hip_stream;
    hipLaunchKernelGGL(k_plan_count, dim3(p.tiles + nadapters + 1), dim3(PTHR), 0, st, p, row_adapter, (int*)plan);
    hipLaunchKernelGGL(k_plan_rows, dim3(nadapters + 1), dim3(PTHR), 0, st, p, (int*)plan);
    return hipGetLastError() == hipSuccess ? SSD_OK : SSD_ERR_LAUNCH;
}

extern "C" size_t ssd_adapter_workspace_bytes(const ssd_adapter_shape_t* shape, int32_t is_backward) {
    if (check_shape(shape) != SSD_OK || shape->rows > SSD_MAX_ADAPTER_ROWS) return 0;
    if (!is_backward) return packed_bytes(shape) + (packs_b(shape) ? factor_bytes(shape, shape->out_dim) : 0) + slice_bytes(shape, false) + 256;
    const Plan p = plan_of(shape->rows, shape->nadapters);
    const size_t slices = slice_bytes(shape, true), parts = part_bytes(p, shape, shape->in_dim) + part_bytes(p, shape, shape->out_dim);
    return 2 * low_bytes(shape) + packed_bytes(shape) + factor_bytes(shape, shape->in_dim) + (slices > parts ? slices : parts) + 256;  // (one is read before the other is written)
}

extern "C" int ssd_adapter_linear_fwd(const ssd_adapter_shape_t* shape, const void* x, const void* w, const void* a, const void* b,
                                      const float* scale, const void* plan, void* out, float* hidden, void* workspace,
                                      size_t workspace_bytes, void* hip_stream) {
    const int rc = check_shape(shape);
    if (rc != SSD_OK) return rc;
    if (shape->rows > SSD_MAX_ADAPTER_ROWS) return SSD_ERR_SHAPE;
    if (shape->rows == 0) return SSD_OK;
    if (!x || !w || !a || !b || !scale || !plan || !out) return SSD_ERR_NULL;
    if (!al(x, 16) || !al(w, 16) || !al(a, 16) || !al(b, 16) || !al(out, 16) || !al(scale, 4) || !al(hidden, 16) || !al(plan, 256)) return SSD_ERR_ARG;
    if (!workspace || !al(workspace, 256) || workspace_bytes < ssd_adapter_workspace_bytes(shape, 0)) return SSD_ERR_WORKSPACE;
    hipStream_t st = (hipStream_t)hip_stream;
    const Plan p = plan_of(shape->rows, shape->nadapters);
    const int* pl = (const int*)plan;
    __bf16* packed = (__bf16*)workspace;
    char *b_packed = (char*)workspace + packed_bytes(shape), *slices = b_packed;
    PackJob pj = {};
    if (packs_b(shape)) {
        pj = pack_of(shape, b, b_packed, shape->out_dim);
        slices += factor_bytes(shape, shape->out_dim);
    }
    const int64_t ldx = shape->x_row_stride ? shape->x_row_stride : shape->in_dim;
    const LowParams lp = {(const __bf16*)x, ldx, (const __bf16*)a, scale, hidden, packed, shape->in_dim, shape->rank};
    if (launch_low_products<false>(lp, p, pl, pj, st) != hipSuccess) return SSD_ERR_LAUNCH;
    const LowRankTerm lr = term_of(p, pl, packed, pj.blocks ? b_packed : b, pj.blocks != 0, shape, shape->out_dim);
    const hipError_t e = launch_linear_low(product_of(shape, false, x, w, out), lr, slices, st);
    return e == hipSuccess ? SSD_OK : SSD_ERR_LAUNCH;
}

extern "C" int ssd_adapter_linear_bwd(const ssd_adapter_shape_t* shape, const void* x, const void* w, const void* a, const void* b,
                                      const float* scale, const void* plan, const void* dout, const float* hidden, void* dx, float* da,
                                      float* db, void* workspace, size_t workspace_bytes, uint32_t flags, void* hip_stream) {
    const int rc = check_shape(shape);
    if (rc != SSD_OK) return rc;
    if (shape->rows > SSD_MAX_ADAPTER_ROWS) return SSD_ERR_SHAPE;
    if (flags & ~(uint32_t)SSD_FLAG_ACCUM_PARAM) return SSD_ERR_ARG;
    if ((da == nullptr) != (db == nullptr)) return SSD_ERR_NULL;
    hipStream_t st = (hipStream_t)hip_stream;
    const bool accumulate = flags & SSD_FLAG_ACCUM_PARAM;
    const size_t size_a = (size_t)shape->nadapters * shape->rank * shape->in_dim, size_b = (size_t)shape->nadapters * shape->rank * shape->out_dim;
    if (!al(da, 16) || !al(db, 16)) return SSD_ERR_ARG;
    if (shape->rows == 0) {
        if (da && !accumulate && (launch_fill_zero(da, size_a, st) != hipSuccess || launch_fill_zero(db, size_b, st) != hipSuccess)) return SSD_ERR_LAUNCH;
        return SSD_OK;
    }
    if (!dx && !da) return SSD_OK;
    if (!a || !b || !scale || !plan || !dout || (dx && !w) || (da && !x)) return SSD_ERR_NULL;
    if (!al(x, 16) || !al(w, 16) || !al(a, 16) || !al(b, 16) || !al(dout, 16) || !al(dx, 16) || !al(scale, 4) || !al(hidden, 16) || !al(plan, 256)) return SSD_ERR_ARG;
    if (!workspace || !al(workspace, 256) || workspace_bytes < ssd_adapter_workspace_bytes(shape, 1)) return SSD_ERR_WORKSPACE;
    const Plan p = plan_of(shape->rows, shape->nadapters);
    const int* pl = (const int*)plan;
    char* ws = (char*)workspace;
    float *g = (float*)ws, *own_h = (float*)(ws + low_bytes(shape));
    __bf16 *packed = (__bf16*)(ws + 2 * low_bytes(shape)), *a_packed = (__bf16*)((char*)packed + packed_bytes(shape));
    float *part_a = (float*)((char*)a_packed + factor_bytes(shape, shape->in_dim)), *part_b = (float*)((char*)part_a + part_bytes(p, shape, shape->in_dim));
    const int64_t ldx = shape->x_row_stride ? shape->x_row_stride : shape->in_dim, ldd = shape->out_row_stride ? shape->out_row_stride : shape->out_dim;
    const LowParams lg = {(const __bf16*)dout, ldd, (const __bf16*)b, scale, da ? g : nullptr, dx ? packed : nullptr, shape->out_dim, shape->rank};
    PackJob pj = {};
    if (dx) pj = pack_of(shape, a, a_packed, shape->in_dim);
    if (launch_low_products<true>(lg, p, pl, pj, st) != hipSuccess) return SSD_ERR_LAUNCH;
    if (dx && launch_linear_low(product_of(shape, true, dout, w, dx), term_of(p, pl, packed, a_packed, true, shape, shape->in_dim), part_a, st) != hipSuccess)
        return SSD_ERR_LAUNCH;
    if (!da) return SSD_OK;
    if (!hidden) {
        const LowParams lh = {(const __bf16*)x, ldx, (const __bf16*)a, scale, own_h, nullptr, shape->in_dim, shape->rank};
        if (launch_low_products<false>(lh, p, pl, PackJob{}, st) != hipSuccess) return SSD_ERR_LAUNCH;
        hidden = own_h;
    }
    GradParams gp;
    gp.job[0] = {(const __bf16*)x, ldx, g, da, part_a, shape->in_dim, (shape->in_dim + GCOLS - 1) / GCOLS};
    gp.job[1] = {(const __bf16*)dout, ldd, hidden, db, part_b, shape->out_dim, (shape->out_dim + GCOLS - 1) / GCOLS};
    gp.rank = shape->rank;
    gp.accumulate = accumulate;
    const hipError_t e = gp.rank <= 16 ? launch_grads_rt<1>(gp, p, pl, st) : gp.rank <= 32 ? launch_grads_rt<2>(gp, p, pl, st) : launch_grads_rt<4>(gp, p, pl, st);
    if (e != hipSuccess) return SSD_ERR_LAUNCH;
    if (!most_slots(p)) return SSD_OK;  // no adapter has several units
    const int64_t b0 = ((int64_t)gp.rank * shape->in_dim + 1023) / 1024, b1 = ((int64_t)gp.rank * shape->out_dim + 1023) / 1024;
    hipLaunchKernelGGL(k_adapter_grads_sum, dim3((unsigned)(b0 + b1), p.max_several()), dim3(256), 0, st, gp, p, pl, (int)b0);
    return hipGetLastError() == hipSuccess ? SSD_OK : SSD_ERR_LAUNCH;
}
