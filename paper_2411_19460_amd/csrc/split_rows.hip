// Products of some tens to hundreds of rows with a low-rank term (adapters): out = x w^T + low up^T, forward (w [N, K]) or the input's
// gradient (w [K, N]).  The tiles of linear.hip, 256 rows high and one to a compute unit, leave most of the chip idle here and walk the
// whole of K one step after another.  These are 32 x 16, 32, 64 or 64 x 64 (16 MT rows, 16 NT columns), and the eight waves of a workgroup share out K in steps
// of 64: a wave fetches a step's rows as 128 contiguous bytes each, U steps at a time, turns them into operands through LDS of its
// own without a barrier, and the waves' sums meet in LDS once, at the end, where they are rounded and leave.  The rows' adapters are
// shared out as well: wave w adds numbers w, w + 8, ... of the tile's.
// What bounds it: the operands' way from the L2 (each element of x is fetched N / (16 NT) times, each of w rows / (16 MT) times) and
// through LDS.  64 rows 5120 -> 2560, rank 32, 24 adapters: 12.8 us (w 26 MB: 2.0 TB/s; LDS works in 38 % of the
// busy cycles, bank conflicts in 10 %); 600 rows, input gradient of 1024 -> 4384: 21.1 us.
#include "low_rank.h"
#include "mfma_common.h"

namespace ssdk {
namespace {

using namespace mf;

constexpr int WAVES = 8, PITCH = 144;  // bytes of a row of a step in LDS: 64 k, and sixteen rows fall into distinct banks

struct SplitParams {
    const __bf16 *x, *w;
    __bf16* out;
    int64_t ldx, ldw, ldo;
    int M, N, K, tiles_m;
};

template <int NT>
constexpr int krow_pitch() { return 32 * NT + 16; }
template <int MT, int NT, bool KROW>
constexpr int wave_lds() { return 16 * MT * PITCH + (KROW ? 64 * krow_pitch<NT>() : 16 * NT * PITCH); }
template <int NT>
constexpr int sum_pitch() { return 16 * NT + 4; }
template <int MT, int NT, bool KROW>
constexpr int split_lds() {
    constexpr int a = WAVES * wave_lds<MT, NT, KROW>(), b = WAVES * 16 * MT * sum_pitch<NT>() * 4;
    return a > b ? a : b;
}

template <int MT, int NT, bool KROW, int U>
__global__ __launch_bounds__(64 * WAVES, 2) void k_split(SplitParams sp, LowRankTerm lr) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6), q = lane >> 4, l16 = lane & 15;
    const int r8 = lane >> 3, c8 = (lane & 7) * 8;  // fetching lanes: eight rows of 64 elements
    // the row tiles of the same columns one after another on one XCD
    const int n = gridDim.x, per = n >> 3, b = blockIdx.x, id = b < 8 * per ? (b & 7) * per + (b >> 3) : b;
    const int m0 = id % sp.tiles_m * 16 * MT, n0 = id / sp.tiles_m * 16 * NT;
    // Rows and columns that do not exist, and k beyond K, are fetched from beyond a descriptor's end: zeros.
    constexpr uint32_t OUT = 0x80000000u;
    const uint32_t ldx = (uint32_t)sp.ldx * 2, ldw = (uint32_t)sp.ldw * 2;
    const rsrc_t rx = make_rows(sp.x + m0 * sp.ldx, sp.M - m0 < 16 * MT ? sp.M - m0 : 16 * MT, ldx);
    const uint32_t x0 = r8 * ldx + c8 * 2;
    // w: 16 NT rows of 64 k, or 64 rows of k of 16 NT columns
    constexpr int CP = 2 * NT, KR = 64 / CP;  // KROW: pieces of a row, rows an access
    const rsrc_t rw = make_rows(sp.w + n0 * sp.ldw, sp.N - n0 < 16 * NT ? sp.N - n0 : 16 * NT, ldw);  // (KROW: not used)
    const uint32_t w0 = !KROW ? r8 * ldw + c8 * 2 : n0 + 8 * (lane % CP) < sp.N ? (lane / CP) * ldw + (n0 + 8 * (lane % CP)) * 2 : OUT;
    char *mx = lds + wv * wave_lds<MT, NT, KROW>(), *mw = mx + 16 * MT * PITCH;
    f32x4 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = (f32x4)(0.f);
    struct Steps {
        bf16x8 x[U][2 * MT], w[U][2 * NT];
    };
    auto load = [&](Steps& b, int k0) {
#pragma unroll
        for (int s = 0; s < U; ++s) {
            const int ks = k0 + 64 * WAVES * s;
            const uint32_t off = ks + c8 < sp.K ? (uint32_t)ks * 2 : OUT;
#pragma unroll
            for (int i = 0; i < 2 * MT; ++i) b.x[s][i] = rows_load(rx, x0 + off + i * 8 * ldx);
            if (KROW) {
                const int left = sp.K - ks;
                const rsrc_t rk = make_rows(sp.w + (int64_t)(left > 0 ? ks : 0) * sp.ldw, left < 0 ? 0 : left < 64 ? left : 64, ldw);
#pragma unroll
                for (int i = 0; i < 2 * NT; ++i) b.w[s][i] = rows_load(rk, w0 + i * KR * ldw);
            } else {
#pragma unroll
                for (int i = 0; i < 2 * NT; ++i) b.w[s][i] = rows_load(rw, w0 + off + i * 8 * ldw);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    auto use = [&](const Steps& b, int k0) {
#pragma unroll
        for (int s = 0; s < U; ++s) {
            if (k0 + 64 * WAVES * s >= sp.K) break;
#pragma unroll
            for (int i = 0; i < 2 * MT; ++i) *(bf16x8*)(mx + (8 * i + r8) * PITCH + 2 * c8) = b.x[s][i];
#pragma unroll
            for (int i = 0; i < 2 * NT; ++i)
                *(bf16x8*)(KROW ? mw + (i * KR + lane / CP) * krow_pitch<NT>() + 16 * (lane % CP) : mw + (8 * i + r8) * PITCH + 2 * c8) = b.w[s][i];
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the wave's own rows: its LDS operations are done in order
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                bf16x8 xo[MT], wo[NT];
#pragma unroll
                for (int i = 0; i < MT; ++i) xo[i] = *(const bf16x8*)(mx + (i * 16 + l16) * PITCH + 64 * h + 16 * q);
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    if (KROW) {
                        const char* p = mw + (32 * h + 8 * q + (l16 >> 2)) * krow_pitch<NT>() + 32 * j + 8 * (l16 & 3);
                        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p);
                        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 4 * krow_pitch<NT>()));
                        wo[j] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
                    } else {
                        wo[j] = *(const bf16x8*)(mw + (j * 16 + l16) * PITCH + 64 * h + 16 * q);
                    }
                }
#pragma unroll
                for (int j = 0; j < NT; ++j)
#pragma unroll
                    for (int i = 0; i < MT; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wo[j], xo[i], acc[i][j], 0, 0, 0);
            }
            asm volatile("" ::: "memory");  // the next step's rows come in behind these reads
        }
    };
    constexpr int NEXT = 64 * WAVES * U;
    Steps a, c;
    int k0 = 64 * wv;
    load(a, k0);
    add_low_rank<MT, NT>(acc, lr, m0, sp.M, n0, sp.N, lane, wv, WAVES);
    for (; k0 < sp.K; k0 += 2 * NEXT) {  // one group of steps is multiplied while the next is under way
        load(c, k0 + NEXT);
        use(a, k0);
        load(a, k0 + 2 * NEXT);
        use(c, k0 + NEXT);
    }
    __syncthreads();
    float* sums = (float*)lds;  // lane -> row l16 of tile i, four consecutive columns
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) *(f32x4*)(sums + (wv * 16 * MT + 16 * i + l16) * sum_pitch<NT>() + 16 * j + 4 * q) = acc[i][j];
    __syncthreads();
    for (int v = tid; v < 16 * MT * 2 * NT; v += 64 * WAVES) {
        const int r = v / (2 * NT), c = 8 * (v % (2 * NT));
        if (m0 + r >= sp.M || n0 + c >= sp.N) continue;
        f32x4 o0 = (f32x4)(0.f), o1 = (f32x4)(0.f);
#pragma unroll
        for (int u = 0; u < WAVES; ++u) {
            const f32x4* p = (const f32x4*)(sums + (u * 16 * MT + r) * sum_pitch<NT>() + c);
            o0 += p[0];
            o1 += p[1];
        }
        bf16x8 o;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = (__bf16)o0[e], o[4 + e] = (__bf16)o1[e];
        *(bf16x8*)(sp.out + (int64_t)(m0 + r) * sp.ldo + n0 + c) = o;
    }
}

template <int MT, int NT, bool KROW, int U>
hipError_t launch(SplitParams sp, const LowRankTerm& lr, hipStream_t st) {
    constexpr int LDS = split_lds<MT, NT, KROW>();
    static bool raised[64];
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return hipErrorInvalidDevice;
    if (!raised[dev]) {
        const hipError_t e = hipFuncSetAttribute((const void*)k_split<MT, NT, KROW, U>, hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
        if (e != hipSuccess) return e;
        raised[dev] = true;
    }
    sp.tiles_m = (sp.M + 16 * MT - 1) / (16 * MT);
    const int tiles_n = (sp.N + 16 * NT - 1) / (16 * NT);
    hipLaunchKernelGGL((k_split<MT, NT, KROW, U>), dim3((unsigned)(sp.tiles_m * tiles_n)), dim3(64 * WAVES), LDS, st, sp, lr);
    return hipGetLastError();
}

template <bool KROW>
hipError_t launch_shape(const SplitParams& sp, int mt, int nt, const LowRankTerm& lr, hipStream_t st) {
    if (mt == 4) return launch<4, 4, KROW, 1>(sp, lr, st);
    return nt == 1 ? launch<2, 1, KROW, 2>(sp, lr, st) : nt == 2 ? launch<2, 2, KROW, 2>(sp, lr, st) : launch<2, 4, KROW, 1>(sp, lr, st);
}

}  // namespace

hipError_t launch_split_rows(bool input_grad, int rows, int K, int N, const void* x, int64_t ldx, const void* w, int64_t ldw, void* out, int64_t ldo, int mt, int nt,
                             const LowRankTerm& lr, hipStream_t st) {
    const SplitParams sp = {(const __bf16*)x, (const __bf16*)w, (__bf16*)out, ldx, ldw, ldo, rows, N, K, 0};
    return input_grad ? launch_shape<true>(sp, mt, nt, lr, st) : launch_shape<false>(sp, mt, nt, lr, st);
}

}  // namespace ssdk
