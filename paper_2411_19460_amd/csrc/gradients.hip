// The global norm of many gradients, and the gradients scaled down to it:
//     S = sum over all tensors and elements of g^2      norm = sqrt(S)      out = g min(1, max_norm / (norm + 1e-6))
// Bound by memory: the gradients go by twice (the second time partly out of the last-level cache) and their result leaves once.  Many
// tensors of any size share a launch: the plan cuts them into pieces of PIECE elements, and workgroups take pieces in turn.
// S is held in fp64 (squares of fp32 values neither overflow nor vanish there), summed in an order that depends on the pieces alone.
#include <string.h>

#include "ssd_internal.h"

namespace ssdk {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int64_t PIECE = 8192;  // elements: a multiple of 16-byte vectors, so that all pieces of a tensor are aligned as it is
constexpr int THR = 256, NORM_WGS = 1024, CLIP_WGS = 2048;
// Up to this many pieces one workgroup of SOLO_THR threads does everything: a launch less costs more than the others' bandwidth brings
// (51 392 values 9.3 -> 7.2 us a call).
constexpr int SOLO_PIECES = 8, SOLO_THR = 1024;
constexpr int64_t STREAM_PIECES = 8192;  // 256 MiB of fp32 gradients

// Device memory of a plan: the workgroups' sums of squares, then the pieces.
struct Piece {
    const void* src;
    void* dst;
    int n, kind;  // kind: bit 0 source bf16, bit 1 result bf16, bit 2 both on 16 bytes
    int pad[2];
};
struct Head {
    double part[NORM_WGS];
};
static_assert(sizeof(Piece) == 32 && sizeof(Head) % 256 == 0, "");

// The pieces of up to TENSORS tensors, which come as kernel arguments.
constexpr int TENSORS = 64;
struct Tensors {
    const void* src[TENSORS];
    void* dst[TENSORS];
    int64_t numel[TENSORS], first[TENSORS];  // first: piece
    int kind[TENSORS];
    int count;
};

__global__ __launch_bounds__(THR) void k_grad_pieces(Tensors t, Piece* pieces) {
    for (int i = blockIdx.y; i < t.count; i += gridDim.y) {
        const int64_t np = (t.numel[i] + PIECE - 1) / PIECE;
        for (int64_t k = (int64_t)blockIdx.x * THR + threadIdx.x; k < np; k += (int64_t)gridDim.x * THR) {
            const int64_t at = k * PIECE, left = t.numel[i] - at;
            Piece p;
            p.src = (const char*)t.src[i] + at * (t.kind[i] & 1 ? 2 : 4);
            p.dst = (char*)t.dst[i] + at * (t.kind[i] & 2 ? 2 : 4);
            p.n = (int)(left < PIECE ? left : PIECE);
            p.kind = t.kind[i];
            p.pad[0] = p.pad[1] = 0;
            pieces[t.first[i] + k] = p;
        }
    }
}

__device__ __forceinline__ double square(float v) { return (double)v * (double)v; }

__device__ __forceinline__ double block_total(double v, double* lds) {  // in every thread
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

// What a thread holds of a piece: ROUNDS times eight consecutive values, raw.  All of it is asked for at once; what lies beyond the end
// of a short piece comes from beyond the descriptor's end, zeros.
constexpr int ROUNDS = PIECE / (8 * THR);
struct Raw {
    u32x4 x[ROUNDS][2];  // bf16: the first of each alone
};
__device__ __forceinline__ int vectors(const Piece& p) { return p.kind & 4 ? p.n / 8 : 0; }  // of eight values; the others one by one (no value on 16 bytes: 21 M fp32 75 us a call instead of 44, bf16 68 instead of 25)

template <bool BF16>
__device__ __forceinline__ void load_raw(Raw& r, const Piece& p, int tid) {
    constexpr int B = BF16 ? 16 : 32;
    const __amdgpu_buffer_rsrc_t src = __builtin_amdgcn_make_buffer_rsrc((void*)p.src, 0, vectors(p) * B, 0x00020000);
#pragma unroll
    for (int l = 0; l < ROUNDS; ++l)
#pragma unroll
        for (int h = 0; h < (BF16 ? 1 : 2); ++h) r.x[l][h] = __builtin_amdgcn_raw_buffer_load_b128(src, (l * THR + tid) * B + 16 * h, 0, 0);
}
__device__ __forceinline__ void load(Raw& r, const Piece& p, int tid) {
    if (p.kind & 1) load_raw<true>(r, p, tid);
    else load_raw<false>(r, p, tid);
}
template <bool BF16>
__device__ __forceinline__ void values(const Raw& r, int l, float (&f)[8]) {
    if constexpr (BF16) {
        const bf16x8 h = __builtin_bit_cast(bf16x8, r.x[l][0]);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = (float)h[e];
    } else {
        const f32x4 lo = __builtin_bit_cast(f32x4, r.x[l][0]), hi = __builtin_bit_cast(f32x4, r.x[l][1]);
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = lo[e], f[4 + e] = hi[e];
    }
}
__device__ __forceinline__ float value(const Piece& p, int i) { return p.kind & 1 ? (float)((const __bf16*)p.src)[i] : ((const float*)p.src)[i]; }

template <bool BF16>
__device__ __forceinline__ double squares_raw(const Raw& r) {
    double s[4] = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
    for (int l = 0; l < ROUNDS; ++l) {
        float f[8];
        values<BF16>(r, l, f);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e & 3] += square(f[e]);
    }
    return (s[0] + s[1]) + (s[2] + s[3]);
}
__device__ __forceinline__ double squares(const Raw& r, const Piece& p, int tid) {
    double s = p.kind & 1 ? squares_raw<true>(r) : squares_raw<false>(r);
    for (int i = vectors(p) * 8 + tid; i < p.n; i += THR) s += square(value(p, i));
    return s;
}

// part[w] = what workgroup w finds in its pieces.  161 M values, 644 MB, 99 us: 6.5 TB/s; 21 M, 85 MB, 13.3 us: 6.4.
__global__ __launch_bounds__(THR) void k_grad_squares(const Piece* __restrict__ pieces, int64_t count, double* part) {
    __shared__ double lds[4];
    double s = 0.0;
    for (int64_t k = blockIdx.x; k < count; k += gridDim.x) {
        const Piece p = pieces[k];
        Raw r;
        load(r, p, threadIdx.x);
        s += squares(r, p, threadIdx.x);
    }
    s = block_total(s, lds);
    if (threadIdx.x == 0) part[blockIdx.x] = s;
}

// The sum of the workgroups' sums, in a fixed order: every workgroup that asks gets the same.
__device__ __forceinline__ double sum_parts(const double* part, int parts, double* lds) {
    double s = 0.0;
    for (int i = threadIdx.x; i < parts; i += THR) s += part[i];
    return block_total(s, lds);
}

__global__ __launch_bounds__(THR) void k_grad_sum(const double* part, int parts, double* sum_sq) {
    __shared__ double lds[4];
    const double s = sum_parts(part, parts, lds);
    if (threadIdx.x == 0) *sum_sq = s;
}

template <bool FROM, bool TO, bool STREAM>
__device__ __forceinline__ void scale_raw(const Raw& r, const Piece& p, float c, int tid) {
    constexpr int B = TO ? 16 : 32;
    const __amdgpu_buffer_rsrc_t dst = __builtin_amdgcn_make_buffer_rsrc(p.dst, 0, vectors(p) * B, 0x00020000);
#pragma unroll
    for (int l = 0; l < ROUNDS; ++l) {
        float f[8];
        values<FROM>(r, l, f);
        const int at = (l * THR + tid) * B;
        if constexpr (TO) {
            bf16x8 o;
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = (__bf16)(f[e] * c);
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, o), dst, at, 0, STREAM ? 2 : 0);
        } else {
            f32x4 lo, hi;
#pragma unroll
            for (int e = 0; e < 4; ++e) lo[e] = f[e] * c, hi[e] = f[4 + e] * c;
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, lo), dst, at, 0, STREAM ? 2 : 0);
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, hi), dst, at + 16, 0, STREAM ? 2 : 0);
        }
    }
}
__device__ __forceinline__ bool stays(const Piece& p, float c) { return p.src == p.dst && c == 1.f; }
template <bool STREAM>
__device__ __forceinline__ void scale(const Raw& r, const Piece& p, float c, int tid) {
    switch (p.kind & 3) {
        case 0: scale_raw<false, false, STREAM>(r, p, c, tid); break;
        case 1: scale_raw<true, false, STREAM>(r, p, c, tid); break;
        case 2: scale_raw<false, true, STREAM>(r, p, c, tid); break;
        default: scale_raw<true, true, STREAM>(r, p, c, tid);
    }
    for (int i = vectors(p) * 8 + tid; i < p.n; i += THR) {
        const float v = value(p, i) * c;
        if (p.kind & 2) ((__bf16*)p.dst)[i] = (__bf16)v;
        else ((float*)p.dst)[i] = v;
    }
}
__device__ __forceinline__ float factor(double norm, float max_norm) {
    if (max_norm == __builtin_inff()) return 1.f;  // no bound: infinite or not a number, the norm is all that is asked for
    const double by = (double)max_norm / (norm + 1e-6);
    return by > 1.0 ? 1.f : (float)by;
}

// The pieces in reverse: what the norm read last is still in the last-level cache.  The sum of squares is *sum_sq, or (null) that of the
// parts.  The factor is worked out in fp64 and rounded once; a NaN in it stays one.  A gradient that is its own result and needs no
// scaling is left alone.  STREAM: results by streaming stores, which leave the last-level cache to the gradients that are still to come.
// They pay where the gradients are more than it holds: 161 M values fp32 -> bf16 295 -> 287 us a call, 21 M fp32 43 -> 49.
// Measured: 161 M values, 644 MB read, 322 MB written, 181 us (5.3 TB/s); 21 M, half of them still in the cache, 29 us.
template <bool STREAM>
__global__ __launch_bounds__(THR) void k_grad_clip(const Piece* __restrict__ pieces, int64_t count, const double* part, int parts, const double* sum_sq, float max_norm,
                                                   float* norm) {
    __shared__ double lds[4];
    const double n = sqrt(sum_sq ? *sum_sq : sum_parts(part, parts, lds));
    const float c = factor(n, max_norm);
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)n;
    for (int64_t k = count - 1 - blockIdx.x; k >= 0; k -= gridDim.x) {
        const Piece p = pieces[k];
        if (stays(p, c)) continue;
        Raw r;
        load(r, p, threadIdx.x);
        __builtin_amdgcn_sched_barrier(0);
        scale<STREAM>(r, p, c, threadIdx.x);
    }
}

// Both in one workgroup: quarters of it have up to two pieces each, which stay in registers in between.
__global__ __launch_bounds__(SOLO_THR) void k_grad_solo(const Piece* __restrict__ pieces, int count, float max_norm, float* norm) {
    __shared__ double lds[SOLO_THR / 64];
    const int tid = threadIdx.x % THR, k0 = __builtin_amdgcn_readfirstlane(threadIdx.x / THR), k1 = k0 + SOLO_THR / THR;
    Piece p0 = {}, p1 = {};
    if (k0 < count) p0 = pieces[k0];
    if (k1 < count) p1 = pieces[k1];
    Raw r0, r1;
    load(r0, p0, tid);
    load(r1, p1, tid);
    __builtin_amdgcn_sched_barrier(0);
    double s = squares(r0, p0, tid) + squares(r1, p1, tid);
    for (int off = 32; off > 0; off >>= 1) s += __shfl_xor(s, off, 64);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
    __syncthreads();  // every gradient has been read
    s = 0.0;
#pragma unroll
    for (int w = 0; w < SOLO_THR / 64; ++w) s += lds[w];
    const double n = sqrt(s);
    const float c = factor(n, max_norm);
    if (norm && threadIdx.x == 0) *norm = (float)n;
    if (!stays(p0, c)) scale<false>(r0, p0, c, tid);
    if (!stays(p1, c)) scale<false>(r1, p1, c, tid);
}
static_assert(SOLO_PIECES == 2 * (SOLO_THR / THR), "");

bool al(const void* p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
int64_t pieces_of(int64_t numel) { return (numel + PIECE - 1) / PIECE; }
unsigned wgs_of(int64_t pieces, int most) { return (unsigned)(pieces < 1 ? 1 : pieces < most ? pieces : most); }
void launch_squares(void* plan, int64_t pieces, hipStream_t st) {
    hipLaunchKernelGGL(k_grad_squares, dim3(wgs_of(pieces, NORM_WGS)), dim3(THR), 0, st, (const Piece*)((Head*)plan + 1), pieces, ((Head*)plan)->part);
}
constexpr int64_t MAX_NUMEL = (int64_t)1 << 48;

}  // namespace
}  // namespace ssdk

using namespace ssdk;

extern "C" size_t ssd_grad_plan_bytes(int32_t ntensors, const ssd_grad_tensor_t* tensors) {
    if (ntensors < 0 || (ntensors && !tensors)) return 0;
    int64_t n = 0;
    for (int32_t i = 0; i < ntensors; ++i) {
        if (tensors[i].numel < 0 || tensors[i].numel > MAX_NUMEL || n > MAX_NUMEL) return 0;
        n += pieces_of(tensors[i].numel);
    }
    return sizeof(Head) + (size_t)n * sizeof(Piece);
}

extern "C" int ssd_grad_plan(int32_t ntensors, const ssd_grad_tensor_t* tensors, void* plan, size_t plan_bytes, int64_t* pieces, void* hip_stream) {
    if (!pieces || !plan || (ntensors > 0 && !tensors)) return SSD_ERR_NULL;
    const size_t need = ssd_grad_plan_bytes(ntensors, tensors);
    if (!need) return SSD_ERR_SHAPE;
    if (!al(plan, 256) || plan_bytes < need) return SSD_ERR_WORKSPACE;
    for (int32_t i = 0; i < ntensors; ++i) {
        const ssd_grad_tensor_t& t = tensors[i];
        if (t.grad_dtype != SSD_F32 && t.grad_dtype != SSD_BF16) return SSD_ERR_DTYPE;
        if (t.out_dtype != SSD_F32 && t.out_dtype != SSD_BF16) return SSD_ERR_DTYPE;
        if (!t.numel) continue;
        if (!t.grad || !t.out) return SSD_ERR_NULL;
        if (!al(t.grad, t.grad_dtype == SSD_BF16 ? 2 : 4) || !al(t.out, t.out_dtype == SSD_BF16 ? 2 : 4)) return SSD_ERR_ARG;
        if (t.grad == t.out && t.grad_dtype != t.out_dtype) return SSD_ERR_ARG;
    }
    hipStream_t st = (hipStream_t)hip_stream;
    Head* head = (Head*)plan;
    Piece* list = (Piece*)(head + 1);
    int64_t n = 0;
    int32_t i = 0;
    do {
        Tensors t;
        memset(&t, 0, sizeof(t));
        int64_t most = 1;
        for (; i < ntensors && t.count < TENSORS; ++i) {
            const ssd_grad_tensor_t& s = tensors[i];
            if (!s.numel) continue;
            const int c = t.count++;
            t.src[c] = s.grad;
            t.dst[c] = s.out;
            t.numel[c] = s.numel;
            t.first[c] = n;
            t.kind[c] = (s.grad_dtype == SSD_BF16 ? 1 : 0) | (s.out_dtype == SSD_BF16 ? 2 : 0) | (al(s.grad, 16) && al(s.out, 16) ? 4 : 0);
            const int64_t np = pieces_of(s.numel);
            most = most > np ? most : np;
            n += np;
        }
        const int64_t gx = (most + THR - 1) / THR;
        hipLaunchKernelGGL(k_grad_pieces, dim3((unsigned)(gx < 1024 ? gx : 1024), t.count ? t.count : 1), dim3(THR), 0, st, t, list);
    } while (i < ntensors);
    *pieces = n;
    return hipGetLastError() == hipSuccess ? SSD_OK : SSD_ERR_LAUNCH;
}

extern "C" int ssd_grad_norm(void* plan, int64_t pieces, double* sum_sq, void* hip_stream) {
    if (!plan || !sum_sq) return SSD_ERR_NULL;
    if (pieces < 0 || !al(sum_sq, 8) || !al(plan, 256)) return SSD_ERR_ARG;
    hipStream_t st = (hipStream_t)hip_stream;
    launch_squares(plan, pieces, st);
    hipLaunchKernelGGL(k_grad_sum, dim3(1), dim3(THR), 0, st, (const double*)plan, (int)wgs_of(pieces, NORM_WGS), sum_sq);
    return hipGetLastError() == hipSuccess ? SSD_OK : SSD_ERR_LAUNCH;
}

extern "C" int ssd_grad_clip(void* plan, int64_t pieces, const double* sum_sq, float max_norm, float* norm, void* hip_stream) {
    if (!plan) return SSD_ERR_NULL;
    if (pieces < 0 || !al(sum_sq, 8) || !al(norm, 4) || !al(plan, 256) || !(max_norm >= 0.f)) return SSD_ERR_ARG;
    hipStream_t st = (hipStream_t)hip_stream;
    if (!sum_sq && pieces <= SOLO_PIECES) {
        hipLaunchKernelGGL(k_grad_solo, dim3(1), dim3(SOLO_THR), 0, st, (const Piece*)((Head*)plan + 1), (int)pieces, max_norm, norm);
        return hipGetLastError() == hipSuccess ? SSD_OK : SSD_ERR_LAUNCH;
    }
    if (!sum_sq) launch_squares(plan, pieces, st);
    const bool stream = pieces > STREAM_PIECES;
    hipLaunchKernelGGL(stream ? k_grad_clip<true> : k_grad_clip<false>, dim3(wgs_of(pieces, CLIP_WGS)), dim3(THR), 0, st, (const Piece*)((Head*)plan + 1), pieces, (const double*)plan,
                       (int)wgs_of(pieces, NORM_WGS), sum_sq, max_norm, norm);
    return hipGetLastError() == hipSuccess ? SSD_OK : SSD_ERR_LAUNCH;
}
