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
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int64_t PIECE = 8192;  // elements: a multiple of 16-byte vectors, so that all pieces of a tensor are aligned as it is
constexpr int THR = 256, MAX_WGS = 2048;

// Device memory of a plan: the counter of finished workgroups, their sums of squares, then the pieces.
struct Piece {
    const void* src;
    void* dst;
    int n, kind;  // kind: bit 0 source bf16, bit 1 result bf16, bit 2 both on 16 bytes
    int pad[2];
};
struct Head {
    unsigned int done;
    unsigned int pad[63];
    double part[MAX_WGS];
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

__global__ __launch_bounds__(THR) void k_grad_pieces(Tensors t, Piece* pieces, Head* head) {
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) head->done = 0;
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

__device__ __forceinline__ double block_total(double v, double* lds) {  // in thread 0
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

template <bool BF16>
__device__ __forceinline__ double piece_squares(const Piece& p) {
    double s = 0.0;
    constexpr int V = BF16 ? 8 : 4;
    int i0 = 0;
    if (p.kind & 4) {
        const int nv = p.n / V;
        for (int v = threadIdx.x; v < nv; v += THR) {
            if (BF16) {
                const bf16x8 x = ((const bf16x8*)p.src)[v];
#pragma unroll
                for (int e = 0; e < 8; ++e) s += square((float)x[e]);
            } else {
                const f32x4 x = ((const f32x4*)p.src)[v];
#pragma unroll
                for (int e = 0; e < 4; ++e) s += square(x[e]);
            }
        }
        i0 = nv * V;
    }
    for (int i = i0 + threadIdx.x; i < p.n; i += THR) s += square(BF16 ? (float)((const __bf16*)p.src)[i] : ((const float*)p.src)[i]);
    return s;
}

// The workgroup that finishes last adds up the sums of all: their order is that of the workgroups, whoever is last.
__global__ __launch_bounds__(THR) void k_grad_norm(const Piece* pieces, int64_t count, Head* head, double* sum_sq) {
    __shared__ double lds[4];
    __shared__ int last;
    double s = 0.0;
    for (int64_t k = blockIdx.x; k < count; k += gridDim.x) {
        const Piece p = pieces[k];
        s += p.kind & 1 ? piece_squares<true>(p) : piece_squares<false>(p);
    }
    s = block_total(s, lds);
    if (threadIdx.x == 0) {
        __hip_atomic_store(&head->part[blockIdx.x], s, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        const unsigned int before = __hip_atomic_fetch_add(&head->done, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT);
        last = before == gridDim.x - 1;
    }
    __syncthreads();
    if (!last) return;
    s = 0.0;
    for (int i = threadIdx.x; i < (int)gridDim.x; i += THR) s += __hip_atomic_load(&head->part[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    s = block_total(s, lds);
    if (threadIdx.x == 0) {
        *sum_sq = s;
        head->done = 0;  // for the next call
    }
}

template <bool FROM, bool TO>
__device__ __forceinline__ void scale_piece(const Piece& p, float c) {
    int i0 = 0;
    if (p.kind & 4) {
        const int nv = p.n / 8;
        for (int v = threadIdx.x; v < nv; v += THR) {
            float f[8];
            if (FROM) {
                const bf16x8 x = ((const bf16x8*)p.src)[v];
#pragma unroll
                for (int e = 0; e < 8; ++e) f[e] = (float)x[e];
            } else {
                const f32x4 x0 = ((const f32x4*)p.src)[2 * v], x1 = ((const f32x4*)p.src)[2 * v + 1];
#pragma unroll
                for (int e = 0; e < 4; ++e) f[e] = x0[e], f[4 + e] = x1[e];
            }
            if (TO) {
                bf16x8 o;
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e] = (__bf16)(f[e] * c);
                ((bf16x8*)p.dst)[v] = o;
            } else {
                f32x4 o0, o1;
#pragma unroll
                for (int e = 0; e < 4; ++e) o0[e] = f[e] * c, o1[e] = f[4 + e] * c;
                ((f32x4*)p.dst)[2 * v] = o0;
                ((f32x4*)p.dst)[2 * v + 1] = o1;
            }
        }
        i0 = nv * 8;
    }
    for (int i = i0 + threadIdx.x; i < p.n; i += THR) {
        const float v = (FROM ? (float)((const __bf16*)p.src)[i] : ((const float*)p.src)[i]) * c;
        if (TO) ((__bf16*)p.dst)[i] = (__bf16)v;
        else ((float*)p.dst)[i] = v;
    }
}

// The pieces in reverse: what the norm read last is still in the last-level cache.  The factor is worked out in fp64 and rounded once;
// a NaN in it stays one.  A gradient that is its own result and needs no scaling is left alone.
__global__ __launch_bounds__(THR) void k_grad_clip(const Piece* pieces, int64_t count, const double* sum_sq, float max_norm, float* norm) {
    const double n = sqrt(*sum_sq), by = (double)max_norm / (n + 1e-6);
    const float c = by > 1.0 ? 1.f : (float)by;
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)n;
    for (int64_t k = count - 1 - blockIdx.x; k >= 0; k -= gridDim.x) {
        const Piece p = pieces[k];
        if (p.src == p.dst && c == 1.f) continue;
        switch (p.kind & 3) {
            case 0: scale_piece<false, false>(p, c); break;
            case 1: scale_piece<true, false>(p, c); break;
            case 2: scale_piece<false, true>(p, c); break;
            default: scale_piece<true, true>(p, c);
        }
    }
}

bool al(const void* p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
int64_t pieces_of(int64_t numel) { return (numel + PIECE - 1) / PIECE; }
unsigned wgs_of(int64_t pieces) { return (unsigned)(pieces < 1 ? 1 : pieces < MAX_WGS ? pieces : MAX_WGS); }
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
        hipLaunchKernelGGL(k_grad_pieces, dim3((unsigned)(gx < 1024 ? gx : 1024), t.count ? t.count : 1), dim3(THR), 0, st, t, list, head);
    } while (i < ntensors);
    *pieces = n;
    return hipGetLastError() == hipSuccess ? SSD_OK : SSD_ERR_LAUNCH;
}

extern "C" int ssd_grad_norm(void* plan, int64_t pieces, double* sum_sq, void* hip_stream) {
    if (!plan || !sum_sq) return SSD_ERR_NULL;
    if (pieces < 0 || !al(sum_sq, 8) || !al(plan, 256)) return SSD_ERR_ARG;
    Head* head = (Head*)plan;
    hipLaunchKernelGGL(k_grad_norm, dim3(wgs_of(pieces)), dim3(THR), 0, (hipStream_t)hip_stream, (const Piece*)(head + 1), pieces, head, sum_sq);
    return hipGetLastError() == hipSuccess ? SSD_OK : SSD_ERR_LAUNCH;
}

extern "C" int ssd_grad_clip(void* plan, int64_t pieces, const double* sum_sq, float max_norm, float* norm, void* hip_stream) {
    if (!plan || !sum_sq) return SSD_ERR_NULL;
    if (pieces < 0 || !al(sum_sq, 8) || !al(norm, 4) || !al(plan, 256) || !(max_norm >= 0.f)) return SSD_ERR_ARG;
    hipLaunchKernelGGL(k_grad_clip, dim3(wgs_of(pieces)), dim3(THR), 0, (hipStream_t)hip_stream, (const Piece*)((Head*)plan + 1), pieces, sum_sq, max_norm, norm);
    return hipGetLastError() == hipSuccess ? SSD_OK : SSD_ERR_LAUNCH;
}
