// The join of a block's output f with the residual stream x around it, and dropout alone:
//     u = f rstd_f post_w     v = dropout(u)     s = alpha x + gate v     out = s rstd_s pre_w          rstd = 1 / sqrt(mean of squares + eps)
// Backward from s and f:
//     t  = ds + rstd_s (dout pre_w - s rstd_s mean(dout pre_w s rstd_s))
//     dx = alpha t      dalpha = sum t x      dgate = sum t v      du = mask gate t
//     df = rstd_f (du post_w - f rstd_f mean(du post_w f rstd_f))      dpost_w = sum du f rstd_f      dpre_w = sum dout s rstd_s
#include <math.h>
#include <string.h>

#include <initializer_list>

#include "column_sums.h"
#include "philox.h"

namespace ssdk {
namespace {

enum { SLOT_POST, SLOT_PRE, SLOT_ALPHA, SLOT_HEAD, SLOT_TAIL, SLOTS };

struct JoinParams {
    const void *x, *f, *s, *dout, *ds;
    void *s_out, *out, *dx, *df;
    const float *post_w, *gate, *alpha, *pre_w;
    float *dpost_w, *dgate, *dalpha, *dpre_w;
    float *part, *stat;  // [parts][SLOTS][dim] sums of the rows of a part; [rows][4] 1/rms and means of each row (struct Row)
    int64_t rows, gate_rows, s_rs, f_rs, o_rs, part_rows, groups;  // groups: eights of a row
    DropJob drop;
    int dim, parts, accumulate;
    float eps;
};

// The sum over a workgroup of 256 threads, in every thread.
__device__ __forceinline__ float block_sum(float v, float* lds) {
    v = wave_total(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

// A row in memory: a descriptor that ends with it, so that lanes behind its end read zeros and write nothing without a branch.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t row_at(const void* p, int64_t first, int dim, int size) {
    return __builtin_amdgcn_make_buffer_rsrc((char*)p + first * size, 0, dim * size, 0x00020000);
}
// Eight consecutive values of a row, zeros behind its end.  VEC: the row is a whole number of eights and lies on 16 bytes.  Else they lie at whatever
// address, and who reaches behind the row's end loads its last eight, which settle() moves into place: it waits for them, so it comes where
// they are used (20000 rows of 2561, bf16, forward and backward: element by element 697 us, the end alone element by element 395, this 378).
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_any __attribute__((aligned(2)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef u32x2 u32x2_any __attribute__((aligned(2)));
typedef unsigned int u32_any __attribute__((aligned(2)));
template <typename T>
struct Eight;
template <>
struct Eight<bf16_t> {
    bf16x8 v;
    template <bool VEC>
    __device__ __forceinline__ void load(const void* p, int64_t first, int dim, int c0) {
        if (VEC) {
            v = __builtin_bit_cast(bf16x8, __builtin_amdgcn_raw_buffer_load_b128(row_at(p, first, dim, 2), c0 * 2, 0, 0));
        } else if (dim >= 8) {
            v = __builtin_bit_cast(bf16x8, *(const u32x4_any*)((const __bf16*)p + first + min(c0, dim - 8)));
        } else {
            v = bf16x8{};
#pragma unroll
            for (int e = 0; e < 7; ++e)
                if (c0 + e < dim) v[e] = ((const __bf16*)p)[first + c0 + e];
        }
    }
    template <bool VEC>
    __device__ __forceinline__ void settle(int dim, int c0) {
        if (VEC || dim < 8 || c0 + 8 <= dim) return;
        const int by = c0 + 8 - dim;
        u32x4 d = __builtin_bit_cast(u32x4, v);
        if (by & 4) d = u32x4{d[2], d[3], 0, 0};
        if (by & 2) d = u32x4{d[1], d[2], d[3], 0};
        if (by & 1) d = u32x4{d[0] >> 16 | d[1] << 16, d[1] >> 16 | d[2] << 16, d[2] >> 16 | d[3] << 16, d[3] >> 16};
        if (by >= 8) d = u32x4{};
        v = __builtin_bit_cast(bf16x8, d);
    }
    template <bool VEC>
    __device__ __forceinline__ void store(void* p, int64_t first, int dim, int c0) const {
        u32x4 d = __builtin_bit_cast(u32x4, v);
        if (VEC) {
            __builtin_amdgcn_raw_buffer_store_b128(d, row_at(p, first, dim, 2), c0 * 2, 0, 0);
            return;
        }
        __bf16* q = (__bf16*)p + first + c0;
        const int n = dim - c0;
        if (n >= 8) {
            *(u32x4_any*)q = d;
        } else if (n > 0) {
            if (n & 4) *(u32x2_any*)q = u32x2{d[0], d[1]}, q += 4, d[0] = d[2], d[1] = d[3];
            if (n & 2) *(u32_any*)q = d[0], q += 2, d[0] = d[1];
            if (n & 1) *(unsigned short*)q = (unsigned short)d[0];
        }
    }
    __device__ __forceinline__ void fetch(const void* p, int64_t first, int dim, int c0) { load<false>(p, first, dim, c0), settle<false>(dim, c0); }
    __device__ __forceinline__ float get(int e) const { return (float)v[e]; }
    __device__ __forceinline__ void set(int e, float f) { v[e] = (__bf16)f; }
};
template <>
struct Eight<float> {
    u32x4 v[2];
    template <bool VEC>
    __device__ __forceinline__ void load(const void* p, int64_t first, int dim, int c0) {
        if (VEC) {
            const __amdgpu_buffer_rsrc_t q = row_at(p, first, dim, 4);
            v[0] = __builtin_amdgcn_raw_buffer_load_b128(q, c0 * 4, 0, 0);
            v[1] = __builtin_amdgcn_raw_buffer_load_b128(q, c0 * 4 + 16, 0, 0);
        } else if (dim >= 8) {
            const u32x4_any* const q = (const u32x4_any*)((const float*)p + first + min(c0, dim - 8));
            v[0] = q[0];
            v[1] = q[1];
        } else {
            v[0] = v[1] = u32x4{};
#pragma unroll
            for (int e = 0; e < 7; ++e)
                if (c0 + e < dim) set(e, ((const float*)p)[first + c0 + e]);
        }
    }
    template <bool VEC>
    __device__ __forceinline__ void settle(int dim, int c0) {
        if (VEC || dim < 8 || c0 + 8 <= dim) return;
        const int by = c0 + 8 - dim;
        if (by & 4) v[0] = v[1], v[1] = u32x4{};
        if (by & 2) v[0] = u32x4{v[0][2], v[0][3], v[1][0], v[1][1]}, v[1] = u32x4{v[1][2], v[1][3], 0, 0};
        if (by & 1) v[0] = u32x4{v[0][1], v[0][2], v[0][3], v[1][0]}, v[1] = u32x4{v[1][1], v[1][2], v[1][3], 0};
        if (by >= 8) v[0] = v[1] = u32x4{};
    }
    template <bool VEC>
    __device__ __forceinline__ void store(void* p, int64_t first, int dim, int c0) const {
        if (VEC) {
            const __amdgpu_buffer_rsrc_t q = row_at(p, first, dim, 4);
            __builtin_amdgcn_raw_buffer_store_b128(v[0], q, c0 * 4, 0, 0);
            __builtin_amdgcn_raw_buffer_store_b128(v[1], q, c0 * 4 + 16, 0, 0);
            return;
        }
        float* q = (float*)p + first + c0;
        const int n = dim - c0;
        if (n >= 8) {
            ((u32x4_any*)q)[0] = v[0];
            ((u32x4_any*)q)[1] = v[1];
        } else if (n > 0) {
            u32x4 d = v[0];
            if (n & 4) *(u32x4_any*)q = d, q += 4, d = v[1];
            if (n & 2) *(u32x2_any*)q = u32x2{d[0], d[1]}, q += 2, d[0] = d[2];
            if (n & 1) *(u32_any*)q = d[0];
        }
    }
    __device__ __forceinline__ void fetch(const void* p, int64_t first, int dim, int c0) { load<false>(p, first, dim, c0), settle<false>(dim, c0); }
    __device__ __forceinline__ float get(int e) const { return __uint_as_float(v[e >> 2][e & 3]); }
    __device__ __forceinline__ void set(int e, float f) { v[e >> 2][e & 3] = __float_as_uint(f); }
};
template <typename T>
__device__ __forceinline__ void zero(Eight<T>& v) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v.set(e, 0.f);
}
// Eight values of a parameter, ones where there is none; without a branch, so that several are asked for at once.
template <bool VEC>
__device__ __forceinline__ void parameter(float (&w)[8], const float* p, int64_t first, int dim, int c0) {
    Eight<float> v;
    v.load<VEC>(p, p ? first : 0, p ? dim : 0, c0);  // no bytes where there is none
    v.settle<VEC>(p ? dim : 0, c0);
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = p ? v.get(e) : 1.f;
}

constexpr int MAX_WAVES = 16;
constexpr int AHEAD_DIM = 8 * 512;        // up to here the backward kernel may have the next row beside the present one
constexpr int ROW_DIM = MAX_WAVES * 512;  // the widest row that a workgroup holds in registers, eight values a thread

// Whether that row finds registers: not beside what settle() needs, nor in 128 of them where all is fp32 and dropped (20000 rows of 2560: 434 us, with
// the next row, which spills, 468; a bf16 stream 240 with it).
template <typename TS, typename TF, bool VEC, bool DROP, bool ALPHA>
constexpr bool ROOM = VEC && (sizeof(TS) + sizeof(TF) < 8 || !DROP || ALPHA);

// Sums of K values over the workgroup, in every thread, with one barrier: `side` alternates between two halves of the exchange, so that a wave
// that is ahead writes where none still reads.  Each row of sixteen lanes takes the waves' sums, one a lane, and adds them by rotations: pairs
// are added in both orders, so every lane gets the same bits.
template <int K>
struct RowLds {
    float v[2][MAX_WAVES][K];
};
template <int CTRL>
__device__ __forceinline__ float rotate_add(float v) {
    return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}
template <int K>
__device__ __forceinline__ void row_sums(RowLds<K>& L, float (&s)[K], int waves, int& side) {
#pragma unroll
    for (int k = 0; k < K; ++k) s[k] = wave_total(s[k]);
    if (waves == 1) return;
    const int lane = threadIdx.x & 63;
    if (lane == 0)
#pragma unroll
        for (int k = 0; k < K; ++k) L.v[side][threadIdx.x >> 6][k] = s[k];
    __syncthreads();
    const int w = lane & 15;
#pragma unroll
    for (int k = 0; k < K; ++k) s[k] = L.v[side][w][k];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        s[k] = w < waves ? s[k] : 0.f;
        s[k] = rotate_add<0x128>(s[k]);  // row_ror:8, 4, 2, 1
        s[k] = rotate_add<0x124>(s[k]);
        s[k] = rotate_add<0x122>(s[k]);
        s[k] = rotate_add<0x121>(s[k]);
    }
    side ^= 1;
}

__device__ __forceinline__ uint32_t keep_bits(const DropJob& d, uint64_t seed, uint64_t offset, int64_t number) {  // bit e: element e stays
    const PhiloxWords w = philox((uint64_t)(d.first + number), offset, seed);
    uint32_t k = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) k |= (philox_bits(w, e) >= d.drop ? 1u : 0u) << e;
    return k;
}

// Rows of up to ROW_DIM values: as many waves as it takes hold a row, eight values a thread, and walk the rows of a part one after
// another, the next one under way while this one is worked on.  No branch hides a store, so that a row's wait
// is for its loads and not for the stores behind them (with branches around them 300 us).  Parameters stay in registers (the gate until it
// changes).  65536 rows of 2560, bf16, dropout: 224 us (1.34 GB, 6.0 TB/s).
template <typename TS, typename TF, bool VEC, bool DROP, bool, bool>  // the last two are the backward kernel's
__global__ __launch_bounds__(64 * MAX_WAVES) void k_join_fwd(JoinParams jp) {
    __shared__ RowLds<1> L;
    const int waves = blockDim.x >> 6, c0 = threadIdx.x * 8, dim = jp.dim;
    const DropJob d = jp.drop;
    const uint64_t seed = DROP ? d.rng[0] : 0, offset = DROP ? d.rng[1] : 0;
    const float inv = 1.f / (float)dim;
    const int64_t r0 = blockIdx.x * jp.part_rows, r1 = r0 + jp.part_rows < jp.rows ? r0 + jp.part_rows : jp.rows;
    int64_t gate_end = (r0 / jp.gate_rows + 1) * jp.gate_rows;  // the first row that the gate in registers is not for
    int side = 0;
    struct In {
        Eight<TS> x;
        Eight<TF> f;
    };
    auto load = [&](In& v, int64_t r) {
        v.x.template load<VEC>(jp.x, r * jp.s_rs, dim, c0);
        v.f.template load<VEC>(jp.f, r * jp.f_rs, dim, c0);
    };
    In next;
    load(next, r0);
    float post[8], alpha[8], pre[8], gate[8];
    parameter<VEC>(post, jp.post_w, 0, dim, c0);
    parameter<VEC>(gate, jp.gate, r0 / jp.gate_rows * dim, dim, c0);
    parameter<VEC>(alpha, jp.alpha, 0, dim, c0);
    parameter<VEC>(pre, jp.pre_w, 0, dim, c0);
    auto row = [&](const In& v, int64_t r) {
        if (r == gate_end) {
            parameter<VEC>(gate, jp.gate, gate_end / jp.gate_rows * dim, dim, c0);
            gate_end += jp.gate_rows;
        }
        const uint32_t keep = DROP ? keep_bits(d, seed, offset, r * jp.groups + threadIdx.x) : 0;
        float rstd_f = 1.f;
        if (jp.post_w) {
            float s[1] = {0.f};
#pragma unroll
            for (int e = 0; e < 8; ++e) s[0] = fmaf(v.f.get(e), v.f.get(e), s[0]);
            row_sums(L, s, waves, side);
            rstd_f = rsqrtf(s[0] * inv + jp.eps);
        }
        Eight<TS> x;
        float s[1] = {0.f};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float u = v.f.get(e) * rstd_f * post[e];
            if (DROP) u = keep >> e & 1 ? u * d.scale : 0.f;
            x.set(e, fmaf(gate[e], u, alpha[e] * v.x.get(e)));
            s[0] = fmaf(x.get(e), x.get(e), s[0]);  // zeros behind the row's end
        }
        x.template store<VEC>(jp.s_out, r * jp.s_rs, dim, c0);
        if (!jp.pre_w) return;
        row_sums(L, s, waves, side);
        const float rstd = rsqrtf(s[0] * inv + jp.eps);
        Eight<TF> o;
#pragma unroll
        for (int e = 0; e < 8; ++e) o.set(e, x.get(e) * rstd * pre[e]);
        o.template store<VEC>(jp.out, r * jp.o_rs, dim, c0);
    };
    for (int64_t r = r0; r < r1; ++r) {
        In v = next;
        load(next, r + 1 < r1 ? r + 1 : r);
        v.x.template settle<VEC>(dim, c0);
        v.f.template settle<VEC>(dim, c0);
        row(v, r);
    }
}

// Backward.  The mean of du post_w f rstd_f is that of three terms of t, whose factors are known once the row's sums are, so that one
// exchange between the waves does: with k = mask gate post_w f rstd_f (rstd_f taken out of the sum)
//     sum k t = sum k ds + rstd_s sum k dout pre_w - rstd_s^2 ms sum k s
// Parameters lie in LDS, each thread's own, since registers decide how many rows a compute unit has under way: three workgroups of five
// waves (128 registers).  AHEAD: the next row comes in while this one is worked on.  65536 rows of 2560, bf16, dropout, three parameters: 453 us
// (2.0 GB, 4.4 TB/s).  When it was chosen, on another card: 486, without AHEAD 509; two workgroups of 146 registers, AHEAD, 676.
template <typename TS, typename TF, bool VEC, bool DROP, bool ALPHA, bool AHEAD>
__global__ __launch_bounds__(AHEAD ? 512 : 64 * MAX_WAVES, AHEAD && ALPHA ? 3 : 4) void k_join_bwd(JoinParams jp) {
    __shared__ RowLds<6> L;
    const int waves = blockDim.x >> 6, c0 = threadIdx.x * 8, dim = jp.dim;
    const DropJob d = jp.drop;
    const uint64_t seed = DROP ? d.rng[0] : 0, offset = DROP ? d.rng[1] : 0;
    const float inv = 1.f / (float)dim;
    extern __shared__ f32x4 own[];  // [parameter][half of a thread's eight][thread]
    enum { POST, PRE, GATE, DPOST, FACTOR = DPOST + AHEAD };  // without AHEAD the sums of dpost stay in registers
    auto put = [&](const float (&w)[8], int i) {
        own[(2 * i) * blockDim.x + threadIdx.x] = f32x4{w[0], w[1], w[2], w[3]};
        own[(2 * i + 1) * blockDim.x + threadIdx.x] = f32x4{w[4], w[5], w[6], w[7]};
    };
    auto fetch = [&](float (&w)[8], int i) {
        const f32x4 lo = own[(2 * i) * blockDim.x + threadIdx.x], hi = own[(2 * i + 1) * blockDim.x + threadIdx.x];
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = lo[e], w[4 + e] = hi[e];
    };
    // dgate = post sum mask t fhat and dpost = gate sum mask t fhat for the rows of a gate: one sum does, taken apart where the gate changes
    float dpost[8] = {}, dpre[8] = {}, dalpha[8] = {}, sum[8] = {};
    if (AHEAD) put(dpost, DPOST);
    const int64_t r0 = blockIdx.x * jp.part_rows, r1 = r0 + jp.part_rows < jp.rows ? r0 + jp.part_rows : jp.rows;
    auto store_sums = [&](float* p, int64_t first, const float (&s)[8], bool add) {
        Eight<float> v;
        zero(v);
        if (add) {
            v.template load<VEC>(p, first, dim, c0);
            v.template settle<VEC>(dim, c0);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) v.set(e, v.get(e) + s[e]);
        v.template store<VEC>(p, first, dim, c0);
    };
    int64_t gate_begin = r0 / jp.gate_rows * jp.gate_rows, gate_end = gate_begin + jp.gate_rows;
    int side = 0;
    struct In {
        Eight<TS> s, ds, x;
        Eight<TF> f, dout;
    };
    auto load = [&](In& v, int64_t r) {
        v.f.template load<VEC>(jp.f, r * jp.f_rs, dim, c0);
        if (jp.pre_w) {
            v.s.template load<VEC>(jp.s, r * jp.s_rs, dim, c0);
            v.dout.template load<VEC>(jp.dout, r * jp.o_rs, dim, c0);
        } else {
            zero(v.s), zero(v.dout);
        }
        if (jp.ds) v.ds.template load<VEC>(jp.ds, r * jp.s_rs, dim, c0);
        else zero(v.ds);
        if (ALPHA) {
            if (jp.dalpha) v.x.template load<VEC>(jp.x, r * jp.s_rs, dim, c0);
            else zero(v.x);
        }
    };
    auto settle = [&](In& v) {  // what was not loaded holds zeros
        v.f.template settle<VEC>(dim, c0);
        v.s.template settle<VEC>(dim, c0);
        v.dout.template settle<VEC>(dim, c0);
        v.ds.template settle<VEC>(dim, c0);
        if (ALPHA) v.x.template settle<VEC>(dim, c0);
    };
    In next;
    if (AHEAD) load(next, r0);
    {
        float w[4][8];
        parameter<VEC>(w[0], jp.post_w, 0, dim, c0);
        parameter<VEC>(w[1], jp.pre_w, 0, dim, c0);
        parameter<VEC>(w[2], jp.gate, r0 / jp.gate_rows * dim, dim, c0);
        if (ALPHA) parameter<VEC>(w[3], jp.alpha, 0, dim, c0);
        put(w[0], POST);
        put(w[1], PRE);
        put(w[2], GATE);
        if (ALPHA) put(w[3], FACTOR);
    }
    auto row = [&](const In& v, int64_t r) {
        if (r == gate_end) {
            float w[8];
            gate_begin = gate_end;
            gate_end += jp.gate_rows;
            parameter<VEC>(w, jp.gate, gate_begin / jp.gate_rows * dim, dim, c0);
            put(w, GATE);
        }
        const uint32_t keep = DROP ? keep_bits(d, seed, offset, r * jp.groups + threadIdx.x) : 0;
        float s[6] = {};
        float post[8], pre[8], gate[8], alpha[8];
        fetch(post, POST);
        fetch(pre, PRE);
        fetch(gate, GATE);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float f = v.f.get(e), y = v.s.get(e), g = v.dout.get(e) * pre[e];
            const float kf = !DROP ? gate[e] * post[e] * f : keep >> e & 1 ? d.scale * gate[e] * post[e] * f : 0.f;
            s[0] = fmaf(f, f, s[0]);
            s[1] = fmaf(y, y, s[1]);
            s[2] = fmaf(g, y, s[2]);
            s[3] = fmaf(kf, v.ds.get(e), s[3]);
            s[4] = fmaf(kf, g, s[4]);
            s[5] = fmaf(kf, y, s[5]);
        }
        row_sums(L, s, waves, side);
        const float rstd_f = jp.post_w ? rsqrtf(s[0] * inv + jp.eps) : 1.f;
        const float rstd_s = jp.pre_w ? rsqrtf(s[1] * inv + jp.eps) : 0.f;
        const float ms = s[2] * inv * rstd_s;
        float mf = jp.post_w ? (s[3] + rstd_s * (s[4] - rstd_s * ms * s[5])) * inv * rstd_f : 0.f;
        // Where ds or dout of a dropped element is not finite, k = 0 times that is no number, though nothing of it enters the mean: there the mean is taken of
        // its own terms.  Every thread of the row has the same mf.
        if (DROP && jp.post_w && !(fabsf(__builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, mf)))) < INFINITY)) {
            float own_terms[6] = {};
            fetch(post, POST);
            fetch(pre, PRE);
            fetch(gate, GATE);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float t = v.ds.get(e) + rstd_s * (v.dout.get(e) * pre[e] - v.s.get(e) * rstd_s * ms);
                if (keep >> e & 1) own_terms[0] = fmaf(d.scale * gate[e] * t * post[e], v.f.get(e), own_terms[0]);
            }
            row_sums(L, own_terms, waves, side);
            mf = own_terms[0] * inv * rstd_f;
        }
        Eight<TS> dx;
        Eight<TF> df;
        fetch(post, POST);
        fetch(pre, PRE);
        fetch(gate, GATE);
        if (ALPHA) fetch(alpha, FACTOR);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float fhat = v.f.get(e) * rstd_f, shat = v.s.get(e) * rstd_s, g = v.dout.get(e);
            const float t = v.ds.get(e) + rstd_s * (g * pre[e] - shat * ms);
            const float mt = !DROP ? t : keep >> e & 1 ? d.scale * t : 0.f, du = gate[e] * mt;
            dx.set(e, ALPHA ? alpha[e] * t : t);
            df.set(e, jp.post_w ? rstd_f * (du * post[e] - fhat * mf) : du);  // f itself is not read without a norm
            sum[e] = !DROP || (keep >> e & 1) ? fmaf(mt, fhat, sum[e]) : sum[e];
            dpre[e] = fmaf(g, shat, dpre[e]);
            if (ALPHA) dalpha[e] = fmaf(t, v.x.get(e), dalpha[e]);
        }
        dx.template store<VEC>(jp.dx, r * jp.s_rs, dim, c0);
        df.template store<VEC>(jp.df, r * jp.f_rs, dim, c0);
        if (r + 1 == gate_end || r + 1 == r1) {
            const bool before = gate_begin < r0, behind = gate_end > r + 1 && r + 1 < jp.rows;
            float dgate[8];
            fetch(post, POST);
            fetch(gate, GATE);
            if (AHEAD) fetch(dpost, DPOST);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                dgate[e] = post[e] * sum[e];
                dpost[e] = fmaf(gate[e], sum[e], dpost[e]);
                sum[e] = 0.f;
            }
            if (AHEAD) put(dpost, DPOST);
            if (jp.dgate) {
                if (before || behind) store_sums(jp.part, ((int64_t)blockIdx.x * SLOTS + (before ? SLOT_HEAD : SLOT_TAIL)) * dim, dgate, false);
                else store_sums(jp.dgate, gate_begin / jp.gate_rows * dim, dgate, jp.accumulate);
            }
        }
    };
    for (int64_t r = r0; r < r1; ++r) {
        In v;
        if (AHEAD) {
            v = next;
            load(next, r + 1 < r1 ? r + 1 : r);
        } else {
            load(v, r);
        }
        if (!VEC) settle(v);
        row(v, r);
    }
    const int64_t part = (int64_t)blockIdx.x * SLOTS * dim;
    if (AHEAD) fetch(dpost, DPOST);
    if (jp.dpost_w) store_sums(jp.part, part + SLOT_POST * dim, dpost, false);
    if (jp.dpre_w) store_sums(jp.part, part + SLOT_PRE * dim, dpre, false);
    if (ALPHA && jp.dalpha) store_sums(jp.part, part + SLOT_ALPHA * dim, dalpha, false);
}

// Rows wider than that: a workgroup a row, eights in turn, the row read again for every sum that needs the one before (20000 rows of 10240,
// bf16, forward and backward: 1695 us, 2.4 TB/s of what has to be moved; with a residual scale, on another card, 1970, element by element 6344).
template <typename TS, typename TF>
__global__ __launch_bounds__(256) void k_join_fwd_wide(JoinParams jp) {
    __shared__ float lds[4];
    const DropJob d = jp.drop;
    const uint64_t seed = d.drop ? d.rng[0] : 0, offset = d.drop ? d.rng[1] : 0;
    const float inv = 1.f / (float)jp.dim;
    const int dim = jp.dim;
    for (int64_t r = blockIdx.x; r < jp.rows; r += gridDim.x) {
        float rstd_f = 1.f, q = 0.f;
        if (jp.post_w) {
            for (int c0 = threadIdx.x * 8; c0 < dim; c0 += 256 * 8) {
                Eight<TF> f;
                f.fetch(jp.f, r * jp.f_rs, dim, c0);
#pragma unroll
                for (int e = 0; e < 8; ++e) q = fmaf(f.get(e), f.get(e), q);
            }
            rstd_f = rsqrtf(block_sum(q, lds) * inv + jp.eps);
        }
        q = 0.f;
        for (int c0 = threadIdx.x * 8; c0 < dim; c0 += 256 * 8) {
            Eight<TF> f;
            Eight<TS> x;
            float post[8], alpha[8], gate[8];
            f.fetch(jp.f, r * jp.f_rs, dim, c0);
            x.fetch(jp.x, r * jp.s_rs, dim, c0);
            parameter<false>(post, jp.post_w, 0, dim, c0);
            parameter<false>(alpha, jp.alpha, 0, dim, c0);
            parameter<false>(gate, jp.gate, r / jp.gate_rows * dim, dim, c0);
            const uint32_t keep = d.drop ? keep_bits(d, seed, offset, r * jp.groups + (c0 >> 3)) : 0xff;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float u = f.get(e) * rstd_f * post[e], v = keep >> e & 1 ? u * d.scale : 0.f;
                x.set(e, fmaf(gate[e], v, alpha[e] * x.get(e)));
                q = fmaf(x.get(e), x.get(e), q);
            }
            x.template store<false>(jp.s_out, r * jp.s_rs, dim, c0);
        }
        if (!jp.pre_w) continue;
        const float rstd = rsqrtf(block_sum(q, lds) * inv + jp.eps);
        for (int c0 = threadIdx.x * 8; c0 < dim; c0 += 256 * 8) {
            Eight<TS> s;
            Eight<TF> o;
            float pre[8];
            s.fetch(jp.s_out, r * jp.s_rs, dim, c0);  // a thread's own
            parameter<false>(pre, jp.pre_w, 0, dim, c0);
#pragma unroll
            for (int e = 0; e < 8; ++e) o.set(e, s.get(e) * rstd * pre[e]);
            o.template store<false>(jp.out, r * jp.o_rs, dim, c0);
        }
    }
}

// Eight elements of the backward pass, from the row's four numbers.
struct Row {
    float rstd_f, rstd_s, ms, mf;
};
struct Elems {
    float t[8], du[8], v[8], fhat[8], shat[8], dout[8], post[8];
    uint32_t keep;  // bit e: element e stays
};
template <typename TS, typename TF>
__device__ __forceinline__ void join_elements(Elems& o, const JoinParams& jp, const Row& w, uint64_t seed, uint64_t offset, int64_t r, int c0) {
    const int dim = jp.dim;
    Eight<TS> ds, s;
    Eight<TF> f, dout;
    float pre[8], gate[8];
    zero(ds), zero(s), zero(dout);
    f.fetch(jp.f, r * jp.f_rs, dim, c0);
    if (jp.ds) ds.fetch(jp.ds, r * jp.s_rs, dim, c0);
    if (jp.pre_w) {
        dout.fetch(jp.dout, r * jp.o_rs, dim, c0);
        s.fetch(jp.s, r * jp.s_rs, dim, c0);
    }
    parameter<false>(pre, jp.pre_w, 0, dim, c0);
    parameter<false>(o.post, jp.post_w, 0, dim, c0);
    parameter<false>(gate, jp.gate, r / jp.gate_rows * dim, dim, c0);
    o.keep = jp.drop.drop ? keep_bits(jp.drop, seed, offset, r * jp.groups + (c0 >> 3)) : 0xff;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const bool on = o.keep >> e & 1;
        o.dout[e] = dout.get(e);
        o.shat[e] = s.get(e) * w.rstd_s;
        o.t[e] = ds.get(e) + w.rstd_s * (o.dout[e] * pre[e] - o.shat[e] * w.ms);
        o.fhat[e] = f.get(e) * w.rstd_f;
        o.du[e] = on ? gate[e] * o.t[e] * jp.drop.scale : 0.f;
        o.v[e] = on ? o.fhat[e] * o.post[e] * jp.drop.scale : 0.f;
    }
}

template <typename TS, typename TF>
__global__ __launch_bounds__(256) void k_join_stats_wide(JoinParams jp) {
    __shared__ float lds[4];
    const uint64_t seed = jp.drop.drop ? jp.drop.rng[0] : 0, offset = jp.drop.drop ? jp.drop.rng[1] : 0;
    const float inv = 1.f / (float)jp.dim;
    const int dim = jp.dim;
    for (int64_t r = blockIdx.x; r < jp.rows; r += gridDim.x) {
        Row w = {1.f, 0.f, 0.f, 0.f};
        float qf = 0.f, qs = 0.f, ps = 0.f;
        for (int c0 = threadIdx.x * 8; c0 < dim; c0 += 256 * 8) {
            Eight<TF> f, dout;
            Eight<TS> s;
            float pre[8];
            zero(f), zero(dout), zero(s);
            if (jp.post_w) f.fetch(jp.f, r * jp.f_rs, dim, c0);
            if (jp.pre_w) {
                s.fetch(jp.s, r * jp.s_rs, dim, c0);
                dout.fetch(jp.dout, r * jp.o_rs, dim, c0);
            }
            parameter<false>(pre, jp.pre_w, 0, dim, c0);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                qf = fmaf(f.get(e), f.get(e), qf);
                qs = fmaf(s.get(e), s.get(e), qs);
                ps = fmaf(dout.get(e) * pre[e], s.get(e), ps);
            }
        }
        if (jp.pre_w) {
            w.rstd_s = rsqrtf(block_sum(qs, lds) * inv + jp.eps);
            w.ms = block_sum(ps, lds) * inv * w.rstd_s;
        }
        if (jp.post_w) {
            w.rstd_f = rsqrtf(block_sum(qf, lds) * inv + jp.eps);
            float p = 0.f;
            for (int c0 = threadIdx.x * 8; c0 < dim; c0 += 256 * 8) {
                Elems o;
                join_elements<TS, TF>(o, jp, w, seed, offset, r, c0);
#pragma unroll
                for (int e = 0; e < 8; ++e) p = fmaf(o.du[e] * o.post[e], o.fhat[e], p);
            }
            w.mf = block_sum(p, lds) * inv;
        }
        if (threadIdx.x == 0) *(Row*)(jp.stat + r * 4) = w;
    }
}

// The sums of a part's rows, a thread eight columns: workgroups along x take columns, along y parts.  A gate whose rows lie inside the part is
// complete; one that began before it or goes on behind it leaves its sum in SLOT_HEAD (it began before) or SLOT_TAIL.
template <typename TS, typename TF>
__global__ __launch_bounds__(64) void k_join_sums_wide(JoinParams jp) {
    const int c0 = (blockIdx.x * 64 + threadIdx.x) * 8, dim = jp.dim;
    if (c0 >= dim) return;
    const uint64_t seed = jp.drop.drop ? jp.drop.rng[0] : 0, offset = jp.drop.drop ? jp.drop.rng[1] : 0;
    const int64_t k = blockIdx.y, r0 = k * jp.part_rows, r1 = r0 + jp.part_rows < jp.rows ? r0 + jp.part_rows : jp.rows;
    const int64_t part = k * SLOTS * dim;
    auto leave = [&](float* p, int64_t first, const float (&s)[8], bool add) {
        Eight<float> v;
        zero(v);
        if (add) v.fetch(p, first, dim, c0);
#pragma unroll
        for (int e = 0; e < 8; ++e) v.set(e, v.get(e) + s[e]);
        v.template store<false>(p, first, dim, c0);
    };
    float post[8] = {}, pre[8] = {}, alpha[8] = {}, gate[8] = {};
    for (int64_t r = r0; r < r1; ++r) {
        Elems o;
        join_elements<TS, TF>(o, jp, *(const Row*)(jp.stat + r * 4), seed, offset, r, c0);
        Eight<TS> x;
        zero(x);
        if (jp.dalpha) x.fetch(jp.x, r * jp.s_rs, dim, c0);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const bool on = o.keep >> e & 1;  // a dropped element adds nothing, whatever f, ds and dout hold
            post[e] = on ? fmaf(o.du[e], o.fhat[e], post[e]) : post[e];
            pre[e] = fmaf(o.dout[e], o.shat[e], pre[e]);
            alpha[e] = fmaf(o.t[e], x.get(e), alpha[e]);
            gate[e] = on ? fmaf(o.t[e], o.v[e], gate[e]) : gate[e];
        }
        if (jp.dgate && (r + 1 == r1 || (r + 1) % jp.gate_rows == 0)) {
            const int64_t q = r / jp.gate_rows;
            const bool before = q * jp.gate_rows < r0, behind = (r + 1) % jp.gate_rows != 0 && r + 1 < jp.rows;
            if (before || behind) leave(jp.part, part + (before ? SLOT_HEAD : SLOT_TAIL) * dim, gate, false);
            else leave(jp.dgate, q * dim, gate, jp.accumulate);
#pragma unroll
            for (int e = 0; e < 8; ++e) gate[e] = 0.f;
        }
    }
    leave(jp.part, part + SLOT_POST * dim, post, false);
    leave(jp.part, part + SLOT_PRE * dim, pre, false);
    leave(jp.part, part + SLOT_ALPHA * dim, alpha, false);
}

template <typename TS, typename TF>
__global__ __launch_bounds__(256) void k_join_bwd_wide(JoinParams jp) {
    const uint64_t seed = jp.drop.drop ? jp.drop.rng[0] : 0, offset = jp.drop.drop ? jp.drop.rng[1] : 0;
    const int dim = jp.dim;
    for (int64_t r = blockIdx.x; r < jp.rows; r += gridDim.x) {
        const Row w = *(const Row*)(jp.stat + r * 4);
        for (int c0 = threadIdx.x * 8; c0 < dim; c0 += 256 * 8) {
            Elems o;
            join_elements<TS, TF>(o, jp, w, seed, offset, r, c0);
            float alpha[8];
            parameter<false>(alpha, jp.alpha, 0, dim, c0);
            Eight<TS> dx;
            Eight<TF> df;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                dx.set(e, alpha[e] * o.t[e]);
                df.set(e, jp.post_w ? w.rstd_f * (o.du[e] * o.post[e] - o.fhat[e] * w.mf) : o.du[e]);
            }
            dx.template store<false>(jp.dx, r * jp.s_rs, dim, c0);
            df.template store<false>(jp.df, r * jp.f_rs, dim, c0);
        }
    }
}

// Adds the parts' sums up: along y the three sums of all rows, then the gates whose rows lie in several parts, found by their number or,
// where there are more gates than parts, by the part behind whose end they go on (each at the part where it begins).  Bound by latency: 3001 rows
// of 1024 (751 parts) 5.9 us, 65536 of 2560 (768) 9.7; sixteen loads in flight 7.9 for 5.9.
__global__ __launch_bounds__(COLSUM_THREADS) void k_join_reduce(JoinParams jp, int by_gate) {
    __shared__ ColsumLds L;
    const int c = blockIdx.x * 64 + (threadIdx.x & 63);
    const bool live = c < jp.dim;
    const int64_t stride = (int64_t)SLOTS * jp.dim;
    float s;
    float* to;
    if (blockIdx.y < 3) {
        to = blockIdx.y == SLOT_POST ? jp.dpost_w : blockIdx.y == SLOT_PRE ? jp.dpre_w : jp.dalpha;
        if (!to) return;
        s = column_sum(L, jp.part + (int64_t)blockIdx.y * jp.dim, jp.parts, stride, c, live);
    } else {
        int64_t k = blockIdx.y - 3, q;  // the gate and the part where it begins
        if (by_gate) {
            q = k;
            k = q * jp.gate_rows / jp.part_rows;
        } else {
            const int64_t edge = (k + 1) * jp.part_rows;
            q = (edge - 1) / jp.gate_rows;
            if (edge % jp.gate_rows == 0 || q * jp.gate_rows < k * jp.part_rows) return;  // ends at the edge, or began in an earlier part
        }
        const int64_t end = (q + 1) * jp.gate_rows < jp.rows ? (q + 1) * jp.gate_rows : jp.rows, last = (end - 1) / jp.part_rows;
        if (last == k) return;  // all in one part, which has written it
        to = jp.dgate + q * jp.dim;
        s = column_sum(L, jp.part + (k + 1) * stride + (int64_t)SLOT_HEAD * jp.dim, last - k, stride, c, live);
        if (threadIdx.x < 64 && live) s += jp.part[k * stride + (int64_t)SLOT_TAIL * jp.dim + c];
    }
    if (threadIdx.x < 64 && live) to[c] = jp.accumulate ? to[c] + s : s;
}

// Dropout alone, a call of the generator and eight values a thread, bound by memory (65536 rows of 5120, bf16: 1.34 GB, 251 us, 5.3 TB/s; an element a
// thread 931).  A workgroup takes 256 consecutive eights; where the first of them lies is worked out once for all.  VEC: rows of whole eights on
// 16 bytes, for bf16 alone: 30000 rows of 2560 forward and backward 125 us, without 131; fp32 232, without 221.
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void k_dropout(const void* x, void* out, int64_t count, int dim, uint32_t groups, int64_t x_rs, int64_t o_rs, DropJob d) {
    const uint64_t seed = d.drop ? d.rng[0] : 0, offset = d.drop ? d.rng[1] : 0;
    for (int64_t n0 = (int64_t)blockIdx.x * 256; n0 < count; n0 += (int64_t)gridDim.x * 256) {
        const int64_t n = n0 + threadIdx.x, first = n0 / groups;
        if (n >= count) return;
        const uint32_t in = (uint32_t)(n0 - first * groups) + threadIdx.x, down = in / groups;
        const int64_t r = first + down;
        const int c0 = (int)(in - down * groups) * 8;
        const uint32_t keep = d.drop ? keep_bits(d, seed, offset, n) : 0xff;
        Eight<T> v;
        if (VEC) v = *(const Eight<T>*)((const T*)x + r * x_rs + c0);
        else v.fetch(x, r * x_rs, dim, c0);
#pragma unroll
        for (int e = 0; e < 8; ++e) v.set(e, keep >> e & 1 ? v.get(e) * d.scale : 0.f);
        if (VEC) *(Eight<T>*)((T*)out + r * o_rs + c0) = v;
        else v.template store<false>(out, r * o_rs, dim, c0);
    }
}

constexpr int64_t MAX_ROWS = (int64_t)1 << 36;
constexpr int MAX_DIM = 1 << 20;
constexpr int64_t MAX_STRIDE = 1 << 24;
constexpr int PARTS_WIDE = 256;

bool al(const void* p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
bool element(int dtype, const void* p) { return al(p, dtype == SSD_BF16 ? 2 : 4); }
size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }
int done() { return hipGetLastError() == hipSuccess ? SSD_OK : SSD_ERR_LAUNCH; }

int check_drop(const ssd_dropout_t* dr, int64_t rows, int64_t groups, DropJob* d) {
    memset(d, 0, sizeof(*d));
    d->scale = 1.f;
    if (!dr) return SSD_OK;
    if (!(dr->p >= 0.f && dr->p <= 1.f)) return SSD_ERR_ARG;
    if (dr->first_row < 0 || dr->first_row > MAX_ROWS) return SSD_ERR_SHAPE;
    const double n = rint((double)dr->p * 65536.0);
    d->drop = (uint32_t)n;
    if (!d->drop) return SSD_OK;
    d->scale = d->drop == 65536u ? 0.f : (float)(65536.0 / (65536.0 - n));
    d->first = dr->first_row * groups;
    d->rng = dr->rng;
    if (!dr->rng) return SSD_ERR_NULL;
    return al(dr->rng, 8) ? SSD_OK : SSD_ERR_ARG;
}

int check(const ssd_join_shape_t* sh, const ssd_join_params_t* pr, const ssd_dropout_t* dr, JoinParams* jp) {
    if (!sh) return SSD_ERR_NULL;
    for (int t : {sh->dtype, sh->stream_dtype})
        if (t != SSD_F32 && t != SSD_BF16) return SSD_ERR_DTYPE;
    if (sh->rows < 0 || sh->rows > MAX_ROWS || sh->dim <= 0 || sh->dim > MAX_DIM || sh->gate_rows < 0) return SSD_ERR_SHAPE;
    if (!(sh->eps >= 0.f) || !(sh->eps <= 3.4e38f)) return SSD_ERR_ARG;
    memset(jp, 0, sizeof(*jp));
    jp->rows = sh->rows;
    jp->dim = sh->dim;
    jp->eps = sh->eps;
    jp->groups = (sh->dim + 7) / 8;
    jp->gate_rows = sh->gate_rows && sh->gate_rows < sh->rows ? sh->gate_rows : sh->rows > 0 ? sh->rows : 1;
    const int64_t given[3] = {sh->stream_row_stride, sh->f_row_stride, sh->out_row_stride};
    int64_t* const to[3] = {&jp->s_rs, &jp->f_rs, &jp->o_rs};
    for (int k = 0; k < 3; ++k) {
        *to[k] = given[k] ? given[k] : sh->dim;
        if (*to[k] < sh->dim || *to[k] > MAX_STRIDE) return SSD_ERR_SHAPE;
    }
    if (pr) jp->post_w = pr->post_w, jp->gate = pr->gate, jp->alpha = pr->alpha, jp->pre_w = pr->pre_w;
    for (const float* p : {jp->post_w, jp->gate, jp->alpha, jp->pre_w})
        if (!al(p, 4)) return SSD_ERR_ARG;
    return check_drop(dr, sh->rows, jp->groups, &jp->drop);
}

// Launches kernel<stream type, type>.
#define JOIN_TYPES(KERNEL, GRID, BLOCK)                                                                                            \
    do {                                                                                                                           \
        const bool sb = sh->stream_dtype == SSD_BF16, fb = sh->dtype == SSD_BF16;                                                  \
        if (sb && fb) hipLaunchKernelGGL((KERNEL<bf16_t, bf16_t>), GRID, BLOCK, 0, st, jp);                                        \
        else if (sb) hipLaunchKernelGGL((KERNEL<bf16_t, float>), GRID, BLOCK, 0, st, jp);                                          \
        else if (fb) hipLaunchKernelGGL((KERNEL<float, bf16_t>), GRID, BLOCK, 0, st, jp);                                          \
        else hipLaunchKernelGGL((KERNEL<float, float>), GRID, BLOCK, 0, st, jp);                                                   \
    } while (0)

// Launches kernel<stream type, type, vectors, dropout, ALPHA and alpha> for rows that a workgroup holds.
#define JOIN_ROWS2(KERNEL, TS, TF, VEC, DROP)                                                                                            \
    do {                                                                                                                                 \
        constexpr bool WITH = BWD && ROOM<TS, TF, VEC, DROP, true>, WITHOUT = BWD && ROOM<TS, TF, VEC, DROP, false>;  /* alpha */         \
        const bool few = jp.dim <= AHEAD_DIM;                                                                                            \
        const size_t lds = BWD ? (size_t)threads * 32 * (3 + (few && (jp.alpha ? WITH : WITHOUT)) + (jp.alpha ? 1 : 0)) : 0;             \
        if (BWD && jp.alpha && few) hipLaunchKernelGGL((KERNEL<TS, TF, VEC, DROP, BWD, WITH>), grid, dim3(threads), lds, st, jp);        \
        else if (BWD && jp.alpha) hipLaunchKernelGGL((KERNEL<TS, TF, VEC, DROP, BWD, false>), grid, dim3(threads), lds, st, jp);         \
        else if (BWD && few) hipLaunchKernelGGL((KERNEL<TS, TF, VEC, DROP, false, WITHOUT>), grid, dim3(threads), lds, st, jp);          \
        else hipLaunchKernelGGL((KERNEL<TS, TF, VEC, DROP, false, false>), grid, dim3(threads), lds, st, jp);                            \
    } while (0)
#define JOIN_ROWS1(KERNEL, TS, TF)                                          \
    do {                                                                    \
        if (vec && jp.drop.drop) JOIN_ROWS2(KERNEL, TS, TF, true, true);    \
        else if (vec) JOIN_ROWS2(KERNEL, TS, TF, true, false);              \
        else if (jp.drop.drop) JOIN_ROWS2(KERNEL, TS, TF, false, true);     \
        else JOIN_ROWS2(KERNEL, TS, TF, false, false);                      \
    } while (0)
#define JOIN_ROWS(KERNEL, IS_BWD)                                                                    \
    do {                                                                                             \
        constexpr bool BWD = IS_BWD;                                                                 \
        const bool sb = sh->stream_dtype == SSD_BF16, fb = sh->dtype == SSD_BF16;                    \
        const dim3 grid(jp.parts);                                                                   \
        const int threads = 64 * ((jp.dim + 511) / 512);                                             \
        if (sb && fb) JOIN_ROWS1(KERNEL, bf16_t, bf16_t);                                            \
        else if (sb) JOIN_ROWS1(KERNEL, bf16_t, float);                                              \
        else if (fb) JOIN_ROWS1(KERNEL, float, bf16_t);                                              \
        else JOIN_ROWS1(KERNEL, float, float);                                                       \
    } while (0)

// Whether all rows lie on 16 bytes and are whole eights.
bool join_vectors(const ssd_join_shape_t* sh, const JoinParams& jp, std::initializer_list<const void*> ptrs) {
    const int ps = sh->stream_dtype == SSD_BF16 ? 8 : 4, pf = sh->dtype == SSD_BF16 ? 8 : 4;
    if (jp.dim % 8 || jp.s_rs % ps || jp.f_rs % pf || jp.o_rs % pf) return false;
    for (const void* p : ptrs)
        if (!al(p, 16)) return false;
    for (const float* p : {jp.post_w, jp.gate, jp.alpha, jp.pre_w, (const float*)jp.dgate})
        if (!al(p, 16)) return false;
    return true;
}
void cut(JoinParams* jp, int64_t most) {  // the rows into parts of equal length, no more than that many
    jp->part_rows = (jp->rows + most - 1) / most;
    jp->parts = (int)((jp->rows + jp->part_rows - 1) / jp->part_rows);
}
// Parts of the rows, a workgroup each: as many as compute units hold at once with 16 waves each, since a part reads the parameters once
// (65536 rows of 2560, bf16, forward: 258 us in 768 parts, 2048 parts 275; 3001 rows of 5120 24.6 and 29.0; 512 values 46.6 and 50.2).
int64_t parts_fwd(const JoinParams& jp) {
    const int64_t waves = (jp.dim + 511) / 512, most = 256 * (16 / waves);
    return jp.rows < most ? jp.rows : most;
}
// Backward, where each part leaves sums of its own: four rows and more a part, once every compute unit has one (300 rows of 2560: with the launch that
// adds the sums up 15.4 us, four rows a part everywhere 18.6; 3001 rows of 1024 22.6, two rows a part 22.5, eight 28).  Up to four parts a
// compute unit, where a row is one wave eight, from eight rows a part on (65536 rows of 512, 256 and 100: 107, 80 and 151 us, with four 121, 101 and 237;
// sixteen 114, 78 and 125, and fp32 streams lose: 126, 131, 142 for 512; rows of two waves lose with eight).
int64_t parts_bwd(const JoinParams& jp) {
    const int64_t waves = (jp.dim + 511) / 512, at = waves <= 8 && jp.alpha ? 12 : 16, most = 256 * (at / waves < 4 ? at / waves : 4);
    const int64_t few = jp.rows < 256 ? jp.rows : 256, fours = (jp.rows + 3) / 4 > few ? (jp.rows + 3) / 4 : few, by = fours < most ? fours : most;
    const int64_t eights = waves > 1 ? 0 : jp.rows / 8 < 2048 ? jp.rows / 8 : 2048;
    return by > eights ? by : eights;
}

unsigned row_grid(int64_t rows) { return (unsigned)(rows < 4096 ? rows : 4096); }

}  // namespace
}  // namespace ssdk

using namespace ssdk;

extern "C" size_t ssd_join_workspace_bytes(const ssd_join_shape_t* sh) {
    JoinParams jp;
    if (check(sh, nullptr, nullptr, &jp) != SSD_OK) return 0;
    int64_t parts = jp.dim <= ROW_DIM ? parts_bwd(jp) : jp.rows < PARTS_WIDE ? jp.rows : PARTS_WIDE;
    if (parts < 1) parts = 1;
    return up256((size_t)parts * SLOTS * jp.dim * 4) + (jp.dim <= ROW_DIM ? 0 : up256((size_t)jp.rows * 16));
}

extern "C" int ssd_join_fwd(const ssd_join_shape_t* sh, const ssd_join_params_t* params, const ssd_dropout_t* dropout, const void* x, const void* f,
                            void* s, void* out, void* hip_stream) {
    JoinParams jp;
    const int rc = check(sh, params, dropout, &jp);
    if (rc != SSD_OK) return rc;
    if (jp.rows == 0) return SSD_OK;
    if (!x || !f || !s || (jp.pre_w && !out)) return SSD_ERR_NULL;
    if (!jp.pre_w && out) return SSD_ERR_ARG;
    if (!element(sh->stream_dtype, x) || !element(sh->stream_dtype, s) || !element(sh->dtype, f) || !element(sh->dtype, out)) return SSD_ERR_ARG;
    jp.x = x, jp.f = f, jp.s_out = s, jp.out = out;
    hipStream_t st = (hipStream_t)hip_stream;
    if (jp.dim <= ROW_DIM) {
        const bool vec = join_vectors(sh, jp, {x, f, s, out});
        cut(&jp, parts_fwd(jp));
        JOIN_ROWS(k_join_fwd, false);
    } else {
        JOIN_TYPES(k_join_fwd_wide, dim3(row_grid(jp.rows)), dim3(256));
    }
    return done();
}

extern "C" int ssd_join_bwd(const ssd_join_shape_t* sh, const ssd_join_params_t* params, const ssd_dropout_t* dropout, const void* x, const void* f,
                            const void* s, const void* dout, const void* ds, void* dx, void* df, const ssd_join_grads_t* grads, void* workspace,
                            size_t workspace_bytes, uint32_t flags, void* hip_stream) {
    JoinParams jp;
    const int rc = check(sh, params, dropout, &jp);
    if (rc != SSD_OK) return rc;
    if (flags & ~(uint32_t)SSD_FLAG_ACCUM_PARAM) return SSD_ERR_ARG;
    jp.accumulate = flags & SSD_FLAG_ACCUM_PARAM ? 1 : 0;
    if (grads) jp.dpost_w = grads->dpost_w, jp.dgate = grads->dgate, jp.dalpha = grads->dalpha, jp.dpre_w = grads->dpre_w;
    const float* const of[4] = {jp.post_w, jp.gate, jp.alpha, jp.pre_w};
    float* const to[4] = {jp.dpost_w, jp.dgate, jp.dalpha, jp.dpre_w};
    for (int k = 0; k < 4; ++k)
        if (!al(to[k], 4) || (to[k] && !of[k])) return SSD_ERR_ARG;
    hipStream_t st = (hipStream_t)hip_stream;
    if (jp.rows == 0) {
        for (int k = 0; k < 4 && !jp.accumulate; ++k)
            if (to[k] && !(k == 1 && sh->gate_rows) && launch_fill_zero(to[k], (size_t)jp.dim, st) != hipSuccess) return SSD_ERR_LAUNCH;
        return SSD_OK;
    }
    if (!f || !dx || !df || (jp.dalpha && !x) || (jp.pre_w ? !s || !dout : !ds)) return SSD_ERR_NULL;
    if (!jp.pre_w && dout) return SSD_ERR_ARG;
    for (const void* p : {x, s, ds, (const void*)dx})
        if (!element(sh->stream_dtype, p)) return SSD_ERR_ARG;
    for (const void* p : {f, dout, (const void*)df})
        if (!element(sh->dtype, p)) return SSD_ERR_ARG;
    if (!workspace || !al(workspace, 256) || workspace_bytes < ssd_join_workspace_bytes(sh)) return SSD_ERR_WORKSPACE;
    jp.x = x, jp.f = f, jp.s = s, jp.dout = dout, jp.ds = ds, jp.dx = dx, jp.df = df;
    jp.part = (float*)workspace;
    const bool sums = jp.dpost_w || jp.dgate || jp.dalpha || jp.dpre_w;
    if (jp.dim <= ROW_DIM) {
        const bool vec = join_vectors(sh, jp, {x, f, s, dout, ds, dx, df});
        cut(&jp, parts_bwd(jp));
        JOIN_ROWS(k_join_bwd, true);
    } else {
        cut(&jp, PARTS_WIDE);
        jp.stat = (float*)((char*)workspace + up256((size_t)jp.parts * SLOTS * jp.dim * 4));
        JOIN_TYPES(k_join_stats_wide, dim3(row_grid(jp.rows)), dim3(256));
        if (sums) JOIN_TYPES(k_join_sums_wide, dim3((jp.dim + 511) / 512, jp.parts), dim3(64));
        JOIN_TYPES(k_join_bwd_wide, dim3(row_grid(jp.rows)), dim3(256));
    }
    if (sums) {
        const int64_t gates = (jp.rows + jp.gate_rows - 1) / jp.gate_rows;
        const int by_gate = gates < jp.parts, split = !jp.dgate || jp.parts == 1 ? 0 : by_gate ? (int)gates : jp.parts - 1;
        hipLaunchKernelGGL(k_join_reduce, dim3((jp.dim + 63) / 64, 3 + split), dim3(COLSUM_THREADS), 0, st, jp, by_gate);
    }
    return done();
}

extern "C" int ssd_dropout(int32_t dtype, int64_t rows, int32_t dim, const void* x, int64_t x_row_stride, void* out, int64_t out_row_stride,
                           const ssd_dropout_t* dropout, void* hip_stream) {
    if (!dropout) return SSD_ERR_NULL;
    if (dtype != SSD_F32 && dtype != SSD_BF16) return SSD_ERR_DTYPE;
    if (rows < 0 || rows > MAX_ROWS || dim <= 0 || dim > MAX_DIM) return SSD_ERR_SHAPE;
    const int64_t x_rs = x_row_stride ? x_row_stride : dim, o_rs = out_row_stride ? out_row_stride : dim, groups = (dim + 7) / 8;
    if (x_rs < dim || o_rs < dim || x_rs > MAX_STRIDE || o_rs > MAX_STRIDE) return SSD_ERR_SHAPE;
    DropJob d;
    const int rc = check_drop(dropout, rows, groups, &d);
    if (rc != SSD_OK) return rc;
    if (rows == 0) return SSD_OK;
    if (!x || !out) return SSD_ERR_NULL;
    if (!element(dtype, x) || !element(dtype, out) || (x == out && x_rs != o_rs)) return SSD_ERR_ARG;
    hipStream_t st = (hipStream_t)hip_stream;
    const int64_t n = rows * groups, most = 16384;
    const dim3 grid((unsigned)(n < most * 256 ? (n + 255) / 256 : most));
    const bool vec = dtype == SSD_BF16 && dim % 8 == 0 && x_rs % 8 == 0 && o_rs % 8 == 0 && al(x, 16) && al(out, 16);
#define DROPOUT(T, VEC) hipLaunchKernelGGL((k_dropout<T, VEC>), grid, dim3(256), 0, st, x, out, n, dim, (uint32_t)groups, x_rs, o_rs, d)
    if (vec) DROPOUT(bf16_t, true);
    else if (dtype == SSD_BF16) DROPOUT(bf16_t, false);
    else DROPOUT(float, false);
#undef DROPOUT
    return done();
}
