// The gated recurrence of a channel, forward, backward and token by token:
//     r = sigmoid(gate_r)   i = sigmoid(gate_i)   la = -rate softplus(lam) r   a = exp(la)   m = sqrt(1 - a^2)
//     h_t = a_t h_{t-1} + m_t i_t x_t                    (h_{t-1} = 0 where a sequence begins)
// Backward, with e_t the adjoint that token t hands to the state in front of it:
//     dh_t = dout_t + e_{t+1}      e_t = a_t dh_t (0 where a sequence begins)
//     dx = dh m i      dgate_i = dh m x i (1 - i)
//     u  = dh (a h_{t-1} la - i x a^2 la / m)            dgate_r = u (1 - r)      dlam = sigmoid(lam) / softplus(lam) sum u
// la / m goes to zero with la, where a and m alone have no finite derivative.
#include <math.h>
#include <string.h>

#include <initializer_list>
#include <type_traits>

#include "chunk_places.h"
#include "column_sums.h"

namespace ssdk {
namespace {

constexpr int KEPT = SSD_GATED_SCAN_CHUNK;  // tokens from one kept state to the next
constexpr int64_t MAX_STRIDE = 1 << 20;
constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;

// sigmoid(z) and 1 - sigmoid(z), both to their own relative precision: 1 / (1 + t) and t / (1 + t), t = e^-z.  z is held above -86, where t is
// finite and the sigmoid as good as 0 (5e-38); a NaN stays one.
struct Sig {
    float s, c;
};
__device__ __forceinline__ Sig sigmoid2(float z) {
    const float t = __builtin_amdgcn_exp2f(__builtin_elementwise_maximum(z, -86.f) * -LOG2E), s = __builtin_amdgcn_rcpf(1.f + t);
    return {s, t * s};
}
__device__ __forceinline__ float sigmoid1(float z) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * -LOG2E)); }

// From log2(a) = l2 <= 0: a, m = sqrt(1 - a^2) and 1 / m.  1 - a^2 = 1 - e^w with w = 2 ln a loses its leading digits near a = 1: above
// w = -1/4 it is -w times a polynomial for (e^w - 1) / w, interpolated at the five Chebyshev points of [-1/4, 0] (off by 7.3e-9 of itself, its coefficients in fp32).
// m is 0 where 1 - a^2 is, and 1 / m is then held at a finite value: what it is multiplied by is 0 too.
struct Decay {
    float a, m, rm;
};
__device__ __forceinline__ Decay decay(float l2) {
    Decay d;
    d.a = __builtin_amdgcn_exp2f(l2);
    constexpr float S = 2.f * LN2;  // the polynomial is in l2 itself, its coefficients times powers of S
    float p = fmaf(l2, 0.00751361f * S * S * S * S, 0.04149065f * S * S * S);
    p = fmaf(l2, p, 0.16665108f * S * S);
    p = fmaf(l2, p, 0.49999951f * S);
    p = fmaf(l2, p, 1.f);
    const float m2 = l2 > -0.25f / S ? l2 * -S * p : fmaf(-d.a, d.a, 1.f);
    d.rm = __builtin_amdgcn_rsqf(fmaxf(m2, 1.17549435e-38f));
    d.m = m2 * d.rm;
    return d;
}
// log2 of the decay of an open gate: -rate softplus(lam) log2(e)
__device__ __forceinline__ float slope_of(float lam, float rate) { return -rate * (fmaxf(lam, 0.f) + log1pf(expf(-fabsf(lam)))) * LOG2E; }
// sigmoid(lam) / softplus(lam): 1 - O(e^lam) for very negative lam, where both vanish
__device__ __forceinline__ float lam_factor(float lam) {
    if (lam < -17.f) return 1.f;
    return 1.f / (1.f + expf(-lam)) / (fmaxf(lam, 0.f) + log1pf(expf(-fabsf(lam))));
}

struct ScanParams {
    const void *x, *gr, *gi, *dout;
    const float *lam, *init, *dfinal, *states_in;
    void *out, *dx, *dgr, *dgi;
    float *final_state, *states, *dinit, *part;  // part: [chunks][Bt][C], the chunks' shares of dlam
    const uint8_t* reset;
    int64_t L, nchunks;  // nchunks: kept states, the backward kernel's chunks
    int64_t x_rs, g_rs, o_rs, dx_rs, dg_rs, x_bs, g_bs, o_bs, dx_bs, dg_bs;
    int Bt, C;
    float rate;
};

// ---- scan over chunks ----------------------------------------------------------------------------------------------------------------
//
// A run of tokens maps the state in front of it to the one behind it: h -> A h + H with A the product of its decays; runs compose.  A workgroup
// takes a chunk of 128 (backward 64) tokens of 64 channels (128 bytes of a bf16 row): a thread 4 channels of K consecutive tokens, whose inputs it reads
// once and keeps, 16 lanes side by side, 4 lanes and then the waves along the tokens.  Runs of threads are composed by exchanges of half
// waves, runs of waves through LDS, and chunks along the sequence through memory, while the values stay in registers:
//   - a workgroup leaves its chunk's (A, H) as one 64-bit word a channel as soon as it has them;
//   - it takes the words of the chunks in front of it in its group of GROUP chunks, and the state behind the group in front;
//   - the last of a group leaves the state behind it.
// So the way along a sequence is one exchange through memory for 2048 (1024) tokens, every state is the same composition whatever came first, and
// the inputs are read once.  A workgroup takes its chunk from a counter of its tile, so that what it waits for is always work of
// workgroups that run already (one counter for all would be the limit: 12 ns a workgroup); the words are set to "not there" (all ones,
// a NaN that no result is written as) by a launch in front.
// A run in which a sequence begins does not hand on what is in front of it: its A is left as CUT, and nothing is multiplied by it.
constexpr int TILE = 64;    // channels of a workgroup
constexpr int GROUP = 16;   // chunks
constexpr int WAVES = 4, K_FWD = 8, K_BWD = 4;  // tokens of a chunk: 4 WAVES K
static_assert(64 * WAVES * (uint64_t)MOST_IN_LINE < (uint64_t)1 << 32, "");
static_assert(4 * WAVES * K_BWD == KEPT && K_FWD % K_BWD == 0 && GROUP % WAVES == 0, "");
constexpr float CUT = -1.f;
constexpr uint32_t NOT_THERE = 0xffffffffu;
constexpr int TICKET = 16;  // words: a counter has 64 bytes of its own
// Looks (of a microsecond or so each) after which a word is taken as it is: it never comes where another call clears the workspace meanwhile,
// and what is not there is a NaN, which the results then are.
constexpr uint32_t MOST_TRIES = 1u << 21;

struct Run {  // of one channel
    float A, H;
};
// first `first`, then `then`
template <bool RESET>
__device__ __forceinline__ Run compose(Run first, Run then) {
    Run r = {first.A * then.A, fmaf(then.A, first.H, then.H)};
    if (RESET) {
        const bool cut = then.A < 0.f;
        r.H = cut ? then.H : r.H;
        r.A = cut || first.A < 0.f ? CUT : r.A;
    }
    return r;
}
template <bool RESET>
__device__ __forceinline__ float apply(Run r, float h) {
    const float v = fmaf(r.A, h, r.H);
    return RESET && r.A < 0.f ? r.H : v;
}

typedef float f32x4 __attribute__((ext_vector_type(4)));
// The runs of four channels, as waves leave them: A, then H.
template <bool RESET>
__device__ __forceinline__ void apply(const f32x4 (&r)[2][16], int q, float (&h)[4]) {
    const f32x4 A = r[0][q], H = r[1][q];
#pragma unroll
    for (int e = 0; e < 4; ++e) h[e] = apply<RESET>(Run{A[e], H[e]}, h[e]);
}

// The values of the lower and the upper of two halves, in both: rows 0, 1 of sixteen lanes (and 2, 3), or the halves of the wave.
struct Pair {
    float lo, hi;
};
template <int STAGE>
__device__ __forceinline__ Pair halves(float v) {
    const unsigned u = __builtin_bit_cast(unsigned, v);
    const auto p = STAGE == 0 ? __builtin_amdgcn_permlane16_swap(u, u, false, false) : __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return {__builtin_bit_cast(float, (unsigned)p[0]), __builtin_bit_cast(float, (unsigned)p[1])};
}
// all: the run of a thread -> of its wave; other: the composition of the lanes in front (BACK: behind, the order turned round).  A is both
// directions' and comes exchanged.
template <bool RESET, bool BACK, int STAGE>
__device__ __forceinline__ Run wave_stage(Pair A, float H, Run& other, int lane) {
    const Pair h = halves<STAGE>(H);
    const Run lo = {A.lo, h.lo}, hi = {A.hi, h.hi}, near = BACK ? hi : lo;
    const bool takes = BACK != (bool)(lane & (STAGE == 0 ? 16 : 32));
    const Run o = STAGE == 0 ? near : compose<RESET>(near, other);
    if (STAGE == 0) other = {1.f, 0.f};
    if (takes) other = o;
    return BACK ? compose<RESET>(hi, lo) : compose<RESET>(lo, hi);
}
template <bool RESET>
__device__ __forceinline__ void wave_runs(Run& all, Run& front, int lane) {
    all = wave_stage<RESET, false, 0>(halves<0>(all.A), all.H, front, lane);
    all = wave_stage<RESET, false, 1>(halves<1>(all.A), all.H, front, lane);
}
// Both directions at once: E is the backward run's second number.
template <bool RESET>
__device__ __forceinline__ void wave_runs(Run& all, float& E, Run& front, Run& behind, int lane) {
    Pair A = halves<0>(all.A);
    E = wave_stage<RESET, true, 0>(A, E, behind, lane).H;
    all = wave_stage<RESET, false, 0>(A, all.H, front, lane);
    A = halves<1>(all.A);
    E = wave_stage<RESET, true, 1>(A, E, behind, lane).H;
    all = wave_stage<RESET, false, 1>(A, all.H, front, lane);
}

// What a launch's workgroups exchange, in its workspace.
struct Chain {
    uint32_t* tickets;  // [Bt tiles], TICKET words apart
    uint64_t* runs;     // [chunk][Bt][Cp]: A, H of a chunk
    uint32_t* ends;     // [group][Bt][Cp]: the state behind a group
    float* slopes;      // [Cp], of the channels that there are
    uint32_t chunks;    // of a sequence
};
// Sets the words to "not there" and the counters to 0, and works out every channel's slope on the way: a launch's time, 2.3 us for 16 chunks of
// 768 channels, 12 for 2048 of 2560.
__global__ __launch_bounds__(256) void k_gated_scan_clear(Chain ch, int64_t side, uint4* words, int64_t n, const float* lam, int C, float rate) {
    const int64_t i0 = (int64_t)blockIdx.x * 256 + threadIdx.x, all = (int64_t)gridDim.x * 256;
    for (int64_t i = i0; i < side; i += all) ch.tickets[i * TICKET] = 0;
    for (int64_t i = i0; i < C; i += all) ch.slopes[i] = slope_of(lam[i], rate);
    for (int64_t i = i0; i < n; i += all) words[i] = make_uint4(NOT_THERE, NOT_THERE, NOT_THERE, NOT_THERE);
}
__device__ __forceinline__ uint32_t word_of(float v) { return v == v ? __builtin_bit_cast(uint32_t, v) : 0x7fc00000u; }
__device__ __forceinline__ void leave(uint64_t* to, Run r) {
    __hip_atomic_store(to, (uint64_t)word_of(r.H) << 32 | word_of(r.A), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void leave(uint32_t* to, float v) { __hip_atomic_store(to, word_of(v), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// A workgroup's place.
struct Place {
    int64_t chunk;  // in the order in which they depend on each other: backward, 0 is the last of the sequence
    int b, c0;
};
template <bool CHAIN>
__device__ __forceinline__ Place take_place(const ScanParams& sp, const Chain& ch, uint32_t* lds) {
    const uint32_t tiles = (uint32_t)((sp.C + TILE - 1) / TILE), side = tiles * sp.Bt, number = number_of(blockIdx.x, blockIdx.y), in = tile_of(number, side);
    uint32_t chunk = number / side;  // where there is one chunk: 0, or a workgroup to spare
    if (CHAIN) {
        if (threadIdx.x == 0) *lds = __hip_atomic_fetch_add(ch.tickets + in * TICKET, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __syncthreads();
        chunk = __builtin_amdgcn_readfirstlane(*lds);
    }
    return {chunk, (int)(in / tiles), (int)(in % tiles) * TILE};
}

// The state that a chunk starts from (backward: the adjoint that comes from behind), of channel `lane` of the tile in the first wave.  The waves
// take GROUP / WAVES chunks of the group each, the first one the state behind the group in front as well, and leaves the one behind this
// group if the chunk (its run: `chunk`) ends it.  from_outside: what the sequence itself starts from.
struct ChainLds {
    float state[TILE];  // what the chunk starts from
    Run runs[WAVES][TILE];
};
template <bool RESET>
__device__ __forceinline__ float gather(ChainLds& L, const Chain& ch, const Place& at, int64_t row, int64_t col, Run chunk, float from_outside, int wv, int lane) {
    constexpr int EACH = GROUP / WAVES;
    const int64_t group = at.chunk / GROUP, before = at.chunk - group * GROUP;
    const int first = wv * EACH;
    uint64_t w[EACH];
    uint32_t s = 0;
    const bool state = wv == 0 && group > 0;
    if (first < before || state) {
        for (uint32_t tries = 0;; ++tries) {
            bool there = true;
            if (state) s = __hip_atomic_load(ch.ends + (group - 1) * row + col, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
            for (int k = 0; k < EACH; ++k)
                if (first + k < before) w[k] = __hip_atomic_load(ch.runs + (group * GROUP + first + k) * row + col, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            if (state) there = s != NOT_THERE;
#pragma unroll
            for (int k = 0; k < EACH; ++k)
                if (first + k < before) there = there && (uint32_t)w[k] != NOT_THERE;
            if (__all(there) || tries == MOST_TRIES) break;
            __builtin_amdgcn_s_sleep(1);
        }
    }
    Run r = {1.f, 0.f};
#pragma unroll
    for (int k = 0; k < EACH; ++k)
        if (first + k < before) r = compose<RESET>(r, Run{__builtin_bit_cast(float, (uint32_t)w[k]), __builtin_bit_cast(float, (uint32_t)(w[k] >> 32))});
    if (wv > 0) L.runs[wv][lane] = r;
    __syncthreads();
    float h = 0.f;
    if (wv == 0) {
        h = apply<RESET>(r, group > 0 ? __builtin_bit_cast(float, s) : from_outside);
#pragma unroll
        for (int k = 1; k < WAVES; ++k) h = apply<RESET>(L.runs[k][lane], h);
        const float end = apply<RESET>(chunk, h);
        if (at.chunk % GROUP == GROUP - 1) leave(ch.ends + group * row + col, end);
    }
    return h;
}

// Keeps the compiler from putting the making of a value off to where it is used, which keeps more values alive than it saves.
__device__ __forceinline__ void made(float& v) { asm volatile("" : "+v"(v)); }

// Rows in memory: a descriptor that ends with them, so that tokens and channels that do not exist, at NOWHERE or behind its end, read zeros and
// write nothing; and the rows as they are.
struct Rows {
    __amdgpu_buffer_rsrc_t q;
    char* p;
    int bytes;
};
// Four channels of one token.  VEC: on four elements' boundary.  Else four that exist go as a vector at whatever address and the last one to
// three of a row element by element (30000 tokens of 2561 channels, bf16, forward and backward, tiles in turn over the XCDs:
// 570 us; all element by element 756).
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef u32x2 u32x2_any __attribute__((aligned(2)));
typedef u32x4 u32x4_any __attribute__((aligned(4)));
constexpr int NOWHERE = 0x7fffffff;
template <typename T>
struct Four;
template <>
struct Four<bf16_t> {
    static constexpr int SIZE = 2;
    bf16x4 v;
    template <bool VEC>
    __device__ __forceinline__ void load(const Rows& rows, int at, int left) {
        if (VEC) {
            v = __builtin_bit_cast(bf16x4, __builtin_amdgcn_raw_buffer_load_b64(rows.q, at, 0, 0));
        } else if (left >= 4 && (unsigned)at + 4 * SIZE <= (unsigned)rows.bytes) {
            v = __builtin_bit_cast(bf16x4, *(const u32x2_any*)(rows.p + at));
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = __builtin_bit_cast(__bf16, __builtin_amdgcn_raw_buffer_load_b16(rows.q, e < left ? at + 2 * e : NOWHERE, 0, 0));
        }
    }
    template <bool VEC>
    __device__ __forceinline__ void store(const Rows& rows, int at, int left) const {
        if (VEC) {
            __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, v), rows.q, at, 0, 0);
        } else if (left >= 4 && (unsigned)at + 4 * SIZE <= (unsigned)rows.bytes) {
            *(u32x2_any*)(rows.p + at) = __builtin_bit_cast(u32x2, v);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(unsigned short, (__bf16)v[e]), rows.q, e < left ? at + 2 * e : NOWHERE, 0, 0);
        }
    }
    __device__ __forceinline__ float get(int e) const { return (float)v[e]; }
    __device__ __forceinline__ void set(int e, float f) { v[e] = (__bf16)f; }
};
template <>
struct Four<float> {
    static constexpr int SIZE = 4;
    f32x4 v;
    template <bool VEC>
    __device__ __forceinline__ void load(const Rows& rows, int at, int left) {
        if (VEC) {
            v = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rows.q, at, 0, 0));
        } else if (left >= 4 && (unsigned)at + 4 * SIZE <= (unsigned)rows.bytes) {
            v = __builtin_bit_cast(f32x4, *(const u32x4_any*)(rows.p + at));
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rows.q, e < left ? at + 4 * e : NOWHERE, 0, 0));
        }
    }
    template <bool VEC>
    __device__ __forceinline__ void store(const Rows& rows, int at, int left) const {
        if (VEC) {
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), rows.q, at, 0, 0);
        } else if (left >= 4 && (unsigned)at + 4 * SIZE <= (unsigned)rows.bytes) {
            *(u32x4_any*)(rows.p + at) = __builtin_bit_cast(u32x4, v);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, (float)v[e]), rows.q, e < left ? at + 4 * e : NOWHERE, 0, 0);
        }
    }
    __device__ __forceinline__ float get(int e) const { return v[e]; }
    __device__ __forceinline__ void set(int e, float f) { v[e] = f; }
};
// The rows of a chunk: `rows` of them from token t0 of batch b.
template <typename T>
__device__ __forceinline__ Rows rows_at(const void* p, int64_t first, int64_t rs, int rows, int C) {
    char* const from = (char*)p + first * Four<T>::SIZE;
    const int bytes = (int)(((rows - 1) * rs + C) * Four<T>::SIZE);
    return {__builtin_amdgcn_make_buffer_rsrc(from, 0, bytes, 0x00020000), from, bytes};
}

// A thread's place in its workgroup of WAVES waves: channels 4 q .. 4 q + 3 of the tile, K tokens from token t on.
template <int K>
struct Lane {
    int lane, wv, c, t, left;  // left: channels from c on that exist
    __device__ __forceinline__ Lane(int c0, int C) {
        lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
        c = c0 + 4 * (lane & 15), t = (wv * 4 + (lane >> 4)) * K, left = C - c;
    }
};
// The bytes of its tokens in rows that far apart.
struct Steps {
    int first, step;
    template <int K>
    __device__ __forceinline__ Steps(const Lane<K>& me, int64_t rs, int size) {
        first = me.left > 0 ? (me.t * (int)rs + me.c) * size : NOWHERE;
        step = me.left > 0 ? (int)rs * size : 0;
    }
    __device__ __forceinline__ int operator[](int j) const { return first + j * step; }
};
// The slopes of a thread's channels; a single chunk has no launch in front, and lanes work out a channel each.
template <bool CHAIN>
__device__ __forceinline__ void slopes(float (&s)[4], const ScanParams& sp, const Chain& ch, int c0, int lane) {
    if (CHAIN) {
        const f32x4 v = *(const f32x4*)(ch.slopes + c0 + 4 * (lane & 15));
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] = v[e];
    } else {
        const float own = c0 + lane < sp.C ? slope_of(sp.lam[c0 + lane], sp.rate) : 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] = __shfl(own, 4 * (lane & 15) + e, 64);
    }
}
// The flags of a thread's K tokens, a byte each, in one load at whatever address where all of them exist.  Asked for in front of the inputs: loads
// come back in order, and the first token needs them.
template <int K>
struct Flags {
    static_assert(K == 4 || K == 8, "");
    uint32_t w[K / 4] = {};
    __device__ __forceinline__ void load(const ScanParams& sp, const Place& at, int64_t t0, int t, int rows) {
        const uint8_t* const from = sp.reset + at.b * sp.L + t0 + t;
        if (t + K <= rows) {
            __builtin_memcpy(w, from, K);
        } else {
#pragma unroll
            for (int j = 0; j < K - 1; ++j)
                if (t + j < rows) w[j >> 2] |= (uint32_t)from[j] << 8 * (j & 3);
        }
    }
    __device__ __forceinline__ bool any() const { return w[0] | w[K / 4 - 1]; }
    __device__ __forceinline__ bool operator[](int j) const { return w[j >> 2] >> 8 * (j & 3) & 0xff; }
};
// Does `work` as it is where a sequence may begin and as it is where none does: few waves of a packed batch hold the beginning of one (3 x 2001
// tokens of 2048 channels, packed, forward and backward: 81 us, with looks for beginnings in every wave 92; not packed 78).
template <bool RESET, typename Work>
__device__ __forceinline__ void either(bool begins, Work work) {
    if (RESET && begins) work(std::true_type());
    else work(std::false_type());
}

// Forward.  Bound by memory and vector units alike (39 instructions a value): 262144 tokens of 2560 channels, bf16, 989 us (5.4 GB, 5.4 TB/s), fp32 1999
// of 768 8.3; 3 x 2001 of 2048 31: two rounds of workgroups, the second half filled.  Four tokens a thread instead of eight double the chain: slower.
template <typename T, bool VEC, bool RESET, bool CHAIN>
__global__ __launch_bounds__(64 * WAVES, 4) void k_gated_scan_fwd(ScanParams sp, Chain ch) {
    constexpr int K = K_FWD, CHUNK = 4 * WAVES * K;
    __shared__ uint32_t place;
    __shared__ f32x4 totals[WAVES][2][16];  // the waves' runs
    __shared__ ChainLds L;
    const Place at = take_place<CHAIN>(sp, ch, &place);
    if (!chunk_there((uint32_t)at.chunk, CHAIN ? ch.chunks : 1)) return;
    const Lane<K> me(at.c0, sp.C);
    const int64_t t0 = at.chunk * CHUNK, Cp = (int64_t)((sp.C + TILE - 1) / TILE) * TILE;
    const int rows = sp.L - t0 < CHUNK ? (int)(sp.L - t0) : CHUNK;
    Flags<K> flags;
    if (RESET) flags.load(sp, at, t0, me.t, rows);
    Four<T> x[K], gr[K], gi[K];
    {
        const Rows qx = rows_at<T>(sp.x, at.b * sp.x_bs + t0 * sp.x_rs, sp.x_rs, rows, sp.C);
        const Rows qr = rows_at<T>(sp.gr, at.b * sp.g_bs + t0 * sp.g_rs, sp.g_rs, rows, sp.C);
        const Rows qi = rows_at<T>(sp.gi, at.b * sp.g_bs + t0 * sp.g_rs, sp.g_rs, rows, sp.C);
        const Steps sg(me, sp.g_rs, Four<T>::SIZE), sx(me, sp.x_rs, Four<T>::SIZE);
#pragma unroll
        for (int j = 0; j < K; ++j) {
            gr[j].template load<VEC>(qr, sg[j], me.left);
            gi[j].template load<VEC>(qi, sg[j], me.left);
            x[j].template load<VEC>(qx, sx[j], me.left);
        }
    }
    const bool begins = RESET && __any(flags.any());  // a sequence, at one of the wave's tokens
    float from_outside = 0.f;
    if (sp.init && me.wv == 0 && at.c0 + me.lane < sp.C) from_outside = sp.init[(int64_t)at.b * sp.C + at.c0 + me.lane];
    float slope[4];
    slopes<CHAIN>(slope, sp, ch, at.c0, me.lane);

    float a[K][4], v[K][4];
#pragma unroll
    for (int j = 0; j < K; ++j) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const Decay d = decay(slope[e] * sigmoid1(gr[j].get(e)));
            a[j][e] = d.a;
            v[j][e] = d.m * sigmoid1(gi[j].get(e)) * x[j].get(e);  // 0 behind the end, where x is
            made(a[j][e]), made(v[j][e]);
        }
        __builtin_amdgcn_sched_barrier(0);  // one token after another, as below
    }
    if (rows < CHUNK)  // tokens behind the end hand the state on
#pragma unroll
        for (int j = 0; j < K; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) a[j][e] = me.t + j < rows ? a[j][e] : 1.f;
    if (begins)
#pragma unroll
        for (int j = 0; j < K; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) a[j][e] = flags[j] ? CUT : a[j][e];
    Run all[4], front[4];
    either<RESET>(begins, [&](auto cuts) {
        constexpr bool CUTS = decltype(cuts)::value;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            all[e] = {a[0][e], v[0][e]};
#pragma unroll
            for (int j = 1; j < K; ++j) all[e] = compose<CUTS>(all[e], Run{a[j][e], v[j][e]});
            wave_runs<CUTS>(all[e], front[e], me.lane);
        }
    });
    if (me.lane < 16) {
        totals[me.wv][0][me.lane] = f32x4{all[0].A, all[1].A, all[2].A, all[3].A};
        totals[me.wv][1][me.lane] = f32x4{all[0].H, all[1].H, all[2].H, all[3].H};
    }
    __syncthreads();
    // of the chunk: channel `lane` of the tile, in the first wave
    Run chunk = {1.f, 0.f};
    const int64_t col = at.b * Cp + at.c0 + me.lane, row = (int64_t)sp.Bt * Cp;
    if (me.wv == 0) {
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const Run r = {((const float*)totals[w][0])[me.lane], ((const float*)totals[w][1])[me.lane]};
            chunk = w == 0 ? r : compose<RESET>(chunk, r);
        }
        if (CHAIN) leave(ch.runs + at.chunk * row + col, chunk);
    }
    const float begin = CHAIN ? gather<RESET>(L, ch, at, row, col, chunk, from_outside, me.wv, me.lane) : from_outside;
    if (me.wv == 0) {
        L.state[me.lane] = begin;
        if (sp.final_state && at.chunk == (sp.L - 1) / CHUNK && at.c0 + me.lane < sp.C) sp.final_state[(int64_t)at.b * sp.C + at.c0 + me.lane] = apply<RESET>(chunk, begin);
    }
    __syncthreads();
    float h[4];
    const int q = me.lane & 15;
    const f32x4 start = ((const f32x4*)L.state)[q];
#pragma unroll
    for (int e = 0; e < 4; ++e) h[e] = start[e];
    for (int w = 0; w < me.wv; ++w) apply<RESET>(totals[w], q, h);
#pragma unroll
    for (int e = 0; e < 4; ++e) h[e] = apply<RESET>(front[e], h[e]);
    if (sp.states && me.t % KEPT == 0 && me.t < rows) {
        float* const to = sp.states + (at.b * sp.nchunks + (t0 + me.t) / KEPT) * sp.C + me.c;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < me.left) to[e] = h[e];
    }
    const Steps so(me, sp.o_rs, Four<T>::SIZE);
    const Rows qo = rows_at<T>(sp.out, at.b * sp.o_bs + t0 * sp.o_rs, sp.o_rs, rows, sp.C);
    either<RESET>(begins, [&](auto cuts) {
#pragma unroll
        for (int j = 0; j < K; ++j) {
            Four<T> o;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                h[e] = apply<decltype(cuts)::value>(Run{a[j][e], v[j][e]}, h[e]);
                o.set(e, h[e]);
            }
            o.template store<VEC>(qo, so[j], me.left);
        }
    });
}

// Backward, chunks from the last to the first.  The states inside the chunk are worked out again from the one that the forward call kept, which
// needs nothing of other chunks; the adjoint is a recurrence of the same form from behind, e_t = a_t (dout_t + e_{t+1}).  Three workgroups a compute unit (168
// registers; four spill and are slower).  262144 tokens of 2560 channels, bf16: 2047 us (9.4 GB, 4.6 TB/s; 74 instructions a value), 3 x 2001 of 2048 46.
template <typename T, bool VEC, bool RESET, bool CHAIN>
__global__ __launch_bounds__(64 * WAVES, 3) void k_gated_scan_bwd(ScanParams sp, Chain ch) {
    constexpr int K = K_BWD, CHUNK = 4 * WAVES * K;
    __shared__ uint32_t place;
    __shared__ f32x4 totals[2][WAVES][2][16];  // the waves' runs, forward and backward
    __shared__ f32x4 sums[WAVES][16];
    __shared__ ChainLds L;
    __shared__ f32x4 later[2][K][64 * WAVES];  // each thread's own
    const Place at = take_place<CHAIN>(sp, ch, &place);
    if (!chunk_there((uint32_t)at.chunk, CHAIN ? ch.chunks : 1)) return;
    const Lane<K> me(at.c0, sp.C);
    const int64_t chunk_at = sp.nchunks - 1 - at.chunk, t0 = chunk_at * CHUNK, Cp = (int64_t)((sp.C + TILE - 1) / TILE) * TILE;
    const int rows = sp.L - t0 < CHUNK ? (int)(sp.L - t0) : CHUNK;
    Flags<K> flags;
    if (RESET) flags.load(sp, at, t0, me.t, rows);
    Four<T> x[K], gr[K], gi[K], dout[K];
    {
        const Rows qx = rows_at<T>(sp.x, at.b * sp.x_bs + t0 * sp.x_rs, sp.x_rs, rows, sp.C);
        const Rows qr = rows_at<T>(sp.gr, at.b * sp.g_bs + t0 * sp.g_rs, sp.g_rs, rows, sp.C);
        const Rows qi = rows_at<T>(sp.gi, at.b * sp.g_bs + t0 * sp.g_rs, sp.g_rs, rows, sp.C);
        const Rows qd = rows_at<T>(sp.dout, at.b * sp.o_bs + t0 * sp.o_rs, sp.o_rs, rows, sp.C);
        const Steps sg(me, sp.g_rs, Four<T>::SIZE), sx(me, sp.x_rs, Four<T>::SIZE), so(me, sp.o_rs, Four<T>::SIZE);
#pragma unroll
        for (int j = 0; j < K; ++j) {
            gr[j].template load<VEC>(qr, sg[j], me.left);
            gi[j].template load<VEC>(qi, sg[j], me.left);
            x[j].template load<VEC>(qx, sx[j], me.left);
            dout[j].template load<VEC>(qd, so[j], me.left);
        }
    }
    const bool begins = RESET && __any(flags.any());
    float from_outside = 0.f, h[4];
    if (sp.dfinal && me.wv == 0 && at.c0 + me.lane < sp.C) from_outside = sp.dfinal[(int64_t)at.b * sp.C + at.c0 + me.lane];
#pragma unroll
    for (int e = 0; e < 4; ++e) h[e] = e < me.left ? sp.states_in[(at.b * sp.nchunks + chunk_at) * sp.C + me.c + e] : 0.f;
    float slope[4];
    slopes<CHAIN>(slope, sp, ch, at.c0, me.lane);

    // Decays; what the results need besides: m i, w1 = a la, w2 = i x a^2 la / m, and, in LDS until the end, x (1 - i) and 1 - r.
    float a[K][4], mi[K][4], w1[K][4], w2[K][4];
#pragma unroll
    for (int j = 0; j < K; ++j) {
        f32x4 k0, k1;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const Sig r = sigmoid2(gr[j].get(e)), i = sigmoid2(gi[j].get(e));
            const float l2 = slope[e] * r.s, la = l2 * LN2, xv = x[j].get(e);
            const Decay d = decay(l2);
            a[j][e] = d.a;
            mi[j][e] = d.m * i.s;
            w1[j][e] = d.a * la;
            w2[j][e] = i.s * xv * d.a * (w1[j][e] * d.rm);
            k0[e] = xv * i.c;
            k1[e] = r.c;
            made(a[j][e]), made(mi[j][e]), made(w1[j][e]), made(w2[j][e]);
        }
        later[0][j][threadIdx.x] = k0;
        later[1][j][threadIdx.x] = k1;
        __builtin_amdgcn_sched_barrier(0);  // one token after another: side by side they need more registers than there are
    }
    if (rows < CHUNK)  // tokens behind the end hand on what comes; x and dout are 0 there, and so is w2
#pragma unroll
        for (int j = 0; j < K; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const bool real = me.t + j < rows;
                a[j][e] = real ? a[j][e] : 1.f;
                w1[j][e] = real ? w1[j][e] : 0.f;
            }
    if (begins)
#pragma unroll
        for (int j = 0; j < K; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) a[j][e] = flags[j] ? CUT : a[j][e];
    // the run of a token forward is (a, m i x), backward, e = a (dout + e), it is (a, a dout)
    Run all[4], front[4], behind[4];
    float E[4];
    either<RESET>(begins, [&](auto cuts) {
        constexpr bool CUTS = decltype(cuts)::value;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            all[e] = {a[0][e], mi[0][e] * x[0].get(e)};
#pragma unroll
            for (int j = 1; j < K; ++j) all[e] = compose<CUTS>(all[e], Run{a[j][e], mi[j][e] * x[j].get(e)});
            E[e] = 0.f;
#pragma unroll
            for (int j = K - 1; j >= 0; --j) {
                const float s = j == K - 1 ? dout[j].get(e) : dout[j].get(e) + E[e];
                E[e] = CUTS && a[j][e] < 0.f ? 0.f : a[j][e] * s;
            }
            wave_runs<CUTS>(all[e], E[e], front[e], behind[e], me.lane);
        }
    });
    if (me.lane < 16) {
        totals[0][me.wv][0][me.lane] = totals[1][me.wv][0][me.lane] = f32x4{all[0].A, all[1].A, all[2].A, all[3].A};
        totals[0][me.wv][1][me.lane] = f32x4{all[0].H, all[1].H, all[2].H, all[3].H};
        totals[1][me.wv][1][me.lane] = f32x4{E[0], E[1], E[2], E[3]};
    }
    __syncthreads();
    Run chunk = {1.f, 0.f};
    const int64_t col = at.b * Cp + at.c0 + me.lane, row = (int64_t)sp.Bt * Cp;
    if (me.wv == 0) {
#pragma unroll
        for (int w = WAVES - 1; w >= 0; --w) {
            const Run r = {((const float*)totals[1][w][0])[me.lane], ((const float*)totals[1][w][1])[me.lane]};
            chunk = w == WAVES - 1 ? r : compose<RESET>(chunk, r);
        }
        if (CHAIN) leave(ch.runs + at.chunk * row + col, chunk);
    }
    // the states in front of the tokens turn w1 h - w2 into what dh is multiplied by
    const int q = me.lane & 15;
    for (int w = 0; w < me.wv; ++w) apply<RESET>(totals[0][w], q, h);
#pragma unroll
    for (int e = 0; e < 4; ++e) h[e] = apply<RESET>(front[e], h[e]);
    either<RESET>(begins, [&](auto cuts) {
        constexpr bool CUTS = decltype(cuts)::value;
#pragma unroll
        for (int j = 0; j < K; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const bool cut = CUTS && a[j][e] < 0.f;
                w1[j][e] = cut ? -w2[j][e] : fmaf(w1[j][e], h[e], -w2[j][e]);
                if (j + 1 < K) h[e] = apply<CUTS>(Run{a[j][e], mi[j][e] * x[j].get(e)}, h[e]);
                made(w1[j][e]);
            }
    });
    const float begin = CHAIN ? gather<RESET>(L, ch, at, row, col, chunk, from_outside, me.wv, me.lane) : from_outside;
    if (me.wv == 0) {
        L.state[me.lane] = begin;
        if (sp.dinit && chunk_at == 0 && at.c0 + me.lane < sp.C) sp.dinit[(int64_t)at.b * sp.C + at.c0 + me.lane] = apply<RESET>(chunk, begin);
    }
    __syncthreads();
    float adj[4], sum[4] = {};
    const f32x4 start = ((const f32x4*)L.state)[q];
#pragma unroll
    for (int e = 0; e < 4; ++e) adj[e] = start[e];
    for (int w = WAVES - 1; w > me.wv; --w) apply<RESET>(totals[1][w], q, adj);
#pragma unroll
    for (int e = 0; e < 4; ++e) adj[e] = apply<RESET>(behind[e], adj[e]);
    const Steps sx(me, sp.dx_rs, Four<T>::SIZE), sg(me, sp.dg_rs, Four<T>::SIZE);
    const Rows qx = rows_at<T>(sp.dx, at.b * sp.dx_bs + t0 * sp.dx_rs, sp.dx_rs, rows, sp.C);
    const Rows qr = rows_at<T>(sp.dgr, at.b * sp.dg_bs + t0 * sp.dg_rs, sp.dg_rs, rows, sp.C);
    const Rows qi = rows_at<T>(sp.dgi, at.b * sp.dg_bs + t0 * sp.dg_rs, sp.dg_rs, rows, sp.C);
#pragma unroll
    for (int j = K - 1; j >= 0; --j) {
        Four<T> ox, orr, oi;
        const f32x4 k0 = later[0][j][threadIdx.x], k1 = later[1][j][threadIdx.x];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bool cut = RESET && a[j][e] < 0.f;
            const float dh = dout[j].get(e) + adj[e], u = dh * w1[j][e], d = dh * mi[j][e];
            ox.set(e, d);
            oi.set(e, d * k0[e]);
            orr.set(e, u * k1[e]);
            sum[e] += u;
            adj[e] = cut ? 0.f : a[j][e] * dh;
        }
        ox.template store<VEC>(qx, sx[j], me.left);
        orr.template store<VEC>(qr, sg[j], me.left);
        oi.template store<VEC>(qi, sg[j], me.left);
    }
    // the chunk's share of dlam
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const Pair s = halves<0>(sum[e]);
        const Pair t = halves<1>(s.lo + s.hi);
        sum[e] = t.lo + t.hi;
    }
    if (me.lane < 16) sums[me.wv][me.lane] = f32x4{sum[0], sum[1], sum[2], sum[3]};
    __syncthreads();
    if (me.wv == 0 && at.c0 + me.lane < sp.C) {
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) s += ((const float*)sums[w])[me.lane];
        sp.part[(chunk_at * sp.Bt + at.b) * sp.C + at.c0 + me.lane] = s;
    }
}

// dlam = sigmoid(lam) / softplus(lam) times the sum of the chunks' sums, in fp64 (there may be thousands) and in a fixed order.  4096 chunks of 2560
// channels 28 us, 96 of 2048 4.7.
__global__ __launch_bounds__(COLSUM_THREADS) void k_gated_scan_dlam(const float* part, int64_t nparts, int C, const float* lam, float* dlam, int accumulate) {
    __shared__ double red[COLSUM_WAVES][64];
    constexpr int U = 8;
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
    double s = 0.0;
    if (c < C) {
        int64_t p = wv;
        for (; p + (U - 1) * COLSUM_WAVES < nparts; p += U * COLSUM_WAVES) {
            float v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = part[(p + u * COLSUM_WAVES) * C + c];
#pragma unroll
            for (int u = 0; u < U; ++u) s += (double)v[u];
        }
        for (; p < nparts; p += COLSUM_WAVES) s += (double)part[p * C + c];
    }
    red[wv][lane] = s;
    __syncthreads();
    if (wv == 0 && c < C) {
        s = 0.0;
#pragma unroll
        for (int w = 0; w < COLSUM_WAVES; ++w) s += red[w][lane];
        const float d = (float)s * lam_factor(lam[c]);
        dlam[c] = accumulate ? dlam[c] + d : d;
    }
}

// A few tokens: four channels of a sequence a thread, token after token, the next token's inputs under way.  Bound by latency: one token of 2560 channels
// 4.2 us, of 64 x 5120 5.2.
template <typename T, bool VEC>
__global__ __launch_bounds__(64) void k_gated_scan_step(ScanParams sp) {
    const int c = (blockIdx.x * 64 + threadIdx.x) * 4, b = blockIdx.y, left = sp.C - c;
    if (left <= 0) return;
    Four<T> nx, nr, ni;
    auto load = [&](int64_t t) {
        nr.template load<VEC>(rows_at<T>(sp.gr, b * sp.g_bs + t * sp.g_rs, 0, 1, sp.C), c * Four<T>::SIZE, left);
        ni.template load<VEC>(rows_at<T>(sp.gi, b * sp.g_bs + t * sp.g_rs, 0, 1, sp.C), c * Four<T>::SIZE, left);
        nx.template load<VEC>(rows_at<T>(sp.x, b * sp.x_bs + t * sp.x_rs, 0, 1, sp.C), c * Four<T>::SIZE, left);
    };
    load(0);
    const int64_t at = (int64_t)b * sp.C + c;
    float h[4], slope[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        h[e] = e < left ? sp.init[at + e] : 0.f;
        slope[e] = e < left ? slope_of(sp.lam[c + e], sp.rate) : 0.f;
    }
    for (int64_t t = 0; t < sp.L; ++t) {
        const Four<T> x = nx, r = nr, i = ni;
        if (t + 1 < sp.L) load(t + 1);
        Four<T> o;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const Decay d = decay(slope[e] * sigmoid1(r.get(e)));
            h[e] = fmaf(d.a, h[e], d.m * sigmoid1(i.get(e)) * x.get(e));
            o.set(e, h[e]);
        }
        o.template store<VEC>(rows_at<T>(sp.out, b * sp.o_bs + t * sp.o_rs, 0, 1, sp.C), c * Four<T>::SIZE, left);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < left) sp.final_state[at + e] = h[e];
}

// A state or its adjoint where there are no tokens: as it came, or zeros.
__global__ __launch_bounds__(256) void k_gated_scan_pass(const float* from, float* to, int64_t n) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) to[i] = from ? from[i] : 0.f;
}

int check(const ssd_gated_scan_shape_t* sh, ScanParams* sp) {
    if (!sh) return SSD_ERR_NULL;
    if (sh->dtype != SSD_F32 && sh->dtype != SSD_BF16) return SSD_ERR_DTYPE;
    if (sh->channels <= 0 || sh->channels > MAX_STRIDE || sh->batch <= 0 || sh->batch > 65535 || sh->seqlen < 0 || sh->seqlen > ((int64_t)1 << 32)) return SSD_ERR_SHAPE;
    if (!(sh->rate > 0.f) || !(sh->rate <= 3.4e38f)) return SSD_ERR_ARG;
    memset(sp, 0, sizeof(*sp));
    sp->C = sh->channels;
    sp->Bt = (int)sh->batch;
    sp->L = sh->seqlen;
    sp->nchunks = (sh->seqlen + KEPT - 1) / KEPT;
    sp->rate = sh->rate;
    sp->reset = sh->seq_reset;
    const int64_t rows[5] = {sh->x_row_stride, sh->gate_row_stride, sh->out_row_stride, sh->dx_row_stride, sh->dgate_row_stride};
    const int64_t batches[5] = {sh->x_batch_stride, sh->gate_batch_stride, sh->out_batch_stride, sh->dx_batch_stride, sh->dgate_batch_stride};
    int64_t* const rs[5] = {&sp->x_rs, &sp->g_rs, &sp->o_rs, &sp->dx_rs, &sp->dg_rs};
    int64_t* const bs[5] = {&sp->x_bs, &sp->g_bs, &sp->o_bs, &sp->dx_bs, &sp->dg_bs};
    for (int k = 0; k < 5; ++k) {
        *rs[k] = rows[k] ? rows[k] : sp->C;
        if (*rs[k] < sp->C || *rs[k] > MAX_STRIDE) return SSD_ERR_SHAPE;
        const int64_t least = sp->L > 0 ? (sp->L - 1) * *rs[k] + sp->C : 0;
        *bs[k] = batches[k] ? batches[k] : sp->L * *rs[k];
        if (sp->Bt > 1 && *bs[k] < least) return SSD_ERR_SHAPE;
        if (*bs[k] < 0 || *bs[k] > ((int64_t)1 << 46)) return SSD_ERR_SHAPE;
    }
    // a workgroup for every chunk and tile
    if (sp->nchunks * sp->Bt * ((sp->C + TILE - 1) / TILE) > 0x7fffffff) return SSD_ERR_SHAPE;
    return SSD_OK;
}

bool al(const void* p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
bool elements(int dtype, std::initializer_list<const void*> ptrs) {
    for (const void* p : ptrs)
        if (!al(p, dtype == SSD_BF16 ? 2 : 4)) return false;
    return true;
}
size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }
// The workspace: counters, slopes, the words of chunks and groups (none for a single chunk), backward the chunks' sums for dlam.
struct Layout {
    size_t tickets, slopes, runs, ends, part, total;
    int64_t Cp, chunks, side;
};
Layout layout(const ScanParams& sp, bool bwd) {
    Layout l;
    l.Cp = (int64_t)((sp.C + TILE - 1) / TILE) * TILE;
    const int64_t chunk = 4 * WAVES * (bwd ? K_BWD : K_FWD);
    l.chunks = (sp.L + chunk - 1) / chunk;
    const size_t row = (size_t)sp.Bt * l.Cp, n = l.chunks > 1 ? (size_t)l.chunks : 0;
    l.side = sp.Bt * (l.Cp / TILE);
    l.tickets = 256;  // a workspace is never empty
    l.slopes = l.tickets + (n ? up256((size_t)l.side * TICKET * 4) : 0);
    l.runs = l.slopes + (n ? up256((size_t)l.Cp * 4) : 0);
    l.ends = l.runs + up256(n * row * 8);
    l.part = l.ends + up256((n + GROUP - 1) / GROUP * row * 4);
    l.total = l.part + (bwd ? up256((size_t)(sp.nchunks > 0 ? sp.nchunks : 1) * sp.Bt * sp.C * 4) : 0);
    return l;
}
Chain chain_of(const Layout& l, void* ws) {
    char* const p = (char*)ws;
    return {(uint32_t*)(p + l.tickets), (uint64_t*)(p + l.runs), (uint32_t*)(p + l.ends), (float*)(p + l.slopes), (uint32_t)l.chunks};
}
// The launch in front, where there are several chunks.
void clear_chain(const ScanParams& sp, const Layout& l, const Chain& ch, hipStream_t st) {
    if (l.chunks <= 1) return;
    const int64_t n = (int64_t)(l.part - l.runs) / 16;
    hipLaunchKernelGGL(k_gated_scan_clear, dim3((unsigned)(n < 1024 * 256 ? (n + 255) / 256 : 1024)), dim3(256), 0, st, ch, l.side, (uint4*)ch.runs, n, sp.lam, sp.C, sp.rate);
}
bool fours(const ScanParams& sp, int dtype, bool bwd, std::initializer_list<const void*> ptrs) {
    for (int64_t v : {(int64_t)sp.C, sp.x_rs, sp.g_rs, sp.o_rs, sp.x_bs, sp.g_bs, sp.o_bs})
        if (v % 4) return false;
    for (int64_t v : {sp.dx_rs, sp.dg_rs, sp.dx_bs, sp.dg_bs})
        if (bwd && v % 4) return false;
    for (const void* p : ptrs)
        if (!al(p, dtype == SSD_BF16 ? 8 : 16)) return false;
    return true;
}
#define SCAN_LAUNCH3(KERNEL, T, VEC, RESET)                                                                          \
    do {                                                                                                             \
        if (lay.chunks > 1) hipLaunchKernelGGL((KERNEL<T, VEC, RESET, true>), grid, block, 0, st, sp, chain);        \
        else hipLaunchKernelGGL((KERNEL<T, VEC, RESET, false>), grid, block, 0, st, sp, chain);                      \
    } while (0)
#define SCAN_LAUNCH2(KERNEL, T)                                       \
    do {                                                              \
        if (vec && sp.reset) SCAN_LAUNCH3(KERNEL, T, true, true);     \
        else if (vec) SCAN_LAUNCH3(KERNEL, T, true, false);           \
        else if (sp.reset) SCAN_LAUNCH3(KERNEL, T, false, true);      \
        else SCAN_LAUNCH3(KERNEL, T, false, false);                   \
    } while (0)
#define SCAN_LAUNCH(KERNEL)                                                                                    \
    do {                                                                                                       \
        const Grid g = grid_of((uint32_t)(lay.chunks * lay.side));                                             \
        const dim3 grid(g.x, g.y), block(64 * WAVES);                                                          \
        if (sh->dtype == SSD_BF16) SCAN_LAUNCH2(KERNEL, bf16_t);                                               \
        else SCAN_LAUNCH2(KERNEL, float);                                                                      \
    } while (0)
unsigned pass_grid(int64_t n) { return (unsigned)(n < 262144 ? (n + 255) / 256 : 1024); }
int done() { return hipGetLastError() == hipSuccess ? SSD_OK : SSD_ERR_LAUNCH; }

}  // namespace
}  // namespace ssdk

using namespace ssdk;

extern "C" size_t ssd_gated_scan_workspace_bytes(const ssd_gated_scan_shape_t* sh, int32_t is_backward) {
    ScanParams sp;
    if (check(sh, &sp) != SSD_OK) return 0;
    return layout(sp, is_backward != 0).total;
}

extern "C" int ssd_gated_scan_fwd(const ssd_gated_scan_shape_t* sh, const void* x, const void* gate_r, const void* gate_i, const float* lam,
                                  const float* init_state, void* out, float* final_state, float* states, void* workspace, size_t workspace_bytes,
                                  void* hip_stream) {
    ScanParams sp;
    const int rc = check(sh, &sp);
    if (rc != SSD_OK) return rc;
    hipStream_t st = (hipStream_t)hip_stream;
    if (!al(init_state, 4) || !al(final_state, 4) || !al(states, 4)) return SSD_ERR_ARG;
    if (sp.L == 0) {
        if (!final_state) return SSD_OK;
        const int64_t n = (int64_t)sp.Bt * sp.C;
        hipLaunchKernelGGL(k_gated_scan_pass, dim3(pass_grid(n)), dim3(256), 0, st, init_state, final_state, n);
        return done();
    }
    if (!x || !gate_r || !gate_i || !lam || !out) return SSD_ERR_NULL;
    if (!elements(sh->dtype, {x, gate_r, gate_i, out}) || !al(lam, 4)) return SSD_ERR_ARG;
    if (!workspace || !al(workspace, 256) || workspace_bytes < ssd_gated_scan_workspace_bytes(sh, 0)) return SSD_ERR_WORKSPACE;
    sp.x = x, sp.gr = gate_r, sp.gi = gate_i, sp.lam = lam, sp.init = init_state, sp.out = out, sp.final_state = final_state, sp.states = states;
    const Layout lay = layout(sp, false);
    const Chain chain = chain_of(lay, workspace);
    const bool vec = fours(sp, sh->dtype, false, {x, gate_r, gate_i, out});
    clear_chain(sp, lay, chain, st);
    SCAN_LAUNCH(k_gated_scan_fwd);
    return done();
}

extern "C" int ssd_gated_scan_bwd(const ssd_gated_scan_shape_t* sh, const void* x, const void* gate_r, const void* gate_i, const float* lam,
                                  const float* states, const void* dout, const float* dfinal_state, void* dx, void* dgate_r, void* dgate_i,
                                  float* dlam, float* dinit_state, void* workspace, size_t workspace_bytes, uint32_t flags, void* hip_stream) {
    ScanParams sp;
    const int rc = check(sh, &sp);
    if (rc != SSD_OK) return rc;
    if (flags & ~(uint32_t)SSD_FLAG_ACCUM_PARAM) return SSD_ERR_ARG;
    if (!dlam) return SSD_ERR_NULL;
    if (!al(dlam, 4) || !al(dinit_state, 4) || !al(dfinal_state, 4) || !al(states, 4)) return SSD_ERR_ARG;
    hipStream_t st = (hipStream_t)hip_stream;
    const int accumulate = flags & SSD_FLAG_ACCUM_PARAM ? 1 : 0;
    if (sp.L == 0) {
        const int64_t n = (int64_t)sp.Bt * sp.C;
        if (dinit_state) hipLaunchKernelGGL(k_gated_scan_pass, dim3(pass_grid(n)), dim3(256), 0, st, dfinal_state, dinit_state, n);
        if (!accumulate) hipLaunchKernelGGL(k_gated_scan_pass, dim3(pass_grid(sp.C)), dim3(256), 0, st, (const float*)nullptr, dlam, (int64_t)sp.C);
        return done();
    }
    if (!x || !gate_r || !gate_i || !lam || !states || !dout || !dx || !dgate_r || !dgate_i) return SSD_ERR_NULL;
    if (!elements(sh->dtype, {x, gate_r, gate_i, dout, dx, dgate_r, dgate_i}) || !al(lam, 4)) return SSD_ERR_ARG;
    if (!workspace || !al(workspace, 256) || workspace_bytes < ssd_gated_scan_workspace_bytes(sh, 1)) return SSD_ERR_WORKSPACE;
    sp.x = x, sp.gr = gate_r, sp.gi = gate_i, sp.lam = lam, sp.states_in = states, sp.dout = dout, sp.dfinal = dfinal_state;
    sp.dx = dx, sp.dgr = dgate_r, sp.dgi = dgate_i, sp.dinit = dinit_state;
    const Layout lay = layout(sp, true);
    const Chain chain = chain_of(lay, workspace);
    sp.part = (float*)((char*)workspace + lay.part);
    const bool vec = fours(sp, sh->dtype, true, {x, gate_r, gate_i, dout, dx, dgate_r, dgate_i});
    clear_chain(sp, lay, chain, st);
    SCAN_LAUNCH(k_gated_scan_bwd);
    if (done() != SSD_OK) return SSD_ERR_LAUNCH;  // there are no shares to add up
    hipLaunchKernelGGL(k_gated_scan_dlam, dim3((sp.C + 63) / 64), dim3(COLSUM_THREADS), 0, st, sp.part, sp.nchunks * sp.Bt, sp.C, lam, dlam, accumulate);
    return done();
}

extern "C" int ssd_gated_scan_step(const ssd_gated_scan_shape_t* sh, const void* x, const void* gate_r, const void* gate_i, const float* lam,
                                   const float* state_in, float* state_out, void* out, void* hip_stream) {
    ScanParams sp;
    const int rc = check(sh, &sp);
    if (rc != SSD_OK) return rc;
    if (sh->seq_reset) return SSD_ERR_ARG;
    if (!state_in || !state_out) return SSD_ERR_NULL;
    if (!al(state_in, 4) || !al(state_out, 4)) return SSD_ERR_ARG;
    hipStream_t st = (hipStream_t)hip_stream;
    const int64_t n = (int64_t)sp.Bt * sp.C;
    if (sp.L == 0) {
        if (state_in != state_out) hipLaunchKernelGGL(k_gated_scan_pass, dim3(pass_grid(n)), dim3(256), 0, st, state_in, state_out, n);
        return done();
    }
    if (!x || !gate_r || !gate_i || !lam || !out) return SSD_ERR_NULL;
    if (!elements(sh->dtype, {x, gate_r, gate_i, out}) || !al(lam, 4)) return SSD_ERR_ARG;
    sp.x = x, sp.gr = gate_r, sp.gi = gate_i, sp.lam = lam, sp.init = state_in, sp.final_state = state_out, sp.out = out;
    const dim3 grid((sp.C + 255) / 256, sp.Bt);
    const bool vec = fours(sp, sh->dtype, false, {x, gate_r, gate_i, out});
    if (sh->dtype == SSD_BF16) {
        if (vec) hipLaunchKernelGGL((k_gated_scan_step<bf16_t, true>), grid, dim3(64), 0, st, sp);
        else hipLaunchKernelGGL((k_gated_scan_step<bf16_t, false>), grid, dim3(64), 0, st, sp);
    } else {
        if (vec) hipLaunchKernelGGL((k_gated_scan_step<float, true>), grid, dim3(64), 0, st, sp);
        else hipLaunchKernelGGL((k_gated_scan_step<float, false>), grid, dim3(64), 0, st, sp);
    }
    return done();
}
