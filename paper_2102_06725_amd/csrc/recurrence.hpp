// recurrence.hpp -- what the kernels of the gated linear recurrence share: gates, lanes, and
// the exchange between workgroups.
//
// h_t = a_t h_(t-1) + u_t is a composition of affine maps, so a stretch of tokens is the pair
// (A, H) of h_out = A h_in + H, and stretches can be computed apart and joined:
//   - a lane holds two neighbouring channels (one 4-byte load of a 16-bit
//     tensor) and walks 16 tokens that it keeps in registers; a wave covers 128
//     channels (or, of 64 channels and fewer, 16 tokens with each of its teams of
//     lanes), and the waves of a workgroup consecutive tokens (a chunk);
//   - the waves exchange their (A, H) through LDS;
//   - chunks exchange theirs through one 64-bit word per channel in the
//     workspace (below).  The inputs are read once, and y is computed from
//     registers.
// Whether a token takes part is the same for a whole wave, so lengths and the end of the
// sequence cost no divergence.
//
// Bound by memory (8 bytes a token and channel forward, 14 backward), and close behind it by
// the vector units: a forward element takes 37 instructions, 4 of them transcendental, which
// alone would take half of the time.  Measured, cold: forward of 8 x 2048 x 1152 36 us (4.2
// TB/s), backward 59 us (4.5 TB/s); forward of 2 x 32768 x 768 93 us (4.3 TB/s; the same
// elements as 512 sequences of 128 tokens, one chunk each, 74 us).  Short calls are bound by
// their launches and one exchange between workgroups: 6 us for one chunk, 10 for two.
//
// Chunks: forward 8 waves of 16 tokens, backward 4 of 16, the most that leave two workgroups to
// a compute unit: what is on its way and what waits for its predecessors are then never the
// same.  With one team a wave the kernels take 123 and 253 registers; with several, whose
// addresses are a lane's own, all 128 and 256, and 7 to 10 (forward) and 2 (backward, from four
// teams on) are kept in memory.  16 waves of 8 tokens, 4 of 32 and 16 of 16 took 103,
// 102 and 98 us where 8 of 16 take 97, chunks of half the tokens 115; backward, 8 waves of 8
// and 16 of 4 took 65 and 66 us where 4 of 16 take 55.
#pragma once

#include <type_traits>

#include "launch.hpp"

namespace nnconv {

// How a call is split.  Chunks of waves * teams * 16 tokens; more than one only with the most
// waves.
struct RecGrid {
    int32_t cols, waves, teams, chunks, gs, groups;
    uint64_t *words;   // [n][chunks][c], null for a single chunk
    uint64_t *states;  // [n][groups][c]
};

constexpr int FWD_WAVES = 8, BWD_WAVES = 4;  // at most
constexpr int TOKENS = 16;                   // of a team
// Up to here a lane walks all tokens, without a barrier (forward of 4096 x 6 x 1152 39 us, 52 as
// a chunk; with 8 tokens 54 and 59, backward 164 and 128).
constexpr int SHORT_T = 6;

// One column of channels and one chunk a workgroup; `blocks` of them.  dtype, and whether p.g
// is given, choose the kernel, and q.waves and q.teams.
void launch_recurrence_fwd_chunks(int dtype, const RecParams &p, const RecGrid &q, uint32_t blocks, hipStream_t st);
void launch_recurrence_bwd_chunks(int dtype, const RecParams &p, const RecGrid &q, uint32_t blocks, hipStream_t st);
// t <= SHORT_T; c = 1.
void launch_recurrence_fwd_short(int dtype, const RecParams &p, hipStream_t st);
void launch_recurrence_bwd_short(int dtype, const RecParams &p, hipStream_t st);
void launch_recurrence_fwd_single(int dtype, const RecParams &p, hipStream_t st);
void launch_recurrence_bwd_single(int dtype, const RecParams &p, hipStream_t st);

constexpr uint64_t NO_WORD = ~0ull;  // a word that is not written yet

namespace {

constexpr int SAVE = NNCONV_RECURRENCE_SAVE;
constexpr int COLS = 128;                 // channels of a wave
constexpr float A_MIN = 0x1p-126f;        // products of gates stay above 0: 0 * inf would be NaN

typedef uint32_t __attribute__((aligned(2))) u32_any;  // 4-byte access at any element

constexpr float LOG2E = 1.4426950408889634f;
constexpr float Z_MAX = 80.f * LOG2E;

// The gate a = sigma(z) and b = 1 - a = sigma(-z), each with a relative error of its own: with a
// near 1 the difference 1 - a would keep few bits of the long memories' rates.  bias is the
// negated bias times log2(e): -z log2(e) is one multiply-add, whose roundings, of the bias's
// product and of log2(e) itself the exponential turns into relative ones.  Both are within (|z| +
// 1.3 |bias| + 0.3 |f| + 5) 2^-24 (the arithmetic emulated with f from a normal distribution and
// biases up to 7: 15 * 2^-24 for b, 5 * 2^-24 for a).  The limits let a NaN through.
__device__ __forceinline__ void gate(float f, float bias, float &a, float &b) {
    float z = __builtin_fmaf(f, -LOG2E, bias);
    z = __builtin_elementwise_minimum(__builtin_elementwise_maximum(z, -Z_MAX), Z_MAX);
    const float e = __builtin_amdgcn_exp2f(z);
    // one Newton step on the reciprocal, whose own error of up to a unit has a sign: a product
    // of a thousand gates near 1 would add it up
    const float d = 1.0f + e, r = __builtin_amdgcn_rcpf(d);
    a = __builtin_fmaf(r, __builtin_fmaf(-d, r, 1.0f), r);
    b = e * a;
}

__device__ __forceinline__ float sigma(float v) {
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(v * -LOG2E));
}

__device__ __forceinline__ int length_of(const RecParams &p, int n) {
    if (!p.lengths) return p.t;
    const int l = p.lengths[n];
    return l < 0 ? 0 : l > p.t ? p.t : l;
}

// The two channels of a lane.  c >= 2: a lane whose second channel would be past the end (the
// last one of an odd count) takes the last two, the first of which is its neighbour's, and
// writes the second alone: the neighbour may be in another workgroup, and states may be updated
// in place. Lanes past the end load the last two and write nothing.
struct Lane {
    uint32_t at;  // first channel
    int k0, k1;   // the channels, for per-channel fp32 arrays and words
    bool both, second;  // channels that it writes
    bool odd;           // c is odd, the same for all lanes

    __device__ __forceinline__ Lane(int c0, int c) {
        at = c0 < c - 2 ? c0 : c - 2;
        both = c0 + 1 < c;
        second = c0 < c;
        odd = c & 1;
        k0 = at;
        k1 = at + 1;
    }
};

template <class T>
__device__ __forceinline__ void unpack(uint32_t v, float o[2]);

template <>
__device__ __forceinline__ void unpack<Half>(uint32_t v, float o[2]) {
    o[0] = from16<Half>(v & 0xFFFFu);
    o[1] = from16<Half>(v >> 16);
}

template <>
__device__ __forceinline__ void unpack<BFloat>(uint32_t v, float o[2]) {
    o[0] = __builtin_bit_cast(float, v << 16);
    o[1] = __builtin_bit_cast(float, v & 0xFFFF0000u);
}

// The token at `row`, an address that is the same for the whole wave: in scalar registers, so
// that an access costs no address arithmetic on the vector units.
typedef __attribute__((address_space(1))) char global_char;

__device__ __forceinline__ global_char *uniform(const void *row) {
    uint64_t v = (uint64_t)row;
    asm("" : "+s"(v));
    return (global_char *)v;
}

typedef __attribute__((address_space(1))) u32_any global_u32_any;
typedef __attribute__((address_space(1))) uint16_t global_u16;

// A lane's two channels of a token.  U: the token is the same for the whole wave.
template <bool U = true>
__device__ __forceinline__ uint32_t load2(const void *row, const Lane &L) {
    global_char *r = U ? uniform(row) : (global_char *)(uintptr_t)row;
    return *(const global_u32_any *)(r + (uint32_t)(2 * L.at));
}

// N tensors' two channels of a token, in one masked region.  full (the same for the wave): all
// its channels exist.
template <class T, int N, bool U = true>
__device__ __forceinline__ void store2(void *const row[N], const Lane &L, bool full, const float v[N][2]) {
    uint32_t q[N];
    global_char *to[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
        q[k] = pack16<T>(v[k][0], v[k][1]);
        to[k] = (U ? uniform(row[k]) : (global_char *)(uintptr_t)row[k]) + (uint32_t)(2 * L.at);
    }
    if (full || L.both)
#pragma unroll
        for (int k = 0; k < N; ++k) __builtin_nontemporal_store(q[k], (global_u32_any *)to[k]);
    if (!full && L.odd)
        if (L.second && !L.both)
#pragma unroll
            for (int k = 0; k < N; ++k) ((global_u16 *)to[k])[1] = (uint16_t)(q[k] >> 16);
}

// Two fp32 values of a per-channel array.
__device__ __forceinline__ void put2(float *to, const Lane &L, float v0, float v1) {
    if (L.both) to[L.k0] = v0;
    if (L.second) to[L.k1] = v1;
}

// Few channels: a wave's lanes are NG teams of 64 / NG, which take S tokens each, one team's
// after the other's; otherwise the wave is one team.
template <int NG>
struct Team {
    static constexpr int LANES = 64 / NG;
    int lane, w;  // in the wave, and the wave
    int c;        // lane in the team
    int r;        // the team among the workgroup's, the same for a wave that is one

    __device__ __forceinline__ Team() {
        lane = threadIdx.x & 63;
        w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        c = NG == 1 ? lane : lane % LANES;
        r = NG == 1 ? w : w * NG + lane / LANES;
    }

    // Place in LDS of team v's value for this lane's channels.
    __device__ __forceinline__ int of(int v) const { return v * LANES + c; }
    __device__ __forceinline__ bool first_of_wave() const { return NG == 1 || lane < LANES; }
    static __device__ __forceinline__ bool all(bool b) { return NG == 1 ? b : (bool)__all(b); }
};

// ---- words between chunks ------------------------------------------------------

// Chunks are taken in the direction of the recurrence: place k of a sequence. Two arrays of
// 64-bit words, all ones until written: the (A, H) of every place, and the state in front of
// every group of 2^gs places: a place waits for the pairs in front of it in its group, all at
// once, and for the group's state, which the last place of the group before hands on.  A word
// is stored and loaded at once, so it needs no flag and no ordering with other memory.  Which
// words are composed, and in which order, depends on the sizes alone, so that results do not
// depend on which workgroup came first.
constexpr int GROUP = 32;  // places of a group at most
constexpr int ROUND = 16;  // rows of words that a workgroup has on their way at once
// Looks at a word that is not there before it is computed.  0 (a build for tests): no word is ever
// looked at but the first group's state, which is there before the call, so that every pair and
// state is computed again.
#ifndef NNCONV_RECURRENCE_LOOKS
#define NNCONV_RECURRENCE_LOOKS 4096
#endif
constexpr int POLLS = NNCONV_RECURRENCE_LOOKS;

__device__ __forceinline__ uint64_t word(float a, float h) {
    return (uint64_t)__builtin_bit_cast(uint32_t, a) |
           ((uint64_t)__builtin_bit_cast(uint32_t, h) << 32);
}

__device__ __forceinline__ float word_a(uint64_t v) { return __builtin_bit_cast(float, (uint32_t)v); }
__device__ __forceinline__ float word_h(uint64_t v) { return __builtin_bit_cast(float, (uint32_t)(v >> 32)); }

__device__ __forceinline__ void put(uint64_t *row, const Lane &L, const float a[2], const float h[2]) {
    if (L.both) __hip_atomic_store(row + L.k0, word(a[0], h[0]), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (L.second) __hip_atomic_store(row + L.k1, word(a[1], h[1]), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// A lane's two words of a row.
struct Words {
    uint64_t v0, v1;

    __device__ __forceinline__ void load(const uint64_t *row, const Lane &L) {
        v0 = __hip_atomic_load(row + L.k0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        v1 = __hip_atomic_load(row + L.k1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }

    // Whether the whole wave has its words.
    __device__ __forceinline__ bool there() const { return POLLS > 0 && !__any(v0 == NO_WORD || v1 == NO_WORD); }

    // Looks again until they are there, POLLS times at most.
    __device__ __forceinline__ bool wait(const uint64_t *row, const Lane &L) {
        for (int k = 0; !there(); ++k) {
            if (k >= POLLS) return false;
            __builtin_amdgcn_s_sleep(1);
            load(row, L);
        }
        return true;
    }

    __device__ __forceinline__ void unpack(float a[2], float h[2]) const {
        a[0] = word_a(v0);
        a[1] = word_a(v1);
        h[0] = word_h(v0);
        h[1] = word_h(v1);
    }
};

__device__ __forceinline__ void compose(float A[2], float H[2], const float a[2], const float h[2]) {
    H[0] = __builtin_fmaf(a[0], H[0], h[0]);
    H[1] = __builtin_fmaf(a[1], H[1], h[1]);
    A[0] = fmaxf(A[0] * a[0], A_MIN);
    A[1] = fmaxf(A[1] * a[1], A_MIN);
}

// The state in front of place k, for all waves.  (ca, ch): the place's own pair, known to wave
// `own`, whose lanes with `writes` publish it.  A word that stays empty for POLLS looks is
// computed here instead (chunk_pair(place, a, h) walks that place's tokens), so that every wait
// ends whatever order the workgroups run in.
template <int W, class F>
__device__ __forceinline__ void carry_in(const RecGrid &q, int n, int32_t c, int k, const Lane &L, bool writes, int w,
                                         int own, const float ca[2], const float ch[2], F chunk_pair,
                                         float out[2]) {
    __shared__ f32x4 pairs[GROUP][64];
    __shared__ float into[2][64];
    const int lane = threadIdx.x & 63, group = 1 << q.gs, g = k >> q.gs, i = k & (group - 1);
    const bool last = i + 1 == group;
    uint64_t *words = q.words + (int64_t)n * q.chunks * c, *states = q.states + (int64_t)n * q.groups * c;
    if (w == own && writes && !last && k + 1 < q.chunks) put(words + (int64_t)k * c, L, ca, ch);
    constexpr int R = ROUND / W;
    for (int j0 = w; j0 < i; j0 += ROUND) {
        Words v[R];
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (j0 + r * W < i) v[r].load(words + (int64_t)(g * group + j0 + r * W) * c, L);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int j = j0 + r * W;
            if (j >= i) break;
            float a[2], h[2];
            if (v[r].wait(words + (int64_t)(g * group + j) * c, L))
                v[r].unpack(a, h);
            else
                chunk_pair(g * group + j, a, h);
            pairs[j][lane] = f32x4{a[0], h[0], a[1], h[1]};
        }
    }
    Words s;
    if (w == own) s.load(states + (int64_t)g * c, L);
    __syncthreads();
    if (w == own) {
        float A[2] = {1.f, 1.f}, H[2] = {0.f, 0.f}, no[2], h[2];
        for (int j = 0; j < i; ++j) {
            const f32x4 e = pairs[j][lane];
            const float ea[2] = {e[0], e[2]}, eh[2] = {e[1], e[3]};
            compose(A, H, ea, eh);
        }
        if (s.wait(states + (int64_t)g * c, L)) {
            s.unpack(no, h);
        } else {
            // from the nearest state there is; the first one was there before the call
            int from = g;
            do {
                from = from > 0 ? from - 1 : 0;
                s.load(states + (int64_t)from * c, L);
            } while (from > 0 && !s.there());
            s.unpack(no, h);
            for (; from < g; ++from) {
                float ga[2] = {1.f, 1.f}, gh[2] = {0.f, 0.f}, a[2], b[2];
                for (int j = 0; j + 1 < group; ++j) {
                    chunk_pair(from * group + j, a, b);
                    compose(ga, gh, a, b);
                }
                chunk_pair(from * group + group - 1, a, b);
                for (int u = 0; u < 2; ++u)
                    h[u] = __builtin_fmaf(a[u], __builtin_fmaf(ga[u], h[u], gh[u]), b[u]);
            }
        }
        h[0] = __builtin_fmaf(A[0], h[0], H[0]);
        h[1] = __builtin_fmaf(A[1], h[1], H[1]);
        if (writes && last && k + 1 < q.chunks) {
            const float next[2] = {__builtin_fmaf(ca[0], h[0], ch[0]), __builtin_fmaf(ca[1], h[1], ch[1])};
            const float zero[2] = {0.f, 0.f};
            put(states + (int64_t)(g + 1) * c, L, zero, next);
        }
        into[0][lane] = h[0];
        into[1][lane] = h[1];
    }
    __syncthreads();
    out[0] = into[0][lane];
    out[1] = into[1][lane];
}

// Kernels by type, gate and teams.
template <class F>
void with_kind(int dtype, bool g, F f) {
    if (dtype == Half::id) {
        if (g) f(Half{}, std::true_type{}); else f(Half{}, std::false_type{});
    } else {
        if (g) f(BFloat{}, std::true_type{}); else f(BFloat{}, std::false_type{});
    }
}

template <int N>
using Int = std::integral_constant<int, N>;

inline dim3 short_grid(const RecParams &p) { return dim3((p.c + COLS - 1) / COLS, p.n < 65535 ? p.n : 65535); }

}  // namespace

}  // namespace nnconv
