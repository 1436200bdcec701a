// recurrence.hip -- gated linear recurrence over the tokens of a sequence,
// channel by channel, forward and backward.
//
// h_t = a_t h_(t-1) + u_t is a composition of affine maps, so a stretch of
// tokens is the pair (A, H) of h_out = A h_in + H, and stretches can be
// computed apart and joined:
//   - a lane holds two neighbouring channels (one 4-byte load of a 16-bit
//     tensor) and walks S tokens that it keeps in registers; a wave covers 128
//     channels, the W waves of a workgroup W * S consecutive tokens (a chunk);
//   - the waves exchange their (A, H) through LDS;
//   - chunks exchange theirs through one 64-bit word per channel in the
//     workspace (below).  The inputs are read once, and y is computed from
//     registers.
// Whether a token takes part is the same for a whole wave, so lengths
// and the end of the sequence cost no divergence.
//
// Bound by memory (8 bytes a token and channel forward, 14 backward), and close behind it by the
// vector units: a forward element takes 37 instructions, 4 of them transcendental, which alone
// would take half of the time.  Measured, cold: forward of 8 x 2048 x 1152
// 37 us (4.1 TB/s), backward 60 us (4.4 TB/s); forward of 2 x 32768 x 768 95 us (4.2 TB/s; the
// same elements as 512 sequences of 128 tokens, one chunk each, 74 us).  Short
// calls are bound by their launches and one exchange between workgroups: 6 us
// for one chunk, 10 for two.
//
// Chunks: forward 8 waves of 16 tokens, backward 4 of 16, the most that leave two
// workgroups to a compute unit (126 and 248 registers): what is on its way and what waits for
// its predecessors are then never the same.  16 waves of 8 tokens, 4 of 32 and 16 of 16 took 103, 102 and
// 98 us where 8 of 16 take 97, chunks of half the tokens 115; backward, 8 waves of 8 and 16 of 4
// took 65 and 66 us where 4 of 16 take 55.
#include <type_traits>

#include "launch.hpp"

namespace nnconv {

namespace {

constexpr int SAVE = NNCONV_RECURRENCE_SAVE;
constexpr int COLS = 128;                 // channels of a wave
constexpr float A_MIN = 0x1p-126f;        // products of gates stay above 0: 0 * inf would be NaN
constexpr int SHORT_T = 16;               // up to here one lane walks all tokens: no exchange, no barrier

typedef uint32_t __attribute__((aligned(2))) u32_any;  // 4-byte access at any element

constexpr float LOG2E = 1.4426950408889634f;
constexpr float Z_MAX = 80.f * LOG2E;

// The gate a = sigma(z) and b = 1 - a = sigma(-z), each to full relative
// precision: with a near 1 the difference 1 - a would keep few bits of the
// long memories' rates.  bias is the negated bias times log2(e): -z log2(e) is one
// multiply-add.  The limits let a NaN through.
__device__ __forceinline__ void gate(float f, float bias, float &a, float &b) {
    float z = __builtin_fmaf(f, -LOG2E, bias);
    z = __builtin_elementwise_minimum(__builtin_elementwise_maximum(z, -Z_MAX), Z_MAX);
    const float e = __builtin_amdgcn_exp2f(z);
    // one Newton step on the reciprocal, whose own error of up to a unit has a sign: a
    // product of a thousand gates near 1 would add it up
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
// last one of an odd count) takes the last two, the first of which is its neighbour's, and writes the second
// alone: the neighbour may be in another workgroup, and states may be updated in place.
// Lanes past the end load the last two and write nothing.
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

// The token at `row`, an address that is the same for the whole wave: in scalar
// registers, so that an access costs no address arithmetic on the vector units.
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

// N tensors' two channels of a token, in one masked region.  full (the same for the wave): all its
// channels exist.
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

// Few channels: a wave's lanes are NG teams of 64 / NG, which take S tokens each, one team's after
// the other's; otherwise the wave is one team.
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

// Chunks are taken in the direction of the recurrence: place k of a sequence.
// Two arrays of 64-bit words, all ones until written: the (A, H) of every place,
// and the state in front of every group of 2^gs places: a place waits for the pairs in front of
// it in its group, all at once, and for the group's state, which the last place of
// the group before hands on.  A word is stored and loaded at
// once, so it needs no flag and no ordering with other memory.  Which words are
// composed, and in which order, depends on the sizes alone, so that results
// do not depend on which workgroup came first.
struct RecGrid {
    int32_t cols, chunks, gs, groups;
    uint64_t *words;   // [n][chunks][c], null for a single chunk
    uint64_t *states;  // [n][groups][c]
};
constexpr int GROUP = 32;  // places of a group at most
constexpr int ROUND = 16;  // rows of words that a workgroup has on their way at once
constexpr uint64_t EMPTY = ~0ull;
constexpr int POLLS = 4096;

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
    __device__ __forceinline__ bool there() const { return !__any(v0 == EMPTY || v1 == EMPTY); }

    // Looks again until they are there, POLLS times at most.
    __device__ __forceinline__ bool wait(const uint64_t *row, const Lane &L) {
        for (int k = 0; !there(); ++k) {
            if (k == POLLS) return false;
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

// Before each split call: every word empty but the states in front of the
// first places.
__global__ __launch_bounds__(256) void recurrence_words_kernel(const RecGrid q, int64_t n, int32_t c,
                                                               const float *init) {
    const int64_t plain = n * q.chunks * c, total = plain + n * q.groups * c;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        uint64_t v = EMPTY;
        if (i >= plain) {
            const int64_t row = (i - plain) / c;
            if (row % q.groups == 0) v = word(0.f, init ? init[row / q.groups * c + (i - plain - row * c)] : 0.f);
        }
        q.words[i] = v;  // the states follow the words
    }
}

__device__ __forceinline__ void compose(float A[2], float H[2], const float a[2], const float h[2]) {
    H[0] = __builtin_fmaf(a[0], H[0], h[0]);
    H[1] = __builtin_fmaf(a[1], H[1], h[1]);
    A[0] = fmaxf(A[0] * a[0], A_MIN);
    A[1] = fmaxf(A[1] * a[1], A_MIN);
}

// The state in front of place k, for all waves.  (ca, ch): the place's own
// pair, known to wave `own`, whose lanes with `writes` publish it.  A word that stays empty for POLLS looks is computed here
// instead (chunk_pair(place, a, h) walks that place's tokens), so that every wait
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

// ---- forward ------------------------------------------------------------------

// Few tokens: a lane walks them all.
template <class T>
__global__ __launch_bounds__(64) void recurrence_fwd_short_kernel(const RecParams p) {
    const int lane = threadIdx.x;
    const Lane L(blockIdx.x * COLS + 2 * lane, p.c);
    for (int64_t n = blockIdx.y; n < p.n; n += gridDim.y) {
        const int len = length_of(p, (int)n);
        float h[2] = {0.f, 0.f}, bias[2] = {0.f, 0.f};
        if (p.h0) {
            h[0] = p.h0[n * p.c + L.k0];
            h[1] = p.h0[n * p.c + L.k1];
        }
        if (p.bias) {
            bias[0] = p.bias[L.k0] * -LOG2E;
            bias[1] = p.bias[L.k1] * -LOG2E;
        }
        const int64_t at = n * p.t * p.ld;
        const uint16_t *x = (const uint16_t *)p.x + at, *f = (const uint16_t *)p.f + at;
        const uint16_t *g = p.g ? (const uint16_t *)p.g + at : nullptr;
        uint16_t *y = (uint16_t *)p.y + n * p.t * p.ldy;
        if (p.saved && p.t > 0) {  // t <= SAVE: one state
            put2(p.saved + n * p.c, L, h[0], h[1]);
        }
        for (int t = 0; t < p.t; ++t) {
            float o[2] = {0.f, 0.f};
            if (t < len) {
                float xv[2], fv[2], gv[2];
                unpack<T>(load2(x + t * p.ld, L), xv);
                unpack<T>(load2(f + t * p.ld, L), fv);
                if (g) unpack<T>(load2(g + t * p.ld, L), gv);
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    float a, b;
                    gate(fv[k], bias[k], a, b);
                    h[k] = a * h[k] + b * xv[k];
                    o[k] = g ? h[k] * (gv[k] * sigma(gv[k])) : h[k];
                }
            }
            void *const row[1] = {y + t * p.ldy};
            store2<T, 1>(row, L, false, &o);
        }
        if (p.ht) put2(p.ht + n * p.c, L, h[0], h[1]);
    }
}

// The pair of a chunk, walked token by token with the arithmetic of the kernel below.
template <class T, int W, int S>
__device__ void walk_fwd(const RecParams &p, int64_t n, const Lane &L, int lo, int len,
                         const float bias[2], float A[2], float H[2]) {
    const int64_t at = n * p.t * p.ld;
    const uint16_t *x = (const uint16_t *)p.x + at, *f = (const uint16_t *)p.f + at;
    A[0] = A[1] = 1.f;
    H[0] = H[1] = 0.f;
    for (int w = 0; w < W; ++w) {
        float a1[2] = {1.f, 1.f}, h1[2] = {0.f, 0.f};
        for (int t = lo + w * S; t < min(lo + w * S + S, len); ++t) {
            float xv[2], fv[2];
            unpack<T>(load2(x + t * p.ld, L), xv);
            unpack<T>(load2(f + t * p.ld, L), fv);
            for (int k = 0; k < 2; ++k) {
                float a, b;
                gate(fv[k], bias[k], a, b);
                h1[k] = __builtin_fmaf(a, h1[k], b * xv[k]);
                a1[k] *= a;
            }
        }
        a1[0] = fmaxf(a1[0], A_MIN);
        a1[1] = fmaxf(a1[1], A_MIN);
        compose(A, H, a1, h1);
    }
}

template <class T, bool G, int W, int S, int NG>
__global__ __launch_bounds__(64 * W, 4) void recurrence_fwd_kernel(const RecParams p, const RecGrid q) {
    static_assert(SAVE % S == 0, "saved states lie at a team's first token");
    constexpr bool U = NG == 1;
    constexpr int TEAMS = W * NG, CHUNK = TEAMS * S;
    const Team<NG> team;
    const int w = team.w;
    const int col = blockIdx.x % q.cols, rest = blockIdx.x / q.cols;
    const int n = rest % p.n, chunk = rest / p.n;
    const Lane L(2 * (col * team.LANES + team.c), p.c);
    const int len = length_of(p, n);
    const int t0 = chunk * CHUNK + team.r * S, last = len > 0 ? len - 1 : 0;
    const int64_t at = (int64_t)n * p.t * p.ld;
    const uint16_t *x = (const uint16_t *)p.x + at, *f = (const uint16_t *)p.f + at;
    const uint16_t *g = G ? (const uint16_t *)p.g + at : nullptr;
    uint32_t xr[S], fr[S], gr[S];
    const bool whole = t0 + S <= len;           // every token takes part
    const bool full = (col + 1) * 2 * team.LANES <= p.c;  // every channel exists
    int64_t o = (int64_t)min(t0, last) * p.ld;
#pragma unroll
    for (int s = 0; s < S; ++s) {
        xr[s] = load2<U>(x + o, L);
        fr[s] = load2<U>(f + o, L);
        o += t0 + s < last ? p.ld : 0;
    }
    float bias[2] = {0.f, 0.f};
    if (p.bias) {
        bias[0] = p.bias[L.k0] * -LOG2E;
        bias[1] = p.bias[L.k1] * -LOG2E;
    }
    float a[S][2], u[S][2], A[2] = {1.f, 1.f}, H[2] = {0.f, 0.f};
#pragma unroll
    for (int s = 0; s < S; ++s) {
        float xv[2], fv[2];
        unpack<T>(xr[s], xv);
        unpack<T>(fr[s], fv);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            float b;
            gate(fv[k], bias[k], a[s][k], b);
            u[s][k] = b * xv[k];
        }
    }
    if (!whole)
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
            for (int k = 0; k < 2; ++k)
                if (t0 + s >= len) {
                    a[s][k] = 1.f;
                    u[s][k] = 0.f;
                }
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            H[k] = __builtin_fmaf(a[s][k], H[k], u[s][k]);
            A[k] *= a[s][k];
        }
    A[0] = fmaxf(A[0], A_MIN);
    A[1] = fmaxf(A[1], A_MIN);
    float h[2] = {0.f, 0.f};
    if (!q.words && p.h0) {  // before the barrier: ht, which another wave writes, may lie on it
        h[0] = p.h0[(int64_t)n * p.c + L.k0];
        h[1] = p.h0[(int64_t)n * p.c + L.k1];
    }
    __shared__ f32x4 part[W * 64];
    part[threadIdx.x] = f32x4{A[0], H[0], A[1], H[1]};
    __syncthreads();
    if (G) {  // not needed before the state is there: on their way during the wait
        o = (int64_t)min(t0, last) * p.ld;
#pragma unroll
        for (int s = 0; s < S; ++s) {
            gr[s] = load2<U>(g + o, L);
            o += t0 + s < last ? p.ld : 0;
        }
    }
    // what the teams in front make of the chunk's first state
    float pa[2] = {1.f, 1.f}, ph[2] = {0.f, 0.f};
    for (int v = 0; v < w * NG + NG - 1; ++v) {
        if (v >= team.r) continue;
        const f32x4 e = part[team.of(v)];
        const float ea[2] = {e[0], e[2]}, eh[2] = {e[1], e[3]};
        compose(pa, ph, ea, eh);
    }
    if (q.words) {
        float ca[2] = {pa[0], pa[1]}, ch[2] = {ph[0], ph[1]};
        compose(ca, ch, A, H);
        if (NG > 1)  // the last team's is the chunk's
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                ca[k] = __shfl(ca[k], 64 - team.LANES + team.c);
                ch[k] = __shfl(ch[k], 64 - team.LANES + team.c);
            }
        carry_in<W>(q, n, p.c, chunk, L, team.first_of_wave(), w, W - 1, ca, ch, [&](int place, float *a2, float *h2) {
            walk_fwd<T, TEAMS, S>(p, n, L, place * CHUNK, len, bias, a2, h2);
        }, h);
    }
    h[0] = pa[0] * h[0] + ph[0];
    h[1] = pa[1] * h[1] + ph[1];
    if (p.saved && t0 % SAVE == 0 && t0 < p.t) {
        float *to = p.saved + ((int64_t)n * ((p.t + SAVE - 1) / SAVE) + t0 / SAVE) * p.c;
        put2(to, L, h[0], h[1]);
    }
    uint16_t *y = (uint16_t *)p.y + (int64_t)n * p.t * p.ldy;
    y += (int64_t)t0 * p.ldy;
    auto finish = [&](auto checked) {
#pragma unroll
        for (int s = 0; s < S; ++s, y += p.ldy) {
            const int t = t0 + s;
            float o[2], gv[2];
            if (G) unpack<T>(gr[s], gv);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                h[k] = a[s][k] * h[k] + u[s][k];
                o[k] = G ? h[k] * (gv[k] * sigma(gv[k])) : h[k];
                if (checked && t >= len) o[k] = 0.f;
            }
            void *const row[1] = {y};
            if (!checked || t < p.t) store2<T, 1, U>(row, L, !checked, &o);
        }
    };
    if (team.all(whole) && full)
        finish(std::false_type{});
    else
        finish(std::true_type{});
    if (p.ht && chunk == q.chunks - 1 && team.r == TEAMS - 1) put2(p.ht + (int64_t)n * p.c, L, h[0], h[1]);
}

// ---- backward -------------------------------------------------------------------

// With own_t = dy_t g_t sigma(g_t), the gradient of h_t is d_t = own_t + r_t, where r_t
// flows in from the right: r_(t-1) = a_t d_t.  So r obeys the same kind
// of recurrence from the last token on, with a_t and a_t own_t.

// r in front of a token; not fused with the product that own is, so that every place that
// computes it gets the same bits.
__device__ __forceinline__ float before_token(float a, float own, float r) {
#pragma clang fp contract(off)
    return a * (own + r);
}

template <class T, bool G>
struct Grad {
    float a[2], b[2], x[2], own[2], dg[2];  // dg without the factor h_t

    __device__ __forceinline__ void make(uint32_t xq, uint32_t fq, uint32_t gq, uint32_t dyq, const float bias[2]) {
        float fv[2], gv[2], dy[2];
        unpack<T>(xq, x);
        unpack<T>(fq, fv);
        unpack<T>(dyq, dy);
        if (G) unpack<T>(gq, gv);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            gate(fv[k], bias[k], a[k], b[k]);
            own[k] = dy[k];
            dg[k] = 0.f;
            if (G) {
                const float s = sigma(gv[k]), sg = gv[k] * s;
                own[k] = dy[k] * sg;
                dg[k] = dy[k] * (s + sg * (1.f - s));
            }
        }
    }

    // A token past the length: the state passes through, nothing else happens.
    __device__ __forceinline__ void pass() {
        a[0] = a[1] = 1.f;
        b[0] = b[1] = x[0] = x[1] = own[0] = own[1] = dg[0] = dg[1] = 0.f;
    }
};

// Few tokens: a lane walks them all, forward for the states (t <= SHORT_T of
// them, in LDS) and back.
template <class T, bool G>
__global__ __launch_bounds__(64) void recurrence_bwd_short_kernel(const RecParams p) {
    __shared__ float hs[SHORT_T][2][64];
    const int lane = threadIdx.x;
    const Lane L(blockIdx.x * COLS + 2 * lane, p.c);
    float bias[2] = {0.f, 0.f};
    if (p.bias) {
        bias[0] = p.bias[L.k0] * -LOG2E;
        bias[1] = p.bias[L.k1] * -LOG2E;
    }
    for (int64_t n = blockIdx.y; n < p.n; n += gridDim.y) {
        const int len = length_of(p, (int)n);
        float r[2] = {0.f, 0.f}, total[2] = {0.f, 0.f};
        if (p.dht) {
            r[0] = p.dht[n * p.c + L.k0];
            r[1] = p.dht[n * p.c + L.k1];
        }
        const int64_t at = n * p.t * p.ld;
        const uint16_t *x = (const uint16_t *)p.x + at, *f = (const uint16_t *)p.f + at;
        const uint16_t *g = G ? (const uint16_t *)p.g + at : nullptr;
        const uint16_t *dy = (const uint16_t *)p.dy + n * p.t * p.ldy;
        uint16_t *dx = (uint16_t *)p.dx + at, *df = (uint16_t *)p.df + at;
        uint16_t *dg = G ? (uint16_t *)p.dg + at : nullptr;
        if (len > 0) {
            float h[2] = {p.saved[n * p.c + L.k0], p.saved[n * p.c + L.k1]};
            for (int t = 0; t < len; ++t) {
                float xv[2], fv[2];
                unpack<T>(load2(x + t * p.ld, L), xv);
                unpack<T>(load2(f + t * p.ld, L), fv);
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    float a, b;
                    gate(fv[k], bias[k], a, b);
                    hs[t][k][lane] = h[k];
                    h[k] = a * h[k] + b * xv[k];
                }
            }
        }
        for (int t = p.t - 1; t >= 0; --t) {
            float out[3][2] = {{0.f, 0.f}, {0.f, 0.f}, {0.f, 0.f}};  // dx, df, dg
            if (t < len) {
                Grad<T, G> e;
                e.make(load2(x + t * p.ld, L), load2(f + t * p.ld, L),
                       G ? load2(g + t * p.ld, L) : 0u, load2(dy + t * p.ldy, L), bias);
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const float before = hs[t][k][lane], d = e.own[k] + r[k];
                    out[0][k] = d * e.b[k];
                    out[1][k] = d * (before - e.x[k]) * (e.a[k] * e.b[k]);
                    if (G) out[2][k] = e.dg[k] * (e.a[k] * before + e.b[k] * e.x[k]);
                    r[k] = e.a[k] * d;
                    total[k] += out[1][k];
                }
            }
            void *const row[3] = {dx + t * p.ld, df + t * p.ld, dg + t * p.ld};
            store2<T, G ? 3 : 2>(row, L, false, out);
        }
        if (p.dh0) put2(p.dh0 + n * p.c, L, r[0], r[1]);
        if (p.part) put2(p.part + n * p.c, L, total[0], total[1]);
    }
}

// The pair of a chunk for r, walked from its last token on with the arithmetic of the kernel below.
template <class T, bool G, int W, int S>
__device__ void walk_bwd(const RecParams &p, int64_t n, const Lane &L, int lo, int len,
                         const float bias[2], float A[2], float R[2]) {
    const int64_t at = n * p.t * p.ld;
    const uint16_t *f = (const uint16_t *)p.f + at;
    const uint16_t *g = G ? (const uint16_t *)p.g + at : nullptr;
    const uint16_t *dy = (const uint16_t *)p.dy + n * p.t * p.ldy;
    A[0] = A[1] = 1.f;
    R[0] = R[1] = 0.f;
    for (int w = W - 1; w >= 0; --w) {
        float a1[2] = {1.f, 1.f}, r1[2] = {0.f, 0.f};
        const int first = lo + w * S;
        for (int t = first; t < min(first + S, len); ++t)
            for (int k = 0; k < 2; ++k) {  // the product in the order of the tokens
                float fv[2], a, b;
                unpack<T>(load2(f + t * p.ld, L), fv);
                gate(fv[k], bias[k], a, b);
                a1[k] *= a;
            }
        for (int t = min(first + S, len) - 1; t >= first; --t) {
            Grad<T, G> e;
            e.make(0u, load2(f + t * p.ld, L), G ? load2(g + t * p.ld, L) : 0u,
                   load2(dy + t * p.ldy, L), bias);
            for (int k = 0; k < 2; ++k) r1[k] = before_token(e.a[k], e.own[k], r1[k]);
        }
        a1[0] = fmaxf(a1[0], A_MIN);
        a1[1] = fmaxf(a1[1], A_MIN);
        compose(A, R, a1, r1);
    }
}

template <class T, bool G, int W, int S, int NG>
__global__ __launch_bounds__(64 * W, 2) void recurrence_bwd_kernel(const RecParams p, const RecGrid q) {
    static_assert((W * S) % SAVE == 0 && SAVE % S == 0, "a chunk is whole saved stretches");
    constexpr int RUN = SAVE / S;  // teams that start from one saved state
    constexpr bool U = NG == 1;
    constexpr int TEAMS = W * NG, CHUNK = TEAMS * S;
    const Team<NG> team;
    const int w = team.w;
    const int col = blockIdx.x % q.cols, rest = blockIdx.x / q.cols;
    const int n = rest % p.n, place = rest / p.n, chunk = q.chunks - 1 - place;  // the last one first
    const Lane L(2 * (col * team.LANES + team.c), p.c);
    const int len = length_of(p, n);
    const int t0 = chunk * CHUNK + team.r * S, last = len > 0 ? len - 1 : 0;
    const int64_t at = (int64_t)n * p.t * p.ld;
    const uint16_t *x = (const uint16_t *)p.x + at, *f = (const uint16_t *)p.f + at;
    const uint16_t *g = G ? (const uint16_t *)p.g + at : nullptr;
    const uint16_t *dy = (const uint16_t *)p.dy + (int64_t)n * p.t * p.ldy;
    uint32_t xr[S], fr[S], gr[S], dr[S];
    const bool whole = t0 + S <= len;           // every token takes part
    const bool full = (col + 1) * 2 * team.LANES <= p.c;  // every channel exists
    int64_t o = (int64_t)min(t0, last) * p.ld;
    dy += (int64_t)min(t0, last) * p.ldy;
#pragma unroll
    for (int s = 0; s < S; ++s) {
        xr[s] = load2<U>(x + o, L);
        fr[s] = load2<U>(f + o, L);
        gr[s] = G ? load2<U>(g + o, L) : 0u;
        dr[s] = load2<U>(dy, L);
        o += t0 + s < last ? p.ld : 0;
        dy += t0 + s < last ? p.ldy : 0;
    }
    float h[2] = {0.f, 0.f}, bias[2] = {0.f, 0.f};
    const int run0 = t0 - team.r % RUN * S;  // first token of the saved stretch
    if (run0 < p.t) {
        const float *from = p.saved + ((int64_t)n * ((p.t + SAVE - 1) / SAVE) + run0 / SAVE) * p.c;
        h[0] = from[L.k0];
        h[1] = from[L.k1];
    }
    if (p.bias) {
        bias[0] = p.bias[L.k0] * -LOG2E;
        bias[1] = p.bias[L.k1] * -LOG2E;
    }
    Grad<T, G> e[S];
    float A[2] = {1.f, 1.f}, H[2] = {0.f, 0.f}, R[2] = {0.f, 0.f};
#pragma unroll
    for (int s = 0; s < S; ++s) {
        e[s].make(xr[s], fr[s], gr[s], dr[s], bias);
        if (!whole && t0 + s >= len) e[s].pass();
    }
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            H[k] = e[s].a[k] * H[k] + e[s].b[k] * e[s].x[k];
            A[k] *= e[s].a[k];
        }
#pragma unroll
    for (int s = S - 1; s >= 0; --s)
#pragma unroll
        for (int k = 0; k < 2; ++k) R[k] = before_token(e[s].a[k], e[s].own[k], R[k]);
    A[0] = fmaxf(A[0], A_MIN);
    A[1] = fmaxf(A[1], A_MIN);
    float r[2] = {0.f, 0.f};
    if (!q.words && p.dht) {  // before the barrier: dh0, which another wave writes, may lie on it
        r[0] = p.dht[(int64_t)n * p.c + L.k0];
        r[1] = p.dht[(int64_t)n * p.c + L.k1];
    }
    __shared__ f32x4 part[W * 64];
    __shared__ float part_r[2][W * 64];
    part[threadIdx.x] = f32x4{A[0], H[0], A[1], H[1]};
    part_r[0][threadIdx.x] = R[0];
    part_r[1][threadIdx.x] = R[1];
    __syncthreads();
    for (int k = 0; k < RUN - 1; ++k) {
        const int v = team.r - team.r % RUN + k;
        if (v >= team.r) continue;
        const f32x4 m = part[team.of(v)];
        h[0] = m[0] * h[0] + m[1];
        h[1] = m[2] * h[1] + m[3];
    }
    // what the teams behind make of the gradient that flows into the chunk
    float pa[2] = {1.f, 1.f}, pr[2] = {0.f, 0.f};
    for (int v = TEAMS - 1; v > w * NG; --v) {
        if (v <= team.r) continue;
        const f32x4 m = part[team.of(v)];
        const float ma[2] = {m[0], m[2]}, mr[2] = {part_r[0][team.of(v)], part_r[1][team.of(v)]};
        compose(pa, pr, ma, mr);
    }
    if (q.words) {
        float ca[2] = {pa[0], pa[1]}, cr[2] = {pr[0], pr[1]};
        compose(ca, cr, A, R);
        if (NG > 1)  // the first team's is the chunk's
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                ca[k] = __shfl(ca[k], team.c);
                cr[k] = __shfl(cr[k], team.c);
            }
        carry_in<W>(q, n, p.c, place, L, team.first_of_wave(), w, 0, ca, cr, [&](int at2, float *a2, float *r2) {
            walk_bwd<T, G, TEAMS, S>(p, n, L, (q.chunks - 1 - at2) * CHUNK, len, bias, a2, r2);
        }, r);
    }
    r[0] = pa[0] * r[0] + pr[0];
    r[1] = pa[1] * r[1] + pr[1];
    float before[S][2];
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            before[s][k] = h[k];
            h[k] = e[s].a[k] * h[k] + e[s].b[k] * e[s].x[k];
        }
    uint16_t *dx = (uint16_t *)p.dx + at, *df = (uint16_t *)p.df + at;
    uint16_t *dg = G ? (uint16_t *)p.dg + at : nullptr;
    float total[2] = {0.f, 0.f};
    o = (int64_t)(t0 + S - 1) * p.ld;
    auto finish = [&](auto checked) {
#pragma unroll
        for (int s = S - 1; s >= 0; --s, o -= p.ld) {
            const int t = t0 + s;
            float out[3][2];  // dx, df, dg
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const Grad<T, G> &m = e[s];
                const float d = m.own[k] + r[k];
                out[0][k] = d * m.b[k];
                out[1][k] = d * (before[s][k] - m.x[k]) * (m.a[k] * m.b[k]);
                out[2][k] = m.dg[k] * (m.a[k] * before[s][k] + m.b[k] * m.x[k]);
                if (checked && t >= len) out[0][k] = out[1][k] = out[2][k] = 0.f;
                r[k] = m.a[k] * d;
                total[k] += out[1][k];
            }
            void *const row[3] = {dx + o, df + o, dg + o};
            if (!checked || t < p.t) store2<T, G ? 3 : 2, U>(row, L, !checked, out);
        }
    };
    if (team.all(whole) && full)
        finish(std::false_type{});
    else
        finish(std::true_type{});
    if (p.dh0 && chunk == 0 && team.r == 0) put2(p.dh0 + (int64_t)n * p.c, L, r[0], r[1]);
    if (p.part) {
        __syncthreads();
        part_r[0][threadIdx.x] = total[0];
        part_r[1][threadIdx.x] = total[1];
        __syncthreads();
        if (w != 0 || !team.first_of_wave()) return;
        for (int v = 1; v < TEAMS; ++v) {
            total[0] += part_r[0][team.of(v)];
            total[1] += part_r[1][team.of(v)];
        }
        float *to = p.part + ((int64_t)n * q.chunks + chunk) * p.c;
        put2(to, L, total[0], total[1]);
    }
}

// ---- one channel: no pairs to load, a lane per sequence walks its tokens ---------

template <class T>
__global__ __launch_bounds__(64) void recurrence_fwd_single_kernel(const RecParams p) {
    const int64_t n = (int64_t)blockIdx.x * 64 + threadIdx.x;
    if (n >= p.n) return;
    const int len = length_of(p, (int)n);
    const float bias = p.bias ? p.bias[0] * -LOG2E : 0.f;
    float h = p.h0 ? p.h0[n] : 0.f;
    const uint16_t *x = (const uint16_t *)p.x + n * p.t * p.ld, *f = (const uint16_t *)p.f + n * p.t * p.ld;
    const uint16_t *g = p.g ? (const uint16_t *)p.g + n * p.t * p.ld : nullptr;
    uint16_t *y = (uint16_t *)p.y + n * p.t * p.ldy;
    for (int64_t t = 0; t < p.t; ++t) {
        if (p.saved && t % SAVE == 0) p.saved[n * ((p.t + SAVE - 1) / SAVE) + t / SAVE] = h;
        float o = 0.f;
        if (t < len) {
            float a, b;
            gate(from16<T>(f[t * p.ld]), bias, a, b);
            h = a * h + b * from16<T>(x[t * p.ld]);
            o = h;
            if (g) {
                const float gv = from16<T>(g[t * p.ld]);
                o = h * (gv * sigma(gv));
            }
        }
        y[t * p.ldy] = (uint16_t)to16<T>(o);
    }
    if (p.ht) p.ht[n] = h;
}

template <class T>
__global__ __launch_bounds__(64) void recurrence_bwd_single_kernel(const RecParams p) {
    __shared__ float hs[SAVE][64];
    const int lane = threadIdx.x;
    const int64_t n = (int64_t)blockIdx.x * 64 + lane;
    if (n >= p.n) return;
    const int len = length_of(p, (int)n);
    const float bias = p.bias ? p.bias[0] * -LOG2E : 0.f;
    const int64_t at = n * p.t * p.ld, stretches = (p.t + SAVE - 1) / SAVE;
    const uint16_t *x = (const uint16_t *)p.x + at, *f = (const uint16_t *)p.f + at;
    const uint16_t *g = p.g ? (const uint16_t *)p.g + at : nullptr;
    const uint16_t *dy = (const uint16_t *)p.dy + n * p.t * p.ldy;
    uint16_t *dx = (uint16_t *)p.dx + at, *df = (uint16_t *)p.df + at;
    uint16_t *dg = p.g ? (uint16_t *)p.dg + at : nullptr;
    float r = p.dht ? p.dht[n] : 0.f, total = 0.f;
    for (int64_t k = stretches - 1; k >= 0; --k) {
        const int64_t lo = k * SAVE, hi = lo + SAVE < p.t ? lo + SAVE : p.t;
        float h = p.saved[n * stretches + k], part = 0.f;
        for (int64_t t = lo; t < hi && t < len; ++t) {
            float a, b;
            hs[t - lo][lane] = h;
            gate(from16<T>(f[t * p.ld]), bias, a, b);
            h = a * h + b * from16<T>(x[t * p.ld]);
        }
        for (int64_t t = hi - 1; t >= lo; --t) {
            float vx = 0.f, vf = 0.f, vg = 0.f;
            if (t < len) {
                float a, b;
                gate(from16<T>(f[t * p.ld]), bias, a, b);
                const float xv = from16<T>(x[t * p.ld]), before = hs[t - lo][lane];
                float own = from16<T>(dy[t * p.ldy]);
                if (g) {
                    const float gv = from16<T>(g[t * p.ld]), s = sigma(gv), sg = gv * s;
                    vg = own * (s + sg * (1.f - s)) * (a * before + b * xv);
                    own *= sg;
                }
                const float d = own + r;
                vx = d * b;
                vf = d * (before - xv) * (a * b);
                r = a * d;
                part += vf;
            }
            dx[t * p.ld] = (uint16_t)to16<T>(vx);
            df[t * p.ld] = (uint16_t)to16<T>(vf);
            if (dg) dg[t * p.ld] = (uint16_t)to16<T>(vg);
        }
        total += part;
    }
    if (p.dh0) p.dh0[n] = r;
    if (p.part) p.part[n] = total;
}

constexpr int FW = 8, FS = 16, BW = 4, BS = 16;  // waves, and tokens of each

// Teams of a wave: as many as leave each the lanes for all channels.
int teams_of(const RecParams &p) { return p.c <= 16 ? 8 : p.c <= 32 ? 4 : p.c <= 64 ? 2 : 1; }

int64_t chunks_of(const RecParams &p, bool backward) {
    const int k = (backward ? BW * BS : FW * FS) * teams_of(p);
    return p.t <= SHORT_T || p.c == 1 ? 1 : ((int64_t)p.t + k - 1) / k;
}

// Places in groups of 2^gs: about as many groups, whose states are handed on
// one after the other, as places in one, whose pairs each place reads.  (Groups of
// 16 throughout: backward of 8 x 2048 x 1152 4 us slower.  Groups of at most 16: forward of 1 x
// 65536 x 256 47 us, 42 with 32.)
RecGrid grid_of(const RecParams &p, bool backward) {
    RecGrid q{};
    const int64_t chunks = chunks_of(p, backward);
    q.cols = (p.c + COLS - 1) / COLS;  // one where a wave is several teams
    q.chunks = (int32_t)chunks;
    while (1 << q.gs < GROUP && chunks >> 2 * q.gs > 1) ++q.gs;
    q.groups = (int32_t)((chunks + (1 << q.gs) - 1) >> q.gs);
    return q;
}

int64_t word_count(const RecParams &p, bool backward) {
    const RecGrid q = grid_of(p, backward);
    return q.chunks > 1 ? (int64_t)p.n * ((int64_t)q.chunks + q.groups) * p.c : 0;
}

// Workgroups of one launch at most: work items of a launch are counted in 32 bits.
constexpr int64_t MOST_BLOCKS = 1 << 22;

// The sequences from n0 on, n of them.
RecParams some(const RecParams &p, bool backward, int64_t n0, int64_t n) {
    RecParams s = p;
    const int64_t in = n0 * p.t * p.ld * 2, out = n0 * p.t * p.ldy * 2, state = n0 * p.c;
    const int64_t stretches = (p.t + SAVE - 1) / SAVE;
    auto move = [](auto &q, int64_t bytes) {
        if (q) q = (std::remove_reference_t<decltype(q)>)((uintptr_t)q + bytes);
    };
    s.n = (int32_t)n;
    for (const void **q : {&s.x, &s.f, &s.g}) move(*q, in);
    for (void **q : {&s.dx, &s.df, &s.dg}) move(*q, in);
    move(s.y, out);
    move(s.dy, out);
    move(s.lengths, n0 * 4);
    for (const float **q : {&s.h0, &s.dht}) move(*q, state * 4);
    for (float **q : {&s.ht, &s.dh0}) move(*q, state * 4);
    move(s.saved, state * stretches * 4);
    move(s.part, state * chunks_of(p, backward) * 4);
    return s;
}

template <class T, bool G, int NG>
void launch_split(const RecParams &s, const RecGrid &q, bool backward, uint32_t blocks, hipStream_t st) {
    if (backward)
        hipLaunchKernelGGL((recurrence_bwd_kernel<T, G, BW, BS, NG>), dim3(blocks), dim3(64 * BW), 0, st, s, q);
    else
        hipLaunchKernelGGL((recurrence_fwd_kernel<T, G, FW, FS, NG>), dim3(blocks), dim3(64 * FW), 0, st, s, q);
}

template <class T, bool G>
hipError_t run(const RecParams &p, bool backward, hipStream_t st) {
    RecGrid q = grid_of(p, backward);
    if (p.c == 1) {
        const dim3 grid((p.n + 63) / 64);
        if (backward)
            hipLaunchKernelGGL((recurrence_bwd_single_kernel<T>), grid, dim3(64), 0, st, p);
        else
            hipLaunchKernelGGL((recurrence_fwd_single_kernel<T>), grid, dim3(64), 0, st, p);
        return hipGetLastError();
    }
    if (p.t <= SHORT_T) {
        const dim3 grid(q.cols, p.n < 65535 ? p.n : 65535);
        if (backward)
            hipLaunchKernelGGL((recurrence_bwd_short_kernel<T, G>), grid, dim3(64), 0, st, p);
        else
            hipLaunchKernelGGL((recurrence_fwd_short_kernel<T>), grid, dim3(64), 0, st, p);
        return hipGetLastError();
    }
    const int64_t each = (int64_t)q.chunks * q.cols, most = each < MOST_BLOCKS ? MOST_BLOCKS / each : 1;
    for (int64_t n0 = 0; n0 < p.n; n0 += most) {
        const RecParams s = some(p, backward, n0, p.n - n0 < most ? p.n - n0 : most);
        if (q.chunks > 1) {  // launches follow each other: they share the words
            q.words = (uint64_t *)p.ws;
            q.states = q.words + (int64_t)s.n * q.chunks * p.c;
            const int64_t nb = (word_count(s, backward) + 255) / 256;
            hipLaunchKernelGGL(recurrence_words_kernel, dim3((uint32_t)(nb < 2048 ? nb : 2048)), dim3(256), 0, st, q,
                               (int64_t)s.n, p.c, backward ? s.dht : s.h0);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
        const uint32_t blocks = (uint32_t)(each * s.n);
        switch (teams_of(p)) {
            case 1: launch_split<T, G, 1>(s, q, backward, blocks, st); break;
            case 2: launch_split<T, G, 2>(s, q, backward, blocks, st); break;
            case 4: launch_split<T, G, 4>(s, q, backward, blocks, st); break;
            default: launch_split<T, G, 8>(s, q, backward, blocks, st); break;
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

// One sequence's workgroups have to fit a launch.
bool recurrence_fits(const RecParams &p) {
    const RecGrid f = grid_of(p, false), b = grid_of(p, true);
    return (int64_t)f.chunks * f.cols <= MOST_BLOCKS && (int64_t)b.chunks * b.cols <= 2 * MOST_BLOCKS;
}

int64_t recurrence_bwd_parts(const RecParams &p) { return p.n * chunks_of(p, true); }

// Words first (8-byte aligned), then, backward, the partial sums of dbias.
size_t recurrence_words_bytes(const RecParams &p, bool backward) {
    return sizeof(uint64_t) * (size_t)word_count(p, backward);
}

size_t recurrence_ws(const RecParams &p, bool backward) {
    const size_t words = recurrence_words_bytes(p, backward);
    if (!backward) return words;
    const int64_t parts = recurrence_bwd_parts(p);
    return words + sizeof(float) * (size_t)((parts + colsum_extra(parts)) * p.c);
}

static hipError_t launch(int dtype, const RecParams &p, bool backward, hipStream_t st) {
    if (p.n <= 0) return hipSuccess;
    if (dtype == Half::id)
        return p.g ? run<Half, true>(p, backward, st) : run<Half, false>(p, backward, st);
    return p.g ? run<BFloat, true>(p, backward, st) : run<BFloat, false>(p, backward, st);
}

hipError_t launch_recurrence_fwd(int dtype, const RecParams &p, hipStream_t st) {
    return launch(dtype, p, false, st);
}

hipError_t launch_recurrence_bwd(int dtype, const RecParams &p, hipStream_t st) {
    return launch(dtype, p, true, st);
}

}  // namespace nnconv
