// embedding.hip -- rows of a table by token number, and the table's gradient.
//
// Forward: a copy with a factor, bound by the bytes.  Backward: the tokens are sorted by number
// (stable, so that the tokens of a row are added in their order and results are the same bits
// every time), spans of sorted tokens are summed by a team of threads each, and rows whose tokens
// reach over several spans are joined from their parts.  The launches that sort wait for their own
// loads and barriers mostly; further workgroups of theirs clear the table meanwhile, the rows that
// tokens name too (32768 tokens of 1152 channels, 32768 rows in fp32: 74 us a
// backward pass, 84 with rows looked up and cleared beside the sums).
#include "launch.hpp"

namespace nnconv {

namespace embedding {

typedef u32x4 __attribute__((aligned(4))) u32x4_any4;
typedef f32x4 __attribute__((aligned(4))) f32x4_any;

template <class T>
__device__ __forceinline__ uint32_t scaled(uint32_t two, float f) {
    return pack16<T>(from16<T>(two) * f, from16<T>(two >> 16) * f);
}

// A thread 8 channels of a row, at any alignment.
template <class T, bool SHORT>
__global__ __launch_bounds__(256) void fwd_kernel(const EmbeddingParams P) {
    const uint32_t per = ((uint32_t)P.c + 7) / 8;
    const int64_t count = P.rows * per;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < count; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / per;
        const int c = (int)(i - r * per) * 8, n = P.c - c;
        const int32_t id = P.ids[r];
        const bool in = (uint32_t)id < (uint32_t)P.v;
        u32x4 v = {};
        if (in) v = row_vector<SHORT>((const uint16_t *)P.table + (int64_t)id * P.c, c, P.c);
#pragma unroll
        for (int d = 0; d < 4; ++d) v[d] = in ? scaled<T>(v[d], P.scale) : 0u;
        uint16_t *y = (uint16_t *)P.y + r * P.c + c;
        if (n >= 8)
            *(u32x4_any *)y = v;
        else
#pragma unroll
            for (int d = 0; d < 7; ++d)
                if (d < n) y[d] = (uint16_t)(v[d >> 1] >> (16 * (d & 1)));
    }
}

// Bytes to clear by the workgroups behind the first `blocks` of a launch, CLEAR_BYTES each.
struct Clear {
    char *p;
    int64_t bytes;  // even
    uint32_t blocks;
};
constexpr int CLEAR_BYTES = 65536;

// Whether this workgroup is one of them.
__device__ __forceinline__ bool cleared(const Clear &c) {
    if (blockIdx.x < c.blocks) return false;
    const int64_t at = (int64_t)(blockIdx.x - c.blocks) * CLEAR_BYTES;
    const int64_t left = c.bytes - at;
    const int n = left < CLEAR_BYTES ? (int)left : CLEAR_BYTES;
    for (int i = threadIdx.x * 16; i + 16 <= n; i += blockDim.x * 16)
        __builtin_nontemporal_store(u32x4{}, (u32x4_any *)(c.p + at + i));
    for (int i = n / 16 * 16 + threadIdx.x * 2; i < n; i += blockDim.x * 2) *(uint16_t *)(c.p + at + i) = 0;
    return true;
}

__global__ __launch_bounds__(256) void clear_kernel(const Clear c) { cleared(c); }

// --- sorting ---------------------------------------------------------------------------
//
// Passes over 8 bits of the number, least first.  A wave takes its tokens in their order; lanes
// with equal digits find each other by ballots, so that a token's place among its equals is its
// order.

constexpr int BITS = 8, BINS = 1 << BITS;

// Number of the token that sorts; padding last.
__device__ __forceinline__ uint32_t key_of(int32_t id, int32_t v) { return (uint32_t)id < (uint32_t)v ? (uint32_t)id : (uint32_t)v; }

// Lanes of the wave that are live and have this lane's digit.
__device__ __forceinline__ uint64_t equals(uint32_t digit, bool live) {
    uint64_t m = __ballot(live);
#pragma unroll
    for (int b = 0; b < BITS; ++b) {
        const bool set = (digit >> b) & 1;
        const uint64_t with = __ballot(set);
        m &= set ? with : ~with;
    }
    return m;
}

// Each token's place among the workgroup's of its digit; `seen` is, behind a barrier, for each wave
// and digit the tokens of the waves before, and `sum` the digit's in all (of thread = digit).
template <int WAVES, int R>
__device__ __forceinline__ uint32_t rank(const uint32_t (&key)[R], const bool (&live)[R], int shift, uint32_t (&place)[R],
                                         uint32_t (*seen)[BINS]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int i = threadIdx.x; i < WAVES * BINS; i += 64 * WAVES) seen[i / BINS][i % BINS] = 0;
    __syncthreads();
#pragma unroll
    for (int s = 0; s < R; ++s) {
        const uint32_t digit = (key[s] >> shift) & (BINS - 1);
        const uint64_t m = equals(digit, live[s]);
        const uint32_t before = __popcll(m & (((uint64_t)1 << lane) - 1));
        // every lane reads the count before the first of its equals adds to it
        place[s] = seen[wave][digit] + before;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (live[s] && before == 0) seen[wave][digit] += (uint32_t)__popcll(m);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    __syncthreads();
    uint32_t sum = 0;
    if (threadIdx.x < BINS) {
        for (int w = 0; w < WAVES; ++w) {
            const uint32_t n = seen[w][threadIdx.x];
            seen[w][threadIdx.x] = sum;
            sum += n;
        }
    }
    return sum;
}

// Sum over the threads before (256 of them), of all of them in `all`.
__device__ __forceinline__ uint32_t scan256(uint32_t n, uint32_t *waves) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t scan = n;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t o = __shfl_up(scan, d);
        if (lane >= d) scan += o;
    }
    if (lane == 63 && wave < 4) waves[wave] = scan;
    __syncthreads();
    uint32_t before = scan - n;
#pragma unroll
    for (int w = 0; w < 3; ++w)
        if (w < wave) before += waves[w];
    return before;
}

// Up to ONE tokens: all passes by one workgroup, through LDS (5003 tokens: 15 us).
constexpr int ONE_ROUNDS = 8, ONE = 1024 * ONE_ROUNDS;

template <int R>
__global__ __launch_bounds__(1024) void sort_one_kernel(const int32_t *ids, int32_t rows, int32_t v, int bits, uint32_t *key_out,
                                                        uint32_t *row_out, const Clear clear) {
    __shared__ uint32_t seen[16][BINS], waves[4];
    __shared__ uint32_t keys[1024 * R];
    __shared__ uint16_t from[1024 * R];
    if (cleared(clear)) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t key[R], row[R], place[R];
    bool live[R];
#pragma unroll
    for (int s = 0; s < R; ++s) {
        const int i = wave * 64 * R + s * 64 + lane;
        live[s] = i < rows;
        key[s] = live[s] ? key_of(ids[i], v) : 0;
        row[s] = (uint32_t)i;
    }
    for (int shift = 0; shift < bits; shift += BITS) {
        const uint32_t sum = rank<16, R>(key, live, shift, place, seen);
        const uint32_t base = scan256(sum, waves);
        if (threadIdx.x < BINS)
            for (int w = 0; w < 16; ++w) seen[w][threadIdx.x] += base;
        __syncthreads();
#pragma unroll
        for (int s = 0; s < R; ++s)
            if (live[s]) {
                const uint32_t to = seen[wave][(key[s] >> shift) & (BINS - 1)] + place[s];
                keys[to] = key[s];
                from[to] = (uint16_t)row[s];
            }
        __syncthreads();
#pragma unroll
        for (int s = 0; s < R; ++s) {
            const int i = wave * 64 * R + s * 64 + lane;
            if (live[s]) {
                key[s] = keys[i];
                row[s] = from[i];
            }
        }
    }
#pragma unroll
    for (int s = 0; s < R; ++s) {
        const int i = wave * 64 * R + s * 64 + lane;
        if (!live[s]) continue;
        key_out[i] = key[s];
        row_out[i] = row[s];
    }
}

// More: a pass counts the digits of each workgroup's tokens and moves them in a second launch, whose
// workgroups add up the counts in front of theirs themselves (32768 tokens, 2 passes: 21 us).
// From MANY workgroups on they would read too much, and a launch between adds the counts up.
constexpr int ROUNDS = 4, MANY = 128;

struct Sort {
    int64_t rows;
    int32_t v, shift, blocks;
    bool summed;                 // counts are places already
    const int32_t *ids;          // first pass
    const uint32_t *key, *row;   // later passes
    uint32_t *key_out, *row_out;
    uint32_t *counts;            // [blocks][BINS]
    Clear clear;
};

template <bool FIRST>
__device__ __forceinline__ uint32_t key_at(const Sort &P, int64_t i) {
    return FIRST ? key_of(P.ids[i], P.v) : P.key[i];
}

template <int WAVES, bool FIRST>
__global__ __launch_bounds__(64 * WAVES) void count_kernel(const Sort P) {
    __shared__ uint32_t seen[WAVES][BINS];
    if (cleared(P.clear)) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t first = (int64_t)blockIdx.x * (64 * WAVES * ROUNDS) + wave * 64 * ROUNDS;
    uint32_t key[ROUNDS], place[ROUNDS];
    bool live[ROUNDS];
#pragma unroll
    for (int s = 0; s < ROUNDS; ++s) {
        const int64_t i = first + s * 64 + lane;
        live[s] = i < P.rows;
        key[s] = live[s] ? key_at<FIRST>(P, i) : 0;
    }
    const uint32_t sum = rank<WAVES, ROUNDS>(key, live, P.shift, place, seen);
    if (threadIdx.x < BINS) P.counts[(int64_t)blockIdx.x * BINS + threadIdx.x] = sum;
}

// counts -> places, by one workgroup of a thread a digit.
__global__ __launch_bounds__(256) void place_kernel(uint32_t *counts, int32_t blocks) {
    __shared__ uint32_t waves[4];
    uint32_t sum = 0;
#pragma unroll 8
    for (int b = 0; b < blocks; ++b) sum += counts[(int64_t)b * BINS + threadIdx.x];
    uint32_t at = scan256(sum, waves);
#pragma unroll 8
    for (int b = 0; b < blocks; ++b) {
        const uint32_t n = counts[(int64_t)b * BINS + threadIdx.x];
        counts[(int64_t)b * BINS + threadIdx.x] = at;
        at += n;
    }
}

template <int WAVES, bool FIRST>
__global__ __launch_bounds__(64 * WAVES) void sort_kernel(const Sort P) {
    __shared__ uint32_t seen[WAVES][BINS], waves[4];
    if (cleared(P.clear)) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t first = (int64_t)blockIdx.x * (64 * WAVES * ROUNDS) + wave * 64 * ROUNDS;
    uint32_t key[ROUNDS], row[ROUNDS], place[ROUNDS];
    bool live[ROUNDS];
#pragma unroll
    for (int s = 0; s < ROUNDS; ++s) {
        const int64_t i = first + s * 64 + lane;
        live[s] = i < P.rows;
        key[s] = live[s] ? key_at<FIRST>(P, i) : 0;
        row[s] = live[s] ? (FIRST ? (uint32_t)i : P.row[i]) : 0;
    }
    uint32_t before = 0, total = 0;
    if (threadIdx.x < BINS) {
        if (P.summed)
            before = P.counts[(int64_t)blockIdx.x * BINS + threadIdx.x];
        else {
#pragma unroll 8
            for (int b = 0; b < P.blocks; ++b) {
                const uint32_t n = P.counts[(int64_t)b * BINS + threadIdx.x];
                total += n;
                before += b < (int)blockIdx.x ? n : 0;
            }
        }
    }
    rank<WAVES, ROUNDS>(key, live, P.shift, place, seen);
    before += scan256(total, waves);
    if (threadIdx.x < BINS)
        for (int w = 0; w < WAVES; ++w) seen[w][threadIdx.x] += before;
    __syncthreads();
#pragma unroll
    for (int s = 0; s < ROUNDS; ++s) {
        if (!live[s]) continue;
        const uint32_t to = seen[wave][(key[s] >> P.shift) & (BINS - 1)] + place[s];
        P.key_out[to] = key[s];
        P.row_out[to] = row[s];
    }
}

// --- sums ------------------------------------------------------------------------------

// Sorted tokens of a team, a multiple of 8: 32, and 8 where there are few and their teams would leave
// most of the chip idle (5003 tokens of 771 channels added to what is there: 33 us a backward pass
// with 8, 40 with 16, 56 with 32; 32768 of 1152: 11 us more with 8 than with 32).
constexpr int SPAN = 32, SMALL_SPAN = 8;
constexpr int64_t FEW_TOKENS = 16384;
constexpr int LEAST_TEAM = 4;   // threads of one, of 8 channels each

struct Sums {
    int64_t rows;
    int32_t c, cp, v, kind;  // cp: c in whole vectors; kind: Half::id, BFloat::id or 2: fp32
    int32_t team, span;      // threads, a power of two; tokens
    const uint32_t *key, *row;
    const uint16_t *dy;
    void *dtable;
    float factor;
    int32_t accumulate;
    int32_t *flag;
    float *part;             // [2 * spans][cp]: of a span, what belongs to the row of the span before, and to the next's
};

// What is at 8 channels of a row of the gradient, fp32 in both or 16 bits in `lo`.
struct Old {
    u32x4 lo, hi;
};

template <bool WIDE, bool SHORT>
__device__ __forceinline__ Old read8(const Sums &P, int64_t j, int c) {
    Old o = {};
    if constexpr (!WIDE) {
        o.lo = row_vector<SHORT>((const uint16_t *)P.dtable + j * P.c, c, P.c);
        return o;
    }
    const uint32_t *row = (const uint32_t *)P.dtable + j * P.c;
    if constexpr (SHORT) {
#pragma unroll
        for (int d = 0; d < 7; ++d)
            if (c + d < P.c) (d < 4 ? o.lo : o.hi)[d & 3] = row[c + d];
        return o;
    }
    // a row's end as its last 8 elements, moved
    const int at = c + 8 <= P.c ? c : P.c - 8;
    o.lo = *(const u32x4_any4 *)(row + at);
    o.hi = *(const u32x4_any4 *)(row + at + 4);
    if (P.c % 8 == 0) return o;
    const int by = c - at;
    if (by & 4) {
        o.lo = o.hi;
        o.hi = u32x4{};
    }
#pragma unroll
    for (int u = 1; u <= 2; u *= 2)
        if (by & u) {
            const u32x4 l = o.lo, h = o.hi;
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                o.lo[d] = d + u < 4 ? l[(d + u) & 3] : h[(d + u) & 3];
                o.hi[d] = d + u < 4 ? h[(d + u) & 3] : 0u;
            }
        }
    return o;
}

// 8 values of row `j` from channel c on to the gradient, added to `old` (zeros without accumulate).
template <class T, bool WIDE>
__device__ __forceinline__ void put8(const Sums &P, int64_t j, int c, const float (&s)[8], const Old &old) {
    const int64_t i = j * P.c + c;
    const int n = P.c - c;
    bool bad = false;
    if constexpr (WIDE) {
        float *o = (float *)P.dtable + i;
        f32x4 lo = __builtin_bit_cast(f32x4, old.lo), hi = __builtin_bit_cast(f32x4, old.hi);
#pragma unroll
        for (int d = 0; d < 4; ++d) {
            lo[d] += s[d] * P.factor;
            hi[d] += s[d + 4] * P.factor;
            // zeros behind the row's end are finite
            bad |= !__builtin_isfinite(lo[d]) | !__builtin_isfinite(hi[d]);
        }
        if (n >= 8) {
            *(f32x4_any *)o = lo;
            *(f32x4_any *)(o + 4) = hi;
        } else
#pragma unroll
            for (int d = 0; d < 7; ++d)
                if (d < n) o[d] = d < 4 ? lo[d & 3] : hi[d & 3];
    } else {
        uint16_t *o = (uint16_t *)P.dtable + i;
        constexpr uint32_t TOP = T::id == Half::id ? 0x7C00u : 0x7F80u;
        u32x4 out;
#pragma unroll
        for (int d = 0; d < 4; ++d) {
            out[d] = pack16<T>(from16<T>(old.lo[d]) + s[2 * d] * P.factor, from16<T>(old.lo[d] >> 16) + s[2 * d + 1] * P.factor);
            bad |= ((out[d] & TOP) == TOP) | (((out[d] >> 16) & TOP) == TOP);
        }
        if (n >= 8)
            *(u32x4_any *)o = out;
        else
#pragma unroll
            for (int d = 0; d < 7; ++d)
                if (d < n) o[d] = (uint16_t)(out[d >> 1] >> (16 * (d & 1)));
    }
    if (bad && P.flag) *P.flag = 1;
}

// Workgroups of teams, a span each: runs of equal numbers.  A run that begins and ends in its span
// is a row's whole sum.  Loads of 8 tokens are on their way at once, and with them of what their rows
// are added to.  Types are compiled in: with them chosen at run time the code of 8 tokens passed the
// instruction cache, 5 us of the 38 that a pass over 5003 tokens of 771 channels took.
template <class T, bool WIDE, bool ACCUMULATE, bool SHORT>
__global__ __launch_bounds__(256) void sum_kernel(const Sums P) {
    __shared__ uint32_t key[256 / LEAST_TEAM * SPAN + 2], row[256 / LEAST_TEAM * SPAN];  // key[0]: the one before
    const int teams = 256 / P.team;
    const int64_t first = (int64_t)blockIdx.x * teams * P.span;
    const int all = P.rows - first < teams * P.span ? (int)(P.rows - first) : teams * P.span;
    for (int i = threadIdx.x; i < all; i += 256) {
        key[i + 1] = P.key[first + i];
        row[i] = P.row[first + i];
    }
    if (threadIdx.x == 0) {
        key[0] = first > 0 ? P.key[first - 1] : ~0u;
        key[all + 1] = first + all < P.rows ? P.key[first + all] : ~0u;
    }
    __syncthreads();
    const int team = threadIdx.x / P.team;
    const int c = ((int)blockIdx.y * 256 + (threadIdx.x & (P.team - 1))) * 8;
    const int begin = team * P.span, n = all - begin < P.span ? all - begin : P.span;
    if (n <= 0 || c >= P.c) return;
    const int64_t span = (int64_t)blockIdx.x * teams + team;
    const uint32_t *k = key + 1 + begin;
    float sum[8] = {};
    bool begun = k[-1] == k[0];  // the run reaches in from the span before
    for (int i0 = 0; i0 < n; i0 += 8) {
        u32x4 v[8];
        Old old[8] = {};
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            v[u] = u32x4{};
            if (i0 + u >= n || k[i0 + u] >= (uint32_t)P.v) continue;  // padding is not read
            if (ACCUMULATE && k[i0 + u + 1] != k[i0 + u]) old[u] = read8<WIDE, SHORT>(P, k[i0 + u], c);
            v[u] = row_vector<SHORT>(P.dy + (int64_t)row[begin + i0 + u] * P.c, c, P.c);
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const int i = i0 + u;
            if (i >= n || k[i] >= (uint32_t)P.v) break;  // padding is sorted last
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                sum[2 * d] += from16<T>(v[u][d]);
                sum[2 * d + 1] += from16<T>(v[u][d] >> 16);
            }
            const bool on = k[i + 1] == k[i];
            if (on && i + 1 < n) continue;
            if (begun || on) {
                float *to = P.part + (2 * span + (begun ? 0 : 1)) * P.cp + c;
                *(f32x4 *)to = f32x4{sum[0], sum[1], sum[2], sum[3]};
                *(f32x4 *)(to + 4) = f32x4{sum[4], sum[5], sum[6], sum[7]};
            } else
                put8<T, WIDE>(P, k[i], c, sum, old[u]);
#pragma unroll
            for (int d = 0; d < 8; ++d) sum[d] = 0.f;
            begun = false;
        }
    }
}

// A workgroup a span: the row whose run begins in it and goes on behind it.  Its teams take a share
// of the spans behind each (a token that pads a batch may be most of it), added up in order.  Bound by
// what one compute unit reads: 2^20 tokens of 1024 channels, nine in ten of one number, 3.0 ms a backward
// pass, 0.79 without a common one.
constexpr int JOIN_THREADS = 1024;

template <class T, bool WIDE, bool ACCUMULATE, bool SHORT>
__global__ __launch_bounds__(JOIN_THREADS) void join_kernel(const Sums P) {
    const int64_t s = blockIdx.x, last = s * P.span + P.span - 1;
    if (last + 1 >= P.rows) return;
    const uint32_t k = P.key[last];
    if (k >= (uint32_t)P.v || P.key[last + 1] != k) return;
    if (s > 0 && P.key[s * P.span] == k && P.key[s * P.span - 1] == k) return;  // begins before
    __shared__ f32x4 sums[2][JOIN_THREADS];
    int64_t more = 0;  // spans behind this one that it reaches into
    for (;; more += 64) {
        const int64_t i = (s + 1 + more + (threadIdx.x & 63)) * P.span;
        const uint64_t in = __ballot(i < P.rows && P.key[i < P.rows ? i : 0] == k);
        if (in != ~(uint64_t)0) {
            more += __builtin_ctzll(~in);
            break;
        }
    }
    const int team = threadIdx.x / P.team, teams = JOIN_THREADS / P.team, at = threadIdx.x & (P.team - 1);
    const int64_t share = (more + teams - 1) / teams, step = 2 * (int64_t)P.cp;
    const int busy = (int)((more + share - 1) / share);
    int64_t i = team * share;
    const int64_t end = i + share < more ? i + share : more;
    const int c = ((int)blockIdx.y * 256 + at) * 8;
    f32x4 lo = {}, hi = {};
    if (c < P.c) {
        const float *from = P.part + (2 * s + 1) * P.cp + c;
        if (team == 0) {
            lo = *(const f32x4 *)from;
            hi = *(const f32x4 *)(from + 4);
        }
        const float *next = P.part + 2 * (s + 1 + i) * P.cp + c;
        for (; i + 8 <= end; i += 8, next += 8 * step) {
            f32x4 a[8], b[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                a[u] = *(const f32x4 *)(next + u * step);
                b[u] = *(const f32x4 *)(next + u * step + 4);
            }
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                lo += a[u];
                hi += b[u];
            }
        }
        for (; i < end; ++i, next += step) {
            lo += *(const f32x4 *)next;
            hi += *(const f32x4 *)(next + 4);
        }
    }
    if (busy > 1) {
        sums[0][threadIdx.x] = lo;
        sums[1][threadIdx.x] = hi;
        __syncthreads();
    }
    if (team > 0 || c >= P.c) return;
    for (int t = 1; t < busy; ++t) {
        lo += sums[0][t * P.team + at];
        hi += sums[1][t * P.team + at];
    }
    const float sum[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    put8<T, WIDE>(P, k, c, sum, ACCUMULATE ? read8<WIDE, SHORT>(P, k, c) : Old{});
}

inline size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }

struct Layout {
    int waves;  // of a sorting workgroup; 0: one workgroup sorts
    int32_t blocks;
    int64_t spans;
    int32_t cp, span;
    size_t key[2], row[2], counts, part, bytes;
};

static Layout layout_of(int64_t rows, int32_t c) {
    Layout l;
    l.waves = rows <= ONE ? 0 : rows <= (int64_t)MANY * 64 * 4 * ROUNDS ? 4 : 16;
    const int64_t tile = 64 * l.waves * ROUNDS;
    l.blocks = l.waves ? (int32_t)((rows + tile - 1) / tile) : 0;
    l.cp = (c + 7) / 8 * 8;
    l.span = rows <= FEW_TOKENS ? SMALL_SPAN : SPAN;
    l.spans = (rows + l.span - 1) / l.span;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t was = at;
        at += align256(bytes);
        return was;
    };
    for (int i = 0; i < 2; ++i) {
        l.key[i] = take((size_t)rows * 4);
        l.row[i] = take((size_t)rows * 4);
    }
    l.counts = take((size_t)l.blocks * BINS * 4);
    l.part = take((size_t)l.spans * 2 * l.cp * 4);
    l.bytes = at;
    return l;
}

// Takes the next of `parts` parts of what is left to clear, behind `blocks` workgroups; the grid.
static dim3 with_clear(Clear &all, Clear &part, uint32_t blocks, int parts) {
    int64_t n = (all.bytes / parts + CLEAR_BYTES - 1) / CLEAR_BYTES * CLEAR_BYTES;
    if (n > all.bytes) n = all.bytes;
    part = {all.p, n, blocks};
    all.p += n;
    all.bytes -= n;
    return dim3(blocks + (uint32_t)((n + CLEAR_BYTES - 1) / CLEAR_BYTES));
}

template <int WAVES, bool FIRST>
static void sort_pass(Sort &q, Clear &all, int parts, hipStream_t st) {
    const dim3 block(64 * WAVES);
    const dim3 counting = with_clear(all, q.clear, (uint32_t)q.blocks, parts);
    hipLaunchKernelGGL((count_kernel<WAVES, FIRST>), counting, block, 0, st, q);
    if (q.summed) hipLaunchKernelGGL(place_kernel, dim3(1), dim3(256), 0, st, q.counts, q.blocks);
    const dim3 sorting = with_clear(all, q.clear, (uint32_t)q.blocks, parts - 1);
    hipLaunchKernelGGL((sort_kernel<WAVES, FIRST>), sorting, block, 0, st, q);
}

template <int WAVES>
static void sort_passes(Sort q, Clear &all, const Layout &l, char *ws, int bits, int &from, hipStream_t st) {
    q.counts = (uint32_t *)(ws + l.counts);
    q.summed = WAVES == 16;
    int parts = 2 * ((bits + BITS - 1) / BITS);
    for (q.shift = 0; q.shift < bits; q.shift += BITS, parts -= 2) {
        q.key = (const uint32_t *)(ws + l.key[from]);
        q.row = (const uint32_t *)(ws + l.row[from]);
        from ^= 1;
        q.key_out = (uint32_t *)(ws + l.key[from]);
        q.row_out = (uint32_t *)(ws + l.row[from]);
        if (q.shift == 0)
            sort_pass<WAVES, true>(q, all, parts, st);
        else
            sort_pass<WAVES, false>(q, all, parts, st);
    }
}

template <int R>
static void sort_one(const Sort &q, Clear &all, const Layout &l, char *ws, int bits, hipStream_t st) {
    Clear part;
    const dim3 grid = with_clear(all, part, 1, 1);
    hipLaunchKernelGGL((sort_one_kernel<R>), grid, dim3(1024), 0, st, q.ids, (int32_t)q.rows, q.v, bits,
                       (uint32_t *)(ws + l.key[0]), (uint32_t *)(ws + l.row[0]), part);
}

template <class T, bool WIDE, bool ACCUMULATE, bool SHORT>
static void launch_sums(const Sums &s, dim3 grid, uint32_t spans, hipStream_t st) {
    hipLaunchKernelGGL((sum_kernel<T, WIDE, ACCUMULATE, SHORT>), grid, dim3(256), 0, st, s);
    if (spans > 1)
        hipLaunchKernelGGL((join_kernel<T, WIDE, ACCUMULATE, SHORT>), dim3(spans, grid.y), dim3(JOIN_THREADS), 0, st, s);
}

template <class T, bool WIDE, bool ACCUMULATE>
static void launch_sums(const Sums &s, dim3 grid, uint32_t spans, hipStream_t st) {
    s.c < 8 ? launch_sums<T, WIDE, ACCUMULATE, true>(s, grid, spans, st) : launch_sums<T, WIDE, ACCUMULATE, false>(s, grid, spans, st);
}

template <class T>
static void launch_sums(const Sums &s, dim3 grid, uint32_t spans, hipStream_t st) {
    if (s.kind == 2)
        s.accumulate ? launch_sums<T, true, true>(s, grid, spans, st) : launch_sums<T, true, false>(s, grid, spans, st);
    else
        s.accumulate ? launch_sums<T, false, true>(s, grid, spans, st) : launch_sums<T, false, false>(s, grid, spans, st);
}

}  // namespace embedding

using namespace embedding;

size_t embedding_ws(int64_t rows, int32_t c) { return rows > 0 ? layout_of(rows, c).bytes : 0; }

hipError_t launch_embedding_fwd(int dtype, const EmbeddingParams &p, hipStream_t st) {
    const int64_t n = (p.rows * ((p.c + 7) / 8) + 255) / 256;
    const dim3 grid((uint32_t)(n < (1 << 20) ? n : (1 << 20)));
    if (dtype == Half::id && p.c < 8)
        hipLaunchKernelGGL((fwd_kernel<Half, true>), grid, dim3(256), 0, st, p);
    else if (dtype == Half::id)
        hipLaunchKernelGGL((fwd_kernel<Half, false>), grid, dim3(256), 0, st, p);
    else if (p.c < 8)
        hipLaunchKernelGGL((fwd_kernel<BFloat, true>), grid, dim3(256), 0, st, p);
    else
        hipLaunchKernelGGL((fwd_kernel<BFloat, false>), grid, dim3(256), 0, st, p);
    return hipGetLastError();
}

hipError_t launch_embedding_bwd(int dtype, const EmbeddingParams &p, hipStream_t st) {
    Sums s;
    s.rows = p.rows;
    s.c = p.c;
    s.v = p.v;
    s.kind = p.dtable_dtype;
    s.dy = (const uint16_t *)p.dy;
    s.dtable = p.dtable;
    s.factor = p.scale * p.inv_loss_scale;
    s.accumulate = p.accumulate;
    s.flag = p.flag;
    char *ws = (char *)p.ws;
    const Layout l = layout_of(p.rows, p.c);
    Clear all = {(char *)p.dtable, p.accumulate ? 0 : (int64_t)p.v * p.c * (p.dtable_dtype == NNCONV_F32 ? 4 : 2), 0};
    if (p.rows == 0) {
        Clear part;
        const dim3 grid = with_clear(all, part, 0, 1);
        if (grid.x == 0) return hipSuccess;
        hipLaunchKernelGGL(clear_kernel, grid, dim3(256), 0, st, part);
        return hipGetLastError();
    }
    int bits = 1;  // of the largest key, which is v
    while (bits < 32 && ((uint32_t)p.v >> bits) != 0) ++bits;
    Sort q = {};
    q.rows = p.rows;
    q.v = p.v;
    q.blocks = l.blocks;
    q.ids = p.ids;
    int from = 0;
    if (l.waves == 4)
        sort_passes<4>(q, all, l, ws, bits, from, st);
    else if (l.waves == 16)
        sort_passes<16>(q, all, l, ws, bits, from, st);
    else if (p.rows <= 1024)
        sort_one<1>(q, all, l, ws, bits, st);
    else if (p.rows <= 4096)
        sort_one<4>(q, all, l, ws, bits, st);
    else
        sort_one<ONE_ROUNDS>(q, all, l, ws, bits, st);
    s.key = (const uint32_t *)(ws + l.key[from]);
    s.row = (const uint32_t *)(ws + l.row[from]);
    s.part = (float *)(ws + l.part);
    s.cp = l.cp;
    s.span = l.span;
    const int32_t vectors = l.cp / 8;
    s.team = LEAST_TEAM;
    while (s.team < vectors && s.team < 256) s.team *= 2;
    const int64_t teams = 256 / s.team;
    const dim3 grid((uint32_t)((l.spans + teams - 1) / teams), (uint32_t)((vectors + 255) / 256));
    if (dtype == Half::id)
        launch_sums<Half>(s, grid, (uint32_t)l.spans, st);
    else
        launch_sums<BFloat>(s, grid, (uint32_t)l.spans, st);
    return hipGetLastError();
}

}  // namespace nnconv
