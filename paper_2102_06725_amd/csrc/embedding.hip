// embedding.hip -- rows of a table by token number, and the table's gradient.
//
// Forward: a copy with a factor, bound by the bytes.  Backward: the tokens are sorted by number
// (stable, so that the tokens of a row are added in their order and results are the same bits
// every time), stretches of SPAN sorted tokens are summed by a workgroup each, and rows whose
// tokens reach over several stretches are joined from their parts.
#include "launch.hpp"

namespace nnconv {

namespace embedding {

template <class T>
__device__ __forceinline__ uint32_t scaled(uint32_t two, float f) {
    return pack16<T>(from16<T>(two) * f, from16<T>(two >> 16) * f);
}

// VEC: rows of whole 16-byte vectors; a thread a vector.  Else a thread an element.
template <class T, bool VEC>
__global__ __launch_bounds__(256) void fwd_kernel(const EmbeddingParams P) {
    const uint32_t per = VEC ? (uint32_t)P.c / 8 : (uint32_t)P.c;
    const int64_t count = P.rows * per;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < count; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / per;
        const uint32_t at = (uint32_t)(i - r * per);
        const int32_t id = P.ids[r];
        const bool in = (uint32_t)id < (uint32_t)P.v;
        if constexpr (VEC) {
            u32x4 v = {};
            if (in) v = *(const u32x4 *)((const uint16_t *)P.table + (int64_t)id * P.c + at * 8);
#pragma unroll
            for (int d = 0; d < 4; ++d) v[d] = in ? scaled<T>(v[d], P.scale) : 0u;
            *(u32x4 *)((uint16_t *)P.y + r * P.c + at * 8) = v;
        } else {
            float v = 0.f;
            if (in) v = from16<T>(((const uint16_t *)P.table)[(int64_t)id * P.c + at]) * P.scale;
            ((uint16_t *)P.y)[i] = in ? (uint16_t)to16<T>(v) : (uint16_t)0;
        }
    }
}

// --- sorting ---------------------------------------------------------------------------
//
// Passes over 8 bits of the number, least first.  A workgroup has TILE tokens, a wave a quarter
// of them in their order; lanes with equal digits find each other by ballots, so that a token's
// place among its equals is its order.

constexpr int BITS = 8, BINS = 1 << BITS, WAVES = 16, TILE = 4096, PER_WAVE = TILE / WAVES;

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

struct Sort {
    int64_t rows;
    int32_t v, shift, blocks;
    const int32_t *ids;          // first pass
    const uint32_t *key, *row;   // later passes
    uint32_t *key_out, *row_out;
    uint32_t *counts;            // [BINS][blocks]
};

// COUNT: the digits of each workgroup's tokens; else their places (counts are running sums then).
template <bool FIRST, bool COUNT>
__global__ __launch_bounds__(64 * WAVES) void sort_kernel(const Sort P) {
    __shared__ uint32_t seen[WAVES][BINS];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int i = threadIdx.x; i < WAVES * BINS; i += 64 * WAVES) seen[i / BINS][i % BINS] = 0;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * TILE + wave * PER_WAVE;
    uint32_t key[PER_WAVE / 64], place[PER_WAVE / 64];
#pragma unroll
    for (int s = 0; s < PER_WAVE / 64; ++s) {
        const int64_t i = first + s * 64 + lane;
        const bool live = i < P.rows;
        key[s] = live ? (FIRST ? key_of(P.ids[i], P.v) : P.key[i]) : 0;
        const uint32_t digit = (key[s] >> P.shift) & (BINS - 1);
        const uint64_t m = equals(digit, live);
        const uint32_t before = __popcll(m & (((uint64_t)1 << lane) - 1));
        // every lane reads the count before the first of its equals adds to it (one wave, in order)
        place[s] = seen[wave][digit] + before;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (live && before == 0) seen[wave][digit] += (uint32_t)__popcll(m);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    __syncthreads();
    if (threadIdx.x < BINS) {
        uint32_t sum = 0;
        for (int w = 0; w < WAVES; ++w) {
            const uint32_t n = seen[w][threadIdx.x];
            seen[w][threadIdx.x] = sum;
            sum += n;
        }
        if constexpr (COUNT)
            P.counts[(int64_t)threadIdx.x * P.blocks + blockIdx.x] = sum;
        else {
            const uint32_t base = P.counts[(int64_t)threadIdx.x * P.blocks + blockIdx.x];
            for (int w = 0; w < WAVES; ++w) seen[w][threadIdx.x] += base;
        }
    }
    if constexpr (!COUNT) {
        __syncthreads();
#pragma unroll
        for (int s = 0; s < PER_WAVE / 64; ++s) {
            const int64_t i = first + s * 64 + lane;
            if (i >= P.rows) continue;
            const uint32_t to = seen[wave][(key[s] >> P.shift) & (BINS - 1)] + place[s];
            P.key_out[to] = key[s];
            P.row_out[to] = FIRST ? (uint32_t)i : P.row[i];
        }
    }
}

// counts -> running sums over (digit, workgroup), by one workgroup.
__global__ __launch_bounds__(1024) void sort_scan_kernel(uint32_t *counts, int64_t n) {
    __shared__ uint32_t wave_sums[16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t carry = 0;
    for (int64_t i0 = 0; i0 < n; i0 += 4096) {
        const int64_t i = i0 + threadIdx.x * 4;
        uint32_t c[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) c[u] = i + u < n ? counts[i + u] : 0;
        uint32_t sum = c[0] + c[1] + c[2] + c[3], scan = sum;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t o = __shfl_up(scan, d);
            if (lane >= d) scan += o;
        }
        if (lane == 63) wave_sums[wave] = scan;
        __syncthreads();
        uint32_t before = carry, all = 0;
#pragma unroll
        for (int w = 0; w < 16; ++w) {
            if (w < wave) before += wave_sums[w];
            all += wave_sums[w];
        }
        before += scan - sum;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (i + u < n) counts[i + u] = before;
            before += c[u];
        }
        carry += all;
        __syncthreads();
    }
}

// --- sums ------------------------------------------------------------------------------

constexpr int SPAN = 64;  // sorted tokens of a workgroup

struct Sums {
    int64_t rows;
    int32_t c, v, kind;     // kind: Half::id, BFloat::id or 2: fp32
    const uint32_t *key, *row;
    const uint16_t *dy;
    void *dtable;
    float factor;
    int32_t accumulate;
    int32_t *flag;
    float *part;            // [2 * spans][c]: of a span, what belongs to the row of the span before, and to the next's
};

__device__ __forceinline__ void put(const Sums &P, int64_t i, float v) {
    v *= P.factor;
    if (P.kind == 2) {
        float *o = (float *)P.dtable + i;
        if (P.accumulate) v += *o;
        *o = v;
        if (P.flag && !__builtin_isfinite(v)) *P.flag = 1;
        return;
    }
    uint16_t *o = (uint16_t *)P.dtable + i;
    if (P.accumulate) v += P.kind == Half::id ? from16<Half>(*o) : from16<BFloat>(*o);
    *o = (uint16_t)(P.kind == Half::id ? to16<Half>(v) : to16<BFloat>(v));
    if (P.flag && !__builtin_isfinite(P.kind == Half::id ? from16<Half>(*o) : from16<BFloat>(*o))) *P.flag = 1;
}

// Workgroup (span, 256 channels): runs of equal numbers.  A run that begins in this span and ends
// in it is a row's whole sum.
template <class T>
__global__ __launch_bounds__(256) void sum_kernel(const Sums P) {
    __shared__ uint32_t key[SPAN + 2], row[SPAN];  // key[0] and key[SPAN + 1]: the neighbours'
    const int64_t at = (int64_t)blockIdx.x * SPAN;
    const int n = P.rows - at < SPAN ? (int)(P.rows - at) : SPAN;
    if (threadIdx.x < (uint32_t)n) {
        key[threadIdx.x + 1] = P.key[at + threadIdx.x];
        row[threadIdx.x] = P.row[at + threadIdx.x];
    }
    if (threadIdx.x == 64) key[0] = at > 0 ? P.key[at - 1] : ~0u;
    if (threadIdx.x == 65) key[n + 1] = at + n < P.rows ? P.key[at + n] : ~0u;
    __syncthreads();
    for (int64_t c = (int64_t)blockIdx.y * 256 + threadIdx.x; c < P.c; c += (int64_t)gridDim.y * 256) {
        float sum = 0.f;
        bool begun = key[0] == key[1];  // the run reaches in from the span before
        for (int i = 0; i < n; ++i) {
            if (key[i + 1] >= (uint32_t)P.v) break;  // padding is sorted last
            sum += from16<T>(P.dy[(int64_t)row[i] * P.c + c]);
            if (key[i + 1] == key[i + 2] && i + 1 < n) continue;
            if (begun)
                P.part[(2 * (int64_t)blockIdx.x) * P.c + c] = sum;
            else if (key[i + 1] == key[i + 2])
                P.part[(2 * (int64_t)blockIdx.x + 1) * P.c + c] = sum;
            else
                put(P, (int64_t)key[i + 1] * P.c + c, sum);
            sum = 0.f;
            begun = false;
        }
    }
}

// Workgroup (span, 256 channels): the row whose run begins in this span and goes on behind it.
__global__ __launch_bounds__(256) void join_kernel(const Sums P, int64_t spans) {
    const int64_t s = blockIdx.x, last = s * SPAN + SPAN - 1;
    if (last + 1 >= P.rows) return;
    const uint32_t k = P.key[last];
    if (k >= (uint32_t)P.v || P.key[last + 1] != k) return;
    if (s * SPAN > 0 && P.key[s * SPAN] == k && P.key[s * SPAN - 1] == k) return;  // begins before
    for (int64_t c = (int64_t)blockIdx.y * 256 + threadIdx.x; c < P.c; c += (int64_t)gridDim.y * 256) {
        float sum = P.part[(2 * s + 1) * P.c + c];
        for (int64_t i = s + 1; i < spans && P.key[i * SPAN] == k; ++i) sum += P.part[2 * i * P.c + c];
        put(P, (int64_t)k * P.c + c, sum);
    }
}

// Rows of the table that no token names.
__global__ __launch_bounds__(256) void clear_kernel(const Sums P) {
    for (int64_t j = blockIdx.x; j < P.v; j += gridDim.x) {
        int64_t lo = 0, hi = P.rows;
        while (lo < hi) {
            const int64_t mid = (lo + hi) / 2;
            if (P.key[mid] < (uint32_t)j)
                lo = mid + 1;
            else
                hi = mid;
        }
        if (lo < P.rows && P.key[lo] == (uint32_t)j) continue;
        for (int64_t c = threadIdx.x; c < P.c; c += 256) {
            if (P.kind == 2)
                ((float *)P.dtable)[j * P.c + c] = 0.f;
            else
                ((uint16_t *)P.dtable)[j * P.c + c] = 0;
        }
    }
}

inline size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }

struct Layout {
    int64_t blocks, spans;
    size_t key[2], row[2], counts, part, bytes;
};

static Layout layout_of(int64_t rows, int32_t c) {
    Layout l;
    l.blocks = (rows + TILE - 1) / TILE;
    l.spans = (rows + SPAN - 1) / SPAN;
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
    l.part = take((size_t)l.spans * 2 * c * 4);
    l.bytes = at;
    return l;
}

}  // namespace embedding

using namespace embedding;

size_t embedding_ws(int64_t rows, int32_t c) { return rows > 0 ? layout_of(rows, c).bytes : 0; }

hipError_t launch_embedding_fwd(int dtype, const EmbeddingParams &p, hipStream_t st) {
    const bool vec = p.c % 8 == 0 && ((uintptr_t)p.table & 15) == 0 && ((uintptr_t)p.y & 15) == 0;
    const int64_t n = (p.rows * (vec ? p.c / 8 : p.c) + 255) / 256;
    const dim3 grid((uint32_t)(n < (1 << 20) ? n : (1 << 20)));
    if (dtype == Half::id) {
        if (vec)
            hipLaunchKernelGGL((fwd_kernel<Half, true>), grid, dim3(256), 0, st, p);
        else
            hipLaunchKernelGGL((fwd_kernel<Half, false>), grid, dim3(256), 0, st, p);
    } else if (vec)
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
    int from = 0;
    if (p.rows > 0) {
        int bits = 1;  // of the largest key, which is v
        while (bits < 32 && ((uint32_t)p.v >> bits) != 0) ++bits;
        Sort q;
        q.rows = p.rows;
        q.v = p.v;
        q.blocks = (int32_t)l.blocks;
        q.ids = p.ids;
        q.counts = (uint32_t *)(ws + l.counts);
        const dim3 grid((uint32_t)l.blocks), block(64 * WAVES);
        for (int shift = 0; shift < bits; shift += BITS) {
            q.shift = shift;
            q.key = (const uint32_t *)(ws + l.key[from]);
            q.row = (const uint32_t *)(ws + l.row[from]);
            from ^= 1;
            q.key_out = (uint32_t *)(ws + l.key[from]);
            q.row_out = (uint32_t *)(ws + l.row[from]);
            if (shift == 0)
                hipLaunchKernelGGL((sort_kernel<true, true>), grid, block, 0, st, q);
            else
                hipLaunchKernelGGL((sort_kernel<false, true>), grid, block, 0, st, q);
            hipLaunchKernelGGL(sort_scan_kernel, dim3(1), dim3(1024), 0, st, q.counts, l.blocks * BINS);
            if (shift == 0)
                hipLaunchKernelGGL((sort_kernel<true, false>), grid, block, 0, st, q);
            else
                hipLaunchKernelGGL((sort_kernel<false, false>), grid, block, 0, st, q);
        }
    }
    s.key = (const uint32_t *)(ws + l.key[from]);
    s.row = (const uint32_t *)(ws + l.row[from]);
    s.part = (float *)(ws + l.part);
    if (!p.accumulate)
        hipLaunchKernelGGL(clear_kernel, dim3((uint32_t)(p.v < 65536 ? p.v : 65536)), dim3(256), 0, st, s);
    if (p.rows > 0) {
        const int64_t cols = (p.c + 255) / 256;
        const dim3 grid((uint32_t)l.spans, (uint32_t)(cols < 64 ? cols : 64));
        if (dtype == Half::id)
            hipLaunchKernelGGL((sum_kernel<Half>), grid, dim3(256), 0, st, s);
        else
            hipLaunchKernelGGL((sum_kernel<BFloat>), grid, dim3(256), 0, st, s);
        hipLaunchKernelGGL(join_kernel, grid, dim3(256), 0, st, s, l.spans);
    }
    return hipGetLastError();
}

}  // namespace nnconv
