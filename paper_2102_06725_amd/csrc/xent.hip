// xent.hip -- softmax cross entropy over a vocabulary, against a label or a teacher's largest
// logits, without the logits in memory: what stands around the matrix products, and the plan.
//
// Training takes the rows in pieces.  A piece's logits are made once (2 rows v c operations), their
// exponentials are kept in 16 bits in a bounded workspace, and the two gradient products (4 rows v
// c) read them as 2^15 (softmax - q).  A form that keeps nothing of the logits would make them
// twice; the 6 bytes that an element moves instead cost less than its 2 c operations from about
// 500 channels up, and below that a piece's few launches are what counts.
#include "xent.hpp"

namespace nnconv {

namespace xent {

constexpr int MOST_TARGETS = 1024;

struct Rows {
    int64_t rows;
    int32_t c, ldx, v, k;
    const uint16_t *x, *w;
    int64_t ldw;
    const int32_t *targets;
    const void *teacher;
    float scale;
    uint16_t *xc;    // [rows][ldx]: x with zeros behind its channels and in rows that do not count
    float *zt, *qt;  // [rows][k]: the targets' logits; what is taken from their softmax
    float *base;     // [rows]: sum q (log q - z); NaN bits NOT_COUNTED in rows that do not count
};

// What `base` holds for a row that does not count.  Arithmetic makes no NaN with these bits.
constexpr uint32_t NOT_COUNTED = 0x7FC0DEADu;

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

// A workgroup a row: the row's copy, the logits of its targets in fp32 (their own sums, since the
// gradient takes q from a softmax value close to it), and the teacher's softmax.
template <class T, class S>
__global__ __launch_bounds__(256) void rows_kernel(const Rows P) {
    const int64_t r = blockIdx.x;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    __shared__ float q[MOST_TARGETS], z[MOST_TARGETS];
    __shared__ float part[4];
    const int k = P.k;
    const int32_t *t = P.targets + r * k;
    const S *teacher = (const S *)P.teacher + r * k;
    // the largest teacher's logit that counts
    float most = -INFINITY;
    bool any = false, nan = false;
    for (int i = lane; i < k; i += 64) {
        const bool in = (uint32_t)t[i] < (uint32_t)P.v;
        float a = 0.f;
        if (P.teacher) {
            if constexpr (sizeof(S) == 4)
                a = teacher[i] * P.scale;
            else
                a = from16<T>(teacher[i]) * P.scale;
        }
        if (!in || a == -INFINITY) continue;
        any = true;
        nan |= !(a == a);
        most = fmaxf(most, a);
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) most = fmaxf(most, __shfl_xor(most, d));
    any = __any(any);
    nan = __any(nan);
    uint16_t *xc = P.xc + r * P.ldx;
    const uint16_t *x = P.x + r * P.c;
    if (!any) {
        for (int c = tid; c < P.ldx; c += 256) xc[c] = 0;
        for (int i = tid; i < k; i += 256) P.zt[r * k + i] = P.qt[r * k + i] = 0.f;
        if (tid == 0) P.base[r] = __builtin_bit_cast(float, NOT_COUNTED);
        return;
    }
    for (int c = tid; c < P.ldx; c += 256) xc[c] = c < P.c ? x[c] : (uint16_t)0;
    // q before its division, and the logits
    float sum = 0.f;
    for (int i = wave; i < k; i += 4) {
        const int32_t j = t[i];
        const bool in = (uint32_t)j < (uint32_t)P.v;
        float a = 0.f;
        if (P.teacher) {
            if constexpr (sizeof(S) == 4)
                a = teacher[i] * P.scale;
            else
                a = from16<T>(teacher[i]) * P.scale;
        }
        const float e = !in || a == -INFINITY ? 0.f : expf(a - most);
        float dot = 0.f;
        if (in) {
            const uint16_t *w = P.w + (int64_t)j * P.ldw;
            for (int c = lane; c < P.c; c += 64) dot = fmaf(from16<T>(x[c]), from16<T>(w[c]), dot);
        }
        dot = wave_sum(dot) * P.scale;
        if (lane == 0) {
            q[i] = e;
            z[i] = dot;
        }
        sum += e;
    }
    if (lane == 0) part[wave] = sum;
    __syncthreads();
    sum = part[0] + part[1] + part[2] + part[3];
    const float log_sum = logf(sum);
    float base = 0.f;
    for (int i = tid; i < k; i += 256) {
        const float e = q[i];
        float taken = 0.f;  // a target that is named twice is taken from once, with both shares
        for (int j = 0; j < k; ++j) taken += t[j] == t[i] ? q[j] : 0.f;
        P.zt[r * k + i] = z[i];
        P.qt[r * k + i] = taken / sum;
        float a = 0.f;
        if (P.teacher) {
            if constexpr (sizeof(S) == 4)
                a = teacher[i] * P.scale;
            else
                a = from16<T>(teacher[i]) * P.scale;
        }
        if (e != 0.f) base += e / sum * (a - most - log_sum - z[i]);
    }
    __syncthreads();
    base = wave_sum(base);
    if (lane == 0) part[wave] = base;
    __syncthreads();
    if (tid == 0) {
        base = part[0] + part[1] + part[2] + part[3];
        if (nan) base = __builtin_nanf("");
        P.base[r] = base;
    }
}

// A wave a row: lse and loss; the tiles' largest logits become the factors of their exponentials.
__global__ __launch_bounds__(256) void join_kernel(int64_t rows, int32_t tiles, float2 *stats, const float *base,
                                                   float *lse, float *loss, float *lse_out, bool train) {
    const int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    if (r >= rows) return;
    float2 *s = stats + r * tiles;
    float most = -INFINITY;
    for (int i = lane; i < tiles; i += 64) most = fmaxf(most, s[i].x);
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) most = fmaxf(most, __shfl_xor(most, d));
    float sum = 0.f;
    for (int i = lane; i < tiles; i += 64) {
        const float2 v = s[i];
        sum += v.y * expf(v.x == most ? 0.f : v.x - most);
    }
    sum = wave_sum(sum);
    const float b = base[r];
    const bool counts = __builtin_bit_cast(uint32_t, b) != NOT_COUNTED;
    const float total = most + logf(sum);
    if (lane == 0) {
        loss[r] = counts ? b + total : 0.f;
        if (lse_out) lse_out[r] = counts ? total : 0.f;
        if (train) lse[r] = total;
    }
    if (!train) return;
    const float over = GRAD_UNIT / sum;
    for (int i = lane; i < tiles; i += 64)
        s[i].x = counts ? over * expf(s[i].x == most ? 0.f : s[i].x - most) : 0.f;
}

struct Scale {
    int32_t v, k, tile, tiles;
    int64_t lde;
    uint16_t *e;
    const float2 *stats;
    const int32_t *targets;
    const float *zt, *qt, *base, *lse;
};

constexpr int SCALE_VECTORS = 4;  // of 8 elements a thread

// e -> 2^15 (softmax - q), a workgroup a stretch of a row: all of it by the tiles' factors, then
// the targets from their own logits.
template <class T>
__global__ __launch_bounds__(256) void scale_kernel(const Scale P) {
    const int64_t r = blockIdx.y;
    const int64_t n0 = (int64_t)blockIdx.x * 256 * 8 * SCALE_VECTORS;
    uint16_t *e = P.e + r * P.lde;
    const float2 *s = P.stats + r * P.tiles;
    const bool counts = __builtin_bit_cast(uint32_t, P.base[r]) != NOT_COUNTED;
#pragma unroll
    for (int i = 0; i < SCALE_VECTORS; ++i) {
        const int64_t n = n0 + (i * 256 + threadIdx.x) * 8;
        if (n >= P.lde) continue;
        u32x4 v = *(const u32x4 *)(e + n);
        const float f = s[n / P.tile].x;
        // a row that does not count has zeros, whatever became of its exponentials
#pragma unroll
        for (int d = 0; d < 4; ++d)
            v[d] = counts ? pack16<T>(unpack_exp<T>(v[d]) * f, unpack_exp<T>(v[d] >> 16) * f) : 0u;
        *(u32x4 *)(e + n) = v;
    }
    if (!counts) return;
    __syncthreads();
    const float lse = P.lse[r];
    for (int i = threadIdx.x; i < P.k; i += 256) {
        const int32_t j = P.targets[r * P.k + i];
        if ((uint32_t)j >= (uint32_t)P.v || j < n0 || j >= n0 + 256 * 8 * SCALE_VECTORS) continue;
        e[j] = (uint16_t)to16<T>(GRAD_UNIT * (expf(P.zt[r * P.k + i] - lse) - P.qt[r * P.k + i]));
    }
}

inline size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }

// Bytes of the exponentials of a piece of rows at most.
constexpr int64_t PIECE_BYTES = (int64_t)1 << 30;
constexpr int CUS = 256;

// A product's tile and, for the gradients, how often its reduction is split.
struct Shape {
    Config cfg;
    int32_t splits;
    int64_t k_split;
};

// 256-row tiles from one tile a compute unit up, else 128-row ones with the reduction split.
static Shape shape_of(int64_t m, int64_t n, int64_t k, bool split) {
    auto tiles = [&](int b) { return ((m + b - 1) / b) * ((n + b - 1) / b); };
    Shape s = {TILE_256, 1, (k + 63) / 64 * 64};
    if (tiles(256) >= CUS) return s;
    s.cfg = TILE_128;
    const int64_t t = tiles(128);
    if (!split || t >= 2 * CUS) return s;
    int64_t splits = 2 * CUS / t;
    const int64_t most = (k + 511) / 512;  // of no less than 512 elements each
    if (splits > most) splits = most;
    if (splits > 16) splits = 16;
    if (splits < 1) splits = 1;
    s.k_split = ((k + splits - 1) / splits + 63) / 64 * 64;
    s.splits = (int32_t)((k + s.k_split - 1) / s.k_split);
    return s;
}

struct Plan {
    int64_t ldx, ldw, lde, piece;
    Shape logits, dx, dw;
    int32_t tiles;  // stats a row
    bool copy_w;
    size_t xc, wc, zt, qt, base, lse, stats, e, part, acc, bytes;
};

static Plan plan_of(const XentParams &p, bool train) {
    Plan q;
    q.ldx = q.ldw = (p.c + 7) / 8 * 8;
    q.copy_w = p.c % 8 != 0;
    q.lde = ((int64_t)p.v + 63) / 64 * 64;
    q.piece = p.rows;
    if (train) {
        const int64_t most = PIECE_BYTES / (2 * q.lde) / 256 * 256;
        if (q.piece > most) q.piece = most > 256 ? most : 256;
        if (q.piece > p.rows) q.piece = p.rows;
    }
    q.logits = shape_of(q.piece, p.v, p.c, false);
    q.dx = shape_of(q.piece, p.c, q.lde, true);
    q.dw = shape_of(p.v, p.c, q.piece, true);
    const int tile = tile_rows(q.logits.cfg);
    q.tiles = (int32_t)(((int64_t)p.v + tile - 1) / tile);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t was = at;
        at += align256(bytes);
        return was;
    };
    q.xc = take((size_t)p.rows * q.ldx * 2);
    q.wc = take(q.copy_w ? (size_t)p.v * q.ldw * 2 : 0);
    q.zt = take((size_t)p.rows * p.k * 4);
    q.qt = take((size_t)p.rows * p.k * 4);
    q.base = take((size_t)p.rows * 4);
    q.stats = take((size_t)q.piece * q.tiles * 8);
    q.lse = q.e = q.part = q.acc = at;
    if (train) {
        q.lse = take((size_t)q.piece * 4);
        q.e = take((size_t)q.piece * q.lde * 2);
        size_t part = q.dx.splits > 1 ? (size_t)q.dx.splits * q.piece * p.c : 0;
        const size_t w = q.dw.splits > 1 ? (size_t)q.dw.splits * p.v * p.c : 0;
        if (p.dw || p.sizes_only) part = part > w ? part : w;
        q.part = take(part * 4);
        q.acc = take(q.piece < p.rows ? (size_t)p.v * p.c * 4 : 0);
    }
    q.bytes = at;
    return q;
}

template <class T>
static void launch_rows(const Rows &r, int teacher_dtype, hipStream_t st) {
    if (r.teacher && teacher_dtype != NNCONV_F32)
        hipLaunchKernelGGL((rows_kernel<T, uint16_t>), dim3((uint32_t)r.rows), dim3(256), 0, st, r);
    else
        hipLaunchKernelGGL((rows_kernel<T, float>), dim3((uint32_t)r.rows), dim3(256), 0, st, r);
}

}  // namespace xent

using namespace xent;

bool xent_fits(const XentParams &p) {
    if (p.k > MOST_TARGETS) return false;
    // a tile's rows are addressed with 31 bits, workgroups with 30
    return p.c <= (1 << 20) && p.v <= (1 << 21) && p.rows <= (1 << 23);
}

size_t xent_ws(const XentParams &p, bool train) {
    XentParams all = p;
    all.sizes_only = true;
    return p.rows == 0 ? 0 : plan_of(all, train).bytes;
}

hipError_t launch_xent(const XentParams &p, bool train, hipStream_t st) {
    if (p.rows == 0) {  // the gradient of no rows
        if (!train || !p.dw || p.accumulate) return hipSuccess;
        Grad g = {};
        g.splits = 1;
        g.k_split = 64;
        g.o = {p.dw, p.dw_dtype, p.c, p.v, 1.0f, nullptr, 0, nullptr, nullptr, nullptr};
        return launch_grad(p.dtype, TILE_128, true, g, st);
    }
    const Plan q = plan_of(p, train);
    char *ws = (char *)p.ws;
    auto at = [&](size_t o) { return (float *)(ws + o); };
    const uint16_t *w = (const uint16_t *)p.w;
    if (q.copy_w) {
        hipError_t e = launch_pad_channels16(p.w, ws + q.wc, p.v, p.c, (int32_t)q.ldw, st);
        if (e != hipSuccess) return e;
        w = (const uint16_t *)(ws + q.wc);
    }
    Rows r;
    r.rows = p.rows;
    r.c = p.c;
    r.ldx = (int32_t)q.ldx;
    r.v = p.v;
    r.k = p.k;
    r.x = (const uint16_t *)p.x;
    r.w = w;
    r.ldw = q.ldw;
    r.targets = p.targets;
    r.teacher = p.teacher;
    r.scale = p.logit_scale;
    r.xc = (uint16_t *)(ws + q.xc);
    r.zt = at(q.zt);
    r.qt = at(q.qt);
    r.base = at(q.base);
    if (p.dtype == Half::id)
        launch_rows<Half>(r, p.teacher_dtype, st);
    else
        launch_rows<BFloat>(r, p.teacher_dtype, st);

    const int tile = tile_rows(q.logits.cfg);
    for (int64_t r0 = 0; r0 < p.rows; r0 += q.piece) {
        const int64_t n = p.rows - r0 < q.piece ? p.rows - r0 : q.piece;
        Logits l;
        l.x = {r.xc + r0 * q.ldx, q.ldx, (int32_t)n};
        l.w = {w, q.ldw, p.v};
        l.k = (int32_t)q.ldx;
        l.scale = p.logit_scale;
        l.stats = (float2 *)(ws + q.stats);
        l.e = train ? (uint16_t *)(ws + q.e) : nullptr;
        l.lde = q.lde;
        hipError_t e = launch_logits(p.dtype, q.logits.cfg, l, st);
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL(join_kernel, dim3((uint32_t)((n + 3) / 4)), dim3(256), 0, st, n, q.tiles, l.stats, r.base + r0,
                           at(q.lse), p.loss + r0, p.lse ? p.lse + r0 : nullptr, train);
        if (!train) continue;
        Scale s;
        s.v = p.v;
        s.k = p.k;
        s.tile = tile;
        s.tiles = q.tiles;
        s.lde = q.lde;
        s.e = l.e;
        s.stats = l.stats;
        s.targets = p.targets + r0 * p.k;
        s.zt = r.zt + r0 * p.k;
        s.qt = r.qt + r0 * p.k;
        s.base = r.base + r0;
        s.lse = at(q.lse);
        constexpr int64_t STRETCH = 256 * 8 * SCALE_VECTORS;
        for (int64_t y0 = 0; y0 < n; y0 += 32768) {  // rows of one launch
            Scale t = s;
            const int64_t ny = n - y0 < 32768 ? n - y0 : 32768;
            t.e += y0 * q.lde;
            t.stats += y0 * q.tiles;
            t.targets += y0 * p.k;
            t.zt += y0 * p.k;
            t.qt += y0 * p.k;
            t.base += y0;
            t.lse += y0;
            const dim3 grid((uint32_t)((q.lde + STRETCH - 1) / STRETCH), (uint32_t)ny);
            if (p.dtype == Half::id)
                hipLaunchKernelGGL((scale_kernel<Half>), grid, dim3(256), 0, st, t);
            else
                hipLaunchKernelGGL((scale_kernel<BFloat>), grid, dim3(256), 0, st, t);
        }
        const float alpha = p.alpha * p.logit_scale / GRAD_UNIT;
        Grad g;
        g.a = {l.e, q.lde, (int32_t)n};
        g.b = {w, q.ldw, (int32_t)q.ldw};
        g.k = p.v;
        g.k_split = q.dx.k_split;
        g.splits = q.dx.splits;
        g.part = at(q.part);
        g.o = {(uint16_t *)p.dx + r0 * p.c, p.dtype, p.c, n, alpha, p.grad_scale, 0, p.flag, nullptr, nullptr};
        e = launch_grad(p.dtype, q.dx.cfg, false, g, st);
        if (e != hipSuccess) return e;
        if (!p.dw) continue;
        g.a = {l.e, q.lde, (int32_t)q.lde};
        g.b = {l.x.p, q.ldx, (int32_t)q.ldx};
        g.k = n;
        g.k_split = q.dw.k_split;
        g.splits = q.dw.splits;
        g.o = {p.dw, p.dw_dtype, p.c, p.v, alpha * p.inv_loss_scale, p.grad_scale, p.accumulate, p.flag,
               r0 > 0 ? at(q.acc) : nullptr, r0 + n < p.rows ? at(q.acc) : nullptr};
        e = launch_grad(p.dtype, q.dw.cfg, true, g, st);
        if (e != hipSuccess) return e;
    }
    return hipGetLastError();
}

}  // namespace nnconv
