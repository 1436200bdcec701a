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

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

struct Rows {
    int64_t rows;
    int32_t c, ldx, v, k;
    const uint16_t *x, *w;
    const int32_t *targets;
    const void *teacher;  // or null: labels
    float scale;
    uint16_t *xc;    // [rows][ldx]: x with zeros behind its channels and in rows that do not count
    uint16_t *wc;    // [v][ldx]: w with zeros behind its channels, or null
    int32_t first_w; // workgroups before those that copy w
    int32_t shares;  // workgroups of a row's targets
    // of a teacher's targets, [rows][k]: products with x, turned where scale is negative; shares; what
    // is taken from their softmax
    float *zt, *qi, *qt;
    float *base;     // [rows]: sum q log q; the bits NOT_COUNTED in rows that do not count
};

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

// Whether this workgroup copies w, 1024 vectors of 8 channels each.
constexpr int COPY_VECTORS = 1024;
__device__ __forceinline__ bool copied_w(const Rows &P) {
    if (blockIdx.x < (uint32_t)P.first_w) return false;
    const uint32_t per = (uint32_t)P.ldx / 8;
    const int64_t first = (int64_t)(blockIdx.x - P.first_w) * COPY_VECTORS, count = (int64_t)P.v * per;
    u32x4 v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int64_t i = first + u * 256 + threadIdx.x, r = i / per;
        if (i < count) v[u] = row_vector(P.w + r * P.c, (int)(i - r * per) * 8, P.c);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int64_t i = first + u * 256 + threadIdx.x;
        if (i < count) *(u32x4 *)(P.wc + i * 8) = v[u];
    }
    return true;
}

// Labels: the copies of x, a thread 8 channels, and of w.
__global__ __launch_bounds__(256) void copy_kernel(const Rows P) {
    if (copied_w(P)) return;
    const uint32_t per = (uint32_t)P.ldx / 8;
    const int64_t count = P.rows * per;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < count; i += (int64_t)P.first_w * 256) {
        const int64_t r = i / per;
        const int c = (int)(i - r * per) * 8;
        const bool in = (uint32_t)P.targets[r] < (uint32_t)P.v;
        *(u32x4 *)(P.xc + r * P.ldx + c) = in ? row_vector(P.x + r * P.c, c, P.c) : u32x4{};
    }
}

template <class T>
__device__ __forceinline__ float dot8(u32x4 a, u32x4 b, float s) {
#pragma unroll
    for (int d = 0; d < 4; ++d) {
        s = fmaf(from16<T>(a[d]), from16<T>(b[d]), s);
        s = fmaf(from16<T>(a[d] >> 16), from16<T>(b[d] >> 16), s);
    }
    return s;
}

// A teacher's logit i, turned where the factor is negative, and whether the entry is left out, which
// its own value says.  The factor comes behind the difference to the largest: before it, what is finite
// may pass fp32.
template <class T, class S>
__device__ __forceinline__ float teacher_logit(const Rows &P, int64_t i, bool &out) {
    float a;
    if constexpr (sizeof(S) == 4)
        a = ((const float *)P.teacher)[i];
    else
        a = from16<T>(((const uint16_t *)P.teacher)[i]);
    out = (uint32_t)P.targets[i] >= (uint32_t)P.v || a == -INFINITY;
    return P.scale < 0.f ? -a : a;
}

// A teacher: workgroups of a row and a share of its targets.  The logits of the targets in fp32 (their own
// sums: the products' tiles have them in many places), LANES lanes each; the first of a row makes
// its copy and the teacher's softmax.  Bound by the gather of the targets' rows of w (4096 x 32 of
// 1152 channels: 302 MB in 58 us); few targets have a wave each, for the latency.  SHORT: fewer than 8
// channels.
template <class T, class S, int LANES, bool SHORT>
__global__ __launch_bounds__(256) void rows_kernel(const Rows P) {
    if (copied_w(P)) return;
    // the rows' first shares, which have more to do, come first, on units of their own
    const int share = (int)(blockIdx.x / (uint32_t)P.rows);
    const int64_t r = blockIdx.x - (uint32_t)share * (uint32_t)P.rows;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int k = P.k;
    const int32_t *t = P.targets + r * k;
    const uint16_t *x = P.x + r * P.c;
    // the largest of the teacher's logits that count
    float most = -INFINITY;
    bool any = false;
    for (int i = lane; i < k; i += 64) {
        bool out;
        const float a = teacher_logit<T, S>(P, r * k + i, out);
        if (out) continue;
        any = true;
        most = fmaxf(most, a);
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) most = fmaxf(most, __shfl_xor(most, d));
    any = __any(any);
    if (share == 0) {
        uint16_t *xc = P.xc + r * P.ldx;
        for (int c = tid * 8; c < P.ldx; c += 2048) *(u32x4 *)(xc + c) = any ? row_vector<SHORT>(x, c, P.c) : u32x4{};
    }
    if (!any) {
        if (share == 0 && tid == 0) P.base[r] = __builtin_bit_cast(float, NOT_COUNTED);
        return;  // nothing is read of the rest
    }
    constexpr int TEAMS = 256 / LANES;
    const int at = tid & (LANES - 1);
    for (int i = share * TEAMS + tid / LANES; i < k; i += TEAMS * P.shares) {
        const int32_t j = t[i];
        float dot = 0.f;
        if ((uint32_t)j < (uint32_t)P.v) {
            const uint16_t *w = P.w + (int64_t)j * P.c;
            for (int c = at * 8; c < P.c; c += LANES * 8)
                dot = dot8<T>(row_vector<SHORT>(x, c, P.c), row_vector<SHORT>(w, c, P.c), dot);
        }
#pragma unroll
        for (int d = LANES / 2; d > 0; d >>= 1) dot += __shfl_xor(dot, d);
        if (at == 0) P.zt[r * k + i] = P.scale < 0.f ? -dot : dot;
    }
    if (share > 0) return;
    __shared__ float q[MOST_TARGETS];
    __shared__ float part[4];
    const float scale = fabsf(P.scale);
    float sum = 0.f;
    for (int i = tid; i < k; i += 256) {
        bool out;
        const float a = teacher_logit<T, S>(P, r * k + i, out);
        const float e = out ? 0.f : expf((a - most) * scale);
        q[i] = e;
        sum += e;
    }
    sum = wave_sum(sum);
    if (lane == 0) part[wave] = sum;
    __syncthreads();
    sum = part[0] + part[1] + part[2] + part[3];
    const float log_sum = logf(sum);
    float base = 0.f;
    for (int i = tid; i < k; i += 256) {
        const float e = q[i];
        float taken = 0.f;  // a target that is named twice is taken from once, with both shares
        for (int j = 0; j < k; ++j) taken += t[j] == t[i] ? q[j] : 0.f;
        P.qi[r * k + i] = e / sum;
        P.qt[r * k + i] = taken / sum;
        bool out;
        if (e != 0.f) base += e / sum * ((teacher_logit<T, S>(P, r * k + i, out) - most) * scale - log_sum);
    }
    __syncthreads();
    base = wave_sum(base);
    if (lane == 0) part[wave] = base;
    __syncthreads();
    if (tid == 0) {
        base = part[0] + part[1] + part[2] + part[3];
        P.base[r] = base == base ? base : __builtin_nanf("");  // a teacher's NaN may have any bits
    }
}

// The tiles' statistics of rows, and what becomes of them.
struct Join {
    int64_t rows;
    int32_t tiles, shift, v, k;  // shift: of a column to its tile
    float scale, unit;          // |logit_scale|, and over log 2: what products count
    const float2 *stats;
    const int32_t *targets;     // [rows][k]
    const float *zt;            // the targets' products
    const float *qi, *qt, *base;  // a teacher's shares and sums (see Rows); null with labels
    float *loss, *lse;          // lse may be null
    uint16_t *e;                // training: [rows][lde]
    int64_t lde, stretch;       // elements of a workgroup
    int32_t parts;              // workgroups of a row
    // [rows][c], or null: x, to be copied with zeros in rows that do not count, in 16-byte vectors
    const uint16_t *x;
    uint16_t *xc;
    int32_t c;
};

// The largest product of a row, and the sum of the exponentials against it, by one wave.
__device__ __forceinline__ void join_row(const float2 *s, int tiles, float unit, float &most, float &sum) {
    const int lane = threadIdx.x & 63;
    most = -INFINITY;
    for (int i = lane; i < tiles; i += 64) most = fmaxf(most, s[i].x);
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) most = fmaxf(most, __shfl_xor(most, d));
    sum = 0.f;
    for (int i = lane; i < tiles; i += 64) {
        const float2 v = s[i];
        sum += v.y * exp2f(v.x == most ? 0.f : (v.x - most) * unit);
    }
    sum = wave_sum(sum);
}

__device__ __forceinline__ bool row_counts(const Join &P, int64_t r) { return Counts{P.targets, P.base, P.v}.of(r); }

// How far a target's product lies below the largest, 0 at least: a teacher's targets have their own
// sums, whose rounding may pass it.
__device__ __forceinline__ float below(float most, float zt) { return zt > most ? 0.f : most - zt; }

// By one wave.
__device__ __forceinline__ void put_loss(const Join &P, int64_t r, bool counts, float most, float log_sum) {
    const int lane = threadIdx.x & 63;
    float loss = 0.f;
    if (P.base && counts) {
        // sum q (log q + lse - z), the terms most - z first
        float z = 0.f;
        for (int i = lane; i < P.k; i += 64) {
            const float q = P.qi[r * P.k + i];
            if (q != 0.f) z += q * below(most, P.zt[r * P.k + i]);
        }
        loss = P.base[r] + wave_sum(z) * P.scale + log_sum * LN2;
    } else if (counts)
        loss = below(most, P.zt[r]) * P.scale + log_sum * LN2;  // near 0 both are small
    if (lane != 0) return;
    P.loss[r] = loss;
    if (P.lse) P.lse[r] = counts ? most * P.scale + log_sum * LN2 : 0.f;
}

// A wave a row.
__global__ __launch_bounds__(256) void join_kernel(const Join P) {
    const int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (r >= P.rows) return;
    float most, sum;
    join_row(P.stats + r * P.tiles, P.tiles, P.unit, most, sum);
    const bool counts = row_counts(P, r);
    put_loss(P, r, counts, most, log2f(sum));
}

// A workgroup a stretch of a row, one or at most SHARE of them: each joins the row's statistics
// itself (a launch for it took 4 us of a small step's 58), all of the stretch is scaled by its
// tiles' factors, then the targets are written from their own logits.  Bound by its 4 bytes an
// element (4.9 TB/s on 1 GiB).
constexpr int64_t STRETCH = 8192, SHARE = 8;

template <class T>
__global__ __launch_bounds__(256) void scale_kernel(const Join P) {
    const int64_t r = blockIdx.x / P.parts;
    const int part = (int)(blockIdx.x - r * P.parts);
    const int64_t n0 = part * P.stretch, n1 = n0 + P.stretch < P.lde ? n0 + P.stretch : P.lde;
    uint16_t *e = P.e + r * P.lde;
    const float2 *s = P.stats + r * P.tiles;
    u32x4 v[4];
    auto load = [&](int64_t i) {
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (i + u * 2048 < n1) v[u] = *(const u32x4 *)(e + i + u * 2048);
    };
    int64_t i = n0 + threadIdx.x * 8;
    load(i);  // on their way meanwhile
    const bool counts = row_counts(P, r);
    float most, sum;
    join_row(s, P.tiles, P.unit, most, sum);
    const float log_sum = log2f(sum), over = GRAD_UNIT / sum;
    if (part == 0 && threadIdx.x < 64) put_loss(P, r, counts, most, log_sum);
    if (P.xc && part == P.parts - 1)
        for (int c = threadIdx.x * 8; c < P.c; c += 2048)
            *(u32x4 *)(P.xc + r * P.c + c) = counts ? *(const u32x4 *)(P.x + r * P.c + c) : u32x4{};
    for (;;) {
        float f[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int64_t n = i + u * 2048;
            const float m = n < n1 ? s[n >> P.shift].x : most;
            f[u] = over * exp2f(m == most ? 0.f : (m - most) * P.unit);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int64_t n = i + u * 2048;
            if (n >= n1) continue;
            // a row that does not count has zeros, whatever became of its exponentials
#pragma unroll
            for (int d = 0; d < 4; ++d)
                v[u][d] = counts ? pack16<T>(unpack_exp<T>(v[u][d]) * f[u], unpack_exp<T>(v[u][d] >> 16) * f[u]) : 0u;
            *(u32x4 *)(e + n) = v[u];
        }
        i += STRETCH;
        if (i >= n1) break;
        load(i);
    }
    if (!counts) return;
    __syncthreads();
    for (int i = threadIdx.x; i < P.k; i += 256) {
        const int32_t j = P.targets[r * P.k + i];
        if ((uint32_t)j >= (uint32_t)P.v || j < n0 || j >= n1) continue;
        const float q = P.qt ? P.qt[r * P.k + i] : 1.f;
        e[j] = (uint16_t)to16<T>(GRAD_UNIT * (exp2f(-below(most, P.zt[r * P.k + i]) * P.unit - log_sum) - q));
    }
}

inline size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }

// Bytes of the exponentials of a piece of rows at most, and in a forward call of the statistics.
constexpr int64_t PIECE_BYTES = (int64_t)1 << 30, STATS_BYTES = (int64_t)1 << 27;
constexpr int64_t MOST_OPERAND = (int64_t)1 << 35;  // elements of x and of w
constexpr int CUS = 256;

// A product's tile and, for the gradients, how often its reduction is split.
struct Shape {
    Config cfg;
    int32_t splits;
    int64_t k_split;
};

// By an estimate of the time in us: rounds of workgroups (one 256 x 256 tile a compute unit, or two
// 128 x 128 ones) of what a reduction element and a tile take, and the sums of the splits.  The
// rates are those of long products, 1200 and 960 TFLOP/s over all units.
static Shape shape_of(int64_t m, int64_t n, int64_t k, bool split) {
    Shape best = {TILE_256, 1, (k + 63) / 64 * 64};
    // Logits that 128 x 128 tiles would keep no more than half the units busy with (300 x 512 of 4096
    // channels: 22 us with 32 x 128 tiles, 31 with 128 x 128; 128 x 16384 of 2048: 28 and 30), and
    // those of up to 32 rows; beyond, the smaller tiles lose (64 x 65536 of 2048: 54 and 49; 512 x 8192
    // of 512: 21 and 12).
    if (!split && (m <= 32 || (m + 127) / 128 * ((n + 127) / 128) <= CUS / 2)) return {TILE_32, 1, best.k_split};
    double least = 1e300;
    for (int c = TILE_256; c <= TILE_128; ++c) {
        const int64_t b = tile_rows((Config)c), slots = c == TILE_256 ? CUS : 2 * CUS;
        const double per_k = c == TILE_256 ? 0.028 : 0.0175, per_tile = c == TILE_256 ? 6.0 : 4.0;
        const int64_t tiles = ((m + b - 1) / b) * ((n + b - 1) / b);
        for (int64_t s = 1; s <= (split ? 16 : 1); ++s) {
            const int64_t ks = ((k + s - 1) / s + 63) / 64 * 64, splits = (k + ks - 1) / ks;
            if (splits != s || (s > 1 && ks < 256)) continue;
            const int64_t rounds = (tiles * splits + slots - 1) / slots;
            // a 128 x 128 tile alone on its unit is faster than beside another
            const double alone = c == TILE_128 && tiles * splits <= CUS ? 0.7 : 1.0;
            double t = (double)rounds * ((double)ks * per_k * alone + per_tile);
            if (splits > 1) t += 3.0 + (double)(m * n) * (8.0 * (double)splits + 4.0) / 5e6;
            if (t < least) {
                least = t;
                best = {(Config)c, (int32_t)splits, ks};
            }
        }
    }
    return best;
}

struct Plan {
    int64_t ldx, ldw, lde, piece;
    Shape logits, dx, dw;
    int32_t tiles;  // stats a row
    bool copy_w, copy_x, late_x;
    size_t xc, wc, zt, qi, qt, base, stats, e, part, part_w, acc, bytes;
};

static Plan plan_of(const XentParams &p, bool train) {
    Plan q;
    q.ldx = q.ldw = (p.c + 7) / 8 * 8;
    q.copy_w = p.c % 8 != 0;
    // rows that do not count may hold NaN, which the product for dw would meet: it reads a copy, made
    // beside a teacher's softmax or, where x is read as it is before, by scale_kernel
    q.copy_x = q.copy_w || p.teacher || ((uintptr_t)p.x & 15) != 0;
    q.late_x = !q.copy_x && train && p.dw;
    q.lde = ((int64_t)p.v + 63) / 64 * 64;
    const int64_t most = (train ? PIECE_BYTES / (2 * q.lde) : STATS_BYTES / (8 * (((int64_t)p.v + 127) / 128))) / 256 * 256;
    q.piece = p.rows;
    if (q.piece > most) q.piece = most > 256 ? most : 256;
    if (q.piece > p.rows) q.piece = p.rows;
    q.logits = shape_of(q.piece, p.v, p.c, false);
    q.dx = shape_of(q.piece, p.c, q.lde, true);
    q.dw = shape_of(p.v, p.c, q.piece, true);
    const int tile = tile_cols(q.logits.cfg);
    q.tiles = (int32_t)(((int64_t)p.v + tile - 1) / tile);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t was = at;
        at += align256(bytes);
        return was;
    };
    q.xc = take(q.copy_x || q.late_x || p.sizes_only ? (size_t)p.rows * q.ldx * 2 : 0);
    q.wc = take(q.copy_w ? (size_t)p.v * q.ldw * 2 : 0);
    q.zt = take((size_t)p.rows * p.k * 4);
    q.qi = take((size_t)p.rows * p.k * 4);
    q.qt = take((size_t)p.rows * p.k * 4);
    q.base = take((size_t)p.rows * 4);
    q.stats = take((size_t)q.piece * q.tiles * 8);
    q.e = q.part = q.part_w = q.acc = at;
    if (train) {
        q.e = take((size_t)q.piece * q.lde * 2);
        q.part = take(q.dx.splits > 1 ? (size_t)q.dx.splits * q.piece * p.c * 4 : 0);
        q.part_w = take(q.dw.splits > 1 ? (size_t)q.dw.splits * p.v * p.c * 4 : 0);
        q.acc = take(q.piece < p.rows ? (size_t)p.v * p.c * 4 : 0);
    }
    q.bytes = at;
    return q;
}

template <class T, class S, int LANES>
static void launch_teacher(Rows r, uint32_t more, hipStream_t st) {
    // few rows: their targets are shared out
    const int64_t most = (r.k + 256 / LANES - 1) / (256 / LANES), want = 1024 / r.rows;
    r.shares = (int32_t)(want < 1 ? 1 : want < most ? want : most);
    r.first_w = (int32_t)r.rows * r.shares;
    const dim3 grid((uint32_t)r.first_w + more);
    if (r.c < 8)
        hipLaunchKernelGGL((rows_kernel<T, S, LANES, true>), grid, dim3(256), 0, st, r);
    else
        hipLaunchKernelGGL((rows_kernel<T, S, LANES, false>), grid, dim3(256), 0, st, r);
}

template <class T, class S>
static void launch_teacher(const Rows &r, uint32_t more, hipStream_t st) {
    // a wave a target while that fills the chip no more than twice
    if (r.rows * r.k <= 2 * CUS * 32)
        launch_teacher<T, S, 64>(r, more, st);
    else
        launch_teacher<T, S, 16>(r, more, st);
}

static void launch_rows(int dtype, int teacher_dtype, Rows r, hipStream_t st) {
    const int64_t vectors = r.wc ? (int64_t)r.v * (r.ldx / 8) : 0;
    const uint32_t more = (uint32_t)((vectors + COPY_VECTORS - 1) / COPY_VECTORS);
    if (!r.teacher) {
        const int64_t n = (r.rows * (r.ldx / 8) + 255) / 256;
        r.first_w = (int32_t)(n < (1 << 20) ? n : (1 << 20));
        hipLaunchKernelGGL(copy_kernel, dim3((uint32_t)r.first_w + more), dim3(256), 0, st, r);
        return;
    }
    const bool wide = teacher_dtype == NNCONV_F32;
    if (dtype == Half::id && wide)
        launch_teacher<Half, float>(r, more, st);
    else if (dtype == Half::id)
        launch_teacher<Half, uint16_t>(r, more, st);
    else if (wide)
        launch_teacher<BFloat, float>(r, more, st);
    else
        launch_teacher<BFloat, uint16_t>(r, more, st);
}

}  // namespace xent

using namespace xent;

bool xent_fits(const XentParams &p) {
    if (p.k > MOST_TARGETS || fabsf(p.logit_scale) > 0x1p127f) return false;  // 1.44 times which fp32 holds
    // a tile's rows are addressed with 31 bits, the threads of a launch with 32
    return p.c <= (1 << 20) && p.v <= (1 << 21) && p.rows <= (1 << 23) && p.rows * p.c <= MOST_OPERAND &&
           (int64_t)p.v * p.c <= MOST_OPERAND;
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
        g.o = {p.dw, p.dw_dtype, p.c, p.v, 1.0f, nullptr, 0, nullptr, nullptr, nullptr, false, {}};
        return launch_grad_w(p.dtype, TILE_128, g, st);
    }
    const Plan q = plan_of(p, train);
    char *ws = (char *)p.ws;
    auto at = [&](size_t o) { return (float *)(ws + o); };
    const uint16_t *w = (const uint16_t *)p.w;
    Rows r;
    r.rows = p.rows;
    r.c = p.c;
    r.ldx = (int32_t)q.ldx;
    r.v = p.v;
    r.k = p.k;
    r.x = (const uint16_t *)p.x;
    r.w = w;
    r.wc = q.copy_w ? (uint16_t *)(ws + q.wc) : nullptr;
    r.targets = p.targets;
    r.teacher = p.teacher;
    r.scale = p.logit_scale;
    r.xc = (uint16_t *)(ws + q.xc);
    r.zt = at(q.zt);
    r.qi = at(q.qi);
    r.qt = at(q.qt);
    r.base = at(q.base);
    const uint16_t *x = (const uint16_t *)p.x;
    if (q.copy_x) {
        launch_rows(p.dtype, p.teacher_dtype, r, st);
        x = r.xc;
        if (q.copy_w) w = r.wc;
    }

    const int tile = tile_cols(q.logits.cfg);
    for (int64_t r0 = 0; r0 < p.rows; r0 += q.piece) {
        const int64_t n = p.rows - r0 < q.piece ? p.rows - r0 : q.piece;
        Logits l;
        l.x = {x + r0 * q.ldx, q.ldx, (int32_t)n};
        l.w = {w, q.ldw, p.v};
        l.k = (int32_t)q.ldx;
        l.unit = p.logit_scale * LOG2E;
        l.labels = p.teacher ? nullptr : p.targets + r0;
        l.zt = r.zt + r0;
        l.stats = (float2 *)(ws + q.stats);
        l.e = train ? (uint16_t *)(ws + q.e) : nullptr;
        l.lde = q.lde;
        // what the last-level cache (256 MB) cannot hold until it is read only drives the operands out
        // of it: 1 GiB of exponentials, streamed, 1.3 % off the whole step; 256 MiB, 1.5 % on
        l.stream = 2 * n * q.lde > ((int64_t)512 << 20);
        hipError_t e = launch_logits(p.dtype, q.logits.cfg, l, st);
        if (e != hipSuccess) return e;
        Join j;
        j.rows = n;
        j.tiles = q.tiles;
        j.shift = tile == 256 ? 8 : 7;
        j.v = p.v;
        j.k = p.k;
        j.scale = fabsf(p.logit_scale);
        j.unit = fabsf(l.unit);
        j.stats = l.stats;
        j.targets = p.targets + r0 * p.k;
        j.zt = r.zt + r0 * p.k;
        j.qi = p.teacher ? r.qi + r0 * p.k : nullptr;
        j.qt = p.teacher ? r.qt + r0 * p.k : nullptr;
        j.base = p.teacher ? r.base + r0 : nullptr;
        j.loss = p.loss + r0;
        j.lse = p.lse ? p.lse + r0 : nullptr;
        j.e = l.e;
        j.lde = q.lde;
        j.x = q.late_x ? x + r0 * p.c : nullptr;
        j.xc = q.late_x ? r.xc + r0 * p.c : nullptr;
        j.c = p.c;
        if (!train) {
            hipLaunchKernelGGL(join_kernel, dim3((uint32_t)((n + 3) / 4)), dim3(256), 0, st, j);
            continue;
        }
        j.stretch = (q.lde + SHARE - 1) / SHARE;
        j.stretch = (j.stretch + STRETCH - 1) / STRETCH * STRETCH;
        j.parts = (int32_t)((q.lde + j.stretch - 1) / j.stretch);
        const dim3 grid((uint32_t)(n * j.parts));  // 2^23 at most: a piece has 2^29 elements, or 256 rows
        if (p.dtype == Half::id)
            hipLaunchKernelGGL((scale_kernel<Half>), grid, dim3(256), 0, st, j);
        else
            hipLaunchKernelGGL((scale_kernel<BFloat>), grid, dim3(256), 0, st, j);
        const float alpha = p.alpha * p.logit_scale / GRAD_UNIT;
        Grad g, d;
        g.a = {l.e, q.lde, (int32_t)n};
        g.b = {w, q.ldw, (int32_t)q.ldw};
        g.k = p.v;
        g.k_split = q.dx.k_split;
        g.splits = q.dx.splits;
        g.part = at(q.part);
        g.o = {(uint16_t *)p.dx + r0 * p.c, p.dtype, p.c, n, alpha, p.grad_scale, 0, p.flag, nullptr, nullptr, true,
               {j.targets, j.base, p.v}};
        d.a = {l.e, q.lde, (int32_t)q.lde};
        d.b = {q.late_x ? j.xc : l.x.p, q.ldx, (int32_t)q.ldx};
        d.k = n;
        d.k_split = q.dw.k_split;
        d.splits = q.dw.splits;
        d.part = at(q.part_w);
        d.o = {p.dw, p.dw_dtype, p.c, p.v, alpha * p.inv_loss_scale, p.grad_scale, p.accumulate, p.flag,
               r0 > 0 ? at(q.acc) : nullptr, r0 + n < p.rows ? at(q.acc) : nullptr, false, {}};
        e = launch_grads(p.dtype, q.dx.cfg, g, q.dw.cfg, p.dw ? &d : nullptr, st);
        if (e != hipSuccess) return e;
    }
    return hipGetLastError();
}

}  // namespace nnconv
