// rmsnorm.hip -- root-mean-square norm over the channels of channel-last rows, with the
// residual's addition in front, a 16-bit or 8-bit output, and its backward pass.
//
// Bound by memory: a row is read once into registers, 8 channels (one 16-byte access) at a
// time, and everything is computed from there.  TPR threads hold a row of up to 8 * V * TPR
// channels, vector k * TPR + i of it in thread i: parts of a wave, a wave, or a workgroup, so
// that short rows fill waves and long ones fit the registers.  Rows of any channel count and
// alignment run on the same kernels: the last vector of a row whose channels are no multiple of
// 8 starts at channel c - 8, and the channels it shares with the one before count once.
//
// Measured: 16384 x 4096 with a residual to 8 bits 84 us (5.6 TB/s); 200704 x 256 forward 66 us
// (6.2 TB/s), backward 65 us and 5 us for the sum of dgain's parts; 12345 x 771 (rows at every
// alignment) 16, 17 and 4 us.
#include <type_traits>

#include "launch.hpp"

namespace nnconv {

namespace {

typedef u32x4 __attribute__((aligned(2))) u32x4_any;  // 16 bytes at any element
typedef u32x2 __attribute__((aligned(1))) u32x2_any;
typedef f32x4 __attribute__((aligned(4))) f32x4_any;

// Value of lane ^ 1, of lane ^ 2, of a lane of the other quad and of the other 8 of a row of 16
// (where all lanes of the quad, or of the 8, hold the same).
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}
constexpr int XOR1 = 0xB1, XOR2 = 0x4E, HALF_MIRROR = 0x141, MIRROR = 0x140;

// Over N neighbouring lanes.
template <int N, class F>
__device__ __forceinline__ float lanes_reduce(float v, F op) {
    if (N >= 2) v = op(v, dpp<XOR1>(v));
    if (N >= 4) v = op(v, dpp<XOR2>(v));
    if (N >= 8) v = op(v, dpp<HALF_MIRROR>(v));
    if (N >= 16) v = op(v, dpp<MIRROR>(v));
    if (N >= 32) v = op(v, __shfl_xor(v, 16));
    if (N >= 64) v = op(v, __shfl_xor(v, 32));
    return v;
}

struct Add {
    __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
};
struct Max {
    __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
};

// Over the TPR threads of a row.  Two rounds that follow each other need buffers of their own.
template <int TPR, class F>
__device__ __forceinline__ float row_reduce(float v, float *buf, F op) {
    v = lanes_reduce<(TPR < 64 ? TPR : 64)>(v, op);
    if constexpr (TPR > 64) {
        if ((threadIdx.x & 63) == 0) buf[threadIdx.x % TPR >> 6] = v;
        __syncthreads();
        v = buf[0];
#pragma unroll
        for (int w = 1; w < TPR / 64; ++w) v = op(v, buf[w]);
    }
    return v;
}

// One vector of a row: where it starts, and its channels below `skip` belong to the vector
// before.
struct Slot {
    int at, skip;
    bool in;
    __device__ __forceinline__ Slot(int vec, int c) {
        const int lo = 8 * vec;
        in = lo < c;
        at = lo < c - 8 ? lo : c - 8;
        skip = in ? lo - at : 8;
    }
};

// What a pass reads or writes once streams past the caches; but rows that do not start on 16
// bytes (ANY) share cache lines between lanes' loads, which then come from the cache.
template <bool ANY>
__device__ __forceinline__ u32x4 load8(const void *p, int64_t i) {
    const u32x4_any *q = (const u32x4_any *)((const uint16_t *)p + i);
    return ANY ? *q : __builtin_nontemporal_load(q);
}

__device__ __forceinline__ void store8(void *p, int64_t i, u32x4 v) {
    __builtin_nontemporal_store(v, (u32x4_any *)((uint16_t *)p + i));
}

// The stored sum, kept in the caches where a training step's backward pass reads it again.
__device__ __forceinline__ void store_sum(const NormParams &p, int64_t i, u32x4 v) {
    if (p.rstd)
        *(u32x4_any *)((uint16_t *)p.sum + i) = v;
    else
        store8(p.sum, i, v);
}

template <class T>
__device__ __forceinline__ void unpack8(u32x4 v, float o[8]) {
#pragma unroll
    for (int d = 0; d < 4; ++d) {
        o[2 * d] = from16<T>(v[d] & 0xFFFFu);
        o[2 * d + 1] = from16<T>(v[d] >> 16);
    }
}

template <class T>
__device__ __forceinline__ u32x4 pack8(const float v[8]) {
    u32x4 r;
#pragma unroll
    for (int d = 0; d < 4; ++d) r[d] = pack16<T>(v[2 * d], v[2 * d + 1]);
    return r;
}

__device__ __forceinline__ void load_gain(const float *g, const Slot &s, float o[8]) {
    const f32x4 a = *(const f32x4_any *)(g + s.at), b = *(const f32x4_any *)(g + s.at + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        o[e] = a[e];
        o[4 + e] = b[e];
    }
}

// Division by a group's scale, max |y| / 448.  A product with a rounded reciprocal is off by an ulp
// or two, which moves a code that lies near a tie; corrected by the product's remainder it is the
// fp32 quotient (three instructions where a division takes ten; 0.7 % of the time at 16384 x 4096, 3 %
// with divisions for the scale and its reciprocal).  The numbers of a tiny group are multiplied
// by 2^64 first, which keeps remainders above the smallest fp32 number.
struct Scale {
    float value, by, inv, up;
    __device__ __forceinline__ explicit Scale(float most) {
        constexpr float part = 1.0f / 448.0f;
        up = most < 0x1p-55f ? 0x1p64f : 1.0f;
        const float m = most * up;
        by = m * part;
        by = __builtin_fmaf(__builtin_fmaf(-by, 448.0f, m), part, by);
        value = up == 1.0f ? by : by * 0x1p-64f;
        if (__builtin_isinf(most)) value = most;
        if (value < 0x1p-126f) value = 0.f;
        inv = __builtin_amdgcn_rcpf(by);
        inv = __builtin_fmaf(__builtin_fmaf(-by, inv, 1.0f), inv, inv);
        if (value == 0.f || __builtin_isinf(value)) by = inv = 0.f;  // the quotients are 0 or NaN
    }
    // y[k] = y[k] / value
    template <int N>
    __device__ __forceinline__ void divide(float (&y)[N]) const {
        if (up != 1.0f)
#pragma unroll
            for (int k = 0; k < N; ++k) y[k] *= up;
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const float q = y[k] * inv;
            y[k] = __builtin_fmaf(__builtin_fmaf(-q, by, y[k]), inv, q);
        }
    }
};

// ---- forward -------------------------------------------------------------------------

template <class T, int TPR, int V, bool TAIL, bool Q8>
__global__ __launch_bounds__(TPR <= 64 ? 256 : TPR) void rmsnorm_fwd_kernel(const NormParams p) {
    constexpr int WG = TPR <= 64 ? 256 : TPR, ROWS = WG / TPR;
    __shared__ float buf[2][TPR > 64 ? TPR / 64 : 1];
    const int t = threadIdx.x % TPR;
    float gain[V][8];
#pragma unroll
    for (int k = 0; k < V; ++k) {
        const Slot s(k * TPR + t, p.c);
        if (s.in) load_gain(p.gain, s, gain[k]);
    }
    const float inv_c = 1.0f / (float)p.c;
    for (int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / TPR; row - threadIdx.x / TPR < p.rows;
         row += (int64_t)gridDim.x * ROWS) {
        const bool live = row < p.rows;  // the rows of a workgroup reduce together
        const int64_t base = row * p.c;
        u32x4 x[V], res[V];
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const Slot s(k * TPR + t, p.c);
            if (!live || !s.in) continue;
            x[k] = load8<TAIL>(p.x, base + s.at);
            if (p.residual) res[k] = load8<TAIL>(p.residual, base + s.at);
        }
        float ss = 0.f;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const Slot s(k * TPR + t, p.c);
            if (!live || !s.in) continue;
            float r[8];
            unpack8<T>(x[k], r);
            if (p.residual) {
                float b[8];
                unpack8<T>(res[k], b);
#pragma unroll
                for (int e = 0; e < 8; ++e) r[e] += b[e];
                x[k] = pack8<T>(r);  // the stream as it is stored
                unpack8<T>(x[k], r);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (!TAIL || e >= s.skip) ss += r[e] * r[e];
        }
        if constexpr (TPR > 64) __syncthreads();  // the buffers' last readers are done
        const float rstd = 1.0f / sqrtf(row_reduce<TPR>(ss, buf[0], Add()) * inv_c + p.eps);
        if (p.rstd && live && t == 0) p.rstd[row] = rstd;
        if constexpr (!Q8) {
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const Slot s(k * TPR + t, p.c);
                if (!live || !s.in) continue;
                float y[8];
                unpack8<T>(x[k], y);
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = y[e] * rstd * gain[k][e];
                if (p.sum) store_sum(p, base + s.at, x[k]);
                store8(p.y, base + s.at, pack8<T>(y));
            }
        } else {
            float y[V][8], most[V], row_most = 0.f;
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const Slot s(k * TPR + t, p.c);
                most[k] = 0.f;
                if (!live || !s.in) continue;
                unpack8<T>(x[k], y[k]);
                if (p.sum) store_sum(p, base + s.at, x[k]);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    y[k][e] = y[k][e] * rstd * gain[k][e];
                    if (!TAIL || e >= s.skip) most[k] = fmaxf(most[k], fabsf(y[k][e]));
                }
                row_most = fmaxf(row_most, most[k]);
            }
            const int wide = p.group / 8;  // threads with one scale: 4, 8 or 16 of a group, or the row
            if (p.groups == 1) {
                row_most = row_reduce<TPR>(row_most, buf[1], Max());
            } else {
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    most[k] = lanes_reduce<4>(most[k], Max());
                    if (wide >= 8) most[k] = fmaxf(most[k], dpp<HALF_MIRROR>(most[k]));
                    if (wide >= 16) most[k] = fmaxf(most[k], dpp<MIRROR>(most[k]));
                }
            }
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const int vec = k * TPR + t;
                const Slot s(vec, p.c);
                if (!live || !s.in) continue;
                const Scale scale(p.groups == 1 ? row_most : most[k]);
                if (p.groups == 1 ? vec == 0 : vec % wide == 0)
                    p.scales[row * p.groups + (p.groups == 1 ? 0 : vec / wide)] = scale.value;
                scale.divide(y[k]);
                int q0 = 0, q1 = 0;
                q0 = __builtin_amdgcn_cvt_pk_fp8_f32(y[k][0], y[k][1], q0, false);
                q0 = __builtin_amdgcn_cvt_pk_fp8_f32(y[k][2], y[k][3], q0, true);
                q1 = __builtin_amdgcn_cvt_pk_fp8_f32(y[k][4], y[k][5], q1, false);
                q1 = __builtin_amdgcn_cvt_pk_fp8_f32(y[k][6], y[k][7], q1, true);
                uint8_t *to = (uint8_t *)p.y + base + s.at;
                if (!TAIL || s.skip == 0) {
                    *(u32x2_any *)to = u32x2{(uint32_t)q0, (uint32_t)q1};
                } else {  // the shared channels may have another scale
#pragma unroll
                    for (int e = 1; e < 8; ++e)
                        if (e >= s.skip) to[e] = (uint8_t)((e < 4 ? q0 : q1) >> (8 * (e & 3)));
                }
            }
        }
    }
}

// Rows that the registers do not hold, and rows of fewer channels than a vector: a workgroup
// per row, which reads it again for the output (and for the scales).
template <class T, bool Q8>
__global__ __launch_bounds__(512) void rmsnorm_fwd_any_kernel(const NormParams p) {
    __shared__ float buf[2][8];
    const int t = threadIdx.x;
    const uint16_t *x = (const uint16_t *)p.x, *res = (const uint16_t *)p.residual;
    uint16_t *sum = (uint16_t *)p.sum;
    for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const int64_t base = row * p.c;
        auto added = [&](int i) {
            if (!res) return from16<T>(x[base + i]);
            return from16<T>(to16<T>(from16<T>(x[base + i]) + from16<T>(res[base + i])) & 0xFFFFu);
        };
        // after the first pass the stored sum, which may lie on x or on the residual
        auto again = [&](int i) { return sum ? from16<T>(sum[base + i]) : added(i); };
        float ss = 0.f;
        for (int i = t; i < p.c; i += 512) {
            const float r = added(i);
            if (sum) sum[base + i] = (uint16_t)to16<T>(r);
            ss += r * r;
        }
        __syncthreads();  // the last row's readers of buf are done; the sum is visible
        const float rstd = 1.0f / sqrtf(row_reduce<512>(ss, buf[0], Add()) / (float)p.c + p.eps);
        if (p.rstd && t == 0) p.rstd[row] = rstd;
        auto y = [&](int i) { return again(i) * rstd * p.gain[i]; };
        auto put8 = [&](int i, const Scale &scale) {
            float q[1] = {y(i)};
            scale.divide(q);
            ((uint8_t *)p.y)[base + i] = (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[0], 0, false);
        };
        if constexpr (!Q8) {
            for (int i = t; i < p.c; i += 512) ((uint16_t *)p.y)[base + i] = (uint16_t)to16<T>(y(i));
        } else if (p.groups == 1) {
            float most = 0.f;
            for (int i = t; i < p.c; i += 512) most = fmaxf(most, fabsf(y(i)));
            const Scale scale(row_reduce<512>(most, buf[1], Max()));
            if (t == 0) p.scales[row] = scale.value;
            for (int i = t; i < p.c; i += 512) put8(i, scale);
        } else {
            for (int g = t >> 6; g < p.groups; g += 8) {  // a wave per group
                const int lo = g * p.group, hi = min(lo + p.group, p.c);
                float most = 0.f;
                for (int i = lo + (t & 63); i < hi; i += 64) most = fmaxf(most, fabsf(y(i)));
                const Scale scale(lanes_reduce<64>(most, Max()));
                if ((t & 63) == 0) p.scales[row * p.groups + g] = scale.value;
                for (int i = lo + (t & 63); i < hi; i += 64) put8(i, scale);
            }
        }
    }
}

// ---- backward ------------------------------------------------------------------------

// dx, and the workgroup's share of dgain: a thread keeps the sums of its channels over all its
// rows in registers, which are added up once, in a fixed order.
template <class T, int TPR, int V, bool TAIL>
__global__ __launch_bounds__(TPR < 512 ? 512 : TPR) void rmsnorm_bwd_kernel(const NormBwdParams p) {
    constexpr int WG = TPR < 512 ? 512 : TPR, ROWS = WG / TPR, LANES = TPR < 64 ? TPR : 64;
    __shared__ float buf[ROWS][TPR > 64 ? TPR / 64 : 1];
    const int t = threadIdx.x % TPR;
    float gain[V][8], acc[V][8];
#pragma unroll
    for (int k = 0; k < V; ++k) {
        const Slot s(k * TPR + t, p.c);
        if (s.in) load_gain(p.gain, s, gain[k]);
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[k][e] = 0.f;
    }
    const float inv_c = 1.0f / (float)p.c;
    for (int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / TPR; row - threadIdx.x / TPR < p.rows;
         row += (int64_t)gridDim.x * ROWS) {
        const bool live = row < p.rows;
        const int64_t base = row * p.c;
        u32x4 x[V], dy[V], ds[V];
        const float rstd = live ? p.rstd[row] : 0.f;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const Slot s(k * TPR + t, p.c);
            if (!live || !s.in) continue;
            x[k] = load8<TAIL>(p.sum, base + s.at);
            dy[k] = load8<TAIL>(p.dy, base + s.at);
            if (p.dsum) ds[k] = load8<TAIL>(p.dsum, base + s.at);  // before any store: dx may lie on it
        }
        float dot = 0.f;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const Slot s(k * TPR + t, p.c);
            if (!live || !s.in) continue;
            float xh[8], d[8];
            unpack8<T>(x[k], xh);
            unpack8<T>(dy[k], d);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (!TAIL || e >= s.skip) {
                    const float m = d[e] * (xh[e] * rstd);
                    dot += gain[k][e] * m;
                    acc[k][e] += m;
                }
        }
        if constexpr (TPR > 64) __syncthreads();  // the buffer's last readers are done
        const float mean = row_reduce<TPR>(dot, buf[threadIdx.x / TPR], Add()) * inv_c;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const Slot s(k * TPR + t, p.c);
            if (!live || !s.in) continue;
            float xh[8], d[8], o[8];
            unpack8<T>(x[k], xh);
            unpack8<T>(dy[k], d);
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = 0.f;
            if (p.dsum) unpack8<T>(ds[k], o);
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] += rstd * (d[e] * gain[k][e] - xh[e] * rstd * mean);
            store8(p.dx, base + s.at, pack8<T>(o));
        }
    }
    if (!p.part) return;
    float *part = p.part + (int64_t)blockIdx.x * p.c;
    if constexpr (ROWS == 1) {
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const Slot s(k * TPR + t, p.c);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e >= s.skip) part[s.at + e] = acc[k][e];
        }
        return;
    }
    // rows of a wave, then the workgroup's TPR-thread teams one after the other
    __shared__ float all[8 * V * TPR];
#pragma unroll
    for (int o = LANES; o < 64; o *= 2)
#pragma unroll
        for (int k = 0; k < V; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[k][e] += __shfl_xor(acc[k][e], o);
    constexpr int TEAM = TPR < 64 ? 64 : TPR;
    for (int team = 0; team < WG / TEAM; ++team) {
        if ((int)(threadIdx.x / TEAM) == team && threadIdx.x % TEAM < TPR)
#pragma unroll
            for (int k = 0; k < V; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float *to = &all[(k * 8 + e) * TPR + t];
                    *to = team ? *to + acc[k][e] : acc[k][e];
                }
        __syncthreads();
    }
    if (threadIdx.x < TPR)
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const Slot s(k * TPR + t, p.c);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e >= s.skip) part[s.at + e] = all[(k * 8 + e) * TPR + t];
        }
}

// Any row length: dx with a workgroup per row that reads it twice, the partial sums of dgain
// with a thread per channel.
template <class T>
__global__ __launch_bounds__(512) void rmsnorm_bwd_any_kernel(const NormBwdParams p) {
    __shared__ float buf[8];
    const uint16_t *r = (const uint16_t *)p.sum, *dy = (const uint16_t *)p.dy, *ds = (const uint16_t *)p.dsum;
    for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const int64_t base = row * p.c;
        const float rstd = p.rstd[row];
        float dot = 0.f;
        for (int i = threadIdx.x; i < p.c; i += 512)
            dot += from16<T>(dy[base + i]) * p.gain[i] * (from16<T>(r[base + i]) * rstd);
        __syncthreads();
        const float mean = row_reduce<512>(dot, buf, Add()) / (float)p.c;
        for (int i = threadIdx.x; i < p.c; i += 512) {
            float v = rstd * (from16<T>(dy[base + i]) * p.gain[i] - from16<T>(r[base + i]) * rstd * mean);
            if (ds) v += from16<T>(ds[base + i]);
            ((uint16_t *)p.dx)[base + i] = (uint16_t)to16<T>(v);
        }
    }
}

template <class T>
__global__ __launch_bounds__(256) void rmsnorm_dgain_any_kernel(const NormBwdParams p) {
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i >= p.c) return;
    const uint16_t *r = (const uint16_t *)p.sum, *dy = (const uint16_t *)p.dy;
    const int64_t per = (p.rows + p.parts - 1) / p.parts;
    const int64_t lo = per * blockIdx.y, hi = lo + per < p.rows ? lo + per : p.rows;
    float s = 0.f;
    for (int64_t k = lo; k < hi; ++k)
        s += from16<T>(dy[k * p.c + i]) * (from16<T>(r[k * p.c + i]) * p.rstd[k]);
    p.part[(int64_t)blockIdx.y * p.c + i] = s;
}

// ---- which kernel ---------------------------------------------------------------------

// Threads of a row and vectors of each.  One vector a thread wherever a workgroup is enough:
// more threads have more loads on their way, and the waits of one row's reduction are covered
// by other workgroups.  Against a wave a row with 4 vectors and 256 threads with 4 (us, forward
// with a residual, 16 bits):
//   2048 channels:  8 rows 4.3 -> 2.6,  8192 rows 27.7 -> 23.8,  32768 rows 100 -> 80
//   8192 channels:  8 rows 4.6 -> 3.1,  8192 rows 102 -> 84,     32768 rows 410 -> 350
// The backward pass keeps sums of dgain in registers and writes them once a workgroup; from
// 2049 channels on it is the faster with two vectors (4096 channels, 32768 rows: 175 us, 186
// with one; 8192 channels: 352 and 369).
// Rows of up to 32 channels take no more threads than they have vectors, to a power of two.
// Against eight a row (us, 400000 rows, forward with a residual and backward):
//   8 channels 16.6 -> 5.3 and 19.2 -> 10.8,  16: 19.3 -> 10.3 and 20.1 -> 15.6,
//   17: 19.7 -> 15.6 and 23.6 -> 20.4,        32: 24.2 -> 19.3 and 22.9 -> 23.3
struct Shape {
    int tpr, v;
};

Shape shape_of(int64_t c, bool backward) {
    if (c < 8 || c > 16384) return {0, 0};
    if (c == 8) return {1, 1};
    if (c <= 16) return {2, 1};
    if (c <= 32) return {4, 1};
    if (c <= 64) return {8, 1};
    if (c <= 128) return {16, 1};
    if (c <= 256) return {32, 1};
    if (c <= 512) return {64, 1};
    if (c <= 1024) return {128, 1};
    if (c <= 2048) return {256, 1};
    if (c <= 4096) return backward ? Shape{256, 2} : Shape{512, 1};
    if (c <= 8192) return backward ? Shape{512, 2} : Shape{1024, 1};
    return backward ? Shape{512, 4} : Shape{1024, 2};
}

template <class F>
void with_shape(Shape s, F f) {
#define SHAPE(t, v_) \
    if (s.tpr == t && s.v == v_) return f(std::integral_constant<int, t>{}, std::integral_constant<int, v_>{})
    SHAPE(1, 1);
    SHAPE(2, 1);
    SHAPE(4, 1);
    SHAPE(8, 1);
    SHAPE(16, 1);
    SHAPE(32, 1);
    SHAPE(64, 1);
    SHAPE(128, 1);
    SHAPE(256, 1);
#undef SHAPE
}

template <class F>
void with_fwd_shape(Shape s, F f) {
    if (s.tpr == 512) return f(std::integral_constant<int, 512>{}, std::integral_constant<int, 1>{});
    if (s.tpr == 1024 && s.v == 1) return f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 1>{});
    if (s.tpr == 1024) return f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 2>{});
    with_shape(s, f);
}

template <class F>
void with_bwd_shape(Shape s, F f) {
    if (s.tpr == 256 && s.v == 2) return f(std::integral_constant<int, 256>{}, std::integral_constant<int, 2>{});
    if (s.tpr == 512 && s.v == 2) return f(std::integral_constant<int, 512>{}, std::integral_constant<int, 2>{});
    if (s.tpr == 512) return f(std::integral_constant<int, 512>{}, std::integral_constant<int, 4>{});
    with_shape(s, f);
}

template <class F>
void with_bool(bool b, F f) {
    if (b)
        f(std::true_type{});
    else
        f(std::false_type{});
}

uint32_t blocks_for(int64_t rows, int per, int64_t most) {
    const int64_t n = (rows + per - 1) / per;
    return (uint32_t)(n < most ? n : most);
}

constexpr int64_t FWD_BLOCKS = 1 << 20, BWD_BLOCKS = 512, BWD_FEW = 128, ANY_PARTS = 256;

template <class T>
void fwd(const NormParams &p, bool q8, hipStream_t st) {
    const Shape s = shape_of(p.c, false);
    with_bool(q8, [&](auto q) {
        if (s.tpr == 0) {
            hipLaunchKernelGGL((rmsnorm_fwd_any_kernel<T, decltype(q)::value>), dim3(blocks_for(p.rows, 1, FWD_BLOCKS)),
                               dim3(512), 0, st, p);
            return;
        }
        with_fwd_shape(s, [&](auto tpr, auto v) {
            constexpr int TPR = decltype(tpr)::value, WG = TPR <= 64 ? 256 : TPR;
            with_bool(p.c % 8 != 0, [&](auto tail) {
                hipLaunchKernelGGL((rmsnorm_fwd_kernel<T, TPR, decltype(v)::value, decltype(tail)::value, decltype(q)::value>),
                                   dim3(blocks_for(p.rows, WG / TPR, FWD_BLOCKS)), dim3(WG), 0, st, p);
            });
        });
    });
}

template <class T>
void bwd(const NormBwdParams &p, hipStream_t st) {
    const Shape s = shape_of(p.c, true);
    if (s.tpr == 0) {
        if (p.part)  // first: dx may lie on dy
            hipLaunchKernelGGL((rmsnorm_dgain_any_kernel<T>), dim3((p.c + 255) / 256, p.parts), dim3(256), 0, st, p);
        hipLaunchKernelGGL((rmsnorm_bwd_any_kernel<T>), dim3(blocks_for(p.rows, 1, FWD_BLOCKS)), dim3(512), 0, st, p);
        return;
    }
    with_bwd_shape(s, [&](auto tpr, auto v) {
        constexpr int TPR = decltype(tpr)::value, WG = TPR < 512 ? 512 : TPR;
        with_bool(p.c % 8 != 0, [&](auto tail) {
            hipLaunchKernelGGL((rmsnorm_bwd_kernel<T, TPR, decltype(v)::value, decltype(tail)::value>), dim3(p.parts), dim3(WG),
                               0, st, p);
        });
    });
}

}  // namespace

// Partial sums of dgain: one per workgroup of the backward pass.
int32_t rmsnorm_bwd_parts(int64_t rows, int32_t c) {
    const Shape s = shape_of(c, true);
    if (s.tpr == 0) return (int32_t)(rows < ANY_PARTS ? rows : ANY_PARTS);
    // at least two rows a team, so that the partial sums stay small beside the rows, unless
    // that leaves few workgroups
    const int64_t each = blocks_for(rows, s.tpr < 512 ? 512 / s.tpr : 1, INT32_MAX), half = each / 2;
    const int64_t few = each < BWD_FEW ? each : BWD_FEW;
    return (int32_t)(half < few ? few : half < BWD_BLOCKS ? half : BWD_BLOCKS);
}

hipError_t launch_rmsnorm_fwd(int dtype, const NormParams &p, bool q8, hipStream_t st) {
    if (p.rows <= 0) return hipSuccess;
    if (dtype == Half::id) fwd<Half>(p, q8, st); else fwd<BFloat>(p, q8, st);
    return hipGetLastError();
}

hipError_t launch_rmsnorm_bwd(int dtype, const NormBwdParams &p, hipStream_t st) {
    if (p.rows <= 0) return hipSuccess;
    if (dtype == Half::id) bwd<Half>(p, st); else bwd<BFloat>(p, st);
    return hipGetLastError();
}

}  // namespace nnconv
