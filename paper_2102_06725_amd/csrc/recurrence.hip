// recurrence.hip -- gated linear recurrence over the tokens of a sequence,
// channel by channel, forward and backward.
#include "launch.hpp"

namespace nnconv {

namespace {

constexpr int SAVE = NNCONV_RECURRENCE_SAVE;

// The gate a = sigma(z) and b = 1 - a = sigma(-z), each to full relative
// precision: with a near 1 the difference 1 - a would keep few bits of the
// long memories' rates.
__device__ __forceinline__ void gate(float f, float bias, float &a, float &b) {
    float z = f + bias;
    z = z > 80.f ? 80.f : z < -80.f ? -80.f : z;  // a NaN stays
    const float e = __expf(-z);
    a = __builtin_amdgcn_rcpf(1.0f + e);
    b = e * a;
}

__device__ __forceinline__ float sigma(float v) {
    return __builtin_amdgcn_rcpf(1.0f + __expf(-v));
}

__device__ __forceinline__ int length_of(const RecParams &p, int n) {
    if (!p.lengths) return p.t;
    const int l = p.lengths[n];
    return l < 0 ? 0 : l > p.t ? p.t : l;
}

// A thread per channel walks the tokens.
template <class T>
__global__ __launch_bounds__(64) void recurrence_fwd_kernel(const RecParams p) {
    const int c = blockIdx.x * 64 + threadIdx.x;
    if (c >= p.c) return;
    for (int64_t n = blockIdx.y; n < p.n; n += gridDim.y) {
        const int len = length_of(p, n);
        float h = p.h0 ? p.h0[n * p.c + c] : 0.f;
        const float bias = p.bias ? p.bias[c] : 0.f;
        const uint16_t *x = (const uint16_t *)p.x + n * p.t * p.ld + c;
        const uint16_t *f = (const uint16_t *)p.f + n * p.t * p.ld + c;
        const uint16_t *g = p.g ? (const uint16_t *)p.g + n * p.t * p.ld + c : nullptr;
        uint16_t *y = (uint16_t *)p.y + n * p.t * p.ldy + c;
        for (int64_t t = 0; t < p.t; ++t) {
            if (p.saved && t % SAVE == 0)
                p.saved[(n * ((p.t + SAVE - 1) / SAVE) + t / SAVE) * p.c + c] = h;
            float out = 0.f;
            if (t < len) {
                float a, b;
                gate(from16<T>(f[t * p.ld]), bias, a, b);
                h = a * h + b * from16<T>(x[t * p.ld]);
                out = h;
                if (g) {
                    const float gv = from16<T>(g[t * p.ld]);
                    out = h * gv * sigma(gv);
                }
            }
            y[t * p.ldy] = (uint16_t)to16<T>(out);
        }
        if (p.ht) p.ht[n * p.c + c] = h;
    }
}

// The same from the last token back; the states inside a stretch of SAVE
// tokens are computed again from the saved one.
template <class T>
__global__ __launch_bounds__(64) void recurrence_bwd_kernel(const RecParams p) {
    __shared__ float hs[SAVE][64];
    const int lane = threadIdx.x;
    const int c = blockIdx.x * 64 + lane;
    if (c >= p.c) return;
    for (int64_t n = blockIdx.y; n < p.n; n += gridDim.y) {
        const int len = length_of(p, n);
        const int64_t chunks = (p.t + SAVE - 1) / SAVE;
        float d = p.dht ? p.dht[n * p.c + c] : 0.f;  // what flows into the state from the right
        const float bias = p.bias ? p.bias[c] : 0.f;
        const int64_t at = n * p.t * p.ld + c;
        const uint16_t *x = (const uint16_t *)p.x + at, *f = (const uint16_t *)p.f + at;
        const uint16_t *g = p.g ? (const uint16_t *)p.g + at : nullptr;
        uint16_t *dx = (uint16_t *)p.dx + at, *df = (uint16_t *)p.df + at;
        uint16_t *dg = p.g ? (uint16_t *)p.dg + at : nullptr;
        const uint16_t *dy = (const uint16_t *)p.dy + n * p.t * p.ldy + c;
        float total = 0.f;
        for (int64_t k = chunks - 1; k >= 0; --k) {
            const int64_t lo = k * SAVE, hi = lo + SAVE < p.t ? lo + SAVE : p.t;
            float h = p.saved[(n * chunks + k) * p.c + c];
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
                    const float ht = a * before + b * xv;
                    float own = from16<T>(dy[t * p.ldy]);
                    if (g) {
                        const float gv = from16<T>(g[t * p.ld]), s = sigma(gv);
                        vg = own * ht * s * (1.0f + gv * (1.0f - s));
                        own = own * gv * s;
                    }
                    d += own;
                    vx = d * b;
                    vf = d * (before - xv) * (a * b);
                    d *= a;
                    total += vf;
                }
                dx[t * p.ld] = (uint16_t)to16<T>(vx);
                df[t * p.ld] = (uint16_t)to16<T>(vf);
                if (dg) dg[t * p.ld] = (uint16_t)to16<T>(vg);
            }
        }
        if (p.dh0) p.dh0[n * p.c + c] = d;
        if (p.part) p.part[n * p.c + c] = total;
    }
}

}  // namespace

int64_t recurrence_bwd_parts(const RecParams &p) { return p.n; }

size_t recurrence_ws(const RecParams &p, bool backward) {
    if (!backward) return 0;
    const int64_t parts = recurrence_bwd_parts(p);
    return sizeof(float) * (size_t)((parts + colsum_extra(parts)) * p.c);
}

hipError_t launch_recurrence_fwd(int dtype, const RecParams &p, hipStream_t st) {
    if (p.n <= 0) return hipSuccess;
    const dim3 grid((p.c + 63) / 64, p.n < 65535 ? p.n : 65535);
    if (dtype == Half::id)
        hipLaunchKernelGGL((recurrence_fwd_kernel<Half>), grid, dim3(64), 0, st, p);
    else
        hipLaunchKernelGGL((recurrence_fwd_kernel<BFloat>), grid, dim3(64), 0, st, p);
    return hipGetLastError();
}

hipError_t launch_recurrence_bwd(int dtype, const RecParams &p, hipStream_t st) {
    if (p.n <= 0) return hipSuccess;
    const dim3 grid((p.c + 63) / 64, p.n < 65535 ? p.n : 65535);
    if (dtype == Half::id)
        hipLaunchKernelGGL((recurrence_bwd_kernel<Half>), grid, dim3(64), 0, st, p);
    else
        hipLaunchKernelGGL((recurrence_bwd_kernel<BFloat>), grid, dim3(64), 0, st, p);
    return hipGetLastError();
}

}  // namespace nnconv
