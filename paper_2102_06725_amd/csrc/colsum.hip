// colsum.hip -- per-channel sums of fp32 partials [parts][c], in a fixed order, with the
// loss-scale step of a parameter gradient.  Bound by the latency of a few rounds of loads: 4 to
// 5 us for 128 to 512 parts.
#include "launch.hpp"

namespace nnconv {

namespace {

constexpr int WAVES = 16;

// 64 channels per workgroup; wave w adds parts w, w + 16, ... in increasing order, eight loads
// in flight, and wave 0 the 16 waves' sums.  With out a null pointer the sums of this
// workgroup's share of the parts go to next.
__global__ __launch_bounds__(64 * WAVES) void colsum_kernel(const float *__restrict__ part,
                                                            int64_t parts, int64_t per, int32_t c,
                                                            float *next, float *out,
                                                            float inv_scale, int accumulate,
                                                            int32_t *flag) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    __shared__ float all[WAVES][64];
    const int64_t lo = per * blockIdx.y, hi = lo + per < parts ? lo + per : parts;
    for (int64_t c0 = (int64_t)blockIdx.x * 64; c0 < c; c0 += (int64_t)gridDim.x * 64) {
        const int64_t i = c0 + lane;
        float s = 0.f;
        if (i < c) {
            int64_t k = lo + w;
            const float *src = part + k * c + i;
            const int64_t step = (int64_t)WAVES * c;
            for (; k + 7 * WAVES < hi; k += 8 * WAVES, src += 8 * step) {
                float v[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) v[u] = src[u * step];
#pragma unroll
                for (int u = 0; u < 8; ++u) s += v[u];
            }
            for (; k < hi; k += WAVES, src += step) s += *src;
        }
        __syncthreads();  // the last channels' sums have been read
        all[w][lane] = s;
        __syncthreads();
        if (w != 0 || i >= c) continue;
        s = all[0][lane];
#pragma unroll
        for (int k = 1; k < WAVES; ++k) s += all[k][lane];
        if (!out) {
            next[(int64_t)blockIdx.y * c + i] = s;
            continue;
        }
        s *= inv_scale;
        if (accumulate) s = out[i] + s;
        out[i] = s;
        if (flag && !__builtin_isfinite(s)) *flag = 1;
    }
}

// Parts that one workgroup sums, more where that would take too many workgroups.
constexpr int64_t PER = 512, MOST = 4096;

int64_t per_group(int64_t parts) {
    const int64_t per = (parts + MOST - 1) / MOST;
    return per < PER ? PER : per;
}

}  // namespace

int64_t colsum_extra(int64_t parts) {
    const int64_t per = per_group(parts);
    return parts > PER ? (parts + per - 1) / per : 0;
}

hipError_t launch_colsum(const float *part, int64_t parts, int32_t c, float *extra, float *out,
                         float inv_scale, int accumulate, int32_t *flag, hipStream_t st) {
    const int64_t cols = ((int64_t)c + 63) / 64;
    const uint32_t nb = (uint32_t)(cols < (1 << 18) ? cols : (1 << 18));
    const int64_t more = colsum_extra(parts);
    if (more > 0) {
        hipLaunchKernelGGL(colsum_kernel, dim3(nb, (uint32_t)more), dim3(64 * WAVES), 0, st, part,
                           parts, per_group(parts), c, extra, (float *)nullptr, 1.0f, 0,
                           (int32_t *)nullptr);
        part = extra;
        parts = more;
    }
    hipLaunchKernelGGL(colsum_kernel, dim3(nb), dim3(64 * WAVES), 0, st, part, parts, parts, c,
                       (float *)nullptr, out, inv_scale, accumulate, flag);
    return hipGetLastError();
}

}  // namespace nnconv
