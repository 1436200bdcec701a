// rmsnorm.hip -- root-mean-square norm over the channels of channel-last rows,
// with the residual's addition in front, a 16-bit or 8-bit output, and its
// backward pass.
#include "launch.hpp"

namespace nnconv {

namespace {

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
    return v;
}

// r of one element, rounded to the storage type.
template <class T>
__device__ __forceinline__ float add_residual(const uint16_t *x, const uint16_t *res, int64_t i,
                                              uint32_t &bits) {
    if (!res) {
        bits = x[i];
        return from16<T>(bits);
    }
    bits = to16<T>(from16<T>(x[i]) + from16<T>(res[i])) & 0xFFFFu;
    return from16<T>(bits);
}

// A wave per row, one element per lane at a time.
template <class T, bool Q8>
__global__ __launch_bounds__(256) void rmsnorm_fwd_kernel(const NormParams p) {
    const int lane = threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= p.rows) return;
    const int64_t base = row * p.c;
    const uint16_t *x = (const uint16_t *)p.x, *res = (const uint16_t *)p.residual;
    float ss = 0.f;
    uint32_t bits;
    for (int i = lane; i < p.c; i += 64) {
        const float r = add_residual<T>(x, res, base + i, bits);
        ss += r * r;
    }
    const float rstd = 1.0f / sqrtf(wave_sum(ss) / (float)p.c + p.eps);
    if (p.rstd && lane == 0) p.rstd[row] = rstd;
    if constexpr (!Q8) {
        for (int i = lane; i < p.c; i += 64) {
            const float r = add_residual<T>(x, res, base + i, bits);
            if (p.sum) ((uint16_t *)p.sum)[base + i] = (uint16_t)bits;
            ((uint16_t *)p.y)[base + i] = (uint16_t)to16<T>(r * rstd * p.gain[i]);
        }
    } else {
        for (int k = 0; k < p.groups; ++k) {
            const int lo = k * p.group, hi = min(lo + p.group, p.c);
            float most = 0.f;
            for (int i = lo + lane; i < hi; i += 64)
                most = fmaxf(most, fabsf(add_residual<T>(x, res, base + i, bits) * rstd * p.gain[i]));
            float scale = wave_max(most) * (1.0f / 448.0f);
            if (scale < 0x1p-126f) scale = 0.f;
            const float inv = scale > 0.f ? 1.0f / scale : 0.f;
            if (lane == 0) p.scales[row * p.groups + k] = scale;
            for (int i = lo + lane; i < hi; i += 64) {
                const float r = add_residual<T>(x, res, base + i, bits);
                if (p.sum) ((uint16_t *)p.sum)[base + i] = (uint16_t)bits;
                const float q = r * rstd * p.gain[i] * inv;
                ((uint8_t *)p.y)[base + i] =
                    (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(q, q, 0, false);
            }
        }
    }
}

// dx: a wave per row.
template <class T>
__global__ __launch_bounds__(256) void rmsnorm_bwd_kernel(const NormBwdParams p) {
    const int lane = threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= p.rows) return;
    const int64_t base = row * p.c;
    const uint16_t *r = (const uint16_t *)p.sum, *dy = (const uint16_t *)p.dy;
    const uint16_t *ds = (const uint16_t *)p.dsum;
    const float rstd = p.rstd[row];
    float dot = 0.f;
    for (int i = lane; i < p.c; i += 64)
        dot += from16<T>(dy[base + i]) * p.gain[i] * (from16<T>(r[base + i]) * rstd);
    const float mean = wave_sum(dot) / (float)p.c;
    for (int i = lane; i < p.c; i += 64) {
        const float xh = from16<T>(r[base + i]) * rstd;
        float v = rstd * (from16<T>(dy[base + i]) * p.gain[i] - xh * mean);
        if (ds) v += from16<T>(ds[base + i]);
        ((uint16_t *)p.dx)[base + i] = (uint16_t)to16<T>(v);
    }
}

// Partial sums of dgain: thread per channel, NORM_PARTS slabs of rows.
template <class T>
__global__ __launch_bounds__(256) void rmsnorm_dgain_kernel(const NormBwdParams p) {
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

template <class T>
void fwd(const NormParams &p, bool q8, hipStream_t st) {
    const dim3 grid((uint32_t)((p.rows + 3) / 4));
    if (q8)
        hipLaunchKernelGGL((rmsnorm_fwd_kernel<T, true>), grid, dim3(256), 0, st, p);
    else
        hipLaunchKernelGGL((rmsnorm_fwd_kernel<T, false>), grid, dim3(256), 0, st, p);
}

template <class T>
void bwd(const NormBwdParams &p, hipStream_t st) {
    if (p.part)  // first: dx may lie on dy
        hipLaunchKernelGGL((rmsnorm_dgain_kernel<T>), dim3((p.c + 255) / 256, p.parts), dim3(256), 0, st, p);
    hipLaunchKernelGGL((rmsnorm_bwd_kernel<T>), dim3((uint32_t)((p.rows + 3) / 4)), dim3(256), 0, st, p);
}

}  // namespace

int32_t rmsnorm_bwd_parts(int64_t rows, int32_t c) {
    return (int32_t)(rows < 256 ? rows : 256);
}

hipError_t launch_rmsnorm_fwd(int dtype, const NormParams &p, bool q8, hipStream_t st) {
    if (p.rows <= 0) return hipSuccess;
    if ((p.rows + 3) / 4 > 0x7FFFFFFF) return hipErrorInvalidValue;
    if (dtype == Half::id) fwd<Half>(p, q8, st); else fwd<BFloat>(p, q8, st);
    return hipGetLastError();
}

hipError_t launch_rmsnorm_bwd(int dtype, const NormBwdParams &p, hipStream_t st) {
    if (p.rows <= 0) return hipSuccess;
    if ((p.rows + 3) / 4 > 0x7FFFFFFF) return hipErrorInvalidValue;
    if (dtype == Half::id) bwd<Half>(p, st); else bwd<BFloat>(p, st);
    return hipGetLastError();
}

}  // namespace nnconv
