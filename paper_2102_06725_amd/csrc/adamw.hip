// adamw.hip -- AdamW over a list of tensors in one launch, with fp32 moments
// or 8-bit ones.
#include "launch.hpp"

namespace nnconv {

namespace {

constexpr int CHUNK = ADAMW_CHUNK;
constexpr int BATCH = 40;  // list entries in one launch's arguments (of at most 4 KB)

struct InitArgs {
    nnconv_adamw_tensor t[BATCH];
    int64_t chunk0[BATCH];  // first chunk of each
};
static_assert(sizeof(InitArgs) + 32 < 4096, "kernel arguments");

// Writes BATCH list entries and the chunks that belong to them.
__global__ __launch_bounds__(256) void adamw_plan_kernel(const InitArgs a, int32_t first,
                                                         int32_t count, AdamwTable tab) {
    for (int32_t k = blockIdx.x; k < count; k += gridDim.x) {
        if (threadIdx.x == 0) tab.tensors[first + k] = a.t[k];
        const int64_t n = (a.t[k].count + CHUNK - 1) / CHUNK;
        for (int64_t i = threadIdx.x; i < n; i += 256)
            tab.chunks[a.chunk0[k] + i] = AdamwChunk{first + k, (int32_t)i};
    }
}

// The random bits of an element: 16 for m, 16 for v.
__device__ __forceinline__ uint32_t dither_bits(uint32_t key, int64_t i) {
    uint32_t h = (uint32_t)i * 0x9E3779B1u + key;
    h = (h ^ (h >> 16)) * 0x2C1B3C6Du;
    h = (h ^ (h >> 15)) * 0x297A2D39u;
    return h ^ (h >> 16);
}

__device__ __forceinline__ float pow2(int e) { return __builtin_bit_cast(float, (uint32_t)(e + 127) << 23); }

// beta^t for t >= 0, in 64 bits by squaring: 1 - beta^t would lose most of
// its bits in 32 for a beta near 1.
__device__ __forceinline__ double power(double b, int32_t t) {
    double r = 1.0;
    for (; t > 0; t >>= 1, b *= b)
        if (t & 1) r *= b;
    return r;
}

// Magnitude of an 8-bit code: TOP largest exponent, LOW smallest, M mantissa
// bits.  y = |x| * 2^-k lies within range; u in (0, 1).
template <int TOP, int LOW, int M, bool KEEP>
__device__ __forceinline__ float round_random(float y, float u) {
    int e = (int)(__builtin_bit_cast(uint32_t, y) >> 23) - 127;
    e = e < LOW ? LOW : e;
    float r = floorf(y * pow2(M - e) + u);
    if (KEEP && r == 0.f && y > 0.f) r = 1.f;
    return fminf(r * pow2(e - M), 1.75f * pow2(TOP));
}

// Exponent k of the smallest power of two that brings `most` within 1.75 * 2^TOP.
template <int TOP>
__device__ __forceinline__ int block_exponent(float most) {
    const uint32_t b = __builtin_bit_cast(uint32_t, most);
    int k = (int)(b >> 23) - 127 - TOP + ((b & 0x7FFFFFu) > 0x600000u);
    if ((b >> 23) == 0) k = -127;  // zero, and what is too small for a scale of its own
    return k < -127 ? -127 : k;
}

__device__ __forceinline__ float load_grad(const nnconv_adamw_tensor &t, int64_t i) {
    if (t.grad_dtype == NNCONV_F32) return ((const float *)t.grad)[i];
    const uint32_t b = ((const uint16_t *)t.grad)[i];
    return t.grad_dtype == NNCONV_F16 ? from16<Half>(b) : from16<BFloat>(b);
}

// A workgroup per chunk, an element per lane at a time; the 64 lanes of a wave
// are one block of 8-bit moments.
__global__ __launch_bounds__(256) void adamw_kernel(const AdamwTable tab, const int32_t *step,
                                                    float lr, float beta1, float beta2, float eps,
                                                    uint32_t seed, const nnconv_loss_scaler *state,
                                                    const int32_t *flag) {
    if (flag && *flag != 0) return;
    const AdamwChunk ch = tab.chunks[blockIdx.x];
    const nnconv_adamw_tensor t = tab.tensors[ch.tensor];
    const int32_t now = *step + 1;
    const float c1 = (float)(1.0 / (1.0 - power(beta1, now)));
    const float c2 = (float)(1.0 / (1.0 - power(beta2, now)));
    const float inv_scale = state ? 1.0f / state->scale : 1.0f;
    const uint32_t key = (uint32_t)ch.tensor * 0x6C8E9CF5u + (uint32_t)now * 0xB5297A4Du + seed * 0x68E31DA4u;
    const int64_t lo = (int64_t)ch.index * CHUNK;
    for (int64_t i = lo + threadIdx.x; i - threadIdx.x < lo + CHUNK && i - (threadIdx.x & 63) < t.count; i += 256) {
        const bool in = i < t.count;
        const int64_t blk = i / NNCONV_ADAMW_BLOCK;
        float w = 0.f, m = 0.f, v = 0.f, g = 0.f;
        const bool f8 = t.state_dtype == NNCONV_F8;
        if (in) {
            w = t.master[i];
            g = load_grad(t, i) * inv_scale;
            if (f8) {
                m = __builtin_amdgcn_cvt_f32_fp8(((const uint8_t *)t.m)[i], 0) * ldexpf(1.0f, t.m_scale[blk] - 127);
                v = __builtin_amdgcn_cvt_f32_bf8(((const uint8_t *)t.v)[i], 0) * ldexpf(1.0f, t.v_scale[blk] - 127);
            } else {
                m = ((const float *)t.m)[i];
                v = ((const float *)t.v)[i];
            }
        }
        m = beta1 * m + (1.0f - beta1) * g;
        v = beta2 * v + (1.0f - beta2) * (g * g);
        w = w - lr * (m * c1 / (sqrtf(v * c2) + eps) + t.weight_decay * w);
        asm volatile("" : "+v"(w));  // the 16-bit copy is the rounding of the stored master
        if (f8) {
            const bool mf = __builtin_isfinite(m), vf = __builtin_isfinite(v);
            float mm = in && mf ? fabsf(m) : 0.f, vm = in && vf ? v : 0.f;
            for (int o = 32; o > 0; o >>= 1) {
                mm = fmaxf(mm, __shfl_xor(mm, o));
                vm = fmaxf(vm, __shfl_xor(vm, o));
            }
            const int km = block_exponent<8>(mm), kv = block_exponent<15>(vm);
            const uint32_t bits = dither_bits(key + (uint32_t)(i >> 32) * 0x7F4A7C15u, i);
            const float um = ((float)(bits & 0xFFFFu) + 0.5f) * 0x1p-16f, uv = ((float)(bits >> 16) + 0.5f) * 0x1p-16f;
            float qm = copysignf(round_random<8, -6, 3, false>(fabsf(m) * pow2(-km), um), m);
            float qv = round_random<15, -14, 2, true>(v * pow2(-kv), uv);
            if (!mf) qm = __builtin_nanf("");
            if (!vf) qv = __builtin_nanf("");
            if (in) {
                ((uint8_t *)t.m)[i] = (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(qm, qm, 0, false);
                ((uint8_t *)t.v)[i] = (uint8_t)__builtin_amdgcn_cvt_pk_bf8_f32(qv, qv, 0, false);
                if ((threadIdx.x & 63) == 0) {
                    t.m_scale[blk] = (uint8_t)(km + 127);
                    t.v_scale[blk] = (uint8_t)(kv + 127);
                }
            }
        } else if (in) {
            ((float *)t.m)[i] = m;
            ((float *)t.v)[i] = v;
        }
        if (in) {
            t.master[i] = w;
            if (t.w16) ((uint16_t *)t.w16)[i] = (uint16_t)(t.w16_dtype == NNCONV_F16 ? to16<Half>(w) : to16<BFloat>(w));
        }
    }
}

__global__ __launch_bounds__(64) void adamw_count_kernel(int32_t *step, const int32_t *flag) {
    if (threadIdx.x == 0 && !(flag && *flag != 0)) *step += 1;
}

}  // namespace

AdamwTable adamw_table(void *buffer, int32_t tensors) {
    AdamwTable t;
    t.tensors = (nnconv_adamw_tensor *)buffer;
    t.chunks = (AdamwChunk *)((char *)buffer + (size_t)tensors * sizeof(nnconv_adamw_tensor));
    return t;
}

hipError_t launch_adamw_plan(const nnconv_adamw_tensor *tensors, int32_t n, const AdamwTable &tab,
                             hipStream_t st) {
    int64_t chunk = 0;
    for (int32_t first = 0; first < n; first += BATCH) {
        InitArgs a{};
        const int32_t count = n - first < BATCH ? n - first : BATCH;
        for (int32_t k = 0; k < count; ++k) {
            a.t[k] = tensors[first + k];
            a.chunk0[k] = chunk;
            chunk += (tensors[first + k].count + CHUNK - 1) / CHUNK;
        }
        hipLaunchKernelGGL(adamw_plan_kernel, dim3(count), dim3(256), 0, st, a, first, count, tab);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_adamw(const AdamwTable &tab, int64_t chunks, int32_t *step, float lr, float beta1,
                        float beta2, float eps, uint32_t seed, const nnconv_loss_scaler *state,
                        const int32_t *flag, hipStream_t st) {
    if (chunks > 0x7FFFFFFF) return hipErrorInvalidValue;
    if (chunks > 0)
        hipLaunchKernelGGL(adamw_kernel, dim3((uint32_t)chunks), dim3(256), 0, st, tab, step, lr,
                           beta1, beta2, eps, seed, state, flag);
    hipLaunchKernelGGL(adamw_count_kernel, dim3(1), dim3(64), 0, st, step, flag);
    return hipGetLastError();
}

}  // namespace nnconv
