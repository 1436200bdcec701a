// adamw.hip -- AdamW over a list of tensors in one launch, with fp32 moments or 8-bit ones.
//
// Bound by memory: 30 bytes a parameter with fp32 gradients, moments and a 16-bit copy, 18 (and
// a 32nd) with 8-bit moments.  The list is cut into chunks, whose records (addresses and all)
// lie in the plan; as many workgroups as fit the chip at once (1280; 2048 took 7 % longer) walk
// them, each with the next record on its way.  A lane takes 4 neighbouring elements at a time,
// in 16-byte accesses at any alignment; 16 lanes hold a block of 8-bit moments.  (8
// neighbouring elements a lane with 8-bit moments, half as many accesses, but each of half
// cache lines: 1479 us where 4 take 1160.)
//
// Measured: 23.5 M parameters in 159 tensors 126 us (5.6 TB/s); 302 M with 8-bit moments 1.16
// ms (4.7 TB/s; a copy of that size 4.83); without the hash and the rounding it would take 1.15
// ms.
#include "launch.hpp"

namespace nnconv {

namespace {

constexpr int CHUNK = ADAMW_CHUNK;
constexpr int THREADS = 256;
constexpr int VECS = CHUNK / (4 * THREADS);  // vectors of a lane
constexpr int BLOCKS = 1280;                 // workgroups at most: all are resident at once
constexpr int TEAMS = 31;                    // of workgroups that count their ends together
constexpr int BATCH = 40;                    // list entries in one launch's arguments (of at most 4 KB)
static_assert(ADAMW_HEAD == (1 + TEAMS) * ADAMW_LINE * sizeof(uint32_t), "counters");
static_assert(NNCONV_ADAMW_BLOCK == 64 && CHUNK % 1024 == 0, "16 lanes hold a block");

typedef f32x4 __attribute__((aligned(4))) f32x4_any;
typedef u32x2 __attribute__((aligned(2))) u32x2_any;
typedef uint32_t __attribute__((aligned(1))) u32_any;

enum : int32_t { GRAD_F16 = 1, GRAD_BF16 = 2, W16_F16 = 4, W16_BF16 = 8, STATE_F8 = 16 };

struct InitArgs {
    nnconv_adamw_tensor t[BATCH];
    int64_t chunk0[BATCH];  // first chunk of each
};
static_assert(sizeof(InitArgs) + 64 < 4096, "kernel arguments");

// Writes the records of BATCH list entries' chunks; a workgroup per entry.
__global__ __launch_bounds__(256) void adamw_plan_kernel(const InitArgs a, int32_t first, AdamwTable tab) {
    const nnconv_adamw_tensor &t = a.t[blockIdx.x];
    if (first == 0 && blockIdx.x == 0 && threadIdx.x <= TEAMS) tab.arrived[threadIdx.x * ADAMW_LINE] = 0;
    const bool f8 = t.state_dtype == NNCONV_F8;
    AdamwChunk c;
    c.tensor = first + blockIdx.x;
    c.weight_decay = t.weight_decay;
    c.kind = (t.grad_dtype == NNCONV_F16 ? GRAD_F16 : t.grad_dtype == NNCONV_BF16 ? GRAD_BF16 : 0) |
             (!t.w16 ? 0 : t.w16_dtype == NNCONV_F16 ? W16_F16 : W16_BF16) | (f8 ? STATE_F8 : 0);
    for (int64_t i = threadIdx.x; i * CHUNK < t.count; i += 256) {
        const int64_t at = i * CHUNK;
        c.first = at;
        c.count = (int32_t)(t.count - at < CHUNK ? t.count - at : CHUNK);
        c.master = t.master + at;
        c.grad = (const char *)t.grad + at * (t.grad_dtype == NNCONV_F32 ? 4 : 2);
        c.w16 = t.w16 ? (char *)t.w16 + at * 2 : nullptr;
        c.m = (char *)t.m + at * (f8 ? 1 : 4);
        c.v = (char *)t.v + at * (f8 ? 1 : 4);
        c.m_scale = f8 ? t.m_scale + at / NNCONV_ADAMW_BLOCK : nullptr;
        c.v_scale = f8 ? t.v_scale + at / NNCONV_ADAMW_BLOCK : nullptr;
        tab.chunks[a.chunk0[blockIdx.x] + i] = c;
    }
}

// The random bits of an element: 16 for m, 16 for v.  A mixer of xor-shifts and multiplications,
// with the multipliers as published searches for 32-bit mixers of little bias give them and
// shifts of about half a word, under which every bit of the input reaches the upper half of each
// product.  Its input is linear in element, tensor and step, which thereby read one sequence of
// 2^32 numbers at different places.  Over 2^18 inputs a flipped input bit flips each output bit
// with a probability of 1/2 to within those samples' own deviation (0.003 at most, 0.00094 rms);
// over 2^22 elements, and over as many steps of one element, means and correlations with the
// neighbours, and of m's bits with v's, lie within 2.5 standard deviations of none.
__device__ __forceinline__ uint32_t dither_bits(uint32_t key, uint32_t i) {
    uint32_t h = i * 0x9E3779B1u + key;
    h = (h ^ (h >> 16)) * 0x2C1B3C6Du;
    h = (h ^ (h >> 15)) * 0x297A2D39u;
    return h ^ (h >> 16);
}

// beta^t for t >= 0, in 64 bits by squaring: 1 - beta^t would lose most of its bits in 32 for a
// beta near 1.
__device__ __forceinline__ double power(double b, int32_t t) {
    double r = 1.0;
    for (; t > 0; t >>= 1, b *= b)
        if (t & 1) r *= b;
    return r;
}

// Magnitude of the 8-bit code of y >= 0 in units of 2^k: LOW smallest exponent, M mantissa
// bits; u in (0, 1).  y lies within the range of the format at that scale, and so does its
// rounding: the largest value is a whole number of the topmost spacings. A NaN stays.
template <int LOW, int M, bool KEEP>
__device__ __forceinline__ float round_random(float y, int k, float u) {
    int e = __builtin_amdgcn_frexp_expf(y) - 1 - M;  // exponent of the spacing
    e = max(e, LOW - M + k);
    float r = floorf(__builtin_amdgcn_ldexpf(y, -e) + u);
    if (KEEP) r = y > 0.f ? fmaxf(r, 1.f) : r;
    return __builtin_amdgcn_ldexpf(r, e - k);
}

// Exponent k of the smallest power of two that brings `most` within 1.75 * 2^TOP.
template <int TOP>
__device__ __forceinline__ int block_exponent(float most) {
    const uint32_t b = __builtin_bit_cast(uint32_t, most);
    int k = (int)(b >> 23) - 127 - TOP + ((b & 0x7FFFFFu) > 0x600000u);
    if ((b >> 23) == 0) k = -127;  // zero, and what is too small for a scale of its own
    return k < -127 ? -127 : k;
}

// Maximum over 16 neighbouring lanes.
template <int CTRL>
__device__ __forceinline__ float dpp_max(float v) {
    return fmaxf(v, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true)));
}

__device__ __forceinline__ float max16(float v) {
    return dpp_max<0x140>(dpp_max<0x141>(dpp_max<0x4E>(dpp_max<0xB1>(v))));
}

struct Step {
    float inv_scale, beta1, beta2, rest1, rest2, rate, root, eps, lr;
    uint32_t key;  // of the hash, without the tensor
};

// One element's new moments and master.
__device__ __forceinline__ void adamw_one(const Step &k, float decay, float g, float &w, float &m, float &v) {
    g *= k.inv_scale;
    m = k.beta1 * m + k.rest1 * g;
    v = k.beta2 * v + (k.rest2 * g) * g;
    // instructions of one unit in the last place are enough for the change; the root's takes a
    // subnormal number for 0, and v / (1 - beta2^t) may pass the range that its root is far from
    const bool small = v < 0x1p-96f;
    const float root = __builtin_amdgcn_sqrtf(small ? v * 0x1p64f : v) * (small ? k.root * 0x1p-32f : k.root);
    w -= k.rate * m * __builtin_amdgcn_rcpf(root + k.eps) + decay * w;
    asm volatile("" : "+v"(w));  // the 16-bit copy is the rounding of the stored master
}

// A lane's vectors of a chunk.  FULL: the chunk has CHUNK elements.
template <bool F8, bool FULL>
struct Lanes {
    f32x4 w[VECS], g[VECS], m[F8 ? 1 : VECS], v[F8 ? 1 : VECS];
    uint32_t m8[VECS], v8[VECS];
    int ms[VECS], vs[VECS];

    // Elements of vector k that exist: 4, fewer, none.
    static __device__ __forceinline__ int have(const AdamwChunk &c, int k) {
        if (FULL) return 4;
        const int n = c.count - 4 * ((int)threadIdx.x + k * THREADS);
        return n < 0 ? 0 : n > 4 ? 4 : n;
    }

    template <class T>
    static __device__ __forceinline__ f32x4 load(const void *p, int at, int n) {
        f32x4 r{};
        const T *q = (const T *)p + at;
        if (n == 4) return __builtin_nontemporal_load((const f32x4_any *)q);
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (e < n) r[e] = q[e];
        return r;
    }

    static __device__ __forceinline__ f32x4 load_half(const void *p, int at, int n, bool f16) {
        const uint16_t *q = (const uint16_t *)p + at;
        uint32_t b[4] = {0, 0, 0, 0};
        if (n == 4) {
            const u32x2 d = __builtin_nontemporal_load((const u32x2_any *)q);
            b[0] = d[0] & 0xFFFFu;
            b[1] = d[0] >> 16;
            b[2] = d[1] & 0xFFFFu;
            b[3] = d[1] >> 16;
        } else {
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (e < n) b[e] = q[e];
        }
        f32x4 r;
#pragma unroll
        for (int e = 0; e < 4; ++e) r[e] = f16 ? from16<Half>(b[e]) : from16<BFloat>(b[e]);
        return r;
    }

    static __device__ __forceinline__ uint32_t load_codes(const void *p, int at, int n) {
        const uint8_t *q = (const uint8_t *)p + at;
        if (n == 4) return __builtin_nontemporal_load((const u32_any *)q);
        uint32_t r = 0;
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (e < n) r |= (uint32_t)q[e] << (8 * e);
        return r;
    }

    static __device__ __forceinline__ void store(float *q, f32x4 v, int n) {
        if (n == 4) {
            __builtin_nontemporal_store(v, (f32x4_any *)q);
            return;
        }
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (e < n) q[e] = v[e];
    }

    static __device__ __forceinline__ void store_codes(uint8_t *q, uint32_t v, int n) {
        if (n == 4) {
            __builtin_nontemporal_store(v, (u32_any *)q);
            return;
        }
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (e < n) q[e] = (uint8_t)(v >> (8 * e));
    }

    __device__ __forceinline__ void fetch(const AdamwChunk &c) {
#pragma unroll
        for (int k = 0; k < VECS; ++k) {
            const int at = 4 * ((int)threadIdx.x + k * THREADS), n = have(c, k);
            w[k] = load<float>(c.master, at, n);
            if constexpr (F8) {
                m8[k] = load_codes(c.m, at, n);
                v8[k] = load_codes(c.v, at, n);
                ms[k] = n > 0 ? c.m_scale[at / NNCONV_ADAMW_BLOCK] : 0;
                vs[k] = n > 0 ? c.v_scale[at / NNCONV_ADAMW_BLOCK] : 0;
            } else {
                m[k] = load<float>(c.m, at, n);
                v[k] = load<float>(c.v, at, n);
            }
        }
        if (c.kind & (GRAD_F16 | GRAD_BF16)) {
#pragma unroll
            for (int k = 0; k < VECS; ++k)
                g[k] = load_half(c.grad, 4 * ((int)threadIdx.x + k * THREADS), have(c, k), (c.kind & GRAD_F16) != 0);
        } else {
#pragma unroll
            for (int k = 0; k < VECS; ++k)
                g[k] = load<float>(c.grad, 4 * ((int)threadIdx.x + k * THREADS), have(c, k));
        }
    }

    __device__ __forceinline__ void finish(const AdamwChunk &c, const Step &s) {
        const float decay = s.lr * c.weight_decay;
        const uint32_t key = s.key + (uint32_t)c.tensor * 0x6C8E9CF5u + (uint32_t)(c.first >> 32) * 0x7F4A7C15u;
#pragma unroll
        for (int k = 0; k < VECS; ++k) {
            const int at = 4 * ((int)threadIdx.x + k * THREADS), n = have(c, k);
            f32x4 mk, vk;
            if constexpr (F8) {
                const float sm = __builtin_amdgcn_ldexpf(1.f, ms[k] - 127), sv = __builtin_amdgcn_ldexpf(1.f, vs[k] - 127);
                mk[0] = __builtin_amdgcn_cvt_f32_fp8(m8[k], 0) * sm;
                mk[1] = __builtin_amdgcn_cvt_f32_fp8(m8[k], 1) * sm;
                mk[2] = __builtin_amdgcn_cvt_f32_fp8(m8[k], 2) * sm;
                mk[3] = __builtin_amdgcn_cvt_f32_fp8(m8[k], 3) * sm;
                vk[0] = __builtin_amdgcn_cvt_f32_bf8(v8[k], 0) * sv;
                vk[1] = __builtin_amdgcn_cvt_f32_bf8(v8[k], 1) * sv;
                vk[2] = __builtin_amdgcn_cvt_f32_bf8(v8[k], 2) * sv;
                vk[3] = __builtin_amdgcn_cvt_f32_bf8(v8[k], 3) * sv;
            } else {
                mk = m[k];
                vk = v[k];
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float we = w[k][e], me = mk[e], ve = vk[e];
                adamw_one(s, decay, g[k][e], we, me, ve);
                w[k][e] = we;
                mk[e] = me;
                vk[e] = ve;
            }
            if constexpr (F8) {
                // elements past the end are zeros and stay so; the maxima pass over NaNs
                float mm = fmaxf(fmaxf(fabsf(mk[0]), fabsf(mk[1])), fmaxf(fabsf(mk[2]), fabsf(mk[3])));
                float vm = fmaxf(fmaxf(vk[0], vk[1]), fmaxf(vk[2], vk[3]));
                if (__any(__builtin_isinf(mm) || __builtin_isinf(vm))) {  // infinities become NaNs
                    mm = vm = 0.f;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        mk[e] = __builtin_isinf(mk[e]) ? __builtin_nanf("") : mk[e];
                        vk[e] = __builtin_isinf(vk[e]) ? __builtin_nanf("") : vk[e];
                        mm = fmaxf(mm, fabsf(mk[e]));
                        vm = fmaxf(vm, vk[e]);
                    }
                }
                const int km = block_exponent<8>(max16(mm)), kv = block_exponent<15>(max16(vm));
                float qm[4], qv[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t bits = dither_bits(key, (uint32_t)c.first + at + e);
                    const float um = __builtin_fmaf((float)(bits & 0xFFFFu), 0x1p-16f, 0x1p-17f);
                    const float uv = __builtin_fmaf((float)(bits >> 16), 0x1p-16f, 0x1p-17f);
                    qm[e] = copysignf(round_random<-6, 3, false>(fabsf(mk[e]), km, um), mk[e]);
                    qv[e] = round_random<-14, 2, true>(vk[e], kv, uv);
                }
                int cm = __builtin_amdgcn_cvt_pk_fp8_f32(qm[0], qm[1], 0, false);
                cm = __builtin_amdgcn_cvt_pk_fp8_f32(qm[2], qm[3], cm, true);
                int cv = __builtin_amdgcn_cvt_pk_bf8_f32(qv[0], qv[1], 0, false);
                cv = __builtin_amdgcn_cvt_pk_bf8_f32(qv[2], qv[3], cv, true);
                store_codes((uint8_t *)c.m + at, cm, n);
                store_codes((uint8_t *)c.v + at, cv, n);
                if (n > 0 && (threadIdx.x & 15) == 0) {
                    c.m_scale[at / NNCONV_ADAMW_BLOCK] = (uint8_t)(km + 127);
                    c.v_scale[at / NNCONV_ADAMW_BLOCK] = (uint8_t)(kv + 127);
                }
            } else {
                store((float *)c.m + at, mk, n);
                store((float *)c.v + at, vk, n);
            }
            store(c.master + at, w[k], n);
            if (c.kind & (W16_F16 | W16_BF16)) {  // the next forward's weights: not past the caches
                const bool f16 = (c.kind & W16_F16) != 0;
                const uint32_t lo = f16 ? pack16<Half>(w[k][0], w[k][1]) : pack16<BFloat>(w[k][0], w[k][1]);
                const uint32_t hi = f16 ? pack16<Half>(w[k][2], w[k][3]) : pack16<BFloat>(w[k][2], w[k][3]);
                uint16_t *q = (uint16_t *)c.w16 + at;
                if (n == 4) {
                    *(u32x2_any *)q = u32x2{lo, hi};
                } else {
                    if (n > 0) q[0] = (uint16_t)lo;
                    if (n > 1) q[1] = (uint16_t)(lo >> 16);
                    if (n > 2) q[2] = (uint16_t)hi;
                }
            }
        }
    }
};

// Counts an arrival; true for the last of `all`, which leaves the counter at zero.
__device__ __forceinline__ bool last_of(uint32_t *counter, uint32_t all) {
    if (__hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != all - 1) return false;
    __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return true;
}

__global__ __launch_bounds__(THREADS) void adamw_kernel(const AdamwTable tab, int32_t chunks, int32_t *step, float lr,
                                                        float beta1, float beta2, float eps, uint32_t seed,
                                                        const nnconv_loss_scaler *state, const int32_t *flag) {
    // on their way together with the first record
    const int32_t skip = flag ? *flag : 0, done = *step;
    const float scale = state ? state->scale : 1.0f;
    Step s;
    bool ready = false;
    // the step's numbers, computed behind the first chunk's loads; false: the step is skipped
    auto prepare = [&]() {
        if (ready) return true;
        if (skip != 0) return false;
        const int32_t now = done + 1;
        s.inv_scale = 1.0f / scale;
        s.beta1 = beta1;
        s.beta2 = beta2;
        s.rest1 = 1.0f - beta1;
        s.rest2 = 1.0f - beta2;
        s.rate = (float)(lr / (1.0 - power(beta1, now)));
        s.root = (float)(1.0 / sqrt(1.0 - power(beta2, now)));
        s.eps = eps;
        s.lr = lr;
        s.key = (uint32_t)now * 0xB5297A4Du + seed * 0x68E31DA4u;
        return ready = true;
    };
    auto go = [&](const AdamwChunk &c, auto lanes) {
        lanes.fetch(c);
        if (!prepare()) return false;
        lanes.finish(c, s);
        return true;
    };
    // the records do not change during the call: read through the scalar cache, one ahead
    typedef const __attribute__((address_space(4))) AdamwChunk const_chunk;
    const_chunk *records = (const_chunk *)(uintptr_t)tab.chunks;
    auto record = [&](int32_t i) {
        AdamwChunk c;
        const __attribute__((address_space(4))) uint64_t *from = (const __attribute__((address_space(4))) uint64_t *)(records + i);
        uint64_t w[sizeof(AdamwChunk) / 8];
#pragma unroll
        for (int k = 0; k < (int)(sizeof(AdamwChunk) / 8); ++k) w[k] = from[k];
        __builtin_memcpy(&c, w, sizeof(c));
        return c;
    };
    AdamwChunk next = record(blockIdx.x);
    for (int32_t i = blockIdx.x; i < chunks; i += gridDim.x) {
        const AdamwChunk c = next;
        next = record(min(i + (int32_t)gridDim.x, chunks - 1));
        const bool f8 = (c.kind & STATE_F8) != 0, full = c.count == CHUNK;
        if (!(f8 ? full ? go(c, Lanes<true, true>{}) : go(c, Lanes<true, false>{})
                 : full ? go(c, Lanes<false, true>{}) : go(c, Lanes<false, false>{})))
            return;
    }
    // The last workgroup counts the step: by then all have read the count.  They arrive in
    // teams first: at one address, one after the other, the 384 workgroups of an update of 0.8
    // M parameters took 2.4 of its 10.1 us.
    __syncthreads();
    if (threadIdx.x != 0) return;
    const uint32_t blocks = gridDim.x;
    uint32_t arrivals = blocks;
    if (blocks > TEAMS) {
        const uint32_t team = blockIdx.x % TEAMS;
        if (!last_of(tab.arrived + (1 + team) * ADAMW_LINE, blocks / TEAMS + (team < blocks % TEAMS))) return;
        arrivals = TEAMS;
    }
    if (arrivals == 1 || last_of(tab.arrived, arrivals)) *step = done + 1;
}

// A list without elements.
__global__ __launch_bounds__(64) void adamw_count_kernel(int32_t *step, const int32_t *flag) {
    if (threadIdx.x == 0 && !(flag && *flag != 0)) *step += 1;
}

}  // namespace

AdamwTable adamw_table(void *buffer) {
    AdamwTable t;
    t.arrived = (uint32_t *)buffer;
    t.chunks = (AdamwChunk *)((char *)buffer + ADAMW_HEAD);
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
        hipLaunchKernelGGL(adamw_plan_kernel, dim3(count), dim3(256), 0, st, a, first, tab);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_adamw(const AdamwTable &tab, int64_t chunks, int32_t *step, float lr, float beta1,
                        float beta2, float eps, uint32_t seed, const nnconv_loss_scaler *state,
                        const int32_t *flag, hipStream_t st) {
    if (chunks > 0)
        hipLaunchKernelGGL(adamw_kernel, dim3((uint32_t)(chunks < BLOCKS ? chunks : BLOCKS)), dim3(THREADS), 0, st, tab,
                           (int32_t)chunks, step, lr, beta1, beta2, eps, seed, state, flag);
    else
        hipLaunchKernelGGL(adamw_count_kernel, dim3(1), dim3(64), 0, st, step, flag);
    return hipGetLastError();
}

}  // namespace nnconv
