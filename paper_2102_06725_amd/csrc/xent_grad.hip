// xent_grad.hip -- the two gradient products of the vocabulary loss, dx = d w and dw = d^T x, with
// d = 2^15 (softmax - q) [rows][v]: w and x are read along their rows, and for dw d is too.
//
// Few tiles split the reduction; the partial sums are added in a fixed order.
#include "xent.hpp"

namespace nnconv {

namespace xent {

__device__ __forceinline__ float read16or32(const void *p, int kind, int64_t i) {
    if (kind == 2) return ((const float *)p)[i];
    const uint32_t b = ((const uint16_t *)p)[i];
    return kind == Half::id ? from16<Half>(b) : from16<BFloat>(b);
}

// One value of the product to where it goes.
__device__ __forceinline__ void put(const GradOut &o, float factor, int64_t i, float v) {
    if (o.prev) v += o.prev[i];
    if (o.keep) {
        o.keep[i] = v;
        return;
    }
    v *= factor;
    if (o.accumulate) v += read16or32(o.out, o.kind, i);
    if (o.kind == 2) {
        ((float *)o.out)[i] = v;
        if (o.flag && !__builtin_isfinite(v)) *o.flag = 1;
        return;
    }
    const uint16_t b = (uint16_t)(o.kind == Half::id ? to16<Half>(v) : to16<BFloat>(v));
    ((uint16_t *)o.out)[i] = b;
    if (o.flag && !__builtin_isfinite(o.kind == Half::id ? from16<Half>(b) : from16<BFloat>(b))) *o.flag = 1;
}

__device__ __forceinline__ float factor_of(const GradOut &o) { return o.scale ? o.alpha * *o.scale : o.alpha; }

template <class T, int BM, int BN, int WM, int WN, int BK, int STAGES, int OCC, bool ATR>
__global__ __launch_bounds__(WM * WN * 64, OCC) void grad_kernel(const Grad P) {
    typedef gemm::Tile<T, BM, BN, WM, WN, BK, STAGES, ATR, true> G;
    constexpr int FM = G::FM, FN = G::FN;
    constexpr int LDS = G::LDS_BYTES < BM * BN * 2 ? BM * BN * 2 : G::LDS_BYTES;
    __shared__ __attribute__((aligned(16))) char lds[LDS];

    const int per = P.tiles_m * P.tiles_n;
    const int id = (int)xcd_remap(blockIdx.x, gridDim.x);
    const int split = id / per;
    int tm, tn;
    tile_of(id - split * per, P.tiles_m, P.tiles_n, tm, tn);
    const int64_t m0 = (int64_t)tm * BM, n0 = (int64_t)tn * BN;
    const int64_t k0 = split * P.k_split, k1 = k0 + P.k_split < P.k ? k0 + P.k_split : P.k;
    G g;
    g.run(P.a, P.b, m0, n0, k0, k1, lds);

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave % WM, wn = wave / WM;
    const int l32 = lane & 31, half = lane >> 5;
    const GradOut &o = P.o;
    const float factor = factor_of(o);
    // whole lines of a 16-bit output go through LDS
    const bool lines = P.splits == 1 && o.kind != 2 && !o.accumulate && !o.prev && !o.keep && o.n % 8 == 0 &&
                       ((uintptr_t)o.out & 15) == 0;
    if (!lines) {
        float *part = P.splits > 1 ? P.part + (int64_t)split * o.m * o.n : nullptr;
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            const int64_t m = m0 + wm * G::WTM + i * 32 + l32;
            if (m >= o.m) continue;
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int u = 0; u < 16; ++u) {
                    const int64_t n = n0 + wn * G::WTN + j * 32 + 8 * (u >> 2) + 4 * half + (u & 3);
                    if (n >= o.n) continue;
                    if (part)
                        part[m * o.n + n] = g.acc[j][i][u];
                    else
                        put(o, factor, m * o.n + n, g.acc[j][i][u]);
                }
        }
        return;
    }
    barrier_lds();  // no wave reads operands any more
    constexpr int CPR = G::WTN / 8, ROWB = G::WTN * 2;
    char *own = lds + wave * (G::WTM * ROWB);
#pragma unroll
    for (int i = 0; i < FM; ++i) {
        const int r = i * 32 + l32;
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const f32x16 &a = g.acc[j][i];
                const u32x2 pk = {pack16<T>(a[4 * q] * factor, a[4 * q + 1] * factor),
                                  pack16<T>(a[4 * q + 2] * factor, a[4 * q + 3] * factor)};
                *(u32x2 *)(own + r * ROWB + (((j * 4 + q) ^ (r & (CPR - 1))) * 16) + half * 8) = pk;
            }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const int c = lane % CPR;
    const int64_t n = n0 + wn * G::WTN + c * 8;
    bool bad = false;
    constexpr uint32_t TOP = T::id == Half::id ? 0x7C00u : 0x7F80u;
#pragma unroll 4
    for (int r = lane / CPR; r < G::WTM; r += 64 / CPR) {
        const int64_t m = m0 + wm * G::WTM + r;
        const u32x4 v = *(const u32x4 *)(own + r * ROWB + (c ^ (r & (CPR - 1))) * 16);
        if (m >= o.m || n >= o.n) continue;
#pragma unroll
        for (int d = 0; d < 4; ++d)
            bad |= (v[d] & TOP) == TOP || ((v[d] >> 16) & TOP) == TOP;
        __builtin_nontemporal_store(v, (u32x4 *)((uint16_t *)o.out + m * o.n + n));
    }
    if (o.flag && bad) *o.flag = 1;
}

// Sums of the splits, in order.
__global__ __launch_bounds__(256) void grad_join_kernel(const float *part, int32_t splits, GradOut o) {
    const int64_t count = o.m * o.n;
    const float factor = factor_of(o);
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < count; i += (int64_t)gridDim.x * 256) {
        float v = part[i];
        for (int s = 1; s < splits; ++s) v += part[s * count + i];
        put(o, factor, i, v);
    }
}

template <class T, int BM, int BN, int WM, int WN, int BK, int STAGES, int OCC>
static hipError_t launch(bool atr, Grad p, hipStream_t st) {
    p.tiles_m = (int32_t)((p.o.m + BM - 1) / BM);
    p.tiles_n = (p.o.n + BN - 1) / BN;
    const int64_t nb = (int64_t)p.tiles_m * p.tiles_n * p.splits;
    if (nb <= 0) return hipSuccess;
    if (nb > 0x3FFFFFFF) return hipErrorInvalidValue;
    if (atr)
        hipLaunchKernelGGL((grad_kernel<T, BM, BN, WM, WN, BK, STAGES, OCC, true>), dim3((uint32_t)nb),
                           dim3(WM * WN * 64), 0, st, p);
    else
        hipLaunchKernelGGL((grad_kernel<T, BM, BN, WM, WN, BK, STAGES, OCC, false>), dim3((uint32_t)nb),
                           dim3(WM * WN * 64), 0, st, p);
    if (p.splits > 1) {
        const int64_t blocks = (p.o.m * p.o.n + 255) / 256;
        hipLaunchKernelGGL(grad_join_kernel, dim3((uint32_t)(blocks < 65536 ? blocks : 65536)), dim3(256), 0, st, p.part,
                           p.splits, p.o);
    }
    return hipGetLastError();
}

template <class T>
static hipError_t launch_t(Config cfg, bool atr, const Grad &p, hipStream_t st) {
    if (cfg == TILE_256) return launch<T, 256, 256, 2, 4, 64, 2, 2>(atr, p, st);
    return launch<T, 128, 128, 2, 2, 64, 2, 2>(atr, p, st);
}

hipError_t launch_grad(int dtype, Config cfg, bool atr, Grad p, hipStream_t st) {
    return dtype == Half::id ? launch_t<Half>(cfg, atr, p, st) : launch_t<BFloat>(cfg, atr, p, st);
}

}  // namespace xent

}  // namespace nnconv
