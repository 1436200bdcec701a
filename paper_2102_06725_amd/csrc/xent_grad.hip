// xent_grad.hip -- the two gradient products of the vocabulary loss, dx = d w and dw = d^T x, with
// d = 2^15 (softmax - q) [rows][v]: w and x are read along their rows, and for dw d is too.
//
// Few tiles split the reduction; the partial sums are added in a fixed order.  The two products are
// independent of each other and run in one launch where both take tiles of one kind, the longer
// reductions first: small ones fill the chip together (512 x 512 x 8192: 17 us for both, 14 and 10 one
// after the other).  Bound by the matrix units: 8192 x 2048 x 65536, both products, 3.41 ms, 1.29 PFLOP/s.
#include "xent.hpp"

namespace nnconv {

namespace xent {

typedef f32x4 __attribute__((aligned(4))) f32x4_any;
typedef u32x2 __attribute__((aligned(2))) u32x2_any;

// Columns n on of row m, 4 or those that are left, to where they go.
__device__ __forceinline__ void put4(const GradOut &o, float factor, int64_t m, int64_t n, f32x4 v) {
    const int64_t i = m * o.n + n;
    const int left = o.n - n < 4 ? (int)(o.n - n) : 4;
    const bool half = o.kind == Half::id;
    if (o.prev) {
        if (left == 4)
            v += *(const f32x4_any *)(o.prev + i);
        else
#pragma unroll
            for (int d = 0; d < 3; ++d)
                if (d < left) v[d] += o.prev[i + d];
    }
    if (o.keep) {
        if (left == 4)
            *(f32x4_any *)(o.keep + i) = v;
        else
#pragma unroll
            for (int d = 0; d < 3; ++d)
                if (d < left) o.keep[i + d] = v[d];
        return;
    }
    v *= factor;
    if (o.by_rows && !__builtin_isfinite(v[0] + v[1] + v[2] + v[3]) && !o.counts.of(m)) v = f32x4{};
    bool bad = false;
    if (o.kind == 2) {
        float *to = (float *)o.out + i;
        if (left == 4) {
            if (o.accumulate) v += *(const f32x4_any *)to;
            *(f32x4_any *)to = v;
        }
#pragma unroll
        for (int d = 0; d < 4; ++d) {
            if (d >= left) continue;
            if (left < 4) {
                if (o.accumulate) v[d] += to[d];
                to[d] = v[d];
            }
            bad |= !__builtin_isfinite(v[d]);
        }
    } else {
        uint16_t *to = (uint16_t *)o.out + i;
        u32x2 b = {};
        if (o.accumulate) {
            if (left == 4)
                b = *(const u32x2_any *)to;
            else
#pragma unroll
                for (int d = 0; d < 3; ++d)
                    if (d < left) b[d >> 1] |= (uint32_t)to[d] << (16 * (d & 1));
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                const uint32_t w = b[d >> 1] >> (16 * (d & 1));
                v[d] += half ? from16<Half>(w) : from16<BFloat>(w);
            }
        }
        b[0] = half ? pack16<Half>(v[0], v[1]) : pack16<BFloat>(v[0], v[1]);
        b[1] = half ? pack16<Half>(v[2], v[3]) : pack16<BFloat>(v[2], v[3]);
        if (left == 4) *(u32x2_any *)to = b;
        const uint32_t top = half ? 0x7C00u : 0x7F80u;
#pragma unroll
        for (int d = 0; d < 4; ++d) {
            const uint32_t w = b[d >> 1] >> (16 * (d & 1));
            if (d >= left) continue;
            if (left < 4) to[d] = (uint16_t)w;
            bad |= (w & top) == top;
        }
    }
    if (bad && o.flag) *o.flag = 1;
}

__device__ __forceinline__ float factor_of(const GradOut &o) { return o.scale ? o.alpha * *o.scale : o.alpha; }

// Workgroup `block` of a product.  ATR: a is read along its rows (the reduction's elements are
// p[k * ld + m]).
template <class T, int BM, int BN, int WM, int WN, int BK, int STAGES, bool ATR>
__device__ __forceinline__ void grad_tile(const Grad &P, uint32_t block, char *lds) {
    typedef gemm::Tile<T, BM, BN, WM, WN, BK, STAGES, ATR, true> G;
    constexpr int FM = G::FM, FN = G::FN;
    const int per = P.tiles_m * P.tiles_n;
    const int id = (int)xcd_remap(block, (uint32_t)(per * P.splits));
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
    barrier_lds();  // no wave reads operands any more
    if (!lines) {
        // 32 rows at a time through the wave's own part of LDS, so that a row's columns are stored
        // side by side (16 partial sums of 512 x 512 after 512
        // products each: 14 us, 21 stored from the registers)
        constexpr int ROWB = G::WTN * 4, CPR = G::WTN / 4;
        char *own = lds + wave * (32 * ROWB);
        float *part = P.splits > 1 ? P.part + (int64_t)split * o.m * o.n : nullptr;
        const GradOut raw = {nullptr, 2, o.n, o.m, 1.f, nullptr, 0, nullptr, nullptr, part, false, {}};
#pragma unroll
        for (int i = 0; i < FM; ++i) {
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const f32x16 &a = g.acc[j][i];
                    const int c = j * 8 + 2 * q + half;
                    *(f32x4 *)(own + l32 * ROWB + ((c ^ (l32 & (CPR - 1))) * 16)) = f32x4{a[4 * q], a[4 * q + 1], a[4 * q + 2], a[4 * q + 3]};
                }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            const int c = lane % CPR;
            const int64_t n = n0 + wn * G::WTN + c * 4;
            for (int r = lane / CPR; r < 32; r += 64 / CPR) {
                const int64_t m = m0 + wm * G::WTM + i * 32 + r;
                const f32x4 v = *(const f32x4 *)(own + r * ROWB + ((c ^ (r & (CPR - 1))) * 16));
                if (m < o.m && n < o.n) put4(part ? raw : o, factor, m, n, v);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
        return;
    }
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
        u32x4 v = *(const u32x4 *)(own + r * ROWB + (c ^ (r & (CPR - 1))) * 16);
        if (m >= o.m || n >= o.n) continue;
        bool here = false;
#pragma unroll
        for (int d = 0; d < 4; ++d)
            here |= (v[d] & TOP) == TOP || ((v[d] >> 16) & TOP) == TOP;
        if (here && o.by_rows && !o.counts.of(m)) {
            v = u32x4{};
            here = false;
        }
        bad |= here;
        __builtin_nontemporal_store(v, (u32x4 *)((uint16_t *)o.out + m * o.n + n));
    }
    if (o.flag && bad) *o.flag = 1;
}

// The two products, the first `blocks` workgroups one's: FIRST says which.
template <class T, int BM, int BN, int WM, int WN, int BK, int STAGES, int OCC>
__global__ __launch_bounds__(WM * WN * 64, OCC) void grads_kernel(const Grad dx, const Grad dw, int32_t blocks, bool dw_first) {
    typedef gemm::Tile<T, BM, BN, WM, WN, BK, STAGES, true, true> G;
    constexpr int LDS = G::LDS_BYTES < BM * BN * 2 ? BM * BN * 2 : G::LDS_BYTES;
    __shared__ __attribute__((aligned(16))) char lds[LDS];
    const bool first = (int)blockIdx.x < blocks;
    const uint32_t block = first ? blockIdx.x : blockIdx.x - blocks;
    if (first == dw_first)
        grad_tile<T, BM, BN, WM, WN, BK, STAGES, true>(dw, block, lds);
    else
        grad_tile<T, BM, BN, WM, WN, BK, STAGES, false>(dx, block, lds);
}

// Sums of the splits, in order, a thread 4 columns.
__device__ __forceinline__ void join(const Grad &P, int64_t first, int64_t step) {
    const GradOut &o = P.o;
    const uint32_t per = ((uint32_t)o.n + 3) / 4;
    const int64_t count = o.m * per, size = o.m * o.n;
    const float factor = factor_of(o);
    for (int64_t i = first; i < count; i += step) {
        const int64_t m = i / per;
        const int n = (int)(i - m * per) * 4;
        const float *p = P.part + m * o.n + n;
        f32x4 v = {};
        if (n + 4 <= o.n) {
            v = *(const f32x4_any *)p;
#pragma unroll 4
            for (int s = 1; s < P.splits; ++s) v += *(const f32x4_any *)(p + s * size);
        } else
#pragma unroll
            for (int d = 0; d < 3; ++d)
                if (n + d < o.n)
                    for (int s = 0; s < P.splits; ++s) v[d] += p[s * size + d];
        put4(o, factor, m, n, v);
    }
}

__global__ __launch_bounds__(256) void grads_join_kernel(const Grad a, const Grad b, int32_t blocks) {
    if ((int)blockIdx.x < blocks)
        join(a, (int64_t)blockIdx.x * 256 + threadIdx.x, (int64_t)blocks * 256);
    else
        join(b, (int64_t)(blockIdx.x - blocks) * 256 + threadIdx.x, (int64_t)(gridDim.x - blocks) * 256);
}

static int32_t join_blocks(const Grad &p) {
    if (p.splits <= 1) return 0;
    const int64_t blocks = (p.o.m * ((p.o.n + 3) / 4) + 255) / 256;
    return (int32_t)(blocks < 65536 ? blocks : 65536);
}

// Either may be null.
template <class T, int BM, int BN, int WM, int WN, int BK, int STAGES, int OCC>
static hipError_t launch(const Grad *dx, const Grad *dw, hipStream_t st) {
    Grad x = {}, w = {};
    int64_t nx = 0, nw = 0;
    auto tiles = [](Grad &p) {
        p.tiles_m = (int32_t)((p.o.m + BM - 1) / BM);
        p.tiles_n = (p.o.n + BN - 1) / BN;
        return (int64_t)p.tiles_m * p.tiles_n * p.splits;
    };
    if (dx) {
        x = *dx;
        nx = tiles(x);
    }
    if (dw) {
        w = *dw;
        nw = tiles(w);
    }
    if (nx + nw <= 0) return hipSuccess;
    // a workgroup has up to 512 threads, a launch 2^32
    if (nx + nw > 0x7FFFFF) return hipErrorInvalidValue;
    // the longer reductions first
    const bool dw_first = nx == 0 || (nw > 0 && w.k_split > x.k_split);
    hipLaunchKernelGGL((grads_kernel<T, BM, BN, WM, WN, BK, STAGES, OCC>), dim3((uint32_t)(nx + nw)), dim3(WM * WN * 64), 0, st,
                       x, w, (int32_t)(dw_first ? nw : nx), dw_first);
    const int32_t jx = nx > 0 ? join_blocks(x) : 0, jw = nw > 0 ? join_blocks(w) : 0;
    if (jx + jw > 0)
        hipLaunchKernelGGL(grads_join_kernel, dim3((uint32_t)(jx + jw)), dim3(256), 0, st, x, w, jx);
    return hipGetLastError();
}

template <class T>
static hipError_t launch_t(Config cfg, const Grad *dx, const Grad *dw, hipStream_t st) {
    if (cfg == TILE_256) return launch<T, 256, 256, 2, 4, 64, 2, 2>(dx, dw, st);
    return launch<T, 128, 128, 2, 4, 64, 2, 4>(dx, dw, st);
}

static hipError_t launch_pair(int dtype, Config cfg, const Grad *dx, const Grad *dw, hipStream_t st) {
    return dtype == Half::id ? launch_t<Half>(cfg, dx, dw, st) : launch_t<BFloat>(cfg, dx, dw, st);
}

hipError_t launch_grads(int dtype, Config cfg, const Grad &dx, Config cfg_w, const Grad *dw, hipStream_t st) {
    if (!dw || cfg == cfg_w) return launch_pair(dtype, cfg, &dx, dw, st);
    const hipError_t e = launch_pair(dtype, cfg, &dx, nullptr, st);
    return e == hipSuccess ? launch_pair(dtype, cfg_w, nullptr, dw, st) : e;
}

hipError_t launch_grad_w(int dtype, Config cfg, const Grad &dw, hipStream_t st) {
    return launch_pair(dtype, cfg, nullptr, &dw, st);
}

}  // namespace xent

}  // namespace nnconv
