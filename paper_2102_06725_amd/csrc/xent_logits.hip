// xent_logits.hip -- logits of a vocabulary by tiles, with the softmax's statistics.
//
// A tile's logits stay in registers: of each row the largest (in the lane's 16 values of each
// block, then its other half's, then the other waves' through LDS) and the sum of the exponentials
// against it go to memory, and in training the exponentials themselves, at most 1, in 16 bits.
// The largest product is taken off before a product is scaled (to units of log 2, as the exponential
// instruction takes them): the largest token's exponential is 1, whatever its logit (taken off after the
// scaling, in one fused step, it would be 2 to the power of that logit's rounding, which passes any
// format from 2^24 on).  Statistics are products, and the label's product is one of the same: a row
// that is sure of its label has loss 0.
//
// What bounds it: the matrix units, and behind each tile about 10 vector instructions a logit, the
// exponential a half of their time, that no other tile of the compute unit covers (256 x 256 tiles
// fill it): 8192 x 65536 logits of 2048 channels with their exponentials in 2.0 ms, 1.10 PFLOP/s, against
// 1.68 for the product dx of the same size.  Smaller tiles, two a compute unit, cover it and lose
// more in the product (6.25 to 6.4 ms a step against 5.84).  Up to 32 rows it is bound by the read of w:
// 16 rows of 2048 channels against 65536 tokens 60 us, 4.5 TB/s, whatever the slices (32 or 64 rows of w a
// wave, 64 or 128 elements, 2 to 6 of them: 60 to 65).
#include "xent.hpp"

namespace nnconv {

namespace xent {

template <class T, int BM, int BN, int WM, int WN, int BK, int STAGES, int OCC, bool KEEP>
__global__ __launch_bounds__(WM * WN * 64, OCC) void logits_kernel(const Logits P) {
    typedef gemm::Tile<T, BM, BN, WM, WN, BK, STAGES, false, false> G;
    constexpr int FM = G::FM, FN = G::FN;
    constexpr int LDS = KEEP && G::LDS_BYTES < BM * BN * 2 ? BM * BN * 2 : G::LDS_BYTES;
    __shared__ __attribute__((aligned(16))) char lds[LDS];
    __shared__ float red[2][WN][BM];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave % WM, wn = wave / WM;
    const int l32 = lane & 31, half = lane >> 5;
    int tm, tn;
    tile_of((int)xcd_remap(blockIdx.x, gridDim.x), P.tiles_m, P.tiles_n, tm, tn);
    const int64_t m0 = (int64_t)tm * BM, n0 = (int64_t)tn * BN;
    const int c0 = wn * G::WTN + 4 * half;  // the lane's first column
    // where the label's logit is among the lane's, if it is
    int label[FM];
#pragma unroll
    for (int i = 0; i < FM; ++i) {
        const int64_t m = m0 + wm * G::WTM + i * 32 + l32;
        label[i] = P.labels && m < P.x.extent ? P.labels[m] : -1;
    }
    G g;
    g.run(P.x, P.w, m0, n0, 0, P.k, lds);

    const int cols = P.w.extent - n0 < BN ? (int)(P.w.extent - n0) : BN;  // of the tile
    if (P.unit < 0.f) {
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int u = 0; u < 16; ++u) g.acc[j][i][u] = -g.acc[j][i][u];
    }
    if (cols < BN) {
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int u = 0; u < 16; ++u)
                if (c0 + j * 32 + 8 * (u >> 2) + (u & 3) >= cols) {
#pragma unroll
                    for (int i = 0; i < FM; ++i) g.acc[j][i][u] = -INFINITY;
                }
    }
    const float unit = fabsf(P.unit);
#pragma unroll
    for (int i = 0; i < FM; ++i) {
        float v = -INFINITY;
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int u = 0; u < 16; ++u) v = fmaxf(v, g.acc[j][i][u]);
        v = fmaxf(v, __shfl_xor(v, 32));
        const int r = wm * G::WTM + i * 32 + l32;
        if (half == 0) red[0][wn][r] = v;
        const int64_t at = label[i] - n0 - c0;
        if (!__any(label[i] >= 0 && at >= 0 && at < G::WTN)) continue;
        bool mine = false;
        float z = 0.f;
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int u = 0; u < 16; ++u)
                if (at == j * 32 + 8 * (u >> 2) + (u & 3)) {
                    mine = true;
                    z = g.acc[j][i][u];
                }
        // another padding than -1 may lie in the tile's empty columns
        if (mine && label[i] < P.w.extent && m0 + r < P.x.extent) P.zt[m0 + r] = z;
    }
    barrier_lds();
#pragma unroll
    for (int i = 0; i < FM; ++i) {
        const int r = wm * G::WTM + i * 32 + l32;
        float v = red[0][0][r];
#pragma unroll
        for (int w = 1; w < WN; ++w) v = fmaxf(v, red[0][w][r]);
        v = v == -INFINITY ? 0.f : v;  // a row of infinitely low logits has sum 0
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int u = 0; u < 16; ++u) {
                const float e = __builtin_amdgcn_exp2f((g.acc[j][i][u] - v) * unit);
                g.acc[j][i][u] = e;
                sum += e;
            }
        sum += __shfl_xor(sum, 32);
        if (half == 0) red[1][wn][r] = sum;
    }
    barrier_lds();
    for (int r = threadIdx.x; r < BM; r += WM * WN * 64) {
        if (m0 + r >= P.x.extent) continue;
        float v = red[0][0][r], s = red[1][0][r];
#pragma unroll
        for (int w = 1; w < WN; ++w) {
            v = fmaxf(v, red[0][w][r]);
            s += red[1][w][r];
        }
        P.stats[(m0 + r) * P.tiles_n + tn] = float2{v, s};
    }
    if constexpr (KEEP) {
        // through the wave's own part of LDS (behind the barriers above no wave reads operands there
        // any more), 16-byte chunks swizzled by row, so that whole lines are stored
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
                    const u32x2 pk = {pack_exp<T>(a[4 * q], a[4 * q + 1]), pack_exp<T>(a[4 * q + 2], a[4 * q + 3])};
                    *(u32x2 *)(own + r * ROWB + (((j * 4 + q) ^ (r & (CPR - 1))) * 16) + half * 8) = pk;
                }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        const int c = lane % CPR;
        const int64_t n = n0 + wn * G::WTN + c * 8;
#pragma unroll 4
        for (int r = lane / CPR; r < G::WTM; r += 64 / CPR) {
            const int64_t m = m0 + wm * G::WTM + r;
            const u32x4 v = *(const u32x4 *)(own + r * ROWB + (c ^ (r & (CPR - 1))) * 16);
            if (m >= P.x.extent || n >= P.lde) continue;
            u32x4 *to = (u32x4 *)(P.e + m * P.lde + n);
            if (P.stream)
                __builtin_nontemporal_store(v, to);
            else
                *to = v;
        }
    }
}

template <class T, int BM, int BN, int WM, int WN, int BK, int STAGES, int OCC>
static hipError_t launch(Logits p, hipStream_t st) {
    p.tiles_m = (int32_t)(((int64_t)p.x.extent + BM - 1) / BM);
    p.tiles_n = (int32_t)(((int64_t)p.w.extent + BN - 1) / BN);
    const int64_t nb = (int64_t)p.tiles_m * p.tiles_n;
    if (nb <= 0) return hipSuccess;
    if (nb > 0x7FFFFF) return hipErrorInvalidValue;  // a launch has 2^32 threads at most
    if (p.e)
        hipLaunchKernelGGL((logits_kernel<T, BM, BN, WM, WN, BK, STAGES, OCC, true>), dim3((uint32_t)nb),
                           dim3(WM * WN * 64), 0, st, p);
    else
        hipLaunchKernelGGL((logits_kernel<T, BM, BN, WM, WN, BK, STAGES, OCC, false>), dim3((uint32_t)nb),
                           dim3(WM * WN * 64), 0, st, p);
    return hipGetLastError();
}

template <class T>
static hipError_t launch_t(Config cfg, const Logits &p, hipStream_t st) {
    if (cfg == TILE_32) return launch<T, 32, 128, 1, 4, 64, 4, 2>(p, st);
    if (cfg == TILE_256) return launch<T, 256, 256, 2, 4, 64, 2, 2>(p, st);
    return launch<T, 128, 128, 2, 4, 64, 2, 4>(p, st);
}

hipError_t launch_logits(int dtype, Config cfg, Logits p, hipStream_t st) {
    return dtype == Half::id ? launch_t<Half>(cfg, p, st) : launch_t<BFloat>(cfg, p, st);
}

}  // namespace xent

}  // namespace nnconv
