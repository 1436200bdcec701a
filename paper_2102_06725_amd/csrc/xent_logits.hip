// xent_logits.hip -- logits of a vocabulary by tiles, with the softmax's statistics.
//
// A tile's logits stay in registers: of each row the largest (in the lane's 16 values of each
// block, then its other half's, then the other waves' through LDS) and the sum of the exponentials
// against it go to memory, and in training the exponentials themselves, at most 1, in 16 bits.
#include "xent.hpp"

namespace nnconv {

namespace xent {

constexpr float LOG2E = 1.4426950408889634f;

template <class T, int BM, int BN, int WM, int WN, int BK, int STAGES, int OCC, bool KEEP>
__global__ __launch_bounds__(WM * WN * 64, OCC) void logits_kernel(const Logits P) {
    typedef gemm::Tile<T, BM, BN, WM, WN, BK, STAGES, false, false> G;
    constexpr int FM = G::FM, FN = G::FN;
    constexpr int ROWB = BN * 2;
    constexpr int LDS = KEEP && G::LDS_BYTES < BM * ROWB ? BM * ROWB : G::LDS_BYTES;
    __shared__ __attribute__((aligned(16))) char lds[LDS];
    __shared__ float red[2][WN][BM];

    int tm, tn;
    tile_of((int)xcd_remap(blockIdx.x, gridDim.x), P.tiles_m, P.tiles_n, tm, tn);
    const int64_t m0 = (int64_t)tm * BM, n0 = (int64_t)tn * BN;
    G g;
    g.run(P.x, P.w, m0, n0, 0, P.k, lds);

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave % WM, wn = wave / WM;
    const int l32 = lane & 31, half = lane >> 5;
    const int cols = P.w.extent - n0 < BN ? (int)(P.w.extent - n0) : BN;  // of the tile
    const int c0 = wn * G::WTN + 4 * half;

    float most[FM];
#pragma unroll
    for (int i = 0; i < FM; ++i) {
        float v = -INFINITY;
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int u = 0; u < 16; ++u) {
                float z = g.acc[j][i][u] * P.scale;
                if (cols < BN && c0 + j * 32 + 8 * (u >> 2) + (u & 3) >= cols) z = -INFINITY;
                g.acc[j][i][u] = z;
                v = fmaxf(v, z);
            }
        most[i] = fmaxf(v, __shfl_xor(v, 32));
        if (half == 0) red[0][wn][wm * G::WTM + i * 32 + l32] = most[i];
    }
    barrier_lds();
#pragma unroll
    for (int i = 0; i < FM; ++i) {
        const int r = wm * G::WTM + i * 32 + l32;
        float v = red[0][0][r];
#pragma unroll
        for (int w = 1; w < WN; ++w) v = fmaxf(v, red[0][w][r]);
        most[i] = v;
        const float from = v == -INFINITY ? 0.f : v;  // a row of infinitely low logits
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int u = 0; u < 16; ++u) {
                const float e = __builtin_amdgcn_exp2f((g.acc[j][i][u] - from) * LOG2E);
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
        // through LDS, 16-byte chunks swizzled by row, so that whole lines are stored
        constexpr int CPR = BN / 8;
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            const int r = wm * G::WTM + i * 32 + l32;
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int c = (wn * G::WTN + j * 32) / 8 + q;
                    const f32x16 &a = g.acc[j][i];
                    const u32x2 pk = {pack_exp<T>(a[4 * q], a[4 * q + 1]), pack_exp<T>(a[4 * q + 2], a[4 * q + 3])};
                    *(u32x2 *)(lds + r * ROWB + ((c ^ (r & 15)) * 16) + half * 8) = pk;
                }
        }
        barrier_lds();
        constexpr int PASS = WM * WN * 64 / CPR;
        const int c = threadIdx.x % CPR;
        for (int r = threadIdx.x / CPR; r < BM; r += PASS) {
            if (m0 + r >= P.x.extent || n0 + c * 8 >= P.lde) continue;
            const u32x4 v = *(const u32x4 *)(lds + r * ROWB + (c ^ (r & 15)) * 16);
            *(u32x4 *)(P.e + (m0 + r) * P.lde + n0 + c * 8) = v;
        }
    }
}

template <class T, int BM, int BN, int WM, int WN, int BK, int STAGES, int OCC>
static hipError_t launch(Logits p, hipStream_t st) {
    p.tiles_m = (int32_t)(((int64_t)p.x.extent + BM - 1) / BM);
    p.tiles_n = (int32_t)(((int64_t)p.w.extent + BN - 1) / BN);
    const int64_t nb = (int64_t)p.tiles_m * p.tiles_n;
    if (nb <= 0) return hipSuccess;
    if (nb > 0x3FFFFFFF) return hipErrorInvalidValue;
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
    if (cfg == TILE_256) return launch<T, 256, 256, 2, 2, 32, 4, 1>(p, st);
    return launch<T, 128, 128, 2, 2, 32, 4, 2>(p, st);
}

hipError_t launch_logits(int dtype, Config cfg, Logits p, hipStream_t st) {
    return dtype == Half::id ? launch_t<Half>(cfg, p, st) : launch_t<BFloat>(cfg, p, st);
}

}  // namespace xent

}  // namespace nnconv
