// gemm_tile.hpp -- the matrix-core product of two 16-bit matrices that the vocabulary loss is
// made of: acc[m][n] = sum over k of A(m, k) B(n, k), fp32 accumulators left in registers for an
// epilogue.
//
// An operand's reduction is either contiguous (element (x, k) at p[x * ld + k]) or its rows are
// (p[k * ld + x]: a gradient product reads its operands along their other axis).  Both are staged
// as they lie, straight into LDS; the second kind is turned by the transposing LDS reads.
//
// The reduction goes through an LDS ring of STAGES slices of BK elements; a wave reads the
// fragments of a 16-deep step while it multiplies those of the step before, and issues the loads
// of a slice between matrix instructions.
//
// Tiles and rates, one product of 8192 x 2048 x 65536 bf16 in its three forms (both along the
// reduction; one across it; both across it), normal values, on a card whose library does 1187, 1134
// and 990 TFLOP/s of them (1270 to 1400 of an 8192^3 one):
//   256 x 256, 4 waves, 32-element slices, 4 of them    -, 1131, 1116
//   the same, 64-element slices, 2 of them              -, 1132, 1083
//   8 waves of 128 x 64, 32-element slices, 4           -, 1198, 1144
//   8 waves of 128 x 64, 64-element slices, 2           -, 1222, 1185     (taken)
//   16 waves of 64 x 64, 64-element slices, 2           -, 1260, 1139     (spills registers)
//   256 x 128, 4 waves, two workgroups a compute unit   -, 891, 1105
//   128 x 128, 4 waves, 64-element slices, 2            -, 968, 984
// (the first form ends in another way, see xent_logits.hip).  The matrix units are busy in 59 % of
// the cycles at 1.94 GHz: the rest is waits at the slices' ends, and a faster tile lowers the clock.
// 128 x 128 tiles run with 8 waves: on short reductions, which are bound by latency, a step of 777 x
// 331 x 5003 takes 50 us with 8 and 52.5 with 4.  64 x 64 ones were not faster anywhere.
#pragma once

#include "launch.hpp"

namespace nnconv {

namespace gemm {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

struct Operand {
    const uint16_t *p;
    int64_t ld;     // elements from a row to the next, a multiple of 8
    int32_t extent; // rows that are not the reduction's; rows past it are read as zeros
};

// A slice's staging of one operand: X rows (or columns) of BK reduction elements.
template <bool TR, int X, int BK, int NW>
struct Stage {
    static constexpr int BYTES = X * BK * 2;
    static constexpr int LOADS = BYTES / (1024 * NW);
    static constexpr int KCH = BK / 8;       // 16-byte chunks of a row along the reduction
    static constexpr int ROWB = X * 2;       // bytes of a row across it
    static_assert(LOADS >= 1 && BYTES % (1024 * NW) == 0, "tile shape");

    const uint16_t *base;
    int64_t step;            // elements from a slice to the next
    uint32_t off[LOADS];     // of the lane's chunk; OOB_OFFSET outside the operand
    int32_t k[LOADS];        // its reduction index within a slice

    // 16-byte chunk swizzle of a row of KCH chunks: a fragment read has 16 rows at one chunk.
    static __device__ __forceinline__ int swz(int r) { return KCH == 8 ? (r >> 1) & 7 : (r >> 2) & 3; }
    static_assert(KCH == 4 || KCH == 8, "swizzle");
    // 64-byte segments of rows across the reduction: the 4 rows of a transposing read fall in
    // four segments of the banks.
    static __device__ __forceinline__ int seg(int p) { return ROWB >= 256 ? p & 3 : (p >> 1) & 1; }

    __device__ __forceinline__ void init(const Operand &o, int64_t x0, int64_t k0, int wave, int lane) {
        if constexpr (TR) {
            base = o.p + k0 * o.ld + x0;
            step = (int64_t)BK * o.ld;
        } else {
            base = o.p + x0 * o.ld + k0;
            step = BK;
        }
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            const int idx = (wave * LOADS + j) * 64 + lane;
            if constexpr (TR) {
                constexpr int CH = X / 8;
                const int r = idx / CH, q = idx % CH;
                const int c = ((((q >> 2) ^ seg(r)) << 2) | (q & 3)) * 8;
                off[j] = x0 + c < o.extent ? (uint32_t)(r * o.ld + c) * 2u : OOB_OFFSET;
                k[j] = r;
            } else {
                const int r = idx / KCH, c = (idx % KCH) ^ swz(r);
                off[j] = x0 + r < o.extent ? (uint32_t)(r * o.ld + c * 8) * 2u : OOB_OFFSET;
                k[j] = c * 8;
            }
        }
    }

    // Load j of the next slice, whose reduction elements from `left` on are zeros.
    __device__ __forceinline__ void load(int j, uint32_t lds, int wave, int left) const {
        const uint64_t a = (uint64_t)base;
        i32x4 d;
        d[0] = __builtin_amdgcn_readfirstlane((int32_t)(uint32_t)a);
        d[1] = __builtin_amdgcn_readfirstlane((int32_t)((uint32_t)(a >> 32) & 0xFFFFu));
        d[2] = (int32_t)MAX_BUFFER_BYTES;
        d[3] = 0x00020000;
        dma16(lds + (uint32_t)((wave * LOADS + j) * 1024), k[j] < left ? off[j] : OOB_OFFSET, d);
    }
    __device__ __forceinline__ void advance() { base += step; }

    // Fragment of the 32 rows from x0 on at the 16-deep step ks: lane l has row l % 32, reduction
    // elements 8 * (l / 32) on.
    static __device__ __forceinline__ u32x4 frag(const char *tile, int x0, int ks, int lane) {
        if constexpr (TR) {
            const int li = lane & 15, gq = lane >> 4;
            const int p = ks * 16 + 8 * (gq >> 1) + (li >> 2);
            const int byte = (x0 + 16 * (gq & 1) + (li & 3) * 4) * 2;
            const uint32_t o0 = p * ROWB + ((((byte >> 6) ^ seg(p)) << 6) | (byte & 63));
            const uint32_t o1 = (p + 4) * ROWB + ((((byte >> 6) ^ seg(p + 4)) << 6) | (byte & 63));
            const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(tile + o0));
            const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(tile + o1));
            const u32x2 lo = __builtin_bit_cast(u32x2, v0), hi = __builtin_bit_cast(u32x2, v1);
            return u32x4{lo[0], lo[1], hi[0], hi[1]};
        } else {
            const int r = x0 + (lane & 31);
            return *(const u32x4 *)(tile + (r * KCH + ((2 * ks + (lane >> 5)) ^ swz(r))) * 16);
        }
    }
};

// The product of a BM x BN tile by WM x WN waves.  Lane l of a wave holds, of each 32 x 32 block
// (j, i), row m = 32 i + l % 32 and columns n = 32 j + 8 e + 4 (l / 32) + {0..3} in elements
// 4 e + {0..3}, from its wave's corner (wm * BM / WM, wn * BN / WN) on.
template <class T, int BM, int BN, int WM, int WN, int BK, int STAGES, bool ATR, bool BTR>
struct Tile {
    static constexpr int NW = WM * WN, WTM = BM / WM, WTN = BN / WN, FM = WTM / 32, FN = WTN / 32;
    typedef Stage<ATR, BM, BK, NW> SA;
    typedef Stage<BTR, BN, BK, NW> SB;
    static constexpr int STAGE_BYTES = SA::BYTES + SB::BYTES;
    static constexpr int LDS_BYTES = STAGES * STAGE_BYTES;
    static constexpr int LOADS = SA::LOADS + SB::LOADS;
    static constexpr int KS = BK / 16;
    static_assert(FM >= 1 && FN >= 1 && KS % 2 == 0 && STAGES >= 2, "tile shape");

    f32x16 acc[FN][FM];

    // Reduction elements [k0, k1), k0 a multiple of BK.  On return no wave's loads are on their
    // way, but other waves may still read `lds`.
    __device__ __forceinline__ void run(const Operand &a, const Operand &b, int64_t m0, int64_t n0,
                                        int64_t k0, int64_t k1, char *lds) {
        const int lane = threadIdx.x & 63;
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int am = (wave % WM) * WTM, bn = (wave / WM) * WTN;
        const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_void *)lds;
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int i = 0; i < FM; ++i) acc[j][i] = f32x16{};
        const int iters = (int)((k1 - k0 + BK - 1) / BK);
        if (iters <= 0) return;
        SA sa;
        SB sb;
        sa.init(a, m0, k0, wave, lane);
        sb.init(b, n0, k0, wave, lane);
        int left = (int)(k1 - k0);  // reduction elements from the next slice to load on
        auto load = [&](int j, int buf) {
            const uint32_t at = lds0 + (uint32_t)(buf * STAGE_BYTES);
            if (j < SA::LOADS)
                sa.load(j, at, wave, left);
            else
                sb.load(j - SA::LOADS, at + SA::BYTES, wave, left);
        };
        // past the end the loads deliver zeros without touching memory and keep the counts even
        auto loaded = [&]() {
            sa.advance();
            sb.advance();
            left -= BK;
        };
        u32x4 fa[2][FM], fb[2][FN];
        auto read = [&](int buf, int ks, int to) {
            const char *st = lds + buf * STAGE_BYTES;
#pragma unroll
            for (int i = 0; i < FM; ++i) fa[to][i] = SA::frag(st, am + i * 32, ks, lane);
#pragma unroll
            for (int j = 0; j < FN; ++j) fb[to][j] = SB::frag(st + SA::BYTES, bn + j * 32, ks, lane);
        };
        auto mma = [&](int at) {
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int i = 0; i < FM; ++i) acc[j][i] = mfma32<T>(fb[at][j], fa[at][i], acc[j][i]);
        };
        auto mma_loads = [&](int at, int buf) {
            constexpr int NM = FM * FN;
            constexpr int EVERY = NM >= 2 * LOADS ? NM / LOADS : 1;
#pragma unroll
            for (int j = 0; j < FN; ++j) {
#pragma unroll
                for (int i = 0; i < FM; ++i) {
                    const int m = j * FM + i;
                    acc[j][i] = mfma32<T>(fb[at][j], fa[at][i], acc[j][i]);
                    if (m % EVERY == 0 && m / EVERY < LOADS) {
                        __builtin_amdgcn_sched_barrier(0);
                        load(m / EVERY, buf);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
            }
#pragma unroll
            for (int l = (NM + EVERY - 1) / EVERY; l < LOADS; ++l) load(l, buf);
        };
        auto slice = [&](int buf) {
#pragma unroll
            for (int ks = 0; ks + 1 < KS; ++ks) {
                read(buf, ks + 1, (ks + 1) & 1);
                mma(ks & 1);
            }
        };
#pragma unroll
        for (int s = 0; s < STAGES; ++s) {
#pragma unroll
            for (int j = 0; j < LOADS; ++j) load(j, s);
            loaded();
        }
        wait_vmcnt<(STAGES - 1) * LOADS>();
        barrier_lds();
        read(0, 0, 0);
        int buf = 0;
        for (int kt = 0; kt + 1 < iters; ++kt) {
            slice(buf);
            // the next slice has landed once at most STAGES - 2 later ones are on their way;
            // behind the barrier no wave reads this slice any more, and its buffer is loaded anew
            __builtin_amdgcn_sched_barrier(0);
            wait_vmcnt<(STAGES - 2) * LOADS>();
            barrier_lds();
            const int next = buf + 1 == STAGES ? 0 : buf + 1;
            read(next, 0, 0);
            mma_loads(1, buf);
            loaded();
            buf = next;
        }
        slice(buf);
        mma(1);
        wait_vmcnt<0>();
    }
};

}  // namespace gemm

}  // namespace nnconv
