// xent.hpp -- the pieces of the vocabulary loss (xent.hip) that run on the matrix cores
// (xent_logits.hip, xent_grad.hip).
//
//   logits   z = scale * x w^T by tiles; of each tile's rows the largest z and the sum of
//            e = exp(z - largest), and in training e in 16 bits
//   join     lse and loss of the tiles' statistics
//   scale    the same, and e -> 2^15 (softmax(z) - q) in the operand type, in place
//   grad     dx = d w, dw = d^T x
#pragma once

#include "gemm_tile.hpp"

namespace nnconv {

namespace xent {

// 2^15: the gradient of a logit lies in [-1, 1]; in fp16 it keeps 11 bits down to 2^-29 then.
constexpr float GRAD_UNIT = 32768.0f;

// How the exponentials, at most 1 since the largest product is taken off before the scale, are kept
// in 16 bits.  For bf16 operands fp16's 11 bits
// are three more than what they are rounded to later.  fp16 operands hold 11 themselves, and two
// such roundings would add to the product's error: without a sign and with 4 exponent bits there
// are 13, down to 2^-14 of the tile's largest, and an absolute error of 2^-28 of it below.
template <class T>
__device__ __forceinline__ uint32_t pack_exp(float lo, float hi) {
    if constexpr (T::id == BFloat::id) return pack16<Half>(lo, hi);
    const uint32_t a = __builtin_bit_cast(uint32_t, lo * 0x1p-112f) + 0x400u;  // 1 has exponent 15
    const uint32_t b = __builtin_bit_cast(uint32_t, hi * 0x1p-112f) + 0x400u;
    return ((a >> 11) & 0xFFFFu) | ((b >> 11) << 16);
}
template <class T>
__device__ __forceinline__ float unpack_exp(uint32_t bits) {
    if constexpr (T::id == BFloat::id) return from16<Half>(bits);
    return __builtin_bit_cast(float, (bits & 0xFFFFu) << 11) * 0x1p112f;
}

struct Logits {
    gemm::Operand x, w;  // [rows][k], [v][k]
    int32_t k;           // reduction elements
    float unit;          // logit_scale / log 2: what a product counts in units of log 2
    const int32_t *labels;  // [rows] or null
    // products here and in the statistics are turned where logit_scale is negative
    float *zt;           // [rows]: the labels' products
    float2 *stats;       // [rows][tiles_n]: largest product, and sum of the exponentials
    uint16_t *e;         // [rows][lde] or null
    int64_t lde;         // a multiple of 64, >= v
    bool stream;         // e past the caches
    int32_t tiles_m, tiles_n;
};

// Where a gradient product goes: out = (accumulate ? out : 0) + alpha * *scale * (acc + prev).
struct GradOut {
    void *out;
    int32_t kind;        // Half::id, BFloat::id or 2: fp32
    int32_t n;           // columns, and elements from a row to the next
    int64_t m;           // rows
    float alpha;
    const float *scale;  // device value or null
    int32_t accumulate;
    int32_t *flag;       // set where a value is not finite, or null
    const float *prev;   // fp32 [m][n] sums of earlier pieces, or null
    float *keep;         // fp32 [m][n]: acc + prev goes here and nowhere else, or null
};

struct Grad {
    gemm::Operand a, b;
    int64_t k;           // reduction elements
    int64_t k_split;     // of each split, a multiple of 64
    int32_t splits;
    float *part;         // fp32 [splits][m][n], splits > 1
    GradOut o;
    int32_t tiles_m, tiles_n;
};

// Tiles of a product: 256 x 256, 128 x 128, and for few logits 32 x 128.
enum Config { TILE_256 = 0, TILE_128 = 1, TILE_32 = 2 };
inline int tile_rows(Config c) { return c == TILE_256 ? 256 : c == TILE_128 ? 128 : 32; }
inline int tile_cols(Config c) { return c == TILE_256 ? 256 : 128; }

hipError_t launch_logits(int dtype, Config cfg, Logits p, hipStream_t st);
// dx = d w and, with dw, dw = d^T x: one launch where both take tiles of one kind.
hipError_t launch_grads(int dtype, Config cfg, const Grad &dx, Config cfg_w, const Grad *dw, hipStream_t st);
hipError_t launch_grad_w(int dtype, Config cfg, const Grad &dw, hipStream_t st);

// Tiles in an order that keeps a group of GROUP_M tile rows together.
constexpr int GROUP_M = 8;
__device__ __forceinline__ void tile_of(int id, int tiles_m, int tiles_n, int &tm, int &tn) {
    const int per = GROUP_M * tiles_n, g = id / per, first = g * GROUP_M;
    const int rows = tiles_m - first < GROUP_M ? tiles_m - first : GROUP_M;
    const int rem = id - g * per;
    tn = rem / rows;
    tm = first + rem - tn * rows;
}

}  // namespace xent

}  // namespace nnconv
