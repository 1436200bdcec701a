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
// in 16 bits: without a sign and with the bits that they need.  What they are rounded to later has 11
// bits down to 2^-29 (fp16 in units of 2^-15): 5 bits of exponent and 12 of a number go to 2^-30 of the
// tile's largest, and on in steps of 2^-41.  bf16 has 8 bits and no such end: 6 bits of exponent, 11 of a
// number, down to 2^-62.  With fewer bits of exponent, rare tokens beside a likely one had gradients
// of 0.
template <class T>
struct Kept {
    static constexpr int EXPONENT = T::id == BFloat::id ? 6 : 5;
    static constexpr int SHIFT = 7 + EXPONENT;  // of an fp32 number's bits behind the exponent's are cut
    // 2^(127 - the exponent of 1), which has all bits
    static constexpr float UNIT = T::id == BFloat::id ? 0x1p64f : 0x1p96f;
};
template <class T>
__device__ __forceinline__ uint32_t pack_exp(float lo, float hi) {
    typedef Kept<T> K;
    const uint32_t a = (__builtin_bit_cast(uint32_t, lo * (1.0f / K::UNIT)) + (1u << (K::SHIFT - 1))) << (16 - K::SHIFT);
    const uint32_t b = (__builtin_bit_cast(uint32_t, hi * (1.0f / K::UNIT)) + (1u << (K::SHIFT - 1))) << (16 - K::SHIFT);
    return __builtin_amdgcn_perm(b, a, 0x07060302);  // the upper halves
}
template <class T>
__device__ __forceinline__ float unpack_exp(uint32_t bits) {
    typedef Kept<T> K;
    return __builtin_bit_cast(float, (bits & 0xFFFFu) << K::SHIFT) * K::UNIT;
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

// What stands for a row that does not count.  Arithmetic makes no NaN with these bits.
constexpr uint32_t NOT_COUNTED = 0x7FC0DEADu;
__device__ __forceinline__ bool counted(float v) { return __builtin_bit_cast(uint32_t, v) != NOT_COUNTED; }

// Which rows count: those whose label is a token, or with a teacher whose sum (see Rows in xent.hip) says so.
struct Counts {
    const int32_t *labels;
    const float *base;
    int32_t v;
    __device__ __forceinline__ bool of(int64_t r) const { return base ? counted(base[r]) : (uint32_t)labels[r] < (uint32_t)v; }
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
    // rows of dx that do not count are 0, where an infinity in w or a factor makes them NaN; looked at only there
    bool by_rows;
    Counts counts;
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
