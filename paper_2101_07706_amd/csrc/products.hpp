// Kernels of the feed-forward block's products: what they share (linear.hip, gated.hip, matrix_grad.hip).
#pragma once
#include "apart.hpp"
#include "matrix_tile.hpp"

namespace csgs {

// act(z) and its derivative.  s(z) as the gates of the residual (residual.hip): e = exp(-z) with what the exponent's rounding loses put back, s = 1 / (1 + e), 1 - s = e s: both
// keep their relative precision.  Phi(z) = erfc(-z / sqrt 2) / 2, without a difference.
struct Activation {
    float a, da;
};
template <int ACT>
__device__ CSGS_INLINE inline Activation activate(float z)
{
    if constexpr (ACT == CSGS_ACT_NONE) return Activation{z, 1.0f};
    if constexpr (ACT == CSGS_ACT_RELU) return Activation{z < 0.0f ? 0.0f : z, z > 0.0f ? 1.0f : 0.0f};     // (NaN stays)
    if constexpr (ACT == CSGS_ACT_GELU) {
        const float phi = 0.5f * erfcf(z * -0.707106781f);
        return Activation{z * phi, phi + z * (0.398942280f * expf(-0.5f * z * z))};
    }
    const float t = z * -1.44269504f;
    const float e = __builtin_amdgcn_exp2f(t) * fminf(1.0f + fmaf(t, -0.693147181f, -z), 2.0f);
    const float s = __builtin_amdgcn_rcpf(1.0f + e), rest = fminf(e * s, 1.0f);
    if constexpr (ACT == CSGS_ACT_SIGMOID) return Activation{s, s * rest};
    return Activation{z * s, s * (1.0f + z * rest)};
}
// f with the activation as a constant: chosen once a block, not once an entry.
template <typename F>
__device__ CSGS_INLINE inline void with_activation(int32_t act, F f)
{
    if (act == CSGS_ACT_NONE) f(std::integral_constant<int, CSGS_ACT_NONE>());
    else if (act == CSGS_ACT_RELU) f(std::integral_constant<int, CSGS_ACT_RELU>());
    else if (act == CSGS_ACT_SIGMOID) f(std::integral_constant<int, CSGS_ACT_SIGMOID>());
    else if (act == CSGS_ACT_SILU) f(std::integral_constant<int, CSGS_ACT_SILU>());
    else f(std::integral_constant<int, CSGS_ACT_GELU>());
}
// Four values of a row as they lie in memory, or what there is of them.
template <typename T>
struct Quad {
    RawPiece<T, 4> raw;
    __device__ void load(const T *p, int n)
    {
        if (n >= 4) {
            raw.load(p);
            return;
        }
#pragma unroll
        for (int w = 0; w < RawPiece<T, 4>::WORDS; ++w) raw.w[w] = 0;
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (i < n) {
                if constexpr (sizeof(T) == 4) raw.w[i] = load_global<uint32_t>(p + i);
                else raw.w[i / 2] |= (uint32_t)load_global<uint16_t>(p + i) << (16 * (i & 1));
            }
    }
    __device__ float value(int i) const { return raw.value(i); }
};
struct Nothing {};
// Four entries of a vector from `col` on, zeros where there is none.
__device__ inline void load_bias(const float *b, int count, float (&x)[4])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = 0.0f;
    if (b && count > 0) load_some(b, count, x);
}

__device__ inline int32_t live_rows(int32_t M, const int32_t *M_dev)
{
    if (!M_dev) return M;
    const int32_t n = *M_dev;
    return n < 0 ? 0 : n < M ? n : M;
}

// Block -> tile.  Blocks are handed to the eight dies in turn: each die takes tiles that follow each other, in bands of TILE_BAND tile rows, column by column, so
// that what its cache holds of both operands is used by its next blocks (bands of 1, 2, 3 and 8 tile rows: within 2 % of each other).
constexpr int TILE_BAND = 4, DIES = 8;
__device__ inline void tile_place(int64_t b, int64_t tiles_m, int64_t tiles_n, int64_t *tm, int64_t *tn)
{
    const int64_t all = tiles_m * tiles_n, each = all / DIES, more = all % DIES, die = b % DIES, turn = b / DIES;
    const int64_t t = die * each + (die < more ? die : more) + turn;
    const int64_t band = t / (TILE_BAND * tiles_n), first = band * TILE_BAND;
    const int64_t high = tiles_m - first < TILE_BAND ? tiles_m - first : TILE_BAND, in = t - first * tiles_n;
    *tm = first + in % high;
    *tn = in / high;
}

// A tile's sums, by `sum(tile)` from zero on: once more where the tile asks for it.
template <class Tile, typename F>
__device__ CSGS_INLINE inline void form_sums(Tile &tile, char *lds, F sum)
{
    tile.clear();
    sum(tile);
    if (tile.settle(lds)) tile.again(lds, sum);
}

// ---------------------------------------------------------------- host side
// Blocks of one launch: the device counts 32 bits of threads, of which a block has 256 where there are many.
constexpr int64_t MOST_BLOCKS = (1 << 24) - 1;
inline Memory matrix_of(int dtype, const void *p, int64_t rows, int64_t cols, int64_t ld) { return matrix_memory(p, rows, cols, ld, dtype == CSGS_F32 ? 4 : 2); }
inline Memory vector_of(const float *p, int64_t n) { return matrix_memory(p, 1, n, n, 4); }
inline Memory count_of(const int32_t *p) { return matrix_memory(p, 1, 1, 1, 4); }
// Whether tiles of `large` entries are the quicker ones: a compute unit's share of them, against tiles of `small` entries, which read LDS twice as often for a product and take
// 1 / 0.85 of the time where both fill the device (us, gated gradient in floats: 4001 rows of 602 by 1111, 576 and 1134 tiles, 300 and 275; 5224 rows of 224 by 760, 492 and 984, 28 and 33).
inline bool larger_tiles(int64_t tiles_large, int64_t large, int64_t tiles_small, int64_t small)
{
    return 0.85 * (double)((tiles_large + 255) / 256 * large) <= (double)((tiles_small + 255) / 256 * small);
}

// matrix_grad.hip
// Sums over rows that blocks left as parts [parts x n], joined in double in their order.
int launch_join_columns(const float *part, int64_t parts, int32_t n, float *out, hipStream_t st);

// C = scale * (A B^T summed over the pairs of operands): what the gradients have of products.
struct OutProduct {
    Operand a[2], b[2];
    int32_t pairs;            // 1, or 2: a[0] b[0] + a[1] b[1]
    int32_t outs;             // 1, or 2: out[i] = a[0] b[i]
    void *out[2];
    int64_t ldo[2];
    int64_t rows, cols, red;
    const int32_t *rows_dev, *red_dev;   // nullable
    float scale;
    bool across;              // both operands lie with their outer index side by side, or both with the reduction
};
// Floats of memory for parts of such a product; does not fall as the sizes grow.
int64_t out_product_floats(int64_t rows, int64_t cols, int64_t red, int outs);
int launch_out_product(const OutProduct &p, int dtype, float *parts, hipStream_t st);

// Rows of the scratch for column sums: a wavefront leaves one for at least 32 rows.
inline int64_t column_parts(int32_t M) { return ((int64_t)M + 31) / 32 + 8; }
}  // namespace csgs
