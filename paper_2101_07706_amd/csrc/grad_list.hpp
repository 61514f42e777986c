// A list of gradients as the kernels see it, and the join of what the blocks of grad_norm_k leave.
#pragma once
#include "common.hpp"

namespace csgs {

constexpr int64_t GRAD_TILE = 8192;
constexpr int GRAD_BLOCKS = 2048;      // most blocks of either kernel
constexpr int64_t GRAD_ENTRIES = 1ll << 40;

// A tensor as the kernels see it.  flat: its rows lie side by side, in g and in out.
struct GradDesc {
    const void *g;
    void *out;
    const int32_t *rows_dev;
    int64_t rows, cols, ldg, ldo, first_tile;
    int32_t dtype, flat;
};
struct GradMem {
    double *partial;      // [GRAD_BLOCKS]
    GradDesc *desc;       // [n]
    int32_t *tile_tensor; // [tiles]
    size_t bytes;
};
__host__ __device__ inline GradMem carve_grads(void *base, int32_t n, int64_t tiles)
{
    GradMem m;
    size_t off = align_up(sizeof(double) * GRAD_BLOCKS, 256);
    m.partial = (double *)base;
    m.desc = (GradDesc *)((char *)base + off);
    off = align_up(off + sizeof(GradDesc) * (size_t)n, 256);
    m.tile_tensor = (int32_t *)((char *)base + off);
    m.bytes = align_up(off + sizeof(int32_t) * (size_t)tiles, 256);
    return m;
}

// The sum, or the larger one with NaN above everything.
template <int KIND>
__device__ inline double add_or_max(double a, double b)
{
    if (KIND != CSGS_GRAD_MAX) return a + b;
    return !(a >= b) && !(a != a) ? b : a;
}
// Joined over the block's 256 threads in a fixed order, the result in every thread: across a wavefront by exchanges, then its four.
template <int KIND>
__device__ inline double block_join(double v, double *lds /*[4]*/)
{
#pragma unroll
    for (int s = WAVE / 2; s > 0; s >>= 1) v = add_or_max<KIND>(v, __shfl_xor(v, s));
    if (lane_id() == 0) lds[threadIdx.x / WAVE] = v;
    __syncthreads();
    return add_or_max<KIND>(add_or_max<KIND>(lds[0], lds[1]), add_or_max<KIND>(lds[2], lds[3]));
}

template <int KIND>
__device__ inline double join_partials(const double *__restrict__ partial, int blocks, double *lds)
{
    double p[GRAD_BLOCKS / 256], s = 0.0;
#pragma unroll
    for (int k = 0; k < GRAD_BLOCKS / 256; ++k) p[k] = k * 256 + (int)threadIdx.x < blocks ? partial[k * 256 + (int)threadIdx.x] : 0.0;
#pragma unroll
    for (int k = 0; k < GRAD_BLOCKS / 256; ++k) s = add_or_max<KIND>(s, p[k]);
    return block_join<KIND>(s, lds);
}
// (kind: the same for all threads)
__device__ inline double join_partials(const double *__restrict__ partial, int blocks, int kind, double *lds)
{
    return kind == CSGS_GRAD_MAX ? join_partials<CSGS_GRAD_MAX>(partial, blocks, lds) : join_partials<CSGS_GRAD_L2>(partial, blocks, lds);
}

inline int grad_blocks(int64_t tiles) { return (int)(tiles < GRAD_BLOCKS ? tiles : GRAD_BLOCKS); }
inline bool list_ok(const csgs_grad_list *l, int kind)
{
    return l && l->base && l->ready && l->n > 0 && l->tiles > 0 && kind >= CSGS_GRAD_L2 && kind <= CSGS_GRAD_MAX;
}

// Leaves a sum per block of the list's entries in its memory (clip.hip).
int launch_grad_norm(const csgs_grad_list *l, int kind, hipStream_t st);

}  // namespace csgs
