// Global norm over the gradients of a network, and clipping by it.
//
// total = (sum |g|^p)^(1/p) or max |g|; c = min(1, max_norm / (total + 1e-6)); out = c g.  Two launches for any number of
// tensors: their entries are cut into tiles of GRAD_TILE, the first kernel leaves one sum per block (in double, four sums a
// thread, joined in a fixed order), every block of the second adds those sums up for itself,
// in the same order, and scales its tiles.  The product with c is formed in double: one rounding.
//
// Bound by memory where the gradients are long, which are read twice (245 M floats: norm 169 us, 5.8 TB/s; scaling 340, 5.8 TB/s), by two launches
// and a chain of four loads (tile, description, row count, entries) where they are short (13 tensors of 3.0 M entries 5 and 7 us).
#include <math.h>
#include "common.hpp"
#include "row_pieces.hpp"

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

constexpr int DESC_PER_LAUNCH = 32;
struct DescBatch {
    GradDesc d[DESC_PER_LAUNCH];
    int64_t end_tile[DESC_PER_LAUNCH];
};
__global__ __launch_bounds__(256) void grad_list_k(DescBatch b, int32_t first, GradDesc *__restrict__ desc, int32_t *__restrict__ tile_tensor)
{
    const int k = (int)blockIdx.x;
    if (threadIdx.x == 0) desc[first + k] = b.d[k];
    for (int64_t t = b.d[k].first_tile + threadIdx.x; t < b.end_tile[k]; t += blockDim.x) tile_tensor[t] = first + k;
}

__device__ inline int64_t live_entries(const GradDesc &d)
{
    int64_t rows = d.rows;
    if (d.rows_dev) {
        const int64_t r = *d.rows_dev;
        rows = r < 0 ? 0 : (r < rows ? r : rows);
    }
    return rows * d.cols;
}

// A tile's entries [beg, end) by the block's threads.  Those of a flat tensor are asked for together, 16 bytes a piece and thread, before the first is
// needed; the others, and what does not fill a piece at the end, one by one when they are.
constexpr int TILE_PIECES = (int)(GRAD_TILE * 4 / (256 * 16));   // of a thread, of floats (half as many of bfloat16)
struct Tile {
    GradDesc d;
    int64_t beg, end, whole;
    u32x4 held[TILE_PIECES];

    __device__ void ask(const GradMem &m, int64_t t)
    {
        d = m.desc[m.tile_tensor[t]];
        const int64_t live = live_entries(d);
        beg = (t - d.first_tile) * GRAD_TILE;
        end = beg + GRAD_TILE < live ? beg + GRAD_TILE : live;
        if (end < beg) end = beg;
        const int V = d.dtype == CSGS_F32 ? 4 : 8;
        whole = d.flat ? end - (end - beg) % V : beg;
        const char *p = (const char *)d.g + beg * (16 / V);
        const int pieces = (int)((whole - beg) / V);
#pragma unroll
        for (int u = 0; u < TILE_PIECES; ++u) {
            const int k = u * 256 + (int)threadIdx.x;
            if (k < pieces) held[u] = load_global<u32x4, 2>(p + (int64_t)k * 16);
        }
    }
    // f(values, where they go)
    template <typename T, typename F>
    __device__ void each(F f) const
    {
        constexpr int V = 16 / (int)sizeof(T);
        const T *g = (const T *)d.g;
        T *out = (T *)d.out;
#pragma unroll
        for (int u = 0; u < TILE_PIECES * 4 / V; ++u) {
            const int64_t e = beg + (u * 256 + (int)threadIdx.x) * V;
            if (e < whole) {
                RawPiece<T, V> r;
                r.w[0] = held[u].x; r.w[1] = held[u].y; r.w[2] = held[u].z; r.w[3] = held[u].w;
                Vec<V> v;
#pragma unroll
                for (int i = 0; i < V; ++i) v.x[i] = r.value(i);
                f(v, out + e);
            }
        }
        if (d.flat) {
            const int64_t e = whole + threadIdx.x;
            if (e < end) f(load_row<T, 1>(g + e), out + e);
            return;
        }
        // (a row and a column of the tile's first entry by one division, the others from there in 32 bits)
        const int64_t r0 = beg / d.cols, c0 = beg - r0 * d.cols;
        for (int32_t x = (int32_t)threadIdx.x; x < (int32_t)(end - beg); x += 256) {
            const int64_t c = c0 + x;
            const int64_t dr = c < d.cols ? 0 : d.cols > GRAD_TILE ? 1 : (int64_t)((uint32_t)c / (uint32_t)d.cols);
            const int64_t r = r0 + dr, col = c - dr * d.cols;
            f(load_row<T, 1>(g + r * d.ldg + col), out + r * d.ldo + col);
        }
    }
};

// The sum, or the larger one with NaN above everything.
template <int KIND>
__device__ inline double add_or_max(double a, double b)
{
    if (KIND != CSGS_GRAD_MAX) return a + b;
    return !(a >= b) && !(a != a) ? b : a;
}
template <int KIND>
__device__ inline double take_in(double a, float x)
{
    const double v = (double)x;
    if (KIND == CSGS_GRAD_L2) return fma(v, v, a);   // (a float's square is exact in double)
    return add_or_max<KIND>(a, fabs(v));
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
__global__ __launch_bounds__(256) void grad_norm_k(GradMem m, int64_t tiles)
{
    __shared__ double lds[4];
    double sum[4] = {0.0, 0.0, 0.0, 0.0};
    for (int64_t t = blockIdx.x; t < tiles; t += gridDim.x) {
        Tile tile;
        tile.ask(m, t);
        auto take = [&](const auto &v, auto *) {
            constexpr int V = (int)(sizeof(v.x) / sizeof(float));
#pragma unroll
            for (int i = 0; i < V; ++i) sum[i % 4] = take_in<KIND>(sum[i % 4], v.x[i]);
        };
        if (tile.d.dtype == CSGS_F32) tile.each<float>(take);
        else tile.each<uint16_t>(take);
    }
    const double own = add_or_max<KIND>(add_or_max<KIND>(sum[0], sum[1]), add_or_max<KIND>(sum[2], sum[3]));
    const double all = block_join<KIND>(own, lds);
    if (threadIdx.x == 0) m.partial[blockIdx.x] = all;
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

__global__ __launch_bounds__(256) void grad_total_k(GradMem m, int blocks, int kind, double *__restrict__ total)
{
    __shared__ double lds[4];
    const double s = join_partials(m.partial, blocks, kind, lds);
    if (threadIdx.x == 0) *total = s;
}

// PAST: outputs too long for the caches go past them, so that what the next pass over the gradients reads is not pushed out.
template <bool PAST>
__global__ __launch_bounds__(256) void grad_scale_k(GradMem m, int64_t tiles, int blocks, int kind, const double *total, float max_norm, float *norm_out,
                                                    int32_t *status)
{
    __shared__ double lds[4];
    // (from the last tile back: those may still be in the cache from the pass before; the first one's entries are on their way meanwhile)
    int64_t t = tiles - 1 - blockIdx.x;
    Tile tile;
    tile.ask(m, t);
    const double s = total ? *total : join_partials(m.partial, blocks, kind, lds);
    const double norm = kind == CSGS_GRAD_L2 ? sqrt(s) : s;
    double coef = (double)max_norm / (norm + 1e-6);
    if (coef > 1.0) coef = 1.0;
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        if (norm_out) *norm_out = (float)norm;
        if (status && !(norm <= 1.7976931348623157e308)) atomicOr(status, CSGS_ST_NONFINITE_GRAD);
    }
    auto give = [&](auto v, auto *out) {
#pragma unroll
        for (float &x : v.x) x = float_to_store<std::remove_pointer_t<decltype(out)>>(coef * (double)x);
        if constexpr (PAST) store_row_past_caches(out, v);
        else store_row(out, v);
    };
    for (;;) {
        if (tile.d.out && (coef != 1.0 || tile.d.out != tile.d.g)) {   // (NaN is not 1)
            if (tile.d.dtype == CSGS_F32) tile.each<float>(give);
            else tile.each<uint16_t>(give);
        }
        t -= gridDim.x;
        if (t < 0) return;
        tile.ask(m, t);
    }
}

// Checks a tensor and describes it; tiles counted on from *tiles.
static int describe(const csgs_grad_tensor &t, int64_t *tiles, GradDesc *d)
{
    if (!t.g || t.rows <= 0 || t.cols <= 0 || t.ldg < t.cols || (t.out && t.ldo < t.cols) || (t.out == t.g && t.ldo != t.ldg)) return CSGS_EINVAL;
    if ((t.dtype != CSGS_F32 && t.dtype != CSGS_BF16) || t.rows > GRAD_ENTRIES / t.cols) return CSGS_EUNSUPPORTED;
    d->g = t.g;
    d->out = t.out;
    d->rows_dev = t.rows_dev;
    d->rows = t.rows;
    d->cols = t.cols;
    d->ldg = t.ldg;
    d->ldo = t.out ? t.ldo : t.ldg;
    d->first_tile = *tiles;
    d->dtype = t.dtype;
    d->flat = t.rows == 1 || (t.ldg == t.cols && d->ldo == t.cols) ? 1 : 0;
    *tiles += (t.rows * t.cols + GRAD_TILE - 1) / GRAD_TILE;
    return *tiles > GRAD_ENTRIES / GRAD_TILE ? CSGS_EUNSUPPORTED : CSGS_OK;
}

static int grad_blocks(int64_t tiles) { return (int)(tiles < GRAD_BLOCKS ? tiles : GRAD_BLOCKS); }
static bool list_ok(const csgs_grad_list *l, int kind)
{
    return l && l->base && l->ready && l->n > 0 && l->tiles > 0 && kind >= CSGS_GRAD_L2 && kind <= CSGS_GRAD_MAX;
}

// Entries from which outputs go past the caches: 256 MB of floats, the memory-side cache (us, through / past: 245 M floats 534 / 517).
constexpr int64_t PAST_TILES = (1ll << 26) / GRAD_TILE;
static int launch_scale(const csgs_grad_list *l, int kind, const double *total, float max_norm, float *norm, int32_t *status, hipStream_t st)
{
    const GradMem m = carve_grads(l->base, l->n, l->tiles);
    const int blocks = grad_blocks(l->tiles);
    if (l->tiles >= PAST_TILES)
        CSGS_LAUNCH(K_GRAD_SCALE, grad_scale_k<true>, dim3((unsigned)blocks), dim3(256), st, m, l->tiles, blocks, kind, total, max_norm, norm, status);
    else
        CSGS_LAUNCH(K_GRAD_SCALE, grad_scale_k<false>, dim3((unsigned)blocks), dim3(256), st, m, l->tiles, blocks, kind, total, max_norm, norm, status);
    CSGS_LAUNCH_CHECK();
    return CSGS_OK;
}
static int launch_norm(const csgs_grad_list *l, int kind, hipStream_t st)
{
    const GradMem m = carve_grads(l->base, l->n, l->tiles);
    const dim3 grid((unsigned)grad_blocks(l->tiles)), block(256);
    if (kind == CSGS_GRAD_L2) CSGS_LAUNCH(K_GRAD_NORM, grad_norm_k<CSGS_GRAD_L2>, grid, block, st, m, l->tiles);
    else if (kind == CSGS_GRAD_L1) CSGS_LAUNCH(K_GRAD_NORM, grad_norm_k<CSGS_GRAD_L1>, grid, block, st, m, l->tiles);
    else CSGS_LAUNCH(K_GRAD_NORM, grad_norm_k<CSGS_GRAD_MAX>, grid, block, st, m, l->tiles);
    CSGS_LAUNCH_CHECK();
    return CSGS_OK;
}

}  // namespace csgs

using namespace csgs;

extern "C" size_t csgs_grad_list_bytes(const csgs_grad_tensor *t, int32_t n)
{
    if (!t || n < 1 || n > 1 << 20) return 0;
    int64_t tiles = 0;
    GradDesc d;
    for (int32_t i = 0; i < n; ++i)
        if (describe(t[i], &tiles, &d) != CSGS_OK) return 0;
    return carve_grads(nullptr, n, tiles).bytes;
}

extern "C" int csgs_grad_list_init(csgs_grad_list *l, const csgs_grad_tensor *t, int32_t n, void *stream)
{
    if (!l || !l->base || ((uintptr_t)l->base & 255) || !t || n < 1 || n > 1 << 20) return CSGS_EINVAL;
    l->ready = 0;
    int64_t tiles = 0;
    GradDesc d;
    for (int32_t i = 0; i < n; ++i) {
        const int rc = describe(t[i], &tiles, &d);
        if (rc != CSGS_OK) return rc;
    }
    const GradMem m = carve_grads(l->base, n, tiles);
    if (l->bytes < m.bytes) return CSGS_EWORKSPACE;
    int64_t at = 0;
    for (int32_t first = 0; first < n; first += DESC_PER_LAUNCH) {
        DescBatch b;
        const int32_t k = n - first < DESC_PER_LAUNCH ? n - first : DESC_PER_LAUNCH;
        for (int32_t i = 0; i < k; ++i) {
            (void)describe(t[first + i], &at, &b.d[i]);
            b.end_tile[i] = at;
        }
        CSGS_LAUNCH(K_GRAD_LIST, grad_list_k, dim3((unsigned)k), dim3(256), (hipStream_t)stream, b, first, m.desc, m.tile_tensor);
        CSGS_LAUNCH_CHECK();
    }
    l->n = n;
    l->tiles = tiles;
    l->ready = 1;
    return CSGS_OK;
}

extern "C" int csgs_grad_norm(const csgs_grad_list *l, int kind, double *total, void *stream)
{
    if (!list_ok(l, kind) || !total) return CSGS_EINVAL;
    const int rc = launch_norm(l, kind, (hipStream_t)stream);
    if (rc != CSGS_OK) return rc;
    CSGS_LAUNCH(K_GRAD_TOTAL, grad_total_k, dim3(1), dim3(256), (hipStream_t)stream, carve_grads(l->base, l->n, l->tiles), grad_blocks(l->tiles), kind, total);
    CSGS_LAUNCH_CHECK();
    return CSGS_OK;
}

extern "C" int csgs_grad_scale(const csgs_grad_list *l, int kind, const double *total, float max_norm, float *norm, int32_t *status, void *stream)
{
    if (!list_ok(l, kind) || !total || !(max_norm > 0.0f)) return CSGS_EINVAL;
    return launch_scale(l, kind, total, max_norm, norm, status, (hipStream_t)stream);
}

extern "C" int csgs_grad_clip(const csgs_grad_list *l, int kind, float max_norm, float *norm, int32_t *status, void *stream)
{
    if (!list_ok(l, kind) || !(max_norm > 0.0f)) return CSGS_EINVAL;
    const int rc = launch_norm(l, kind, (hipStream_t)stream);
    return rc != CSGS_OK ? rc : launch_scale(l, kind, nullptr, max_norm, norm, status, (hipStream_t)stream);
}
