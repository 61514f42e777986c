// csgs_linear: y = alpha act(a w + bias) + beta r, and its gradient.
//
// One product with its epilogue: a, w and r are read and y is written once, 2 M K N operations.  For wide layers bound by the matrix cores, by the clock under them, and by what of a
// tile's copies and outputs nothing hides (65536 rows of 4096 by 1024 in bfloat16: 521 us, 1056 TFLOP/s, 542 on a slower card; matrix cores busy 54 % of the cycles at 1.6 GHz with the
// counters on); for narrow ones (K or N up to some hundred) by the rows' bytes, for few rows by the launch and the way through a tile's sum (one row of 1024 by 1024: 8 us).
//
// Gradient, t = alpha dy .* act'(a w + bias): act' needs the product again (4 M K N are da and dw, 2 M K N this), which is cheaper than 4 bytes of each entry kept in the forward pass and leaves
// the forward call nothing to keep.  t is written once, in the operands' type: for bfloat16 a rounding of half a step, 2^-8 relative, of each term of da and dw, which the
// matrix cores ask for.  Column sums for dbias and dr come from the same registers, before that rounding.  Without an activation t is dy but for a factor: da and dw are formed from
// dy itself where the types are the same, else linear_dy_k rounds it (65536 rows of 1024, float to bfloat16 with sums: 116 us with dr).
#include "products.hpp"
#include "direct_tile.hpp"
#include "split_tile.hpp"

namespace csgs {

struct LinearArgs {
    Operand a, w;
    int32_t M, K, N, act;
    const int32_t *M_dev;
    const float *bias;
    const void *r, *dy;
    int64_t ldr, lddy, ldy, lddr, ldt;
    float alpha, beta;
    void *y, *dr, *t;
    float *columns;              // nullable: a row of column sums for each wavefront's rows
    int64_t tiles_m, tiles_n;
};

// GRAD = false: y.  GRAD = true: t = alpha dy act'(a w + bias) as an operand of the gradients' products, its column sums, dr = beta dy.
template <class Tile, typename T, typename TY, bool GRAD>
__global__ __launch_bounds__(Tile::THREADS, Tile::WAVES) void linear_k(LinearArgs p)
{
    constexpr int BM = Tile::ROWS, BN = Tile::COLS, WM = Tile::WAVES_M, WN = Tile::WAVES_N;
    __shared__ __attribute__((aligned(128))) char lds[Tile::LDS_BYTES];
    int64_t tm, tn;
    tile_place(blockIdx.x, p.tiles_m, p.tiles_n, &tm, &tn);
    const int64_t m0 = tm * BM, n0 = tn * BN, rows = live_rows(p.M, p.M_dev);
    if (m0 >= rows && !(GRAD && p.columns)) return;
    Tile tile;
    form_sums(tile, lds, [&](auto &t) CSGS_INLINE {
        if (m0 < rows) t.accumulate(lds, p.a, &p.w, m0, rows, n0, p.N, 0, p.K);
    });
    float sums[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    // (this lane's columns and what is left of them; rows of the tile that count)
    const int mine = Tile::my_column(), left = (int)(p.N - n0 < BN ? p.N - n0 : BN) - mine, count = left < 0 ? 0 : left < 4 ? left : 4;
    const int high = m0 < rows ? (int)(rows - m0 < BM ? rows - m0 : BM) : 0;
    const TY *beside = (const TY *)(GRAD ? p.dy : p.r);
    const int64_t ld = GRAD ? p.lddy : p.ldr;
    if (beside) beside += m0 * ld + n0;
    float bias[4];
    load_bias(p.bias + n0 + mine, p.bias ? count : 0, bias);
    const auto ask = [&](int m, int n) CSGS_INLINE {
        Quad<TY> x;
        x.load(beside + m * ld + n, beside && m < high ? count : 0);
        return x;
    };
    with_activation(p.act, [&](auto act) CSGS_INLINE {
        constexpr int ACT = decltype(act)::value;
        tile.each(lds, ask, [&](int m, int n, const float(&v)[1][4], const Quad<TY> &held) CSGS_INLINE {
            if (m >= high || count == 0) return;
            const int64_t row = m0 + m, col = n0 + n;
            float z[4], x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) z[i] = v[0][i] + bias[i];
            if constexpr (!GRAD) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    z[i] = p.alpha * activate<ACT>(z[i]).a;
                    if (p.r) z[i] += p.beta * held.value(i);
                }
                store_some((TY *)p.y + row * p.ldy + col, count, z);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    x[i] = held.value(i);
                    z[i] = i < count ? p.alpha * x[i] * activate<ACT>(z[i]).da : 0.0f;
                    sums[i] += z[i];
                    x[i] *= p.beta;
                }
                if (p.t) store_some((T *)p.t + row * p.ldt + col, count, z);
                if (p.dr) store_some((TY *)p.dr + row * p.lddr + col, count, x);
            }
        });
    });
    if (GRAD && p.columns)
        Tile::columns(sums, [&](int n, const float(&s)[4]) CSGS_INLINE {
            const int64_t col = n0 + n, rest = p.N - col;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < rest) p.columns[(tm * WM + Tile::my_wave() / WN) * p.N + col + i] = s[i];
        });
}

// Without an activation t is dy but for a factor.  A pass over dy: t in the operands' type, dr, column sums of alpha dy (a block's 64 rows at a time).
constexpr int DY_ROWS = 64;
template <typename T, typename TY>
__global__ __launch_bounds__(256) void linear_dy_k(LinearArgs p)
{
    __shared__ float lds[4][64][4];
    const int lane = (int)threadIdx.x & 63, group = (int)threadIdx.x >> 6;
    const int64_t rows = live_rows(p.M, p.M_dev), part = blockIdx.x / p.tiles_n, col = ((int64_t)(blockIdx.x % p.tiles_n) * 64 + lane) * 4, rest = p.N - col;
    const int count = rest >= 4 ? 4 : rest > 0 ? (int)rest : 0;
    float sums[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (count)
        for (int64_t row = part * DY_ROWS + group, k = 0; k < DY_ROWS / 4 && row < rows; row += 4, ++k) {
            float x[4], t[4];
            load_some((const TY *)p.dy + row * p.lddy + col, count, x);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                t[i] = p.alpha * x[i];
                sums[i] += t[i];
                x[i] *= p.beta;
            }
            if (p.t) store_some((T *)p.t + row * p.ldt + col, count, t);
            if (p.dr) store_some((TY *)p.dr + row * p.lddr + col, count, x);
        }
    if (!p.columns) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) lds[group][lane][i] = sums[i];
    __syncthreads();
    if (group == 0)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < count) p.columns[part * p.N + col + i] = (lds[0][lane][i] + lds[1][lane][i]) + (lds[2][lane][i] + lds[3][lane][i]);
}

template <class Tile, typename T, typename TY, bool GRAD>
static int launch_shape(LinearArgs p, int64_t *parts, hipStream_t st)
{
    constexpr int BM = Tile::ROWS, BN = Tile::COLS, WM = Tile::WAVES_M;
    p.tiles_m = ((int64_t)p.M + BM - 1) / BM;
    p.tiles_n = ((int64_t)p.N + BN - 1) / BN;
    *parts = p.tiles_m * WM;
    if (p.tiles_m * p.tiles_n > MOST_BLOCKS) return CSGS_EUNSUPPORTED;
    CSGS_LAUNCH(K_LINEAR, (linear_k<Tile, T, TY, GRAD>), dim3((unsigned)(p.tiles_m * p.tiles_n)), dim3(Tile::THREADS), st, p);
    CSGS_LAUNCH_CHECK();
    return CSGS_OK;
}
template <typename T, typename TY, bool GRAD>
static int launch_types(const LinearArgs &p, int64_t *parts, hipStream_t st)
{
    const auto tiles = [&](int64_t m, int64_t n) { return (p.M + m - 1) / m * ((p.N + n - 1) / n); };
    // Tiles of 256 by 256 straight to LDS, one block a compute unit; those of 128 by 128 are held two a compute unit, 512 at once: the larger ones are taken where the smaller ones
    // would need a second round (us, 1024 by 1024, large and small: 6400 rows 35 and 30, 9600 rows 36 and 43, 16384 rows 42 and 55; 12800 rows of 4096 by 1024 102 and 194).
    if constexpr (sizeof(T) == 2)
        if (tiles(256, 256) > 128 && direct_operand(p.a, false, p.M, p.K, 256) && direct_operand(p.w, true, p.N, p.K, 256))
            return launch_shape<DirectTile<256, 256, 2, 4, false, true, 1, 128, 2>, T, TY, GRAD>(p, parts, st);
    if (larger_tiles(tiles(128, 128), 128 * 128, tiles(64, 64), 64 * 64)) return launch_shape<AnyTile<T, 128, 128, 2, 2, false, true, 1>, T, TY, GRAD>(p, parts, st);
    // Few tiles and long sums: groups of a block's wavefronts take a tile's chunks in turn (us, without and with: one row of 1024 by 1024 15 and 8, in floats 31 and 16; 1024 rows of 1024 by
    // 1024, 256 tiles, 11.6 and 9.8; 2048 rows, 512 tiles, 13.6 and 17.1).  Eight groups on half the rows as long as those tiles have a unit each (us, four groups and eight: 128 rows of 4096
    // by 1024 22 and 17; 1024 of 1024 by 512, 128 tiles, floats 21 and 18; 1024 of 1024 by 1024, floats 23 and 33).
    if (p.K >= 256 && (p.M <= 32 || tiles(64, 64) <= 128)) return launch_shape<AnyTile<T, 32, 64, 1, 2, false, true, 1, 8>, T, TY, GRAD>(p, parts, st);
    if (p.K >= 256 && tiles(64, 64) <= 256) return launch_shape<AnyTile<T, 64, 64, 2, 2, false, true, 1, 4>, T, TY, GRAD>(p, parts, st);
    return launch_shape<AnyTile<T, 64, 64, 2, 2, false, true, 1>, T, TY, GRAD>(p, parts, st);
}
template <bool GRAD>
static int launch_linear(const LinearArgs &p, int dtype, int y_dtype, int64_t *parts, hipStream_t st)
{
    if (dtype == CSGS_F32) return launch_types<float, float, GRAD>(p, parts, st);
    if (y_dtype == CSGS_F32) return launch_types<uint16_t, float, GRAD>(p, parts, st);
    return launch_types<uint16_t, uint16_t, GRAD>(p, parts, st);
}
static int launch_dy(LinearArgs p, int dtype, int y_dtype, int64_t *parts, hipStream_t st)
{
    *parts = ((int64_t)p.M + DY_ROWS - 1) / DY_ROWS;
    p.tiles_n = ((int64_t)p.N + 255) / 256;
    if (*parts * p.tiles_n > MOST_BLOCKS) return CSGS_EUNSUPPORTED;
    const dim3 grid((unsigned)(*parts * p.tiles_n)), block(256);
    if (dtype == CSGS_F32) CSGS_LAUNCH(K_LINEAR_DY, (linear_dy_k<float, float>), grid, block, st, p);
    else if (y_dtype == CSGS_F32) CSGS_LAUNCH(K_LINEAR_DY, (linear_dy_k<uint16_t, float>), grid, block, st, p);
    else CSGS_LAUNCH(K_LINEAR_DY, (linear_dy_k<uint16_t, uint16_t>), grid, block, st, p);
    CSGS_LAUNCH_CHECK();
    return CSGS_OK;
}

static int check(const csgs_linear_args *p, LinearArgs *a)
{
    if (!p || p->M <= 0 || p->K <= 0 || p->N <= 0 || !p->a || !p->w || p->lda < p->K || p->ldw < p->N || (p->r && p->ldr < p->N)) return CSGS_EINVAL;
    if (p->act < CSGS_ACT_NONE || p->act > CSGS_ACT_GELU) return CSGS_EINVAL;
    const bool same = p->dtype == p->y_dtype && (p->dtype == CSGS_F32 || p->dtype == CSGS_BF16);
    if (!same && !(p->dtype == CSGS_BF16 && p->y_dtype == CSGS_F32)) return CSGS_EUNSUPPORTED;
    *a = LinearArgs{};
    a->a = Operand{p->a, p->lda};
    a->w = Operand{p->w, p->ldw};
    a->M = p->M;
    a->K = p->K;
    a->N = p->N;
    a->act = p->act;
    a->M_dev = p->M_dev;
    a->bias = p->bias;
    a->r = p->r;
    a->ldr = p->ldr;
    a->alpha = p->alpha;
    a->beta = p->beta;
    return CSGS_OK;
}

// What both calls read, as memory.
struct LinearMemory {
    Memory a, w, bias, count;
    explicit LinearMemory(const csgs_linear_args *p)
        : a(matrix_of(p->dtype, p->a, p->M, p->K, p->lda)), w(matrix_of(p->dtype, p->w, p->K, p->N, p->ldw)), bias(vector_of(p->bias, p->N)), count(count_of(p->M_dev))
    {
    }
};

// Scratch of the gradient: t, rows of column sums, parts of the products.
struct LinearScratch {
    void *t;
    float *columns, *parts;
    size_t bytes;
};
static LinearScratch carve_linear(void *base, int32_t M, int32_t K, int32_t N, int dtype)
{
    LinearScratch s;
    size_t off = align_up((size_t)M * (size_t)N * (dtype == CSGS_F32 ? 4 : 2), 256);
    s.t = base;
    s.columns = (float *)((char *)base + off);
    off = align_up(off + (size_t)column_parts(M) * (size_t)N * 4, 256);
    s.parts = (float *)((char *)base + off);
    const int64_t da = out_product_floats(M, K, N, 1), dw = out_product_floats(K, N, M, 1);
    s.bytes = align_up(off + (size_t)(da > dw ? da : dw) * 4, 256);
    return s;
}

}  // namespace csgs

using namespace csgs;

extern "C" int csgs_linear(const csgs_linear_args *p, void *y, int64_t ldy, void *stream)
{
    LinearArgs a;
    const int rc = check(p, &a);
    if (rc != CSGS_OK) return rc;
    if (!y || ldy < p->N) return CSGS_EINVAL;
    const LinearMemory at(p);
    const Memory out = matrix_of(p->y_dtype, y, p->M, p->N, ldy), r = matrix_of(p->y_dtype, p->r, p->M, p->N, p->ldr);
    if (y == p->r && ldy != p->ldr) return CSGS_EINVAL;
    if (spans_too_much({at.a, at.w, out, r})) return CSGS_EUNSUPPORTED;
    if (!outputs_apart({at.a, at.w, at.bias, at.count, y == p->r ? Memory{} : r}, {out})) return CSGS_EINVAL;
    a.y = y;
    a.ldy = ldy;
    int64_t parts;
    return launch_linear<false>(a, p->dtype, p->y_dtype, &parts, (hipStream_t)stream);
}

extern "C" size_t csgs_linear_grad_scratch_bytes(int32_t M, int32_t K, int32_t N, int dtype)
{
    if (M <= 0 || K <= 0 || N <= 0 || (dtype != CSGS_F32 && dtype != CSGS_BF16)) return 0;
    return carve_linear(nullptr, M, K, N, dtype).bytes;
}

extern "C" int csgs_linear_grad(const csgs_linear_args *p, const void *dy, int64_t lddy, void *da, int64_t ldda, void *dw, int64_t lddw, float *dbias, void *dr,
                                int64_t lddr, void *scratch, size_t scratch_bytes, void *stream)
{
    LinearArgs a;
    int rc = check(p, &a);
    if (rc != CSGS_OK) return rc;
    if (!dy || lddy < p->N || (da && ldda < p->K) || (dw && lddw < p->N) || (dr && lddr < p->N) || (!da && !dw && !dbias && !dr)) return CSGS_EINVAL;
    if ((dbias && !p->bias) || (dr && !p->r) || (dr == dy && lddr != lddy)) return CSGS_EINVAL;
    const LinearMemory at(p);
    const Memory in = matrix_of(p->y_dtype, dy, p->M, p->N, lddy), out_a = matrix_of(p->dtype, da, p->M, p->K, ldda), out_w = matrix_of(p->dtype, dw, p->K, p->N, lddw),
                 out_b = vector_of(dbias, p->N), out_r = matrix_of(p->y_dtype, dr, p->M, p->N, lddr);
    if (spans_too_much({at.a, at.w, in, out_a, out_w, out_r})) return CSGS_EUNSUPPORTED;
    const Memory dy_beside_dr = dr == dy ? Memory{} : in;
    if (!outputs_apart({at.a, at.w, at.bias, at.count, dy_beside_dr}, {out_a, out_w, out_b, out_r})) return CSGS_EINVAL;
    if (!scratch || ((uintptr_t)scratch & 255)) return CSGS_EINVAL;
    const LinearScratch s = carve_linear(scratch, p->M, p->K, p->N, p->dtype);
    if (scratch_bytes < s.bytes) return CSGS_EWORKSPACE;
    if (!outputs_apart({at.a, at.w, at.bias, at.count, in, out_a, out_w, out_b, out_r}, {Memory{scratch, 1, (int64_t)s.bytes, 0}})) return CSGS_EINVAL;
    hipStream_t st = (hipStream_t)stream;
    a.dy = dy;
    a.lddy = lddy;
    a.dr = dr;
    a.lddr = lddr;
    a.ldt = p->N;
    a.columns = dbias ? s.columns : nullptr;
    int64_t parts = 0;
    Operand t{s.t, p->N};
    float scale = 1.0f;
    // (of an activation's derivative dr knows nothing)
    const bool plain = p->act == CSGS_ACT_NONE || (!da && !dw && !dbias), direct = plain && p->dtype == p->y_dtype;
    if (direct) {                   // (t is dy itself, its factor that of the products)
        t = Operand{dy, lddy};
        scale = p->alpha;
    } else {
        a.t = plain && !da && !dw ? nullptr : s.t;
        rc = plain ? launch_dy(a, p->dtype, p->y_dtype, &parts, st) : launch_linear<true>(a, p->dtype, p->y_dtype, &parts, st);
        if (rc != CSGS_OK) return rc;
    }
    if (da) {
        OutProduct o{};
        o.a[0] = t;
        o.b[0] = a.w;
        o.pairs = o.outs = 1;
        o.out[0] = da;
        o.ldo[0] = ldda;
        o.rows = p->M;
        o.cols = p->K;
        o.red = p->N;
        o.rows_dev = p->M_dev;
        o.scale = scale;
        o.across = false;
        rc = launch_out_product(o, p->dtype, s.parts, st);
        if (rc != CSGS_OK) return rc;
    }
    if (dw) {
        OutProduct o{};
        o.a[0] = a.a;
        o.b[0] = t;
        o.pairs = o.outs = 1;
        o.out[0] = dw;
        o.ldo[0] = lddw;
        o.rows = p->K;
        o.cols = p->N;
        o.red = p->M;
        o.red_dev = p->M_dev;
        o.scale = scale;
        o.across = true;
        rc = launch_out_product(o, p->dtype, s.parts, st);
        if (rc != CSGS_OK) return rc;
    }
    if (direct && (dbias || dr)) {   // (after the products: dr may be dy)
        rc = launch_dy(a, p->dtype, p->y_dtype, &parts, st);
        if (rc != CSGS_OK) return rc;
    }
    return dbias ? launch_join_columns(s.columns, parts, p->N, dbias, st) : CSGS_OK;
}
