// csgs_gated: h = act(x wg + bg) .* (x wu + bu), and its gradient.
//
// Both projections in one kernel: a tile of x serves both products, whose entries meet in one lane's registers, so that neither g nor u (8 M N bytes each way in floats) reaches memory.
// 4 M K N operations, bound as csgs_linear (65536 rows of 1024 by 4096 in bfloat16: 1117 us, 985 TFLOP/s, 1157 on a slower card; matrix cores busy 49 % of the cycles at 1.7 GHz); a single row is bound by the weights' bytes and the way through a
// tile's sum (16.8 MB, 11.5 us).
//
// Gradient: g and u formed again (4 M K N beside the 8 M K N of dx, dwg and dwu), tg = dh .* u .* act'(g) and tu = dh .* act(g) written once in the operands' type (for bfloat16 a
// rounding of half a step, 2^-8 relative, of each term, which the matrix cores ask for), their column sums from registers before that; dx as one sum over both pairs, dwg and dwu
// by one launch (65536 rows: 3146 us, 1049 TFLOP/s, 3317 on a slower card).
#include "products.hpp"
#include "direct_tile.hpp"
#include "split_tile.hpp"

namespace csgs {

struct GatedArgs {
    Operand x, w[2];
    int32_t M, K, N, act;
    const int32_t *M_dev;
    const float *b[2];
    const void *dh;
    int64_t lddh, ldh, ldt;
    void *h, *t[2];
    float *columns[2];           // nullable: a row of column sums for each wavefront's rows
    int64_t tiles_m, tiles_n;
};

// GRAD = false: h.  GRAD = true: tg and tu as operands of the gradients' products, and their column sums.
template <class Tile, typename T, bool GRAD>
__global__ __launch_bounds__(Tile::THREADS, Tile::WAVES) void gated_k(GatedArgs p)
{
    constexpr int BM = Tile::ROWS, BN = Tile::COLS, WM = Tile::WAVES_M, WN = Tile::WAVES_N;
    __shared__ __attribute__((aligned(128))) char lds[Tile::LDS_BYTES];
    int64_t tm, tn;
    tile_place(blockIdx.x, p.tiles_m, p.tiles_n, &tm, &tn);
    const int64_t m0 = tm * BM, n0 = tn * BN, rows = live_rows(p.M, p.M_dev);
    const bool columns = GRAD && (p.columns[0] || p.columns[1]);
    if (m0 >= rows && !columns) return;
    Tile tile;
    form_sums(tile, lds, [&](auto &t) CSGS_INLINE {
        if (m0 < rows) t.accumulate(lds, p.x, p.w, m0, rows, n0, p.N, 0, p.K);
    });
    float sums[2][4] = {};
    // (this lane's columns and what is left of them; rows of the tile that count)
    const int mine = Tile::my_column(), left = (int)(p.N - n0 < BN ? p.N - n0 : BN) - mine, count = left < 0 ? 0 : left < 4 ? left : 4;
    const int high = m0 < rows ? (int)(rows - m0 < BM ? rows - m0 : BM) : 0;
    float bias[2][4];
#pragma unroll
    for (int b = 0; b < 2; ++b) load_bias(p.b[b] + n0 + mine, p.b[b] ? count : 0, bias[b]);
    const auto ask = [&](int m, int n) CSGS_INLINE {
        if constexpr (GRAD) {
            Quad<T> x;
            x.load((const T *)p.dh + (m0 + m) * p.lddh + n0 + n, m < high ? count : 0);
            return x;
        } else {
            return Nothing{};
        }
    };
    with_activation(p.act, [&](auto act) CSGS_INLINE {
        constexpr int ACT = decltype(act)::value;
        tile.each(lds, ask, [&](int m, int n, const float(&v)[2][4], const auto &held) CSGS_INLINE {
            if (m >= high || count == 0) return;
            const int64_t row = m0 + m, col = n0 + n;
            float t[2][4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float g = v[0][i] + bias[0][i], u = v[1][i] + bias[1][i];
                const Activation a = activate<ACT>(g);
                if constexpr (!GRAD) {
                    t[0][i] = a.a * u;
                } else {
                    t[0][i] = i < count ? held.value(i) * u * a.da : 0.0f;
                    t[1][i] = i < count ? held.value(i) * a.a : 0.0f;
                    sums[0][i] += t[0][i];
                    sums[1][i] += t[1][i];
                }
            }
            if constexpr (!GRAD) {
                store_some((T *)p.h + row * p.ldh + col, count, t[0]);
            } else {
                store_some((T *)p.t[0] + row * p.ldt + col, count, t[0]);
                store_some((T *)p.t[1] + row * p.ldt + col, count, t[1]);
            }
        });
    });
    if constexpr (GRAD)
#pragma unroll
        for (int b = 0; b < 2; ++b)
            if (p.columns[b])
                Tile::columns(sums[b], [&](int n, const float(&s)[4]) CSGS_INLINE {
                    const int64_t col = n0 + n, rest = p.N - col;
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (i < rest) p.columns[b][(tm * WM + Tile::my_wave() / WN) * p.N + col + i] = s[i];
                });
}

template <class Tile, typename T, bool GRAD>
static int launch_shape(GatedArgs p, int64_t *parts, hipStream_t st)
{
    constexpr int BM = Tile::ROWS, BN = Tile::COLS, WM = Tile::WAVES_M;
    p.tiles_m = ((int64_t)p.M + BM - 1) / BM;
    p.tiles_n = ((int64_t)p.N + BN - 1) / BN;
    *parts = p.tiles_m * WM;
    if (p.tiles_m * p.tiles_n > MOST_BLOCKS) return CSGS_EUNSUPPORTED;
    CSGS_LAUNCH(K_GATED, (gated_k<Tile, T, GRAD>), dim3((unsigned)(p.tiles_m * p.tiles_n)), dim3(Tile::THREADS), st, p);
    CSGS_LAUNCH_CHECK();
    return CSGS_OK;
}
template <typename T, bool GRAD>
static int launch_types(const GatedArgs &p, int64_t *parts, hipStream_t st)
{
    const auto tiles = [&](int64_t m, int64_t n) { return (p.M + m - 1) / m * ((p.N + n - 1) / n); };
    // Tiles of 256 rows by 128 columns of both matrices, one block a compute unit, where smaller ones would need a second round (us, 1024 by 1024, large and small: 3200 rows 29 and 25, 4800
    // rows 30 and 37, 8192 rows 37 and 50); for the gradient, which writes twice as much and reads dh, of 128 rows, two blocks: one forms
    // products while the other writes (us, 65536 rows of 1024 by 4096: forward 1043 and 1092, gradient with its products 3182 and 3121; on another card
    // 1109 and 1101, 3205 and 3136).
    if constexpr (sizeof(T) == 2)
        if (tiles(256, 128) > 128 && direct_operand(p.x, false, p.M, p.K, 256) && direct_operand(p.w[0], true, p.N, p.K, 128) && direct_operand(p.w[1], true, p.N, p.K, 128))
            return launch_shape<std::conditional_t<GRAD, DirectTile<128, 128, 2, 2, false, true, 2, 64, 3>, DirectTile<256, 128, 2, 4, false, true, 2, 128, 2>>, T, GRAD>(p, parts, st);
    if (larger_tiles(tiles(128, 64), 128 * 64, tiles(64, 64), 64 * 64)) return launch_shape<AnyTile<T, 128, 64, 2, 2, false, true, 2>, T, GRAD>(p, parts, st);
    // (groups of wavefronts as for csgs_linear; us, without and with: one row of 1024 by 4096 17.4 and 11.3, in floats 46 and 24; 128 rows of 1024 by 1024 in floats 49 and 34, on half the
    // rows 24.  Two matrices' tiles in three planes leave LDS for fewer groups)
    if (p.K >= 256 && (p.M <= 32 || tiles(64, 64) <= 128)) return launch_shape<AnyTile<T, 32, 64, 1, 2, false, true, 2, sizeof(T) == 4 ? 4 : 8>, T, GRAD>(p, parts, st);
    if (p.K >= 256 && tiles(64, 64) <= 256) return launch_shape<AnyTile<T, 64, 64, 2, 2, false, true, 2, sizeof(T) == 4 ? 2 : 4>, T, GRAD>(p, parts, st);
    return launch_shape<AnyTile<T, 64, 64, 2, 2, false, true, 2>, T, GRAD>(p, parts, st);
}
template <bool GRAD>
static int launch_gated(const GatedArgs &p, int dtype, int64_t *parts, hipStream_t st)
{
    return dtype == CSGS_F32 ? launch_types<float, GRAD>(p, parts, st) : launch_types<uint16_t, GRAD>(p, parts, st);
}

static int check(const csgs_gated_args *p, GatedArgs *a)
{
    if (!p || p->M <= 0 || p->K <= 0 || p->N <= 0 || !p->x || !p->wg || !p->wu || p->ldx < p->K || p->ldwg < p->N || p->ldwu < p->N) return CSGS_EINVAL;
    if (p->act < CSGS_ACT_NONE || p->act > CSGS_ACT_GELU) return CSGS_EINVAL;
    if (p->dtype != CSGS_F32 && p->dtype != CSGS_BF16) return CSGS_EUNSUPPORTED;
    *a = GatedArgs{};
    a->x = Operand{p->x, p->ldx};
    a->w[0] = Operand{p->wg, p->ldwg};
    a->w[1] = Operand{p->wu, p->ldwu};
    a->M = p->M;
    a->K = p->K;
    a->N = p->N;
    a->act = p->act;
    a->M_dev = p->M_dev;
    a->b[0] = p->bg;
    a->b[1] = p->bu;
    return CSGS_OK;
}

// What both calls read, as memory.
struct GatedMemory {
    Memory x, wg, wu, bg, bu, count;
    explicit GatedMemory(const csgs_gated_args *p)
        : x(matrix_of(p->dtype, p->x, p->M, p->K, p->ldx)), wg(matrix_of(p->dtype, p->wg, p->K, p->N, p->ldwg)), wu(matrix_of(p->dtype, p->wu, p->K, p->N, p->ldwu)),
          bg(vector_of(p->bg, p->N)), bu(vector_of(p->bu, p->N)), count(count_of(p->M_dev))
    {
    }
};

struct GatedScratch {
    void *t[2];
    float *columns[2], *parts;
    size_t bytes;
};
static GatedScratch carve_gated(void *base, int32_t M, int32_t K, int32_t N, int dtype)
{
    GatedScratch s;
    size_t off = 0;
    for (int i = 0; i < 2; ++i) {
        s.t[i] = (char *)base + off;
        off = align_up(off + (size_t)M * (size_t)N * (dtype == CSGS_F32 ? 4 : 2), 256);
    }
    for (int i = 0; i < 2; ++i) {
        s.columns[i] = (float *)((char *)base + off);
        off = align_up(off + (size_t)column_parts(M) * (size_t)N * 4, 256);
    }
    s.parts = (float *)((char *)base + off);
    const int64_t dx = out_product_floats(M, K, N, 1), dw = out_product_floats(K, N, M, 2);
    s.bytes = align_up(off + (size_t)(dx > dw ? dx : dw) * 4, 256);
    return s;
}

}  // namespace csgs

using namespace csgs;

extern "C" int csgs_gated(const csgs_gated_args *p, void *h, int64_t ldh, void *stream)
{
    GatedArgs a;
    const int rc = check(p, &a);
    if (rc != CSGS_OK) return rc;
    if (!h || ldh < p->N) return CSGS_EINVAL;
    const GatedMemory at(p);
    const Memory out = matrix_of(p->dtype, h, p->M, p->N, ldh);
    if (spans_too_much({at.x, at.wg, at.wu, out})) return CSGS_EUNSUPPORTED;
    if (!outputs_apart({at.x, at.wg, at.wu, at.bg, at.bu, at.count}, {out})) return CSGS_EINVAL;
    a.h = h;
    a.ldh = ldh;
    int64_t parts;
    return launch_gated<false>(a, p->dtype, &parts, (hipStream_t)stream);
}

extern "C" size_t csgs_gated_grad_scratch_bytes(int32_t M, int32_t K, int32_t N, int dtype)
{
    if (M <= 0 || K <= 0 || N <= 0 || (dtype != CSGS_F32 && dtype != CSGS_BF16)) return 0;
    return carve_gated(nullptr, M, K, N, dtype).bytes;
}

extern "C" int csgs_gated_grad(const csgs_gated_args *p, const void *dh, int64_t lddh, void *dx, int64_t lddx, void *dwg, int64_t lddwg, void *dwu, int64_t lddwu,
                               float *dbg, float *dbu, void *scratch, size_t scratch_bytes, void *stream)
{
    GatedArgs a;
    int rc = check(p, &a);
    if (rc != CSGS_OK) return rc;
    if (!dh || lddh < p->N || (dx && lddx < p->K) || (dwg && lddwg < p->N) || (dwu && lddwu < p->N)) return CSGS_EINVAL;
    if ((!dx && !dwg && !dwu && !dbg && !dbu) || (dbg && !p->bg) || (dbu && !p->bu)) return CSGS_EINVAL;
    const GatedMemory at(p);
    const Memory in = matrix_of(p->dtype, dh, p->M, p->N, lddh), out_x = matrix_of(p->dtype, dx, p->M, p->K, lddx), out_g = matrix_of(p->dtype, dwg, p->K, p->N, lddwg),
                 out_u = matrix_of(p->dtype, dwu, p->K, p->N, lddwu), out_bg = vector_of(dbg, p->N), out_bu = vector_of(dbu, p->N);
    if (spans_too_much({at.x, at.wg, at.wu, in, out_x, out_g, out_u})) return CSGS_EUNSUPPORTED;
    if (!outputs_apart({at.x, at.wg, at.wu, at.bg, at.bu, at.count, in}, {out_x, out_g, out_u, out_bg, out_bu})) return CSGS_EINVAL;
    if (!scratch || ((uintptr_t)scratch & 255)) return CSGS_EINVAL;
    const GatedScratch s = carve_gated(scratch, p->M, p->K, p->N, p->dtype);
    if (scratch_bytes < s.bytes) return CSGS_EWORKSPACE;
    if (!outputs_apart({at.x, at.wg, at.wu, at.bg, at.bu, at.count, in, out_x, out_g, out_u, out_bg, out_bu}, {Memory{scratch, 1, (int64_t)s.bytes, 0}})) return CSGS_EINVAL;
    hipStream_t st = (hipStream_t)stream;
    a.dh = dh;
    a.lddh = lddh;
    a.ldt = p->N;
    a.t[0] = s.t[0];
    a.t[1] = s.t[1];
    a.columns[0] = dbg ? s.columns[0] : nullptr;
    a.columns[1] = dbu ? s.columns[1] : nullptr;
    int64_t parts;
    rc = launch_gated<true>(a, p->dtype, &parts, st);
    if (rc != CSGS_OK) return rc;
    if (dx) {
        OutProduct o{};
        for (int i = 0; i < 2; ++i) {
            o.a[i] = Operand{s.t[i], p->N};
            o.b[i] = a.w[i];
        }
        o.pairs = 2;
        o.outs = 1;
        o.out[0] = dx;
        o.ldo[0] = lddx;
        o.rows = p->M;
        o.cols = p->K;
        o.red = p->N;
        o.rows_dev = p->M_dev;
        o.scale = 1.0f;
        o.across = false;
        rc = launch_out_product(o, p->dtype, s.parts, st);
        if (rc != CSGS_OK) return rc;
    }
    if (dwg || dwu) {
        OutProduct o{};
        o.a[0] = a.x;
        void *out[2] = {dwg, dwu};
        const int64_t ld[2] = {lddwg, lddwu};
        for (int i = 0; i < 2; ++i)
            if (out[i]) {
                o.b[o.outs] = Operand{s.t[i], p->N};
                o.out[o.outs] = out[i];
                o.ldo[o.outs++] = ld[i];
            }
        o.pairs = 1;
        o.rows = p->K;
        o.cols = p->N;
        o.red = p->M;
        o.red_dev = p->M_dev;
        o.scale = 1.0f;
        o.across = true;
        rc = launch_out_product(o, p->dtype, s.parts, st);
        if (rc != CSGS_OK) return rc;
    }
    if (dbg) {
        rc = launch_join_columns(s.columns[0], parts, p->N, dbg, st);
        if (rc != CSGS_OK) return rc;
    }
    return dbu ? launch_join_columns(s.columns[1], parts, p->N, dbu, st) : CSGS_OK;
}
