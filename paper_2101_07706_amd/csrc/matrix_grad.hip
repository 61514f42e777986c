// Products of the gradients: da = t w^T (both operands with the reduction side by side) and dw = a^T t (both with the outer index side by side).
//
// dw's sums run over the rows, its output is small: few tiles, so that the sum is cut into parts, one a block, left in float and joined in double in their order (no atomics: two
// calls give the same bits).  Operands with the outer index side by side go to LDS as they lie and are transposed by the reads from there.  Bound by the matrix cores
// (65536 rows, 4096 by 1024 in bfloat16: da 606 us, 907 TFLOP/s, busy 47 % of the cycles; dw in 4 parts 470, 1170 TFLOP/s, busy 68 %, and their join 15: a block of dw forms 256 chunks of k
// between its start and its outputs, which nothing hides, one of da 16).
#include "products.hpp"
#include "direct_tile.hpp"
#include "split_tile.hpp"

namespace csgs {

struct OutArgs {
    Operand a[2], b[2];
    void *out[2];
    int64_t ldo[2];
    int64_t rows, cols, red, part_len;
    const int32_t *rows_dev, *red_dev;
    int32_t pairs, parts, outs;
    float scale;
    float *part;
    int64_t tiles_m, tiles_n;
};

template <class Tile, typename T>
__global__ __launch_bounds__(Tile::THREADS, Tile::WAVES) void out_product_k(OutArgs p)
{
    constexpr int BM = Tile::ROWS, BN = Tile::COLS;
    __shared__ __attribute__((aligned(128))) char lds[Tile::LDS_BYTES];
    int64_t tm, tn;
    tile_place(blockIdx.x, p.tiles_m, p.tiles_n, &tm, &tn);
    const int64_t m0 = tm * BM, n0 = tn * BN;
    const int64_t rows = p.rows_dev ? live_rows((int32_t)p.rows, p.rows_dev) : p.rows, red = p.red_dev ? live_rows((int32_t)p.red, p.red_dev) : p.red;
    if (m0 >= rows) return;
    const int which = (int)blockIdx.z;
    const int64_t k0 = (int64_t)blockIdx.y * p.part_len, end = k0 + p.part_len, k1 = end < red ? end : red;
    Tile tile;
    form_sums(tile, lds, [&](auto &t) CSGS_INLINE {
        for (int i = 0; i < p.pairs; ++i) t.accumulate(lds, p.a[i], &p.b[p.outs > 1 ? which : i], m0, rows, n0, p.cols, k0, k1);
    });
    float *part = p.part ? p.part + ((int64_t)which * p.parts + blockIdx.y) * p.rows * p.cols : nullptr;
    const int mine = Tile::my_column(), left = (int)(p.cols - n0 < BN ? p.cols - n0 : BN) - mine, count = left < 0 ? 0 : left < 4 ? left : 4;
    const int high = (int)(rows - m0 < BM ? rows - m0 : BM);
    const auto none = [](int, int) CSGS_INLINE { return Nothing{}; };
    if (part)
        tile.each(lds, none, [&](int m, int n, const float(&v)[1][4], Nothing) CSGS_INLINE {
            if (m < high && count) store_some(part + (m0 + m) * p.cols + n0 + n, count, v[0]);
        });
    else
        tile.each(lds, none, [&](int m, int n, const float(&v)[1][4], Nothing) CSGS_INLINE {
            float x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = p.scale * v[0][i];
            if (m < high && count) store_some((T *)p.out[which] + (m0 + m) * p.ldo[which] + n0 + n, count, x);
        });
}

// out = scale * the sum of the parts, in double in their order.
template <typename T>
__global__ __launch_bounds__(256) void join_parts_k(const float *__restrict__ part, int32_t parts, int64_t rows, int64_t cols, const int32_t *rows_dev, float scale,
                                                    OutArgs p)
{
    const int which = (int)blockIdx.y;
    const int64_t live = rows_dev ? live_rows((int32_t)rows, rows_dev) : rows, quads = (cols + 3) / 4, n = live * quads, stride = rows * cols;
    const float *from = part + (int64_t)which * parts * stride;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / quads, col = (i - row * quads) * 4, rest = cols - col;
        const int count = rest < 4 ? (int)rest : 4;
        double s[4] = {0.0, 0.0, 0.0, 0.0};
        for (int32_t k = 0; k < parts; ++k) {
            float x[4];
            load_some(from + k * stride + row * cols + col, count, x);
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e] += (double)x[e];
        }
        float x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = float_to_store<T>((double)scale * s[e]);
        store_some((T *)p.out[which] + row * p.ldo[which] + col, count, x);
    }
}

constexpr int JOIN_ROWS = 16;
__global__ __launch_bounds__(64 * JOIN_ROWS) void join_columns_k(const float *__restrict__ part, int64_t parts, int32_t n, float *__restrict__ out)
{
    __shared__ double lds[JOIN_ROWS][64];
    const int lane = (int)threadIdx.x & 63, group = (int)threadIdx.x >> 6;
    const int64_t col = (int64_t)blockIdx.x * 64 + lane;
    double s = 0.0;
    if (col < n) {
        // (eight of a group's rows on their way at a time)
        int64_t p = group;
        for (; p + 7 * JOIN_ROWS < parts; p += 8 * JOIN_ROWS) {
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = part[(p + i * JOIN_ROWS) * n + col];
#pragma unroll
            for (int i = 0; i < 8; ++i) s += (double)x[i];
        }
        for (; p < parts; p += JOIN_ROWS) s += (double)part[p * n + col];
    }
    lds[group][lane] = s;
    __syncthreads();
    if (group == 0 && col < n) {
        for (int g = 1; g < JOIN_ROWS; ++g) s += lds[g][lane];
        out[col] = (float)s;
    }
}

int launch_join_columns(const float *part, int64_t parts, int32_t n, float *out, hipStream_t st)
{
    CSGS_LAUNCH(K_JOIN_COLUMNS, join_columns_k, dim3((unsigned)((n + 63) / 64)), dim3(64 * JOIN_ROWS), st, part, parts, n, out);
    CSGS_LAUNCH_CHECK();
    return CSGS_OK;
}

// Parts of a sum: each of at least PART_MIN terms, for at most PART_FLOATS floats beside one part.
constexpr int64_t PART_MIN = 512, PART_FLOATS = 16ll << 20;
int64_t out_product_floats(int64_t rows, int64_t cols, int64_t red, int outs)
{
    const int64_t one = rows * cols * outs, most = (red + PART_MIN - 1) / PART_MIN;
    return most > 1 + PART_FLOATS / one ? one + PART_FLOATS : most * one;
}
// The number of parts for which the rounds of blocks that the device holds at once (`slots`), times the length of a part, are fewest; of those within 5 % the fewest parts.
// (us, gradient of 4096 by 1024 on 65536 rows, 64 tiles: 4 parts, one round, 1158; 8 parts, two rounds, 1338.)
static int64_t parts_of(int64_t rows, int64_t cols, int64_t red, int outs, int64_t blocks, int64_t slots)
{
    const int64_t one = rows * cols * outs, room = 1 + PART_FLOATS / one;
    int64_t most = (red + PART_MIN - 1) / PART_MIN, best = 1;
    if (most > room) most = room;
    if (most > 2 * slots / blocks) most = 2 * slots / blocks;
    double least = (double)((blocks + slots - 1) / slots);
    for (int64_t n = 2; n <= most; ++n) {
        const double cost = (double)((blocks * n + slots - 1) / slots) / (double)n;
        if (cost < 0.95 * least) {
            least = cost;
            best = n;
        }
    }
    return best;
}

template <class Tile, typename T>
static int launch_shape(const OutProduct &p, float *parts, hipStream_t st)
{
    constexpr int BM = Tile::ROWS, BN = Tile::COLS;
    OutArgs a{};
    for (int i = 0; i < 2; ++i) {
        a.a[i] = p.a[i];
        a.b[i] = p.b[i];
        a.out[i] = p.out[i];
        a.ldo[i] = p.ldo[i];
    }
    a.rows = p.rows;
    a.cols = p.cols;
    a.red = p.red;
    a.rows_dev = p.rows_dev;
    a.red_dev = p.red_dev;
    a.pairs = p.pairs;
    a.outs = p.outs;
    a.scale = p.scale;
    a.tiles_m = (p.rows + BM - 1) / BM;
    a.tiles_n = (p.cols + BN - 1) / BN;
    const int64_t blocks = a.tiles_m * a.tiles_n;
    if (blocks > MOST_BLOCKS) return CSGS_EUNSUPPORTED;
    constexpr int64_t BK = Tile::BK;
    constexpr int64_t SLOTS = 256 * (Tile::LDS_BYTES > 80 * 1024 ? 1 : 2);
    int64_t n = parts_of(p.rows, p.cols, p.red, p.outs, blocks * p.outs, SLOTS);
    a.part_len = ((p.red + n - 1) / n + BK - 1) / BK * BK;
    n = (p.red + a.part_len - 1) / a.part_len;
    a.parts = (int32_t)n;
    a.part = n > 1 ? parts : nullptr;
    CSGS_LAUNCH(K_OUT_PRODUCT, (out_product_k<Tile, T>), dim3((unsigned)blocks, (unsigned)n, (unsigned)p.outs), dim3(Tile::THREADS), st, a);
    CSGS_LAUNCH_CHECK();
    if (n > 1) {
        const int64_t quads = p.rows * ((p.cols + 3) / 4), need = (quads + 255) / 256;
        CSGS_LAUNCH(K_JOIN_PARTS, join_parts_k<T>, dim3((unsigned)(need < 2048 ? need : 2048), (unsigned)p.outs), dim3(256), st, parts, a.parts, p.rows, p.cols, p.rows_dev,
                    p.scale, a);
        CSGS_LAUNCH_CHECK();
    }
    return CSGS_OK;
}

template <typename T, bool ACROSS>
static int launch_sides(const OutProduct &p, float *parts, hipStream_t st)
{
    const int64_t most = (p.red + PART_MIN - 1) / PART_MIN;
    const auto tiles = [&](int64_t m, int64_t n) { return (p.rows + m - 1) / m * ((p.cols + n - 1) / n) * p.outs; };
    if constexpr (sizeof(T) == 2) {
        // As for the forward products, and where the parts of a long sum make up for few tiles (us, 1024 by 1024, tiles of 256 and of 128: da of 6400 rows 35 and 28, of 9600 30 and 45; dw
        // of 8192 rows, 16 tiles and 16 possible parts, 44 and 37, of 16384 54 and 58).
        bool direct = tiles(256, 256) > 128 || tiles(256, 256) * most >= 512;
        for (int i = 0; direct && i < 2; ++i) {
            if (i < p.pairs) direct = direct_operand(p.a[i], ACROSS, p.rows, p.red, 256);
            if (direct && (i < p.pairs || i < p.outs)) direct = direct_operand(p.b[i], ACROSS, p.cols, p.red, 256);
        }
        if (direct) return launch_shape<DirectTile<256, 256, 2, 4, ACROSS, ACROSS, 1, 128, 2>, T>(p, parts, st);
    }
    // (us, floats, 512 by 512, tiles of 128 and of 64: da of 8192 rows, 256 tiles, 41 and 35, dw of 16384 rows, 16 tiles and 32 possible parts, 68 and 79; gradient of 4001 rows of 602 by
    // 1111 with both matrices, da 160 tiles and 3 possible parts, 272 and 291)
    if (tiles(128, 128) * most >= 384) return launch_shape<AnyTile<T, 128, 128, 2, 2, ACROSS, ACROSS, 1>, T>(p, parts, st);
    // (four groups of wavefronts take a tile's chunks in turn; us, without and with: da of 1024 rows, 256 columns, sums of 1024, floats 23 and 16, of 4096 rows, 512 tiles and parts, 29 and 23;
    // dw of 1400 rows of 37 by 6 23 and 13; of 4096 rows of 256 by 256 in bfloat16 12.4 and 12.4)
    if (tiles(64, 64) * most <= 512) return launch_shape<AnyTile<T, 64, 64, 2, 2, ACROSS, ACROSS, 1, 4>, T>(p, parts, st);
    return launch_shape<AnyTile<T, 64, 64, 2, 2, ACROSS, ACROSS, 1>, T>(p, parts, st);
}

int launch_out_product(const OutProduct &p, int dtype, float *parts, hipStream_t st)
{
    if (dtype == CSGS_F32) return p.across ? launch_sides<float, true>(p, parts, st) : launch_sides<float, false>(p, parts, st);
    return p.across ? launch_sides<uint16_t, true>(p, parts, st) : launch_sides<uint16_t, false>(p, parts, st);
}

}  // namespace csgs
