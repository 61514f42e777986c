// csgs_norm_residual: y = beta x + alpha a(gate) .* N(h), u = N(y) per row, and its gradient.
//
// With hat(v) = (v - m) r, r = 1 / sqrt(mean((v - m)^2) + eps), N(v) = w .* hat(v) + b, and t the gradient of hat(v), the gradient of v is
//     r (t - mean(t) - hat .* mean(t .* hat))          (RMS: without mean(t))
// so with d = dL/dy as a whole = dy + the gradient through u's norm, n = N(h), a = a(gate):
//     dx = beta d,   dgate = alpha d .* n .* a'(gate),   dn = alpha d .* a,   dh = the gradient through h's norm of dn,
//     dpost_w = sum over rows of dn .* hat(h),  dpost_b = sum dn,  dpre_w = sum du .* hat(y),  dpre_b = sum du.
// The gradient forms everything again from the forward's inputs: reading x again costs the same bytes as reading y, and no statistics need
// be kept.  Row sums, statistics and everything between are in fp32, one rounding per output.  Both directions move a few bytes per operation:
// bound by memory where there are many rows (us and TB/s of what has to move; a large copy reaches 4.8 to 5.2: 131072 rows of 256 floats 129, 5.2; gradient
// of 65536 rows of 1024, stream in floats, block in bfloat16, 290, 5.1; of 16384 rows of 2048 floats 201, 5.3; of 8192 rows of 4096 in bfloat16 143, 3.8; of
// 4096 rows of 8192 floats 282, 3.8),
// by the latency of a row's loads and of four to six sums over it one after the other where there are few (256 rows of 64 3.1; gradient of 8192
// rows of 256 17.9, of 1999 rows of 602 15.9, two launches each).  Times that stand beside a choice below are those it was made by; the present gates take 1.4 % more.
#include "common.hpp"
#include "row_pieces.hpp"

namespace csgs {

// Two forms: rows in registers (residual_rows_k), and rows walked over several times (residual_k), for fewer columns than a piece and more than the
// registers of a block hold.

struct ResidualArgs {
    int32_t M, F;
    const int32_t *M_dev;
    const void *x, *h, *gate;
    int64_t ldx, ldh, ldg;
    const float *post_w, *post_b, *pre_w, *pre_b;
    int32_t post, pre, act;
    float eps, alpha, beta;
};

// a(g) and its derivative.  e = exp(-g) = 2^t exp(-g - t ln 2) with t = -g log2(e) rounded: the second factor is 1 plus a difference that an fma gives whole, so
// that the rounding of t, |g| halves of an ulp of e, does not stay in it.  s(g) = 1 / (1 + e), 1 - s(g) = e / (1 + e): not by a difference, which would lose
// the derivative of a gate that is nearly open.  The hardware's exponential and reciprocal are within an ulp: s is within 8 * 2^-24 of itself, s (1 - s) within 13,
// and |g| / 20 more by what a float leaves of ln 2 (s below 2^-126: 0).  fminf gives its other argument for NaN: where e is infinite or g is, there is nothing to
// correct, and 1 - s is 1.  (Geometric mean over 64 sizes and gates, both directions: 1.4 % more time than by __expf(-g) and s (1 - s), at most 4 to 5 %; by expf 8 %.)
struct Gate {
    float a, da;
};
__device__ inline Gate gate_of(float g, int32_t act)
{
    if (act == CSGS_GATE_LINEAR) return Gate{g, 1.0f};
    const float t = g * -1.44269504f;
    const float e = __builtin_amdgcn_exp2f(t) * fminf(1.0f + fmaf(t, -0.693147181f, -g), 2.0f);
    const float s = __builtin_amdgcn_rcpf(1.0f + e), rest = fminf(e * s, 1.0f);
    if (act == CSGS_GATE_SIGMOID) return Gate{s, s * rest};
    return Gate{g * s, s * (1.0f + g * rest)};
}

constexpr int RES_BLOCK = 256;
// Sum over the block, the same in every thread.
__device__ inline float block_sum(float v, float *lds /*[RES_BLOCK / WAVE]*/)
{
#pragma unroll
    for (int s = WAVE / 2; s > 0; s >>= 1) v += __shfl_xor(v, s);
    __syncthreads();
    if (lane_id() == 0) lds[threadIdx.x / WAVE] = v;
    __syncthreads();
    float r = 0.0f;
#pragma unroll
    for (int w = 0; w < RES_BLOCK / WAVE; ++w) r += lds[w];
    return r;
}

struct Stats {
    float m, r;
};
// Mean and 1 / deviation of the values v(f) of a row.
template <typename V>
__device__ inline Stats row_stats(V v, int32_t F, int32_t kind, float eps, float *lds)
{
    if (kind == CSGS_NORM_NONE) return Stats{0.0f, 1.0f};
    float m = 0.0f;
    if (kind == CSGS_NORM_LAYER) {
        float s = 0.0f;
        for (int32_t f = (int32_t)threadIdx.x; f < F; f += RES_BLOCK) s += v(f);
        m = block_sum(s, lds) / (float)F;
    }
    float q = 0.0f;
    for (int32_t f = (int32_t)threadIdx.x; f < F; f += RES_BLOCK) {
        const float c = v(f) - m;
        q += c * c;
    }
    return Stats{m, 1.0f / sqrtf(block_sum(q, lds) / (float)F + eps)};
}

// A row's inputs as functions of the column.
template <typename TS, typename TB>
struct Row {
    const ResidualArgs &a;
    int64_t r;
    Stats h_stats;
    __device__ float x(int32_t f) const { return a.x ? load_row<TS, 1>((const TS *)a.x + r * a.ldx + f).x[0] : 0.0f; }
    __device__ float h(int32_t f) const { return load_row<TB, 1>((const TB *)a.h + r * a.ldh + f).x[0]; }
    __device__ Gate gate(int32_t f) const
    {
        if (!a.gate) return Gate{1.0f, 0.0f};
        const float g = a.ldg ? load_row<TB, 1>((const TB *)a.gate + r * a.ldg + f).x[0] : ((const float *)a.gate)[f];
        return gate_of(g, a.act);
    }
    __device__ float hat(int32_t f) const { return (h(f) - h_stats.m) * h_stats.r; }
    __device__ float n(int32_t f) const { return hat(f) * (a.post_w ? a.post_w[f] : 1.0f) + (a.post_b ? a.post_b[f] : 0.0f); }
    __device__ float y(int32_t f) const { return a.beta * x(f) + (a.h ? a.alpha * gate(f).a * n(f) : 0.0f); }
};

// A block takes a row and reads it from memory or the caches each time it is needed (4096 rows of 8192 floats 371 us, rows in registers 137).
template <typename TS, typename TB>
__global__ __launch_bounds__(RES_BLOCK) void residual_k(ResidualArgs a, TS *y, int64_t ldy, TB *u, int64_t ldu)
{
    __shared__ float lds[RES_BLOCK / WAVE];
    const int32_t M = resolve_count(a.M, a.M_dev);
    for (int64_t r = blockIdx.x; r < M; r += gridDim.x) {
        Row<TS, TB> row{a, r, Stats{0.0f, 1.0f}};
        if (a.h) row.h_stats = row_stats([&](int32_t f) { return row.h(f); }, a.F, a.post, a.eps, lds);
        Stats s{0.0f, 1.0f};
        if (u) s = row_stats([&](int32_t f) { return row.y(f); }, a.F, a.pre, a.eps, lds);
        __syncthreads();   // an output may lie on an input: everybody has read the row
        for (int32_t f = (int32_t)threadIdx.x; f < a.F; f += RES_BLOCK) {
            const float v = row.y(f);
            if (u) store_row<TB, 1>(u + r * ldu + f, Vec<1>{{(v - s.m) * s.r * (a.pre_w ? a.pre_w[f] : 1.0f) + (a.pre_b ? a.pre_b[f] : 0.0f)}});
            if (y) store_row<TS, 1>(y + r * ldy + f, Vec<1>{{v}});
        }
    }
}

// ---------------------------------------------------------------- rows in registers
// G lanes take a row, N pieces of V columns each; what a lane holds of the vectors (weights, sums over rows) stays in registers
// from row to row.  Rows start on any element.  RAGGED: V does not divide the width; the last piece then ends with the row and
// overlaps the one before: the values that both hold are computed twice, alike, and count once in sums.  All of a row's inputs are asked for
// before any is widened: with a piece widened where it was loaded the branches waited for each other's loads (gradient of 65536 rows of 1024
// in mixed types 438 us for 302).

// Sum over the G lanes of a row, the same bits in each of them: every step adds two lanes' values that are each other's
// counterparts, first in fours (quad_perm), then mirrored in eights and rows of 16, then rows and halves of the wavefront exchanged.
template <int CTRL>
__device__ inline float add_counterpart(float v)
{
    return v + __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xF, 0xF, true));
}
template <int G>
__device__ inline float lanes_sum(float v)
{
    static_assert(G >= 4, "lanes of a row");
    v = add_counterpart<0xB1>(v);                            // quad_perm:[1,0,3,2]
    v = add_counterpart<0x4E>(v);                            // quad_perm:[2,3,0,1]
    if constexpr (G >= 8) v = add_counterpart<0x141>(v);     // row_half_mirror
    if constexpr (G >= 16) v = add_counterpart<0x140>(v);    // row_mirror
    if constexpr (G >= 32) {
        const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(p[0]) + __uint_as_float(p[1]);
    }
    if constexpr (G >= 64) {
        const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(p[0]) + __uint_as_float(p[1]);
    }
    return v;
}
// Sums of K values over a row's lanes; with G above 64 over the block, through LDS (turn: the two halves of `lds` in turn, so that one barrier a
// sum is enough).
template <int G, int K>
__device__ inline void row_sums(float (&v)[K], float *lds /*[2][G / WAVE][2]*/, int &turn)
{
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = lanes_sum<G>(v[k]);
    if constexpr (G > WAVE) {
        float *l = lds + turn * (2 * G / WAVE);
        turn ^= 1;
        if (lane_id() == 0)
#pragma unroll
            for (int k = 0; k < K; ++k) l[2 * (threadIdx.x / WAVE) + k] = v[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            v[k] = l[k];
#pragma unroll
            for (int w = 1; w < G / WAVE; ++w) v[k] += l[2 * w + k];
        }
    }
}
// Threads of a block: rows of up to 64 lanes share one.
template <int G>
constexpr int row_block() { return G > WAVE ? G : RES_BLOCK; }

// The columns that a lane holds: piece n begins at col(n); its first skip(n) values belong to the piece before.
template <int V, int G, int N, bool RAGGED>
struct Cols {
    int32_t F;
    int lane;   // of the row's
    __device__ int32_t begin(int n) const { return (lane + n * G) * V; }
    __device__ bool active(int n) const { return begin(n) < F; }
    __device__ int32_t col(int n) const { return RAGGED && begin(n) > F - V ? F - V : begin(n); }
    __device__ int32_t skip(int n) const { return RAGGED ? begin(n) - col(n) : 0; }
    // Lanes without a piece read the row's last one again.
    __device__ int32_t load_col(int n) const { return begin(n) > F - V ? F - V : begin(n); }
    template <typename T>
    __device__ void ask(RawPiece<T, V> (&p)[N], const T *row) const
    {
#pragma unroll
        for (int n = 0; n < N; ++n) p[n].load(row + load_col(n));
    }
    template <typename T>
    __device__ void widen(float (&v)[N * V], const RawPiece<T, V> (&p)[N]) const
    {
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int i = 0; i < V; ++i) v[n * V + i] = p[n].value(i);
    }
    __device__ void load_or(float (&v)[N * V], const float *row, float otherwise) const
    {
        if (row) {
            RawPiece<float, V> p[N];
            ask(p, row);
            return widen(v, p);
        }
#pragma unroll
        for (int i = 0; i < N * V; ++i) v[i] = otherwise;
    }
    template <typename T>
    __device__ void store(T *row, const float (&v)[N * V]) const
    {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            Vec<V> p;
#pragma unroll
            for (int i = 0; i < V; ++i) p.x[i] = v[n * V + i];
            if (active(n)) store_row<T, V>(row + col(n), p);
        }
    }
    // Sum of term(i) over the lane's own values.
    template <typename T>
    __device__ float sum(T term) const
    {
        float s = 0.0f;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            float p = 0.0f;
            const int32_t sk = skip(n);
#pragma unroll
            for (int i = 0; i < V; ++i) p += RAGGED && i < sk ? 0.0f : term(n * V + i);
            s += active(n) ? p : 0.0f;
        }
        return s;
    }
};

// Mean and 1 / deviation of a row.
template <int G, typename C, int NV>
__device__ inline Stats stats_of(const float (&v)[NV], const C &c, float inv_F, int32_t kind, float eps, float *lds, int &turn)
{
    if (kind == CSGS_NORM_NONE) return Stats{0.0f, 1.0f};
    float m[1] = {0.0f}, q[1];
    if (kind == CSGS_NORM_LAYER) {
        m[0] = c.sum([&](int i) { return v[i]; });
        row_sums<G>(m, lds, turn);
        m[0] *= inv_F;
    }
    q[0] = c.sum([&](int i) { return (v[i] - m[0]) * (v[i] - m[0]); });
    row_sums<G>(q, lds, turn);
    return Stats{m[0], rsqrtf(q[0] * inv_F + eps)};
}

template <typename TS, typename TB, int V, int G, int N, bool RAGGED>
__global__ __launch_bounds__(row_block<G>()) void residual_rows_k(ResidualArgs a, TS *y, int64_t ldy, TB *u, int64_t ldu)
{
    constexpr int NV = N * V;
    __shared__ float lds[4 * row_block<G>() / WAVE];
    int turn = 0;
    const int32_t M = resolve_count(a.M, a.M_dev);
    const Cols<V, G, N, RAGGED> c{a.F, (int)threadIdx.x % G};
    const float inv_F = 1.0f / (float)a.F;
    float pw[NV], pb[NV], qw[NV], qb[NV], gv[NV];
    c.load_or(pw, a.post_w, 1.0f);
    c.load_or(pb, a.post_b, 0.0f);
    c.load_or(qw, a.pre_w, 1.0f);
    c.load_or(qb, a.pre_b, 0.0f);
    c.load_or(gv, a.gate && !a.ldg ? (const float *)a.gate : nullptr, 0.0f);
    constexpr int ROWS = row_block<G>() / G;
    const int group = (int)threadIdx.x / G;
    for (int64_t r0 = (int64_t)blockIdx.x * ROWS; r0 < M; r0 += (int64_t)gridDim.x * ROWS) {
        const bool live = r0 + group < M;
        const int64_t r = live ? r0 + group : M - 1;
        float v[NV], h[NV];
        RawPiece<TS, V> rx[N];
        RawPiece<TB, V> rh[N], rg[N];
        if (a.h) c.ask(rh, (const TB *)a.h + r * a.ldh);
        if (a.ldg) c.ask(rg, (const TB *)a.gate + r * a.ldg);
        if (a.x) c.ask(rx, (const TS *)a.x + r * a.ldx);
        c.widen(h, rh);
        if (a.ldg) c.widen(gv, rg);
        c.widen(v, rx);
#pragma unroll
        for (int i = 0; i < NV; ++i) v[i] = a.x ? a.beta * v[i] : 0.0f;
        if (a.h) {
            const Stats s = stats_of<G>(h, c, inv_F, a.post, a.eps, lds, turn);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const float n = (h[i] - s.m) * s.r * pw[i] + pb[i];
                v[i] += a.alpha * (a.gate ? gate_of(gv[i], a.act).a * n : n);
            }
        }
        Stats s{0.0f, 1.0f};
        if (u) s = stats_of<G>(v, c, inv_F, a.pre, a.eps, lds, turn);
        if (G > WAVE) __syncthreads();   // an output may lie on an input: everybody has read the row
        if (!live) continue;
        if (y) c.store(y + r * ldy, v);
        if (u) {
#pragma unroll
            for (int i = 0; i < NV; ++i) v[i] = (v[i] - s.m) * s.r * qw[i] + qb[i];
            c.store(u + r * ldu, v);
        }
    }
}

// Sums over rows: every block leaves one row of sums per vector, in fp32 over its share of the rows, which a second kernel adds up in double, in
// order.
enum { COL_POST_W = 0, COL_POST_B, COL_PRE_W, COL_PRE_B, COL_GATE, COL_KINDS };
constexpr int COL_BLOCKS = 1024;   // most blocks
__host__ inline int col_blocks(int32_t M) { return M < COL_BLOCKS ? M : COL_BLOCKS; }
// Blocks of the gradient with rows in registers: about as many as the device holds at a time, by the registers that N pieces take (us, 256 / 512 /
// 1024 / 1536 blocks: 8192 rows of 256, a piece a lane, 21.7 / 19.0 / 19.2 / 22.2; 1999 rows of 602, three pieces, 16.9 / 17.6 / 17.8 / 17.8; 256 / 512:
// 8192 rows of 4096, 512 lanes, 194 / 205).
template <int G, int N>
constexpr int grad_blocks() { return (G > WAVE && N == 1) || G == 128 || G < 32 ? 1024 : (G == 512 || (G == 64 && N >= 3) ? 256 : 512); }

struct ResidualGrad {
    const void *dy, *du;
    void *dx, *dh, *dgate;
    int64_t lddy, lddu, lddx, lddh, lddg;
    float *part;      // [COL_KINDS][blocks][F]
    int32_t want[COL_KINDS];
};

template <typename TS, typename TB>
__global__ __launch_bounds__(RES_BLOCK) void residual_grad_k(ResidualArgs a, ResidualGrad g)
{
    __shared__ float lds[RES_BLOCK / WAVE];
    const int32_t M = resolve_count(a.M, a.M_dev), F = a.F;
    auto part = [&](int k, int32_t f) -> float & { return g.part[((int64_t)k * gridDim.x + blockIdx.x) * F + f]; };
    for (int k = 0; k < COL_KINDS; ++k)
        if (g.want[k])
            for (int32_t f = (int32_t)threadIdx.x; f < F; f += RES_BLOCK) part(k, f) = 0.0f;
    for (int64_t r = blockIdx.x; r < M; r += gridDim.x) {
        Row<TS, TB> row{a, r, Stats{0.0f, 1.0f}};
        if (a.h) row.h_stats = row_stats([&](int32_t f) { return row.h(f); }, F, a.post, a.eps, lds);
        Stats s{0.0f, 1.0f};
        if (g.du) s = row_stats([&](int32_t f) { return row.y(f); }, F, a.pre, a.eps, lds);
        auto du = [&](int32_t f) { return load_row<TB, 1>((const TB *)g.du + r * g.lddu + f).x[0]; };
        auto du_w = [&](int32_t f) { return du(f) * (a.pre_w ? a.pre_w[f] : 1.0f); };
        auto y_hat = [&](int32_t f) { return (row.y(f) - s.m) * s.r; };
        float t1 = 0.0f, t2 = 0.0f;
        if (g.du) {
            for (int32_t f = (int32_t)threadIdx.x; f < F; f += RES_BLOCK) {
                const float t = du_w(f);
                t1 += t;
                t2 += t * y_hat(f);
            }
            t1 = a.pre == CSGS_NORM_LAYER ? block_sum(t1, lds) / (float)F : 0.0f;
            t2 = block_sum(t2, lds) / (float)F;
        }
        auto d = [&](int32_t f) {
            float v = g.dy ? load_row<TS, 1>((const TS *)g.dy + r * g.lddy + f).x[0] : 0.0f;
            if (g.du) v += s.r * (du_w(f) - t1 - y_hat(f) * t2);
            return v;
        };
        float p1 = 0.0f, p2 = 0.0f;
        if (a.h && a.post != CSGS_NORM_NONE) {
            for (int32_t f = (int32_t)threadIdx.x; f < F; f += RES_BLOCK) {
                const float t = a.alpha * d(f) * row.gate(f).a * (a.post_w ? a.post_w[f] : 1.0f);
                p1 += t;
                p2 += t * row.hat(f);
            }
            p1 = a.post == CSGS_NORM_LAYER ? block_sum(p1, lds) / (float)F : 0.0f;
            p2 = block_sum(p2, lds) / (float)F;
        }
        __syncthreads();
        for (int32_t f = (int32_t)threadIdx.x; f < F; f += RES_BLOCK) {
            const float v = d(f);
            if (g.want[COL_PRE_W]) part(COL_PRE_W, f) += du(f) * y_hat(f);
            if (g.want[COL_PRE_B]) part(COL_PRE_B, f) += du(f);
            if (a.h) {
                const Gate gt = row.gate(f);
                const float t = a.alpha * v, dn = t * gt.a, hat = row.hat(f), dg = t * row.n(f) * gt.da;
                const float dh = a.post != CSGS_NORM_NONE ? row.h_stats.r * (dn * (a.post_w ? a.post_w[f] : 1.0f) - p1 - hat * p2) : dn;
                if (g.want[COL_POST_W]) part(COL_POST_W, f) += dn * hat;
                if (g.want[COL_POST_B]) part(COL_POST_B, f) += dn;
                if (g.want[COL_GATE]) part(COL_GATE, f) += dg;
                if (g.dgate && a.ldg) store_row<TB, 1>((TB *)g.dgate + r * g.lddg + f, Vec<1>{{dg}});
                if (g.dh) store_row<TB, 1>((TB *)g.dh + r * g.lddh + f, Vec<1>{{dh}});
            }
            if (g.dx) store_row<TS, 1>((TS *)g.dx + r * g.lddx + f, Vec<1>{{a.beta * v}});
        }
    }
}

// The same with the row in registers.  BIAS: sums of post_b or pre_b are wanted; GATE_ROW: those of a gate for all rows.
template <typename TS, typename TB, int V, int G, int N, bool RAGGED, bool BIAS, bool GATE_ROW>
__global__ __launch_bounds__(row_block<G>(), 2) void residual_grad_rows_k(ResidualArgs a, ResidualGrad g)
{
    constexpr int NV = N * V, ROWS = row_block<G>() / G;
    __shared__ float lds[4 * row_block<G>() / WAVE];
    __shared__ float sums[ROWS > 1 ? ROWS : 1][ROWS > 1 ? G * NV : 1];
    int turn = 0;
    const int32_t M = resolve_count(a.M, a.M_dev);
    const Cols<V, G, N, RAGGED> c{a.F, (int)threadIdx.x % G};
    const float inv_F = 1.0f / (float)a.F;
    // (the vectors' weights: in registers, or of rows of many pieces in LDS, where each lane reads what it wrote: 24 to 48 registers fewer, of at most 256
    // that let a block of 512 be there at all and two of 256.  8192 rows of 4096 in bfloat16 217 us, 141 so)
    constexpr bool IN_LDS = G > WAVE && N >= 3;
    __shared__ float held[IN_LDS ? 3 : 1][IN_LDS ? G * NV : 1];
    float pw[IN_LDS ? 1 : NV], pb[IN_LDS ? 1 : NV], qw[IN_LDS ? 1 : NV], gv[NV], s_pw[NV], s_pb[BIAS ? NV : 1], s_qw[NV], s_qb[BIAS ? NV : 1], s_g[GATE_ROW ? NV : 1];
    auto place = [&](int i) { return i / V * (G * V) + (int)threadIdx.x % G * V + i % V; };
    auto keep = [&](auto &reg, int k, const float *row, float otherwise) {
        if constexpr (IN_LDS) {
            float t[NV];
            c.load_or(t, row, otherwise);
#pragma unroll
            for (int i = 0; i < NV; ++i) held[k][place(i)] = t[i];
        } else c.load_or(reg, row, otherwise);
    };
    keep(pw, 0, a.post_w, 1.0f);
    keep(pb, 1, a.post_b, 0.0f);
    keep(qw, 2, a.pre_w, 1.0f);
    auto post_w = [&](int i) { if constexpr (IN_LDS) return held[0][place(i)]; else return pw[i]; };
    auto post_b = [&](int i) { if constexpr (IN_LDS) return held[1][place(i)]; else return pb[i]; };
    auto pre_w = [&](int i) { if constexpr (IN_LDS) return held[2][place(i)]; else return qw[i]; };
    c.load_or(gv, a.gate && !a.ldg ? (const float *)a.gate : nullptr, 0.0f);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        s_pw[i] = s_qw[i] = 0.0f;
        if constexpr (BIAS) s_pb[i] = s_qb[i] = 0.0f;
        if constexpr (GATE_ROW) s_g[i] = 0.0f;
    }
    const int group = (int)threadIdx.x / G;
    for (int64_t r0 = (int64_t)blockIdx.x * ROWS; r0 < M; r0 += (int64_t)gridDim.x * ROWS) {
        const bool live = r0 + group < M;
        const int64_t r = live ? r0 + group : M - 1;
        float v[NV], h[NV], du[NV], d[NV];
        RawPiece<TS, V> rx[N], rdy[N];
        RawPiece<TB, V> rh[N], rg[N], rdu[N];
        if (a.h) c.ask(rh, (const TB *)a.h + r * a.ldh);
        if (a.ldg) c.ask(rg, (const TB *)a.gate + r * a.ldg);
        if (a.x) c.ask(rx, (const TS *)a.x + r * a.ldx);
        if (g.du) c.ask(rdu, (const TB *)g.du + r * g.lddu);
        if (g.dy) c.ask(rdy, (const TS *)g.dy + r * g.lddy);
        c.widen(h, rh);
        if (a.ldg) c.widen(gv, rg);
        c.widen(v, rx);
        c.widen(du, rdu);
        c.widen(d, rdy);
        if (!g.dy)
#pragma unroll
            for (int i = 0; i < NV; ++i) d[i] = 0.0f;
        Stats hs{0.0f, 1.0f};
        if (a.h) hs = stats_of<G>(h, c, inv_F, a.post, a.eps, lds, turn);
#pragma unroll
        for (int i = 0; i < NV; ++i) h[i] = a.h ? (h[i] - hs.m) * hs.r : 0.0f;   // from here on hat(h)
        constexpr int KEPT = N == 1 ? NV : 1;
        Gate kept[KEPT];   // where there are registers for it
        if (N == 1 && a.gate)
#pragma unroll
            for (int i = 0; i < KEPT; ++i) kept[i] = gate_of(gv[i], a.act);
        if (g.du) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                v[i] = a.x ? a.beta * v[i] : 0.0f;
                if (a.h) {
                    const float n = h[i] * post_w(i) + post_b(i);
                    v[i] += a.alpha * (a.gate ? (N == 1 ? kept[i % KEPT] : gate_of(gv[i], a.act)).a * n : n);
                }
            }
            const Stats s = stats_of<G>(v, c, inv_F, a.pre, a.eps, lds, turn);
#pragma unroll
            for (int i = 0; i < NV; ++i) v[i] = (v[i] - s.m) * s.r;              // hat(y)
            float t[2];
            t[0] = c.sum([&](int i) { return du[i] * pre_w(i) * v[i]; });
            t[1] = a.pre == CSGS_NORM_LAYER ? c.sum([&](int i) { return du[i] * pre_w(i); }) : 0.0f;
            row_sums<G>(t, lds, turn);
            t[0] *= inv_F;
            t[1] *= inv_F;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                d[i] += s.r * (du[i] * pre_w(i) - t[1] - v[i] * t[0]);
            }
            if (live)
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    s_qw[i] += du[i] * v[i];
                    if constexpr (BIAS) s_qb[i] += du[i];
                }
        }
        float t[2] = {0.0f, 0.0f};
        if (a.h) {
            // dn in v (hat(y) is done with), dgate in du
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const float e = a.alpha * d[i];
                Gate gt{1.0f, 0.0f};
                if (a.gate) gt = N == 1 ? kept[i % KEPT] : gate_of(gv[i], a.act);
                v[i] = e * gt.a;
                du[i] = e * (h[i] * post_w(i) + post_b(i)) * gt.da;
            }
            if (live)
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    s_pw[i] += v[i] * h[i];
                    if constexpr (BIAS) s_pb[i] += v[i];
                    if constexpr (GATE_ROW) s_g[i] += du[i];
                }
#pragma unroll
            for (int i = 0; i < NV; ++i) v[i] *= post_w(i);
            if (a.post != CSGS_NORM_NONE) {
                t[0] = c.sum([&](int i) { return v[i] * h[i]; });
                t[1] = a.post == CSGS_NORM_LAYER ? c.sum([&](int i) { return v[i]; }) : 0.0f;
                row_sums<G>(t, lds, turn);
                t[0] *= inv_F;
                t[1] *= inv_F;
            }
        }
        if (G > WAVE) __syncthreads();
        if (!live) continue;
        if (a.h) {
            if (g.dgate && a.ldg) c.store((TB *)g.dgate + r * g.lddg, du);
            if (g.dh) {
#pragma unroll
                for (int i = 0; i < NV; ++i) v[i] = a.post != CSGS_NORM_NONE ? hs.r * (v[i] - t[1] - h[i] * t[0]) : v[i];
                c.store((TB *)g.dh + r * g.lddh, v);
            }
        }
        if (g.dx) {
#pragma unroll
            for (int i = 0; i < NV; ++i) d[i] *= a.beta;
            c.store((TS *)g.dx + r * g.lddx, d);
        }
    }
    // sums over the block's rows
    auto leave = [&](int k, const float (&v)[NV]) {
        if (!g.want[k]) return;
        float *part = g.part + ((int64_t)k * gridDim.x + blockIdx.x) * a.F;
        if constexpr (ROWS == 1) {
            c.store(part, v);
        } else {
            __syncthreads();
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (c.active(n)) sums[group][c.col(n) + i] = v[n * V + i];
            __syncthreads();
            for (int32_t f = (int32_t)threadIdx.x; f < a.F; f += RES_BLOCK) {
                float s = sums[0][f];
#pragma unroll 16
                for (int w = 1; w < ROWS; ++w) s += sums[w][f];
                part[f] = s;
            }
        }
    };
    leave(COL_POST_W, s_pw);
    leave(COL_PRE_W, s_qw);
    if constexpr (BIAS) {
        leave(COL_POST_B, s_pb);
        leave(COL_PRE_B, s_qb);
    }
    if constexpr (GATE_ROW) leave(COL_GATE, s_g);
}

struct ColOut {
    float *out[COL_KINDS];
};
// A block takes 64 columns of a vector; its wavefronts take the parts in turn.  (512 parts of 256 columns 4 us, a launch's latency.)
constexpr int COL_WAVES = 16;
__global__ __launch_bounds__(COL_WAVES * WAVE) void col_sums_k(const float *__restrict__ part, int blocks, int32_t F, ColOut o)
{
    __shared__ double lds[COL_WAVES][WAVE];
    const int k = (int)blockIdx.y, wave = (int)threadIdx.x / WAVE, lane = lane_id();
    if (!o.out[k]) return;
    const int32_t f = (int32_t)blockIdx.x * WAVE + lane;
    double s = 0.0;
    if (f < F) {
        const float *p = part + (int64_t)k * blocks * F + f;
#pragma unroll 8
        for (int b = wave; b < blocks; b += COL_WAVES) s += (double)p[(int64_t)b * F];
    }
    lds[wave][lane] = s;
    __syncthreads();
    if (wave != 0 || f >= F) return;
#pragma unroll
    for (int w = 1; w < COL_WAVES; ++w) s += lds[w][lane];
    o.out[k][f] = (float)s;
}

static int open_residual(const csgs_residual *r, ResidualArgs *a)
{
    if (!r || r->M <= 0 || r->F <= 0 || (!r->x && !r->h) || (r->x && r->ldx < r->F) || (r->h && r->ldh < r->F) || (r->gate && !r->h) ||
        (r->gate && r->ldg != 0 && r->ldg < r->F) || !(r->eps >= 0.0f) || r->post < CSGS_NORM_NONE || r->post > CSGS_NORM_LAYER ||
        r->pre < CSGS_NORM_NONE || r->pre > CSGS_NORM_LAYER || r->gate_act < CSGS_GATE_LINEAR || r->gate_act > CSGS_GATE_SILU)
        return CSGS_EINVAL;
    const bool same = r->x_dtype == r->h_dtype && (r->x_dtype == CSGS_F32 || r->x_dtype == CSGS_BF16);
    if ((!same && !(r->x_dtype == CSGS_F32 && r->h_dtype == CSGS_BF16)) || r->F > 1 << 30) return CSGS_EUNSUPPORTED;   // (a column and a block's step in 32 bits)
    *a = ResidualArgs{r->M, r->F, r->M_dev, r->x, r->h, r->gate, r->ldx, r->ldh, r->gate ? r->ldg : 0, r->post_w, r->post_b, r->pre_w, r->pre_b,
                      r->post, r->pre, r->gate_act, r->eps, r->alpha, r->beta};
    if (a->post == CSGS_NORM_NONE) a->post_w = a->post_b = nullptr;
    if (a->pre == CSGS_NORM_NONE) a->pre_w = a->pre_b = nullptr;
    return CSGS_OK;
}

// Calls f with the row's layout as constants: lanes, pieces a lane, and whether the width is no multiple of a piece.  As few lanes as hold the row
// in one piece, then up to three pieces a lane, then a block per row, of as few lanes as that takes: what counts there is how many rows a compute unit
// holds and how many lanes have nothing to do (us, gradient: 1999 rows of 602, 64 lanes with three pieces 16.9, 256 with one 21; 24000 rows of 1100 in
// bfloat16, 256 lanes with two 207, 128 with three 146, floats 200 / 181; 8192 rows of 2500 floats, 512 with two 175, 256 with three 135; 8192 of 5000,
// 1024 with two 1021, spilling, 512 with three 283; 4096 of 8192, 1024 with two 569, 512 with four 269; 131072 rows of 16, 16 lanes, four of them
// busy, 32, 4 lanes 21).
// ONE: 256 lanes with one piece rather than 128 with two, the gradient with a block of bfloat16 (65536 rows of 1024 in bfloat16 239 and 256, in floats
// 457 and 413; forward 150 and 136, 274 and 266).  FOUR: 256 lanes with four pieces rather than 512 with two, where the registers suffice: the
// gradient with a block of bfloat16 and no bias (8192 rows of 4096 in bfloat16 138 and 175, with a bias 210 and 176; floats 245 and 221).
template <int V, bool ONE, bool FOUR, typename F>
static bool with_layout(int32_t width, F f)
{
    if (width < V) return false;
    const bool ragged = width % V != 0;
    auto go = [&](auto lanes, auto pieces) {
        if (ragged) f(lanes, pieces, std::true_type{});
        else f(lanes, pieces, std::false_type{});
        return true;
    };
    using std::integral_constant;
    const int pieces = (width + V - 1) / V;
    if (pieces <= 4) return go(integral_constant<int, 4>{}, integral_constant<int, 1>{});
    if (pieces <= 8) return go(integral_constant<int, 8>{}, integral_constant<int, 1>{});
    if (pieces <= 16) return go(integral_constant<int, 16>{}, integral_constant<int, 1>{});
    if (pieces <= 32) return go(integral_constant<int, 32>{}, integral_constant<int, 1>{});
    if (pieces <= 64) return go(integral_constant<int, 64>{}, integral_constant<int, 1>{});
    if (pieces <= 128) return go(integral_constant<int, 64>{}, integral_constant<int, 2>{});
    if (pieces <= 192) return go(integral_constant<int, 64>{}, integral_constant<int, 3>{});
    if constexpr (ONE)
        if (pieces <= 256) return go(integral_constant<int, 256>{}, integral_constant<int, 1>{});
    if (pieces <= 256) return go(integral_constant<int, 128>{}, integral_constant<int, 2>{});
    if (pieces <= 384) return go(integral_constant<int, 128>{}, integral_constant<int, 3>{});
    if (pieces <= 512) return go(integral_constant<int, 256>{}, integral_constant<int, 2>{});
    if (pieces <= 768) return go(integral_constant<int, 256>{}, integral_constant<int, 3>{});
    if constexpr (FOUR)
        if (pieces <= 1024) return go(integral_constant<int, 256>{}, integral_constant<int, 4>{});
    if (pieces <= 1024) return go(integral_constant<int, 512>{}, integral_constant<int, 2>{});
    if (pieces <= 1536) return go(integral_constant<int, 512>{}, integral_constant<int, 3>{});
    if (pieces <= 2048) return go(integral_constant<int, 512>{}, integral_constant<int, 4>{});
    return false;
}

template <typename TS, typename TB>
static void launch_residual(const ResidualArgs &a, void *y, int64_t ldy, void *u, int64_t ldu, hipStream_t st)
{
    const bool done = with_layout<4, false, false>(a.F, [&](auto lanes, auto pieces, auto ragged) {
        constexpr int G = decltype(lanes)::value, N = decltype(pieces)::value;
        constexpr int ROWS = row_block<G>() / G;
        const int64_t need = ((int64_t)a.M + ROWS - 1) / ROWS;
        const unsigned blocks = (unsigned)(need < 2048 ? need : 2048);
        CSGS_LAUNCH(K_RESIDUAL, (residual_rows_k<TS, TB, 4, G, N, decltype(ragged)::value>), dim3(blocks), dim3(row_block<G>()), st, a, (TS *)y, ldy, (TB *)u, ldu);
    });
    if (done) return;
    const unsigned blocks = (unsigned)(a.M < 4096 ? a.M : 4096);
    CSGS_LAUNCH(K_RESIDUAL, (residual_k<TS, TB>), dim3(blocks), dim3(RES_BLOCK), st, a, (TS *)y, ldy, (TB *)u, ldu);
}
// Returns the number of blocks, each of which has left a row of sums.
template <typename TS, typename TB>
static int launch_residual_grad(const ResidualArgs &a, const ResidualGrad &g, hipStream_t st)
{
    int blocks = col_blocks(a.M);
    const bool bias = g.want[COL_POST_B] || g.want[COL_PRE_B], row = g.want[COL_GATE];
    auto launch = [&](auto values, auto lanes, auto pieces, auto ragged) {
        constexpr int V = decltype(values)::value, G = decltype(lanes)::value, N = decltype(pieces)::value, ROWS = row_block<G>() / G;
        constexpr bool R = decltype(ragged)::value;
        const int64_t need = ((int64_t)a.M + ROWS - 1) / ROWS;
        constexpr int MOST = grad_blocks<G, N>();
        static_assert(MOST <= COL_BLOCKS, "room for the sums");
        blocks = (int)(need < MOST ? need : MOST);
        const dim3 grid((unsigned)blocks), block(row_block<G>());
        if constexpr (!(G == 256 && N == 4)) {
            if (bias && row) CSGS_LAUNCH(K_RESIDUAL_GRAD, (residual_grad_rows_k<TS, TB, V, G, N, R, true, true>), grid, block, st, a, g);
            else if (bias) CSGS_LAUNCH(K_RESIDUAL_GRAD, (residual_grad_rows_k<TS, TB, V, G, N, R, true, false>), grid, block, st, a, g);
            if (bias) return;
        }
        if (row) CSGS_LAUNCH(K_RESIDUAL_GRAD, (residual_grad_rows_k<TS, TB, V, G, N, R, false, true>), grid, block, st, a, g);
        else CSGS_LAUNCH(K_RESIDUAL_GRAD, (residual_grad_rows_k<TS, TB, V, G, N, R, false, false>), grid, block, st, a, g);
    };
    using std::integral_constant;
    // Rows of bfloat16 alone that 16 to 64 lanes hold in one piece of eight (us, pieces of four / eight: 131072 rows of 64 33.5 / 37.5, of 100 66 / 58, of
    // 250 158 / 128; 65536 of 512 136 / 123; 32768 of 1000 160 / 171).
    if constexpr (sizeof(TS) == 2) {
        if (a.F > 64 && a.F <= 512) {
            auto eight = [&](auto lanes) {
                if (a.F % 8) launch(integral_constant<int, 8>{}, lanes, integral_constant<int, 1>{}, std::true_type{});
                else launch(integral_constant<int, 8>{}, lanes, integral_constant<int, 1>{}, std::false_type{});
            };
            if (a.F <= 128) eight(integral_constant<int, 16>{});
            else if (a.F <= 256) eight(integral_constant<int, 32>{});
            else eight(integral_constant<int, 64>{});
            return blocks;
        }
    }
    auto four = [&](auto lanes, auto pieces, auto ragged) { launch(integral_constant<int, 4>{}, lanes, pieces, ragged); };
    bool done = false;
    if constexpr (sizeof(TB) == 2) done = !bias && with_layout<4, true, true>(a.F, four);
    if (!done && !with_layout<4, sizeof(TB) == 2, false>(a.F, four))
        CSGS_LAUNCH(K_RESIDUAL_GRAD, (residual_grad_k<TS, TB>), dim3((unsigned)blocks), dim3(RES_BLOCK), st, a, g);
    return blocks;
}

}  // namespace csgs

using namespace csgs;

extern "C" int csgs_norm_residual(const csgs_residual *r, void *y, int64_t ldy, void *u, int64_t ldu, void *stream)
{
    ResidualArgs a;
    const int rc = open_residual(r, &a);
    if (rc != CSGS_OK) return rc;
    if ((!y && !u) || (y && ldy < a.F) || (u && ldu < a.F) || (u && a.pre == CSGS_NORM_NONE)) return CSGS_EINVAL;
    hipStream_t st = (hipStream_t)stream;
    if (r->h_dtype == CSGS_F32) launch_residual<float, float>(a, y, ldy, u, ldu, st);
    else if (r->x_dtype == CSGS_F32) launch_residual<float, uint16_t>(a, y, ldy, u, ldu, st);
    else launch_residual<uint16_t, uint16_t>(a, y, ldy, u, ldu, st);
    CSGS_LAUNCH_CHECK();
    return CSGS_OK;
}

extern "C" size_t csgs_norm_residual_grad_scratch_bytes(int32_t M, int32_t F)
{
    if (M <= 0 || F <= 0) return 0;
    return align_up(sizeof(float) * COL_KINDS * (size_t)col_blocks(M) * (size_t)F, 256);
}

extern "C" int csgs_norm_residual_grad(const csgs_residual *r, const void *dy, int64_t lddy, const void *du, int64_t lddu, void *dx, int64_t lddx, void *dh,
                                       int64_t lddh, void *dgate, int64_t lddg, float *dpost_w, float *dpost_b, float *dpre_w, float *dpre_b, void *scratch,
                                       size_t scratch_bytes, void *stream)
{
    ResidualArgs a;
    const int rc = open_residual(r, &a);
    if (rc != CSGS_OK) return rc;
    if ((!dy && !du) || (dy && lddy < a.F) || (du && (lddu < a.F || a.pre == CSGS_NORM_NONE)) || (dx && (lddx < a.F || !a.x)) ||
        (dh && (lddh < a.F || !a.h)) || (dgate && (!a.gate || (a.ldg && lddg < a.F))) || (dpost_w && (!a.h || a.post == CSGS_NORM_NONE)) ||
        (dpost_b && (!a.h || a.post == CSGS_NORM_NONE)) || ((dpre_w || dpre_b) && !du) || !scratch || ((uintptr_t)scratch & 255))
        return CSGS_EINVAL;
    if (scratch_bytes < csgs_norm_residual_grad_scratch_bytes(a.M, a.F)) return CSGS_EWORKSPACE;
    hipStream_t st = (hipStream_t)stream;
    ResidualGrad g{dy, du, dx, dh, dgate, lddy, lddu, lddx, lddh, lddg, (float *)scratch, {}};
    ColOut o{{dpost_w, dpost_b, dpre_w, dpre_b, dgate && !a.ldg ? (float *)dgate : nullptr}};
    bool any = false;
    for (int k = 0; k < COL_KINDS; ++k) any |= (g.want[k] = o.out[k] ? 1 : 0) != 0;
    const int blocks = r->h_dtype == CSGS_F32   ? launch_residual_grad<float, float>(a, g, st)
                       : r->x_dtype == CSGS_F32 ? launch_residual_grad<float, uint16_t>(a, g, st)
                                                : launch_residual_grad<uint16_t, uint16_t>(a, g, st);
    CSGS_LAUNCH_CHECK();
    if (any) {
        CSGS_LAUNCH(K_COL_SUMS, col_sums_k, dim3((unsigned)((a.F + WAVE - 1) / WAVE), COL_KINDS), dim3(COL_WAVES * WAVE), st, (const float *)scratch, blocks, a.F, o);
        CSGS_LAUNCH_CHECK();
    }
    return CSGS_OK;
}
