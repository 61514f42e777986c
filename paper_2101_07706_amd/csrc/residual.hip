// csgs_norm_residual: y = beta x + alpha a(gate) .* N(h), u = N(y) per row, and its gradient.
//
// With hat(v) = (v - m) r, r = 1 / sqrt(mean((v - m)^2) + eps), N(v) = w .* hat(v) + b, and t the gradient of hat(v), the gradient of v is
//     r (t - mean(t) - hat .* mean(t .* hat))          (RMS: without mean(t))
// so with d = dL/dy as a whole = dy + the gradient through u's norm, n = N(h), a = a(gate):
//     dx = beta d,   dgate = alpha d .* n .* a'(gate),   dn = alpha d .* a,   dh = the gradient through h's norm of dn,
//     dpost_w = sum over rows of dn .* hat(h),  dpost_b = sum dn,  dpre_w = sum du .* hat(y),  dpre_b = sum du.
// The gradient forms everything again from the forward's inputs: reading x and the row again costs the same bytes as reading y
// and no statistics need be kept.  Both directions move a few bytes per operation: bound by memory.
#include "common.hpp"
#include "row_pieces.hpp"

namespace csgs {

struct ResidualArgs {
    int32_t M, F;
    const int32_t *M_dev;
    const void *x, *h, *gate;
    int64_t ldx, ldh, ldg;
    const float *post_w, *post_b, *pre_w, *pre_b;
    int32_t post, pre, act;
    float eps, alpha, beta;
};

// a(g) and its derivative.
struct Gate {
    float a, da;
};
__device__ inline Gate gate_of(float g, int32_t act)
{
    if (act == CSGS_GATE_LINEAR) return Gate{g, 1.0f};
    const float s = 1.0f / (1.0f + __expf(-g));
    if (act == CSGS_GATE_SIGMOID) return Gate{s, s * (1.0f - s)};
    return Gate{g * s, s * (1.0f + g * (1.0f - s))};
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

// Sums over rows: every block leaves one row of sums per vector, which a second kernel adds up.
enum { COL_POST_W = 0, COL_POST_B, COL_PRE_W, COL_PRE_B, COL_GATE, COL_KINDS };
constexpr int COL_BLOCKS = 512;   // most blocks
__host__ inline int col_blocks(int32_t M) { return M < COL_BLOCKS ? M : COL_BLOCKS; }

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
                const float dh = row.h_stats.r * (dn * (a.post_w ? a.post_w[f] : 1.0f) - p1 - hat * p2);
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

struct ColOut {
    float *out[COL_KINDS];
};
__global__ __launch_bounds__(256) void col_sums_k(const float *__restrict__ part, int blocks, int32_t F, ColOut o)
{
    const int k = (int)blockIdx.y;
    const int32_t f = (int32_t)(blockIdx.x * blockDim.x + threadIdx.x);
    if (!o.out[k] || f >= F) return;
    double s = 0.0;
    for (int b = 0; b < blocks; ++b) s += (double)part[((int64_t)k * blocks + b) * F + f];
    o.out[k][f] = (float)s;
}

static int open_residual(const csgs_residual *r, ResidualArgs *a)
{
    if (!r || r->M <= 0 || r->F <= 0 || (!r->x && !r->h) || (r->x && r->ldx < r->F) || (r->h && r->ldh < r->F) || (r->gate && !r->h) ||
        (r->gate && r->ldg != 0 && r->ldg < r->F) || !(r->eps >= 0.0f) || r->post < CSGS_NORM_NONE || r->post > CSGS_NORM_LAYER ||
        r->pre < CSGS_NORM_NONE || r->pre > CSGS_NORM_LAYER || r->gate_act < CSGS_GATE_LINEAR || r->gate_act > CSGS_GATE_SILU)
        return CSGS_EINVAL;
    const bool same = r->x_dtype == r->h_dtype && (r->x_dtype == CSGS_F32 || r->x_dtype == CSGS_BF16);
    if (!same && !(r->x_dtype == CSGS_F32 && r->h_dtype == CSGS_BF16)) return CSGS_EUNSUPPORTED;
    *a = ResidualArgs{r->M, r->F, r->M_dev, r->x, r->h, r->gate, r->ldx, r->ldh, r->gate ? r->ldg : 0, r->post_w, r->post_b, r->pre_w, r->pre_b,
                      r->post, r->pre, r->gate_act, r->eps, r->alpha, r->beta};
    if (a->post == CSGS_NORM_NONE) a->post_w = a->post_b = nullptr;
    if (a->pre == CSGS_NORM_NONE) a->pre_w = a->pre_b = nullptr;
    return CSGS_OK;
}

template <typename TS, typename TB>
static void launch_residual(const ResidualArgs &a, void *y, int64_t ldy, void *u, int64_t ldu, hipStream_t st)
{
    const unsigned blocks = (unsigned)(a.M < 4096 ? a.M : 4096);
    CSGS_LAUNCH(K_RESIDUAL, (residual_k<TS, TB>), dim3(blocks), dim3(RES_BLOCK), st, a, (TS *)y, ldy, (TB *)u, ldu);
}
template <typename TS, typename TB>
static void launch_residual_grad(const ResidualArgs &a, const ResidualGrad &g, hipStream_t st)
{
    CSGS_LAUNCH(K_RESIDUAL_GRAD, (residual_grad_k<TS, TB>), dim3((unsigned)col_blocks(a.M)), dim3(RES_BLOCK), st, a, g);
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
    if (r->h_dtype == CSGS_F32) launch_residual_grad<float, float>(a, g, st);
    else if (r->x_dtype == CSGS_F32) launch_residual_grad<float, uint16_t>(a, g, st);
    else launch_residual_grad<uint16_t, uint16_t>(a, g, st);
    CSGS_LAUNCH_CHECK();
    if (any) {
        CSGS_LAUNCH(K_COL_SUMS, col_sums_k, dim3((unsigned)((a.F + 255) / 256), COL_KINDS), dim3(256), st, (const float *)scratch, col_blocks(a.M), a.F, o);
        CSGS_LAUNCH_CHECK();
    }
    return CSGS_OK;
}
