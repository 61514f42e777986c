// One step of AdamW over all tensors of a network, states in 32 or in 8 bits.
//
// Every entry is read and written once: p, g, m, v in, p, m, v (and a bfloat16 copy of p) out, 28 bytes an entry with float states and 16 with
// states in 8 bits, and some 60 operations: bound by memory where the tensors are long, by one launch (two with clipping) and a chain of four
// loads (tile, description, row, entries) where they are short.  (100 M entries with bfloat16 gradients and copies, clipped: 581 us with the pass for the norm, 4.9 TB/s; 51 M with
// states in 8 bits 253 us, 3.2 TB/s: their codes cost as many operations as the step; a toy network 11 us, both launches.)  Clipping costs no pass of its own: the blocks join what grad_norm_k left and
// multiply g by the factor here.
//
// A piece of work is a segment: up to 256 entries of a row, four a lane, by 1 << lane_bits lanes (the fewest that hold a row, at most a wavefront).
// It is also the block of entries that shares an exponent where states are held in 8 bits, so that a block's largest value is a join over
// those lanes.  g' = c g, m and v are formed in double (eight operations): which of two codes a state next to their border gets does then not
// depend on how c g was rounded.
#include <math.h>
#include <new>
#include "apart.hpp"
#include "common.hpp"
#include "grad_list.hpp"
#include "row_pieces.hpp"

namespace csgs {

constexpr int ADAM_U = 2;              // segments of a thread in one tile, all asked for before the first is worked on
constexpr int ADAM_BLOCKS = 1024;      // what the device holds at once (us, the kernel alone, 1024, 2048 and 8192: 51 M entries with 8-bit states 253, 255 and 268, 120 K rows of a table 108, 110 and 124)
constexpr int64_t ADAM_ENTRIES = 1ll << 40;

struct AdamDesc {
    void *p, *m, *v;
    uint16_t *copy;
    const void *g;
    uint8_t *m_exp, *v_exp;
    const int32_t *ids, *n_dev;
    int64_t rows, cols, n, ldp, ldcopy, ldg, first_tile, blocks;   // blocks: of a row
    int32_t p_dtype, g_dtype, state, lane_bits;
    float weight_decay, lr_scale;
};
// Blocks that are done are counted in DONE_GROUPS places, and full groups in one more: additions to one place follow each other at 45 ns.
constexpr int DONE_GROUPS = 64, DONE_STEP = 16;
struct AdamMem {
    uint32_t *done;       // [DONE_GROUPS + 1], DONE_STEP apart: 0 between calls
    AdamDesc *desc;       // [n]
    int32_t *tile_tensor; // [tiles]
    size_t bytes;
};
__host__ __device__ inline AdamMem carve_adamw(void *base, int32_t n, int64_t tiles)
{
    AdamMem m;
    size_t off = align_up(sizeof(uint32_t) * DONE_STEP * (DONE_GROUPS + 1), 256);
    m.done = (uint32_t *)base;
    m.desc = (AdamDesc *)((char *)base + off);
    off = align_up(off + sizeof(AdamDesc) * (size_t)n, 256);
    m.tile_tensor = (int32_t *)((char *)base + off);
    m.bytes = align_up(off + sizeof(int32_t) * (size_t)tiles, 256);
    return m;
}

constexpr int ADAM_PER_LAUNCH = 16;
struct AdamBatch {
    AdamDesc d[ADAM_PER_LAUNCH];
    int64_t end_tile[ADAM_PER_LAUNCH];
};
__global__ __launch_bounds__(256) void adamw_list_k(AdamBatch b, int32_t first, AdamMem m)
{
    const int k = (int)blockIdx.x;
    if (threadIdx.x == 0) {
        m.desc[first + k] = b.d[k];
    }
    if (first + k == 0 && threadIdx.x <= DONE_GROUPS) m.done[threadIdx.x * DONE_STEP] = 0;
    for (int64_t t = b.d[k].first_tile + threadIdx.x; t < b.end_tile[k]; t += blockDim.x) m.tile_tensor[t] = first + k;
}

// ---------------------------------------------------------------- states in 8 bits
// Codes as csgs.h states them, four in a word.  With E the exponent field of the block's largest value: m 2^(134 - E) is below 256 (e4m3 holds 448),
// v 2^(127 - E) below 2.
__device__ inline uint32_t encode_first(const float (&x)[4], int32_t E)
{
    if (E == 0 || E == 255) return 0;
    int32_t w = 0;
    w = __builtin_amdgcn_cvt_pk_fp8_f32(ldexpf(x[0], 134 - E), ldexpf(x[1], 134 - E), w, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(ldexpf(x[2], 134 - E), ldexpf(x[3], 134 - E), w, true);
    return (uint32_t)w;
}
__device__ inline uint32_t encode_second(const float (&x)[4], int32_t E)
{
    if (E == 0 || E == 255) return 0;
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t b = __float_as_uint(ldexpf(x[i], 127 - E));
        int32_t c = (int32_t)((b + 0x7FFFFu + ((b >> 20) & 1u)) >> 20) - 769;
        c = c < 1 ? 1 : c > 255 ? 255 : c;
        w |= (x[i] > 0.0f ? (uint32_t)c : 0u) << (8 * i);
    }
    return w;
}
// (a block that holds a value that is not finite: all of it times NaN)
__device__ inline float block_scale(int32_t E, int32_t of) { return E == 255 ? __uint_as_float(0x7FC00000u) : ldexpf(1.0f, E - of); }
__device__ inline void decode_first(uint32_t w, int32_t E, float (&x)[4])
{
    const float scale = block_scale(E, 134);
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    x[0] = lo[0] * scale;
    x[1] = lo[1] * scale;
    x[2] = hi[0] * scale;
    x[3] = hi[1] * scale;
}
__device__ inline void decode_second(uint32_t w, int32_t E, float (&x)[4])
{
    const float scale = block_scale(E, 127);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t c = (w >> (8 * i)) & 255u;
        x[i] = (c ? __uint_as_float((c + 769u) << 20) : 0.0f) * scale;
    }
}
// Exponent fields of the largest of the lanes' values, of two kinds at once, over the 1 << bits lanes of a segment (the same in all of them).  Lane exchanges in
// the vector unit within four lanes, eight and a row of sixteen, by way of the LDS beyond.
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
template <int CTRL>
__device__ inline u16x2 larger_of_lanes(u16x2 e)
{
    return __builtin_elementwise_max(e, __builtin_bit_cast(u16x2, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, e), CTRL, 15, 15, true)));
}
__device__ inline void block_exponents(const float (&m)[4], const float (&v)[4], int bits, int32_t *Em, int32_t *Ev)
{
    uint32_t a = 0, b = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t x = __float_as_uint(m[i]) & 0x7FFFFFFFu, y = __float_as_uint(v[i]) & 0x7FFFFFFFu;
        a = x > a ? x : a;
        b = y > b ? y : b;
    }
    u16x2 e = {(uint16_t)(a >> 23), (uint16_t)(b >> 23)};
    if (bits > 0) e = larger_of_lanes<0xB1>(e);       // lanes 1 0 3 2
    if (bits > 1) e = larger_of_lanes<0x4E>(e);       // lanes 2 3 0 1
    if (bits > 2) e = larger_of_lanes<0x141>(e);      // eight lanes the other way round
    if (bits > 3) e = larger_of_lanes<0x140>(e);      // sixteen
    for (int s = 4; s < bits; ++s) e = __builtin_elementwise_max(e, __builtin_bit_cast(u16x2, __shfl_xor(__builtin_bit_cast(int, e), 1 << s)));
    *Em = e.x;
    *Ev = e.y;
}

// ---------------------------------------------------------------- the step
struct AdamArgs {
    double beta1, beta2, log_beta1, log_beta2;
    double eps;
    float lr, max_norm;
    int32_t kind, blocks;         // blocks: of clip_partial
    const float *lr_dev;
    int32_t *step;
    const double *clip_partial, *total;
    float *norm;
    int32_t *status;
};
// With f = 1 - beta1^t and r = sqrt(1 - beta2^t):  m / f / (sqrt(v) / r + eps) = m (r / f) / (sqrt(v) + eps r).
struct AdamNow {
    double beta1, beta2, add1, add2;      // (1 - beta1) c, (1 - beta2) c^2
    float lr, eps, gain;                  // eps r, r / f
};
// The hardware's root is within an ulp, for what is not below its range.
__device__ inline float root_of(float v)
{
    const bool small = v < 1.26217745e-29f;       // 2^-96
    const float r = __builtin_amdgcn_sqrtf(small ? v * 1.84467441e19f : v);
    return small ? r * 2.32830644e-10f : r;
}

__device__ inline uint32_t load_codes(const uint8_t *p, int n)
{
    if (n >= 4) return load_global<uint32_t, 1>(p);
    uint32_t w = 0;
    for (int i = 0; i < n; ++i) w |= (uint32_t)load_global<uint8_t>(p + i) << (8 * i);
    return w;
}
__device__ inline void store_codes(uint8_t *p, int n, uint32_t w)
{
    if (n >= 4) {
        store_global<uint32_t, 1>(p, w);
        return;
    }
    for (int i = 0; i < n; ++i) store_global<uint8_t>(p + i, (uint8_t)(w >> (8 * i)));
}

// The id in front of ids[j] that counts, the ones that are passed over left out, or -1: what ids[j] has to be above.  Usually its neighbour.  Behind a run of ids that are passed over a
// lane looks at NEAR_IDS of them, then its whole wavefront at FAR_IDS at a time (us, 300 rows of 100 behind a million ids of -1: one by one
// 116000, so 1800).  For all lanes of a wavefront.
constexpr int NEAR_IDS = 8, FAR_STEPS = 4, FAR_IDS = FAR_STEPS * WAVE;
__device__ inline int32_t id_before(const int32_t *ids, int64_t rows, int64_t j, bool ask)
{
    const auto counts = [&](int32_t id) { return id >= 0 && id < rows; };
    int32_t before = -1;
    int64_t k = ask ? j - 1 : -1;
    for (int i = 0; i < NEAR_IDS && k >= 0; ++i, --k) {
        const int32_t id = load_global<int32_t>(ids + k);
        if (counts(id)) {
            before = id;
            k = -1;
        }
    }
    for (uint64_t todo; (todo = __ballot(k >= 0)) != 0;) {
        const int first = __builtin_ctzll(todo), lane = (int)threadIdx.x & (WAVE - 1);
        const int64_t from = (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int32_t)k, first) |
                                       (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int32_t)(k >> 32), first) << 32);
        int32_t found = -1;
        for (int64_t at = from; at >= 0 && found < 0; at -= FAR_IDS) {
            int32_t id[FAR_STEPS];
#pragma unroll
            for (int i = 0; i < FAR_STEPS; ++i) {
                const int64_t mine = at - i * WAVE - lane;
                id[i] = mine >= 0 ? load_global<int32_t>(ids + mine) : -1;
            }
#pragma unroll
            for (int i = 0; i < FAR_STEPS; ++i) {
                const uint64_t some = __ballot(counts(id[i]));
                if (found < 0 && some) found = __builtin_amdgcn_readlane(id[i], __builtin_ctzll(some));
            }
        }
        if (k == from) {      // (all lanes of that row)
            before = found;
            k = -1;
        }
    }
    return before;
}

// A lane's four entries of a segment.
struct Place {
    int64_t row, block, state, at;    // row of p (-1: none), block of it; entry of the states and of the row
    int n;
};
__device__ inline Place place_of(const AdamDesc &d, int64_t seg, int64_t live, int lane, int64_t *g_row, int32_t *status)
{
    Place o;
    const bool one = d.blocks == 1;
    int64_t j = one ? seg : d.n == 1 ? (seg >= d.blocks ? 1 : 0) : ((seg | d.blocks) >> 32) ? seg / d.blocks : (int64_t)((uint32_t)seg / (uint32_t)d.blocks);
    o.block = seg - j * d.blocks;
    o.row = j;
    if (j >= live) {
        o.row = -1;
    } else if (d.ids) {
        const int32_t id = d.ids[j];
        o.row = id < d.rows ? id : -1;      // (below 0: none)
    }
    if (d.ids) {      // (two lanes that write one row would race)
        const int32_t before = id_before(d.ids, d.rows, j, o.row >= 0);
        if (o.row >= 0 && before >= o.row) {
            o.row = -1;
            if (status && lane == 0) atomicOr(status, CSGS_ST_BAD_NODE_ID);
        }
    }
    *g_row = j;
    o.at = o.block * CSGS_STATE_BLOCK + 4 * lane;
    const int64_t rest = d.cols - o.at;
    o.n = o.row < 0 || rest <= 0 ? 0 : rest < 4 ? (int)rest : 4;
    o.state = o.row * d.cols + o.at;
    return o;
}

template <typename TP, typename TG, bool SMALL>
__device__ inline void adam_tile(const AdamDesc &d, int64_t tile, const AdamNow &now, int32_t *status)
{
    const int bits = d.lane_bits, lane = (int)threadIdx.x & ((1 << bits) - 1), per = 256 >> bits;
    int64_t live = d.n;
    if (d.n_dev) {
        const int64_t r = *d.n_dev;
        live = r < 0 ? 0 : r < live ? r : live;
    }
    Place at[ADAM_U];
    float p[ADAM_U][4], g[ADAM_U][4], m[ADAM_U][4], v[ADAM_U][4];
    uint32_t mc[ADAM_U], vc[ADAM_U], me[ADAM_U], ve[ADAM_U];
#pragma unroll
    for (int u = 0; u < ADAM_U; ++u) {
        int64_t j;
        at[u] = place_of(d, (tile * ADAM_U + u) * per + ((int)threadIdx.x >> bits), live, lane, &j, status);
        const int n = at[u].n;
        if (n > 0) {
            load_some((const TP *)d.p + at[u].row * d.ldp + at[u].at, n, p[u]);
            load_some((const TG *)d.g + j * d.ldg + at[u].at, n, g[u]);
            if constexpr (SMALL) {
                mc[u] = load_codes((const uint8_t *)d.m + at[u].state, n);
                vc[u] = load_codes((const uint8_t *)d.v + at[u].state, n);
                me[u] = d.m_exp[at[u].row * d.blocks + at[u].block];
                ve[u] = d.v_exp[at[u].row * d.blocks + at[u].block];
            } else {
                load_some((const float *)d.m + at[u].state, n, m[u]);
                load_some((const float *)d.v + at[u].state, n, v[u]);
            }
        }
    }
    const float lr = now.lr * d.lr_scale;
#pragma unroll
    for (int u = 0; u < ADAM_U; ++u) {
        const int n = at[u].n;
        if constexpr (SMALL) {
            if (n > 0) {
                decode_first(mc[u], (int32_t)me[u], m[u]);
                decode_second(vc[u], (int32_t)ve[u], v[u]);
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (i >= n) {
                m[u][i] = v[u][i] = 0.0f;
                continue;
            }
            const double x = (double)g[u][i];      // (its square is exact)
            m[u][i] = (float)fma(now.beta1, (double)m[u][i], now.add1 * x);
            v[u][i] = (float)fma(now.beta2, (double)v[u][i], now.add2 * (x * x));
            const float step = m[u][i] * now.gain * __builtin_amdgcn_rcpf(root_of(v[u][i]) + now.eps);
            p[u][i] -= lr * (step + d.weight_decay * p[u][i]);
        }
        if constexpr (SMALL) {
            // (lanes of a segment have one row, and are all here or none of them)
            int32_t Em, Ev;
            block_exponents(m[u], v[u], bits, &Em, &Ev);
            if (n > 0) {
                store_codes((uint8_t *)d.m + at[u].state, n, encode_first(m[u], Em));
                store_codes((uint8_t *)d.v + at[u].state, n, encode_second(v[u], Ev));
                if (lane == 0) {
                    d.m_exp[at[u].row * d.blocks + at[u].block] = (uint8_t)Em;
                    d.v_exp[at[u].row * d.blocks + at[u].block] = (uint8_t)Ev;
                }
            }
        } else if (n > 0) {
            store_some((float *)d.m + at[u].state, n, m[u]);
            store_some((float *)d.v + at[u].state, n, v[u]);
        }
        if (n > 0) {
            store_some((TP *)d.p + at[u].row * d.ldp + at[u].at, n, p[u]);
            if (d.copy) store_some(d.copy + at[u].row * d.ldcopy + at[u].at, n, p[u]);
        }
    }
}

__global__ __launch_bounds__(256, 4) void adamw_k(AdamMem m, int64_t tiles, AdamArgs a)
{
    __shared__ double lds[4];
    AdamNow now;
    double c = 1.0;
    bool take = true;
    if (a.clip_partial || a.total) {
        const double s = a.total ? *a.total : join_partials(a.clip_partial, a.blocks, a.kind, lds);
        const double norm = a.kind == CSGS_GRAD_L2 ? sqrt(s) : s;
        c = (double)a.max_norm / (norm + 1e-6);
        if (!(c < 1.0)) c = 1.0;
        take = norm <= 1.7976931348623157e308;
        if (blockIdx.x == 0 && threadIdx.x == 0) {
            if (a.norm) *a.norm = (float)norm;
            if (a.status && !take) atomicOr(a.status, CSGS_ST_NONFINITE_GRAD);
        }
    }
    // (the counter is advanced by the block that ends last, and a block ends behind a barrier of its wavefronts: each of them has read it by then)
    const int32_t before = __builtin_amdgcn_readfirstlane(*a.step);
    const double t = (double)(before < 0 ? 0 : before) + 1.0;
    const double r = sqrt(-expm1(t * a.log_beta2));
    now.beta1 = a.beta1;
    now.beta2 = a.beta2;
    now.add1 = (1.0 - a.beta1) * c;
    now.add2 = (1.0 - a.beta2) * c * c;
    now.gain = (float)(-r / expm1(t * a.log_beta1));
    now.eps = (float)(a.eps * r);
    now.lr = a.lr_dev ? a.lr * *a.lr_dev : a.lr;
    if (take)
        for (int64_t k = blockIdx.x; k < tiles; k += gridDim.x) {
            const AdamDesc d = m.desc[__builtin_amdgcn_readfirstlane(m.tile_tensor[k])];      // (its own copy: what is stored cannot change it)
            const int64_t tile = k - d.first_tile;
            if (d.state == CSGS_STATE_8BIT) {
                if (d.p_dtype == CSGS_F32) {
                    if (d.g_dtype == CSGS_F32) adam_tile<float, float, true>(d, tile, now, a.status);
                    else adam_tile<float, uint16_t, true>(d, tile, now, a.status);
                } else {
                    if (d.g_dtype == CSGS_F32) adam_tile<uint16_t, float, true>(d, tile, now, a.status);
                    else adam_tile<uint16_t, uint16_t, true>(d, tile, now, a.status);
                }
            } else {
                if (d.p_dtype == CSGS_F32) {
                    if (d.g_dtype == CSGS_F32) adam_tile<float, float, false>(d, tile, now, a.status);
                    else adam_tile<float, uint16_t, false>(d, tile, now, a.status);
                } else {
                    if (d.g_dtype == CSGS_F32) adam_tile<uint16_t, float, false>(d, tile, now, a.status);
                    else adam_tile<uint16_t, uint16_t, false>(d, tile, now, a.status);
                }
            }
        }
    // Every wavefront has read the counter for itself: none is counted before all of its block have.
    __syncthreads();
    if (threadIdx.x == 0) {
        const uint32_t blocks = gridDim.x, group = blockIdx.x % DONE_GROUPS, groups = blocks < DONE_GROUPS ? blocks : DONE_GROUPS;
        const auto last_of = [&](uint32_t place, uint32_t n) {
            uint32_t *at = m.done + place * DONE_STEP;
            // (relaxed: nothing that the blocks have written is handed on, and the counter was read in front of the barrier; a release would write back a die's cache)
            if (__hip_atomic_fetch_add(at, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1 != n) return false;
            *at = 0;
            return true;
        };
        if (last_of(group, (blocks - group + DONE_GROUPS - 1) / DONE_GROUPS) && last_of(DONE_GROUPS, groups))
            if (take && before < 0x7FFFFFFF) *a.step = (before < 0 ? 0 : before) + 1;
    }
}

// Values of 8-bit states and back; segments as above.
template <bool WRITE>
__global__ __launch_bounds__(256) void state_k(uint8_t *codes, uint8_t *exps, int which, int64_t rows, int64_t cols, int64_t blocks, int bits, float *values,
                                               int64_t ld)
{
    const int lane = (int)threadIdx.x & ((1 << bits) - 1), per = 256 >> bits;
    const int64_t segs = rows * blocks;
    // (all lanes of a wavefront go round together: the join below asks for each of them)
    for (int64_t s0 = (int64_t)blockIdx.x * per; s0 < segs; s0 += (int64_t)gridDim.x * per) {
        const int64_t seg = s0 + ((int)threadIdx.x >> bits);
        const int64_t row = blocks == 1 ? seg : seg / blocks, block = seg - row * blocks, at = block * CSGS_STATE_BLOCK + 4 * lane;
        const int64_t rest = cols - at;
        const int n = seg >= segs || rest <= 0 ? 0 : rest < 4 ? (int)rest : 4;
        float x[4] = {0.0f, 0.0f, 0.0f, 0.0f}, none[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if constexpr (WRITE) {
            if (n > 0) load_some((const float *)values + row * ld + at, n, x);
            if (which == CSGS_STATE_SECOND)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (x[i] < 0.0f) x[i] = 0.0f;
            int32_t E, unused;
            block_exponents(x, none, bits, &E, &unused);
            if (n > 0) {
                store_codes(codes + row * cols + at, n, which == CSGS_STATE_FIRST ? encode_first(x, E) : encode_second(x, E));
                if (lane == 0) exps[seg] = (uint8_t)E;
            }
        } else if (n > 0) {
            const uint32_t w = load_codes(codes + row * cols + at, n);
            const int32_t E = exps[seg];
            if (which == CSGS_STATE_FIRST) decode_first(w, E, x);
            else decode_second(w, E, x);
            store_some(values + row * ld + at, n, x);
        }
    }
}

static int lane_bits_of(int64_t cols)
{
    int bits = 0;
    while (bits < 6 && ((int64_t)4 << bits) < cols) ++bits;
    return bits;
}

// Checks a tensor and describes it; tiles counted on from *tiles.
static int describe(const csgs_adamw_tensor &t, int64_t *tiles, AdamDesc *d)
{
    if (!t.p || !t.g || !t.m || !t.v || t.rows <= 0 || t.cols <= 0 || t.n <= 0 || t.ldp < t.cols || t.ldg < t.cols || (t.copy && t.ldcopy < t.cols))
        return CSGS_EINVAL;
    if (t.copy == t.p || t.m == t.v || t.m == t.p || t.v == t.p || t.g == t.p || (!t.ids && t.n != t.rows)) return CSGS_EINVAL;
    if (!(t.weight_decay >= 0.0f) || !(t.lr_scale >= 0.0f)) return CSGS_EINVAL;
    if ((t.p_dtype != CSGS_F32 && t.p_dtype != CSGS_BF16) || (t.g_dtype != CSGS_F32 && t.g_dtype != CSGS_BF16)) return CSGS_EUNSUPPORTED;
    if (t.state != CSGS_STATE_F32 && t.state != CSGS_STATE_8BIT) return CSGS_EUNSUPPORTED;
    const bool small = t.state == CSGS_STATE_8BIT;
    if (small ? (!t.m_exp || !t.v_exp || t.m_exp == t.v_exp) : (t.m_exp || t.v_exp)) return CSGS_EINVAL;
    if (t.rows > ADAM_ENTRIES / t.cols || t.n > ADAM_ENTRIES / t.cols || (t.ids && (t.rows > 0x7FFFFFFF || t.n > 0x7FFFFFFF))) return CSGS_EUNSUPPORTED;
    d->p = t.p;
    d->m = t.m;
    d->v = t.v;
    d->copy = (uint16_t *)t.copy;
    d->g = t.g;
    d->m_exp = t.m_exp;
    d->v_exp = t.v_exp;
    d->ids = t.ids;
    d->n_dev = t.n_dev;
    d->rows = t.rows;
    d->cols = t.cols;
    d->n = t.n;
    d->ldp = t.ldp;
    d->ldcopy = t.copy ? t.ldcopy : t.cols;
    d->ldg = t.ldg;
    // rows that lie side by side everywhere are one long row, whose segments are all full
    if (!t.ids && !t.n_dev && t.ldp == t.cols && t.ldg == t.cols && d->ldcopy == t.cols && (!small || t.cols % CSGS_STATE_BLOCK == 0)) {
        d->cols = t.rows * t.cols;
        d->rows = d->n = 1;
    }
    d->first_tile = *tiles;
    d->blocks = (d->cols + CSGS_STATE_BLOCK - 1) / CSGS_STATE_BLOCK;
    d->p_dtype = t.p_dtype;
    d->g_dtype = t.g_dtype;
    d->state = t.state;
    d->lane_bits = lane_bits_of(d->cols);
    d->weight_decay = t.weight_decay;
    d->lr_scale = t.lr_scale;
    const int64_t per = (int64_t)ADAM_U * (256 >> d->lane_bits);
    *tiles += (d->n * d->blocks + per - 1) / per;
    return *tiles > ADAM_ENTRIES / CSGS_STATE_BLOCK ? CSGS_EUNSUPPORTED : CSGS_OK;
}

// What a step reads and writes of tensor i.  (A tensor's own exponents are not compared with the rest of it: whoever allocates them knows them from its entries.)
static bool hold(const csgs_adamw_tensor &t, int32_t i, std::vector<Held> &all)
{
    const bool small = t.state == CSGS_STATE_8BIT;
    const int64_t blocks = (t.cols + CSGS_STATE_BLOCK - 1) / CSGS_STATE_BLOCK, p = t.p_dtype == CSGS_F32 ? 4 : 2, g = t.g_dtype == CSGS_F32 ? 4 : 2, state = small ? 1 : 4;
    const Held held[] = {
        {matrix_memory(t.p, t.rows, t.cols, t.ldp, p), i, true, false},
        {matrix_memory(t.copy, t.rows, t.cols, t.ldcopy, 2), i, true, false},
        {matrix_memory(t.m, t.rows, t.cols, t.cols, state), i, true, false},
        {matrix_memory(t.v, t.rows, t.cols, t.cols, state), i, true, false},
        {matrix_memory(t.m_exp, t.rows, blocks, blocks, 1), i, true, true},
        {matrix_memory(t.v_exp, t.rows, blocks, blocks, 1), i, true, true},
        {matrix_memory(t.g, t.n, t.cols, t.ldg, g), i, false, false},
        {matrix_memory(t.ids, 1, t.n, t.n, 4), i, false, false},
        {matrix_memory(t.n_dev, 1, 1, 1, 4), i, false, false},
    };
    for (const Held &h : held) {
        if (!h.at.p) continue;
        if (spans_too_much(h.at)) return false;
        all.push_back(h);
    }
    return true;
}
// Checks and counts all of a list's tensors.  What a step writes belongs to one of them and lies apart from what it reads: two blocks would write it at once, or one read it late.
static int describe_all(const csgs_adamw_tensor *t, int32_t n, int64_t *tiles)
{
    *tiles = 0;
    AdamDesc d;
    try {
        std::vector<Held> all;
        all.reserve((size_t)n * 9);
        for (int32_t i = 0; i < n; ++i) {
            const int rc = describe(t[i], tiles, &d);
            if (rc != CSGS_OK) return rc;
            if (!hold(t[i], i, all)) return CSGS_EUNSUPPORTED;
        }
        const Lie lie = all_apart(all);
        return lie == Lie::APART ? CSGS_OK : lie == Lie::MEET ? CSGS_EINVAL : CSGS_EUNSUPPORTED;
    } catch (const std::bad_alloc &) {
        return CSGS_EWORKSPACE;
    }
}

}  // namespace csgs

using namespace csgs;

extern "C" size_t csgs_adamw_list_bytes(const csgs_adamw_tensor *t, int32_t n)
{
    int64_t tiles;
    if (!t || n < 1 || n > 1 << 20 || describe_all(t, n, &tiles) != CSGS_OK) return 0;
    return carve_adamw(nullptr, n, tiles).bytes;
}

extern "C" int csgs_adamw_list_init(csgs_adamw_list *l, const csgs_adamw_tensor *t, int32_t n, void *stream)
{
    if (!l || !l->base || ((uintptr_t)l->base & 255) || !t || n < 1 || n > 1 << 20) return CSGS_EINVAL;
    l->ready = 0;
    int64_t tiles;
    const int rc = describe_all(t, n, &tiles);
    if (rc != CSGS_OK) return rc;
    const AdamMem m = carve_adamw(l->base, n, tiles);
    if (l->bytes < m.bytes) return CSGS_EWORKSPACE;
    int64_t at = 0;
    for (int32_t first = 0; first < n; first += ADAM_PER_LAUNCH) {
        AdamBatch b;
        const int32_t k = n - first < ADAM_PER_LAUNCH ? n - first : ADAM_PER_LAUNCH;
        for (int32_t i = 0; i < k; ++i) {
            (void)describe(t[first + i], &at, &b.d[i]);
            b.end_tile[i] = at;
        }
        CSGS_LAUNCH(K_ADAMW_LIST, adamw_list_k, dim3((unsigned)k), dim3(256), (hipStream_t)stream, b, first, m);
        CSGS_LAUNCH_CHECK();
    }
    l->n = n;
    l->tiles = tiles;
    l->ready = 1;
    return CSGS_OK;
}

extern "C" int csgs_adamw(const csgs_adamw_list *l, const csgs_adamw_args *a, void *stream)
{
    if (!l || !l->base || !l->ready || l->n < 1 || l->tiles < 1 || !a || !a->step) return CSGS_EINVAL;
    if (!(a->beta1 >= 0.0 && a->beta1 < 1.0) || !(a->beta2 >= 0.0 && a->beta2 < 1.0) || !(a->eps >= 0.0) || !(a->lr >= 0.0f)) return CSGS_EINVAL;
    if (a->clip && a->total) return CSGS_EINVAL;
    if (a->clip || a->total) {
        if (!(a->max_norm > 0.0f) || a->kind < CSGS_GRAD_L2 || a->kind > CSGS_GRAD_MAX || (a->clip && !list_ok(a->clip, a->kind))) return CSGS_EINVAL;
    } else if (a->norm) {
        return CSGS_EINVAL;
    }
    hipStream_t st = (hipStream_t)stream;
    AdamArgs k{};
    k.beta1 = a->beta1;
    k.beta2 = a->beta2;
    k.log_beta1 = log(a->beta1);      // (of 0: -infinity, whose power is 0 for every step)
    k.log_beta2 = log(a->beta2);
    k.lr = a->lr;
    k.eps = a->eps;
    k.max_norm = a->max_norm;
    k.kind = a->kind;
    k.lr_dev = a->lr_dev;
    k.step = a->step;
    k.total = a->total;
    k.norm = a->norm;
    k.status = a->status;
    if (a->clip) {
        const int rc = launch_grad_norm(a->clip, a->kind, st);
        if (rc != CSGS_OK) return rc;
        k.clip_partial = carve_grads(a->clip->base, a->clip->n, a->clip->tiles).partial;
        k.blocks = grad_blocks(a->clip->tiles);
    }
    const int64_t blocks = l->tiles < ADAM_BLOCKS ? l->tiles : ADAM_BLOCKS;
    CSGS_LAUNCH(K_ADAMW, adamw_k, dim3((unsigned)blocks), dim3(256), st, carve_adamw(l->base, l->n, l->tiles), l->tiles, k);
    CSGS_LAUNCH_CHECK();
    return CSGS_OK;
}

static int state_ok(const void *codes, const void *exps, const void *values, int which, int64_t rows, int64_t cols, int64_t ld)
{
    if (!codes || !exps || !values || rows <= 0 || cols <= 0 || ld < cols || (which != CSGS_STATE_FIRST && which != CSGS_STATE_SECOND)) return CSGS_EINVAL;
    if (rows > ADAM_ENTRIES / cols) return CSGS_EUNSUPPORTED;
    const int64_t blocks = (cols + CSGS_STATE_BLOCK - 1) / CSGS_STATE_BLOCK;
    const Memory c = matrix_memory(codes, rows, cols, cols, 1), e = matrix_memory(exps, rows, blocks, blocks, 1), v = matrix_memory(values, rows, cols, ld, 4);
    if (spans_too_much({c, e, v})) return CSGS_EUNSUPPORTED;
    return outputs_apart({}, {c, e, v}) ? CSGS_OK : CSGS_EINVAL;
}
static dim3 state_grid(int64_t segs, int bits)
{
    const int64_t per = 256 >> bits, need = (segs + per - 1) / per;
    return dim3((unsigned)(need < 8192 ? need : 8192));
}

extern "C" int csgs_state_read(const uint8_t *codes, const uint8_t *exps, int which, int64_t rows, int64_t cols, float *values, int64_t ld, void *stream)
{
    const int rc = state_ok(codes, exps, values, which, rows, cols, ld);
    if (rc != CSGS_OK) return rc;
    const int bits = lane_bits_of(cols);
    const int64_t blocks = (cols + CSGS_STATE_BLOCK - 1) / CSGS_STATE_BLOCK;
    CSGS_LAUNCH(K_STATE_READ, state_k<false>, state_grid(rows * blocks, bits), dim3(256), (hipStream_t)stream, (uint8_t *)codes, (uint8_t *)exps, which, rows, cols,
                blocks, bits, values, ld);
    CSGS_LAUNCH_CHECK();
    return CSGS_OK;
}

extern "C" int csgs_state_write(const float *values, int64_t ld, int which, int64_t rows, int64_t cols, uint8_t *codes, uint8_t *exps, void *stream)
{
    const int rc = state_ok(codes, exps, values, which, rows, cols, ld);
    if (rc != CSGS_OK) return rc;
    const int bits = lane_bits_of(cols);
    const int64_t blocks = (cols + CSGS_STATE_BLOCK - 1) / CSGS_STATE_BLOCK;
    CSGS_LAUNCH(K_STATE_WRITE, state_k<true>, state_grid(rows * blocks, bits), dim3(256), (hipStream_t)stream, codes, exps, which, rows, cols, blocks, bits,
                (float *)values, ld);
    CSGS_LAUNCH_CHECK();
    return CSGS_OK;
}
