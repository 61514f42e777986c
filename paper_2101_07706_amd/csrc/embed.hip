// csgs_embed: rows of a learned table by id, scaled, and the table's gradient by sorted ids.
//
// Forward: out[t] = s T[i_t].  Gradient: dT[v] = s sum_{t : i_t = v} G[t].  The positions t are sorted by id (stable, least
// significant digit first), so that the positions of a row lie side by side, in order; a row is then summed by one wavefront
// and written once.
#include "common.hpp"
#include "row_pieces.hpp"

namespace csgs {

// ---------------------------------------------------------------- lookup
template <typename TI, typename TO>
__global__ __launch_bounds__(256) void embed_k(const TI *T, int64_t ld, int64_t rows, int32_t F, const int32_t *__restrict__ ids,
                                               int32_t n_cap, const int32_t *__restrict__ n_dev, float scale, TO *out, int64_t ldo)
{
    const int32_t n = resolve_count(n_cap, n_dev);
    const int lane = lane_id();
    const int64_t waves = (int64_t)gridDim.x * (blockDim.x / WAVE);
    for (int64_t t = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) / WAVE; t < n; t += waves) {
        const int64_t id = ids[t];
        const bool ok = id >= 0 && id < rows;
        for (int32_t f = lane; f < F; f += WAVE) {
            Vec<1> v{{0.0f}};
            if (ok) v.x[0] = scale * load_row<TI, 1>(T + id * ld + f).x[0];
            store_row<TO, 1>(out + t * ldo + f, v);
        }
    }
}

// ---------------------------------------------------------------- positions sorted by id
// A pass sorts by one digit of up to 8 bits.  At most SORT_TILES blocks take consecutive tiles of the entries: the first kernel
// counts a tile's digits, the second one adds up what lies before its own (the counts of all tiles, at most 64 K of them)
// and places its entries.  No block waits for another.
constexpr int SORT_TILES = 256, SORT_BLOCK = 256, SORT_WAVES = SORT_BLOCK / WAVE, DIGITS = 256;
constexpr int32_t SORT_TILE_MIN = 2048;

struct EmbedScratch {
    uint32_t *key[2], *pos[2];   // [n] entries, used in turn
    uint32_t *hist;              // [DIGITS * SORT_TILES] of a pass
    uint32_t *heads;             // [SORT_TILES] different ids that begin in a tile
    int32_t *seg_key, *seg_start, *n_seg;   // [n], [n + 1], [1]: the different ids, where their positions begin, how many
    size_t bytes;
};
__host__ inline EmbedScratch carve_embed(void *base, int64_t n, int32_t F)
{
    EmbedScratch s;
    size_t off = 0;
    auto take = [&](size_t bytes) {
        const size_t o = off;
        off = align_up(off + bytes, 256);
        return (char *)base + o;
    };
    for (int i = 0; i < 2; ++i) {
        s.key[i] = (uint32_t *)take((size_t)n * 4);
        s.pos[i] = (uint32_t *)take((size_t)n * 4);
    }
    s.hist = (uint32_t *)take(sizeof(uint32_t) * DIGITS * SORT_TILES);
    s.heads = (uint32_t *)take(sizeof(uint32_t) * SORT_TILES);
    s.seg_key = (int32_t *)take((size_t)n * 4);
    s.seg_start = (int32_t *)take((size_t)(n + 1) * 4);
    s.n_seg = (int32_t *)take(4);
    s.bytes = off;
    (void)F;
    return s;
}

// Where the entries of a pass come from: the caller's ids in the first one (ids outside the table take the key `rows`, behind
// all others), the entries of the pass before in the others.
struct SortIn {
    const int32_t *ids;
    const uint32_t *key, *pos;
    uint32_t rows;
    __device__ uint32_t get(int64_t i, uint32_t *p) const
    {
        if (ids) {
            const uint32_t id = (uint32_t)ids[i];
            *p = (uint32_t)i;
            return id < rows ? id : rows;
        }
        *p = pos[i];
        return key[i];
    }
    __device__ uint32_t get(int64_t i) const
    {
        if (!ids) return key[i];
        const uint32_t id = (uint32_t)ids[i];
        return id < rows ? id : rows;
    }
};

__global__ __launch_bounds__(SORT_BLOCK) void sort_count_k(SortIn in, int32_t n_cap, const int32_t *__restrict__ n_dev, int32_t tile, int shift,
                                                           uint32_t mask, uint32_t *__restrict__ hist)
{
    __shared__ uint32_t count[DIGITS];
    const int32_t n = resolve_count(n_cap, n_dev);
    const int64_t beg = (int64_t)blockIdx.x * tile;
    const int64_t end = beg + tile < n ? beg + tile : n;
    count[threadIdx.x] = 0;
    __syncthreads();
    for (int64_t i = beg + threadIdx.x; i < end; i += SORT_BLOCK) atomicAdd(&count[(in.get(i) >> shift) & mask], 1u);
    __syncthreads();
    hist[threadIdx.x * SORT_TILES + blockIdx.x] = count[threadIdx.x];
}

// The lanes of the wavefront whose digit is this lane's own (lanes that take part).
__device__ inline uint64_t same_digit(uint32_t digit, bool active, int bits)
{
    uint64_t peers = __ballot(active);
    for (int b = 0; b < bits; ++b) {
        const bool bit = (digit >> b) & 1u;
        const uint64_t with = __ballot(active && bit);
        peers &= bit ? with : ~with;
    }
    return peers;
}

__global__ __launch_bounds__(SORT_BLOCK) void sort_place_k(SortIn in, int32_t n_cap, const int32_t *__restrict__ n_dev, int32_t tile, int tiles,
                                                           int shift, int bits, const uint32_t *__restrict__ hist,
                                                           uint32_t *__restrict__ key_out, uint32_t *__restrict__ pos_out)
{
    __shared__ uint32_t at[SORT_WAVES][DIGITS];   // a wavefront's entries by digit, then the next place of each
    __shared__ uint32_t scan[17];
    const int32_t n = resolve_count(n_cap, n_dev);
    const int64_t beg = (int64_t)blockIdx.x * tile;
    const int64_t end = beg + tile < n ? beg + tile : n;
    if (beg >= end) return;
    const uint32_t mask = (1u << bits) - 1;
    const int tid = (int)threadIdx.x, lane = lane_id(), wave = tid / WAVE;
    const int64_t share = tile / SORT_WAVES;   // a multiple of 64
    const int64_t w_beg = beg + wave * share, w_end = w_beg + share < end ? w_beg + share : end;
    for (int w = 0; w < SORT_WAVES; ++w) at[w][tid] = 0;
    // entries with a smaller digit, and of this digit in earlier tiles
    uint32_t before = 0, all = 0;
    for (int t = 0; t < tiles; ++t) {
        const uint32_t c = hist[tid * SORT_TILES + t];
        before += t < (int)blockIdx.x ? c : 0u;
        all += c;
    }
    __syncthreads();
    for (int64_t i = w_beg + lane; i < w_end; i += WAVE) atomicAdd(&at[wave][(in.get(i) >> shift) & mask], 1u);
    uint32_t total;
    const uint32_t smaller = block_exclusive_scan<uint32_t>(all, scan, &total);   // (its barriers: the counts are complete)
    uint32_t next = smaller + before;
    for (int w = 0; w < SORT_WAVES; ++w) {
        const uint32_t c = at[w][tid];
        at[w][tid] = next;
        next += c;
    }
    __syncthreads();
    for (int64_t i0 = w_beg; i0 < w_end; i0 += WAVE) {
        const int64_t i = i0 + lane;
        const bool active = i < w_end;
        uint32_t p = 0;
        const uint32_t k = active ? in.get(i, &p) : 0u;
        const uint32_t digit = (k >> shift) & mask;
        const uint64_t peers = same_digit(digit, active, bits);
        const uint32_t rank = (uint32_t)__popcll(peers & ((1ull << lane) - 1ull));
        uint32_t dst = 0;
        if (active) dst = *(volatile uint32_t *)&at[wave][digit] + rank;
        __builtin_amdgcn_wave_barrier();
        if (active && rank == 0) *(volatile uint32_t *)&at[wave][digit] = dst + (uint32_t)__popcll(peers);
        __builtin_amdgcn_wave_barrier();
        if (active && dst < (uint32_t)n) {
            key_out[dst] = k;
            pos_out[dst] = p;
        }
    }
}

// ---------------------------------------------------------------- the different ids
__device__ inline bool is_head(const uint32_t *__restrict__ key, int64_t i, uint32_t rows) { return key[i] < rows && (i == 0 || key[i - 1] != key[i]); }

__global__ __launch_bounds__(SORT_BLOCK) void heads_count_k(const uint32_t *__restrict__ key, int32_t n_cap, const int32_t *__restrict__ n_dev,
                                                            int32_t tile, uint32_t rows, uint32_t *__restrict__ heads)
{
    __shared__ uint32_t scan[17];
    const int32_t n = resolve_count(n_cap, n_dev);
    const int64_t beg = (int64_t)blockIdx.x * tile;
    const int64_t end = beg + tile < n ? beg + tile : n;
    uint32_t c = 0, total;
    for (int64_t i = beg + threadIdx.x; i < end; i += SORT_BLOCK) c += is_head(key, i, rows) ? 1u : 0u;
    block_exclusive_scan<uint32_t>(c, scan, &total);
    if (threadIdx.x == 0) heads[blockIdx.x] = total;
}

__global__ __launch_bounds__(SORT_BLOCK) void heads_place_k(const uint32_t *__restrict__ key, int32_t n_cap, const int32_t *__restrict__ n_dev,
                                                            int32_t tile, int tiles, uint32_t rows, const uint32_t *__restrict__ heads,
                                                            int32_t *__restrict__ seg_key, int32_t *__restrict__ seg_start,
                                                            int32_t *__restrict__ n_seg, int32_t *__restrict__ n_seg_out)
{
    __shared__ uint32_t scan[17];
    const int32_t n = resolve_count(n_cap, n_dev);
    const int64_t beg = (int64_t)blockIdx.x * tile;
    const int64_t end = beg + tile < n ? beg + tile : n;
    uint32_t all, total;
    const uint32_t c = (int)threadIdx.x < tiles ? heads[threadIdx.x] : 0u;
    block_exclusive_scan<uint32_t>(c, scan, &all);
    block_exclusive_scan<uint32_t>((int)threadIdx.x < (int)blockIdx.x ? c : 0u, scan, &total);
    uint32_t base = total;
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        *n_seg = (int32_t)all;
        if (n_seg_out) *n_seg_out = (int32_t)all;
    }
    for (int64_t i0 = beg; i0 < end; i0 += SORT_BLOCK) {
        const int64_t i = i0 + threadIdx.x;
        const bool head = i < end && is_head(key, i, rows);
        const uint32_t at = base + block_exclusive_scan<uint32_t>(head ? 1u : 0u, scan, &total);
        base += total;
        if (head) {
            seg_key[at] = (int32_t)key[i];
            seg_start[at] = (int32_t)i;
        }
        if (i < end && key[i] < rows && (i + 1 == n || key[i + 1] >= rows)) seg_start[all] = (int32_t)(i + 1);
    }
}

// ---------------------------------------------------------------- sums
template <typename TD>
__global__ __launch_bounds__(256) void rows_zero_k(TD *d, int64_t ldd, int64_t rows, int32_t F)
{
    const int64_t waves = (int64_t)gridDim.x * (blockDim.x / WAVE);
    for (int64_t r = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) / WAVE; r < rows; r += waves)
        for (int32_t f = lane_id(); f < F; f += WAVE) store_row<TD, 1>(d + r * ldd + f, Vec<1>{{0.0f}});
}

// compact: segment j's sum goes to row j, else to row seg_key[j].
template <typename TG, typename TD>
__global__ __launch_bounds__(256) void embed_sum_k(const TG *G, int64_t ldg, int32_t F, const uint32_t *__restrict__ pos,
                                                   const int32_t *__restrict__ seg_key, const int32_t *__restrict__ seg_start,
                                                   const int32_t *__restrict__ n_seg, float scale, int compact, int accumulate, TD *d, int64_t ldd)
{
    const int32_t n = *n_seg;
    const int64_t waves = (int64_t)gridDim.x * (blockDim.x / WAVE);
    for (int64_t j = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) / WAVE; j < n; j += waves) {
        const int32_t beg = seg_start[j], end = seg_start[j + 1];
        TD *row = d + (compact ? j : (int64_t)seg_key[j]) * ldd;
        for (int32_t f = lane_id(); f < F; f += WAVE) {
            double sum = 0.0;
            for (int32_t i = beg; i < end; ++i) sum += (double)load_row<TG, 1>(G + (int64_t)pos[i] * ldg + f).x[0];
            sum *= (double)scale;
            if (accumulate) sum += (double)load_row<TD, 1>(row + f).x[0];
            store_row<TD, 1>(row + f, Vec<1>{{(float)sum}});
        }
    }
}

static unsigned wave_blocks(int64_t n)
{
    const int64_t b = (n + 3) / 4;
    return (unsigned)(b < 1 ? 1 : (b < 4096 ? b : 4096));
}

static bool elem_type(int t) { return t == CSGS_F32 || t == CSGS_BF16; }

template <typename TG, typename TD>
static int embed_grad_sums(const EmbedScratch &s, int last, const int32_t *seg_key, int64_t n, const void *G, int64_t ldg, int32_t F, float scale,
                           int compact, int accumulate, void *d, int64_t ldd, int64_t rows, hipStream_t st)
{
    if (!compact && !accumulate) {
        CSGS_LAUNCH(K_EMBED_ZERO, rows_zero_k<TD>, dim3(wave_blocks(rows)), dim3(256), st, (TD *)d, ldd, rows, F);
        CSGS_LAUNCH_CHECK();
    }
    CSGS_LAUNCH(K_EMBED_SUM, (embed_sum_k<TG, TD>), dim3(wave_blocks(n)), dim3(256), st, (const TG *)G, ldg, F, s.pos[last], seg_key, s.seg_start, s.n_seg,
                scale, compact, accumulate, (TD *)d, ldd);
    CSGS_LAUNCH_CHECK();
    return CSGS_OK;
}

// uniq, n_uniq: null in the dense form.
static int embed_grad(const int32_t *ids, int64_t n, const int32_t *n_dev, const void *G, int64_t ldg, int32_t F, int g_dtype, float scale, int accumulate,
                      int64_t rows, int32_t *uniq, int32_t *n_uniq, void *d, int64_t ldd, int d_dtype, void *scratch, size_t scratch_bytes, void *stream)
{
    if (!ids || n <= 0 || !G || F <= 0 || ldg < F || rows <= 0 || !d || ldd < F || !scratch || ((uintptr_t)scratch & 255) || (accumulate & ~1)) return CSGS_EINVAL;
    if (!elem_type(g_dtype) || !elem_type(d_dtype) || n > INT32_MAX || rows > INT32_MAX) return CSGS_EUNSUPPORTED;
    const EmbedScratch s = carve_embed(scratch, n, F);
    if (scratch_bytes < s.bytes) return CSGS_EWORKSPACE;
    hipStream_t st = (hipStream_t)stream;
    const int64_t even = ((n + SORT_TILES - 1) / SORT_TILES + SORT_BLOCK - 1) / SORT_BLOCK * SORT_BLOCK;
    const int32_t tile = (int32_t)(even < SORT_TILE_MIN ? SORT_TILE_MIN : even);
    const int tiles = (int)((n + tile - 1) / tile);
    int key_bits = 0;
    while ((rows >> key_bits) != 0) ++key_bits;   // the key `rows` too
    const int passes = (key_bits + 7) / 8, bits = (key_bits + passes - 1) / passes;
    for (int p = 0; p < passes; ++p) {
        const SortIn in{p == 0 ? ids : nullptr, p == 0 ? nullptr : s.key[(p + 1) & 1], p == 0 ? nullptr : s.pos[(p + 1) & 1], (uint32_t)rows};
        CSGS_LAUNCH(K_EMBED_COUNT, sort_count_k, dim3((unsigned)tiles), dim3(SORT_BLOCK), st, in, (int32_t)n, n_dev, tile, p * bits, (1u << bits) - 1, s.hist);
        CSGS_LAUNCH(K_EMBED_PLACE, sort_place_k, dim3((unsigned)tiles), dim3(SORT_BLOCK), st, in, (int32_t)n, n_dev, tile, tiles, p * bits, bits, s.hist, s.key[p & 1], s.pos[p & 1]);
        CSGS_LAUNCH_CHECK();
    }
    const int last = (passes - 1) & 1;
    int32_t *seg_key = uniq ? uniq : s.seg_key;
    CSGS_LAUNCH(K_EMBED_HEADS, heads_count_k, dim3((unsigned)tiles), dim3(SORT_BLOCK), st, s.key[last], (int32_t)n, n_dev, tile, (uint32_t)rows, s.heads);
    CSGS_LAUNCH(K_EMBED_HEADS, heads_place_k, dim3((unsigned)tiles), dim3(SORT_BLOCK), st, s.key[last], (int32_t)n, n_dev, tile, tiles, (uint32_t)rows, s.heads,
                seg_key, s.seg_start, s.n_seg, n_uniq);
    CSGS_LAUNCH_CHECK();
    const int compact = uniq ? 1 : 0;
    if (g_dtype == CSGS_F32)
        return d_dtype == CSGS_F32 ? embed_grad_sums<float, float>(s, last, seg_key, n, G, ldg, F, scale, compact, accumulate, d, ldd, rows, st)
                                   : embed_grad_sums<float, uint16_t>(s, last, seg_key, n, G, ldg, F, scale, compact, accumulate, d, ldd, rows, st);
    return d_dtype == CSGS_F32 ? embed_grad_sums<uint16_t, float>(s, last, seg_key, n, G, ldg, F, scale, compact, accumulate, d, ldd, rows, st)
                               : embed_grad_sums<uint16_t, uint16_t>(s, last, seg_key, n, G, ldg, F, scale, compact, accumulate, d, ldd, rows, st);
}

template <typename TI, typename TO>
static void launch_embed(const void *T, int64_t ld, int64_t rows, int32_t F, const int32_t *ids, int32_t n, const int32_t *n_dev, float scale, void *out,
                         int64_t ldo, hipStream_t st)
{
    CSGS_LAUNCH(K_EMBED, (embed_k<TI, TO>), dim3(wave_blocks(n)), dim3(256), st, (const TI *)T, ld, rows, F, ids, n, n_dev, scale, (TO *)out, ldo);
}

}  // namespace csgs

using namespace csgs;

extern "C" int csgs_embed(const void *T, int64_t ld, int64_t rows, int32_t F, int dtype, const int32_t *ids, int64_t n, const int32_t *n_dev, float scale,
                          void *out, int64_t ldo, int out_dtype, void *stream)
{
    if (!T || rows <= 0 || F <= 0 || ld < F || !ids || n <= 0 || !out || ldo < F) return CSGS_EINVAL;
    if (!elem_type(dtype) || !elem_type(out_dtype) || n > INT32_MAX) return CSGS_EUNSUPPORTED;
    hipStream_t st = (hipStream_t)stream;
    if (dtype == CSGS_F32) {
        if (out_dtype == CSGS_F32) launch_embed<float, float>(T, ld, rows, F, ids, (int32_t)n, n_dev, scale, out, ldo, st);
        else launch_embed<float, uint16_t>(T, ld, rows, F, ids, (int32_t)n, n_dev, scale, out, ldo, st);
    } else {
        if (out_dtype == CSGS_F32) launch_embed<uint16_t, float>(T, ld, rows, F, ids, (int32_t)n, n_dev, scale, out, ldo, st);
        else launch_embed<uint16_t, uint16_t>(T, ld, rows, F, ids, (int32_t)n, n_dev, scale, out, ldo, st);
    }
    CSGS_LAUNCH_CHECK();
    return CSGS_OK;
}

extern "C" size_t csgs_embed_grad_scratch_bytes(int64_t n, int64_t rows, int32_t F)
{
    if (n <= 0 || n > INT32_MAX || rows <= 0 || rows > INT32_MAX || F <= 0) return 0;
    return carve_embed(nullptr, n, F).bytes;
}

extern "C" int csgs_embed_grad(const int32_t *ids, int64_t n, const int32_t *n_dev, const void *G, int64_t ldg, int32_t F, int g_dtype, float scale,
                               int accumulate, void *dT, int64_t ldd, int64_t rows, int d_dtype, void *scratch, size_t scratch_bytes, void *stream)
{
    return embed_grad(ids, n, n_dev, G, ldg, F, g_dtype, scale, accumulate, rows, nullptr, nullptr, dT, ldd, d_dtype, scratch, scratch_bytes, stream);
}

extern "C" int csgs_embed_grad_rows(const int32_t *ids, int64_t n, const int32_t *n_dev, const void *G, int64_t ldg, int32_t F, int g_dtype, float scale,
                                    int64_t rows, int32_t *uniq, int32_t *n_uniq, void *dR, int64_t ldd, int d_dtype, void *scratch, size_t scratch_bytes,
                                    void *stream)
{
    if (!uniq || !n_uniq) return CSGS_EINVAL;
    return embed_grad(ids, n, n_dev, G, ldg, F, g_dtype, scale, 0, rows, uniq, n_uniq, dR, ldd, d_dtype, scratch, scratch_bytes, stream);
}
