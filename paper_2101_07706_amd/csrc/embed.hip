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

// Sorted positions are summed in chunks of a fixed number, whatever ids they hold (see chunk_sums_k): as many as leave a
// million values of the sums at a time (1024 wavefronts of 16 bytes a lane), 8 to 64, no more than the lanes that take a row.
__host__ inline int32_t chunk_of(int64_t n, int32_t F)
{
    const int32_t most = F <= 128 ? 16 : (F <= 256 ? 32 : 64);
    int32_t c = 8;
    while (c < most && n / (2 * c) * F >= 1 << 20) c *= 2;
    return c;
}

struct EmbedScratch {
    uint32_t *key[2], *pos[2];   // [n] entries, used in turn
    uint32_t *hist;              // [DIGITS * SORT_TILES] of a pass
    uint32_t *heads;             // [SORT_TILES] different ids that begin in a tile
    uint32_t *rank;              // [n] of an entry's id among the different ones
    double *part;                // [chunks][2][F] sums of rows that go on across chunks
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
    s.rank = (uint32_t *)take((size_t)n * 4);
    const int32_t chunk = chunk_of(n, F);
    s.part = (double *)take(sizeof(double) * 2 * (size_t)((n + chunk - 1) / chunk) * (size_t)F);
    s.bytes = off;
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
                                                            uint32_t *__restrict__ rank, int32_t *__restrict__ uniq, int32_t *__restrict__ n_uniq)
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
    if (blockIdx.x == 0 && threadIdx.x == 0) *n_uniq = (int32_t)all;
    for (int64_t i0 = beg; i0 < end; i0 += SORT_BLOCK) {
        const int64_t i = i0 + threadIdx.x;
        const bool head = i < end && is_head(key, i, rows);
        const uint32_t before = base + block_exclusive_scan<uint32_t>(head ? 1u : 0u, scan, &total);
        base += total;
        if (head) uniq[before] = (int32_t)key[i];
        if (i < end) rank[i] = before + (head ? 1u : 0u) - 1u;
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

// The piece of V columns that a lane holds; where V does not divide F, the row's last piece is read from F - V on and its first `skip`
// values are the piece's before.
template <int V>
struct Piece1 {
    int32_t col, skip;
    bool active;
    __device__ Piece1(int32_t index, int32_t F)
    {
        active = (int64_t)index * V < F;
        col = !active ? 0 : (index * V > F - V ? F - V : index * V);
        skip = active ? index * V - col : 0;
    }
};

// Where the sums go: row `rank` of the compact form, row `key` of the dense one.
struct SumOut {
    const uint32_t *rank;   // null: dense
    void *d;
    int64_t ldd;
    float scale;
    int32_t accumulate;
};
template <typename TD, int V>
__device__ inline void write_sum(const SumOut &o, uint32_t row, const Piece1<V> &pc, const double (&acc)[V])
{
    if (!pc.active) return;
    TD *d = (TD *)o.d + (int64_t)row * o.ldd + pc.col;
    Vec<V> v{};
    if (pc.skip == 0) {
        if (o.accumulate) v = load_row<TD, V>(d);
#pragma unroll
        for (int i = 0; i < V; ++i) v.x[i] = (float)(acc[i] * (double)o.scale + (double)v.x[i]);
        store_row<TD, V>(d, v);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i >= pc.skip) {
                const float old = o.accumulate ? load_row<TD, 1>(d + i).x[0] : 0.0f;
                store_row<TD, 1>(d + i, Vec<1>{{(float)(acc[i] * (double)o.scale + (double)old)}});
            }
    }
}
// Partial sums of chunk c: slot 1 of a row that begins in it and goes on, slot 0 of one that began before it.
template <int V>
__device__ inline void write_part(double *part, const Piece1<V> &pc, const double (&acc)[V])
{
    if (!pc.active) return;
#pragma unroll
    for (int i = 0; i < V; ++i) part[pc.col + i] = acc[i];   // (values of two pieces: the same from both)
}

// Value of lane `from` of the G lanes that work together.
template <int G>
__device__ inline uint32_t from_lane(uint32_t v, int from)
{
    if constexpr (G == WAVE) return (uint32_t)__builtin_amdgcn_readlane((int)v, from);
    return (uint32_t)__shfl((int)v, from, G);
}

// G lanes take a chunk of sorted positions: the rows of G that they point to are added up in order, eight on their way at a time; a
// table row all of whose positions lie in the chunk is written at once, parts of others go to `part`.  The work per chunk does not
// depend on how often an id occurs.
template <typename TG, typename TD, int V, int G>
__global__ __launch_bounds__(256) void chunk_sums_k(const TG *g, int64_t ldg, int32_t F, const uint32_t *__restrict__ key, const uint32_t *__restrict__ pos,
                                                    int32_t n_cap, const int32_t *__restrict__ n_dev, uint32_t rows, int32_t chunk,
                                                    double *__restrict__ part, SumOut o)
{
    constexpr int U = 8;
    const int32_t n = resolve_count(n_cap, n_dev);
    const int lane = (int)threadIdx.x % G;
    const int64_t c = ((int64_t)blockIdx.x * 256 + threadIdx.x) / G;
    const int64_t beg = c * chunk;
    const int64_t end = beg + chunk < n ? beg + chunk : n;
    const int len = end > beg ? (int)(end - beg) : 0;
    const uint32_t NONE = 0xFFFFFFFFu;
    uint32_t k = NONE, p = 0, rk = 0;
    if (lane < len) {
        k = key[beg + lane];
        p = pos[beg + lane];
        if (o.rank) rk = o.rank[beg + lane];
    }
    const uint32_t row = o.rank ? rk : k;
    const uint32_t before = len > 0 && beg > 0 ? key[beg - 1] : NONE, after = len > 0 && end < n ? key[end] : NONE;
    const uint32_t prev = (uint32_t)__shfl_up((int)k, 1, G);
    const uint32_t next = (uint32_t)__shfl_down((int)k, 1, G);
    const bool valid = lane < len && k < rows;
    const bool last = valid && (lane == len - 1 ? after != k : next != k);      // the row's last position
    const bool first = valid && (lane == 0 ? before != k : prev != k);
    const int shift = (int)(threadIdx.x & (WAVE - 1)) / G * G;
    const uint64_t lanes = G == WAVE ? ~0ull : (1ull << (G % WAVE)) - 1ull;
    const uint64_t m_valid = (__ballot(valid) >> shift) & lanes, m_last = (__ballot(last) >> shift) & lanes, m_first = (__ballot(first) >> shift) & lanes;
    const int count = __popcll(m_valid);
    const Piece1<V> pc((int32_t)(blockIdx.y * G + lane), F);
    double acc[V];
#pragma unroll
    for (int i = 0; i < V; ++i) acc[i] = 0.0;
    bool inside = true;    // the row's sum began in this chunk
    for (int i0 = 0; i0 < chunk; i0 += U) {
        if (__ballot(i0 < count) == 0) break;
        RawPiece<TG, V> r[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u < count ? i0 + u : (count > 0 ? count - 1 : 0);
            r[u].load(g + (int64_t)from_lane<G>(p, i) * ldg + pc.col);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u;
            if (i < count) {
                if ((m_first >> i) & 1ull) inside = true;
                else if (i == 0) inside = false;
#pragma unroll
                for (int j = 0; j < V; ++j) acc[j] += (double)r[u].value(j);
                const bool ends = (m_last >> i) & 1ull;
                if (ends || i == count - 1) {
                    if (ends && inside) write_sum<TD, V>(o, from_lane<G>(row, i), pc, acc);
                    else write_part<V>(part + (2 * c + (inside ? 1 : 0)) * F, pc, acc);
#pragma unroll
                    for (int j = 0; j < V; ++j) acc[j] = 0.0;
                }
            }
        }
    }
}

// Table rows that go on across chunks: a wavefront per chunk looks whether one begins in it, and adds up its parts in order; one
// of more than JOIN_LONG chunks is left to the whole block, whose groups of G lanes take consecutive shares of the parts.
constexpr int JOIN_WAVES = 16, JOIN_LONG = 32;
template <typename TD, int V, int G>
__global__ __launch_bounds__(JOIN_WAVES * WAVE) void chunk_join_k(int32_t F, const uint32_t *__restrict__ key, int32_t n_cap,
                                                                  const int32_t *__restrict__ n_dev, uint32_t rows, int32_t chunk,
                                                                  const double *__restrict__ part, SumOut o)
{
    constexpr int GROUPS = JOIN_WAVES * WAVE / G, U = 8;
    __shared__ int64_t long_parts[JOIN_WAVES];
    __shared__ double lds[GROUPS][G * V];
    const int32_t n = resolve_count(n_cap, n_dev);
    const int lane = lane_id(), wave = (int)threadIdx.x / WAVE, sub = lane % G, group = (int)threadIdx.x / G;
    const Piece1<V> pc((int32_t)(blockIdx.y * G + sub), F);
    const int64_t c0 = (int64_t)blockIdx.x * JOIN_WAVES, c = c0 + wave;
    const int64_t beg = c * chunk, end = beg + chunk;
    int64_t parts = 0;     // chunks after c that the row is in
    uint32_t k = 0;
    if (end < n) {
        k = key[end - 1];
        const bool begins = key[beg] != k || beg == 0 || key[beg - 1] != k;
        if (k < rows && begins && key[end] == k) {
            for (;;) {
                const int64_t at = (c + 1 + parts + lane) * chunk;
                const uint64_t m = __ballot(at < n && key[at < n ? at : n - 1] == k);
                const int run = m == ~0ull ? WAVE : __ffsll((unsigned long long)~m) - 1;
                parts += run;
                if (run < WAVE) break;
            }
        }
    }
    auto add = [&](double (&acc)[V], const double *p) {
#pragma unroll
        for (int i = 0; i < V; ++i) acc[i] += p[pc.col + i];
    };
    double acc[V];
    if (parts > 0 && parts <= JOIN_LONG && lane < G) {
#pragma unroll
        for (int i = 0; i < V; ++i) acc[i] = 0.0;
        add(acc, part + (2 * c + 1) * F);
#pragma unroll 4
        for (int64_t t = 1; t <= parts; ++t) add(acc, part + 2 * (c + t) * F);
        write_sum<TD, V>(o, o.rank ? o.rank[end - 1] : k, pc, acc);
    }
    if (lane == 0) long_parts[wave] = parts > JOIN_LONG ? parts : 0;
    __syncthreads();
    for (int w = 0; w < JOIN_WAVES; ++w) {
        const int64_t m = long_parts[w];
        if (m == 0) continue;
        const int64_t cw = c0 + w, share = (m + GROUPS - 1) / GROUPS;
        const int64_t t0 = 1 + group * share, t1 = t0 + share <= m + 1 ? t0 + share : m + 1;
#pragma unroll
        for (int i = 0; i < V; ++i) acc[i] = 0.0;
        if (group == 0) add(acc, part + (2 * cw + 1) * F);
#pragma unroll U
        for (int64_t t = t0; t < t1; ++t) add(acc, part + 2 * (cw + t) * F);
#pragma unroll
        for (int i = 0; i < V; ++i) lds[group][sub * V + i] = acc[i];
        __syncthreads();
        if (group == 0) {
            for (int q = 1; q < GROUPS; ++q)
#pragma unroll
                for (int i = 0; i < V; ++i) acc[i] += lds[q][sub * V + i];
            const int64_t at = (cw + 1) * chunk - 1;
            write_sum<TD, V>(o, o.rank ? o.rank[at] : key[at], pc, acc);
        }
        __syncthreads();
    }
}

static unsigned wave_blocks(int64_t n)
{
    const int64_t b = (n + 3) / 4;
    return (unsigned)(b < 1 ? 1 : (b < 4096 ? b : 4096));
}

static bool elem_type(int t) { return t == CSGS_F32 || t == CSGS_BF16; }

struct SumIn {
    const void *g;
    int64_t ldg;
    int32_t F;
    const uint32_t *key, *pos;
    int32_t n;
    const int32_t *n_dev;
    uint32_t rows;
    double *part;
};
template <typename TG, typename TD, int V, int G>
static void launch_sums(const SumIn &in, const SumOut &o, hipStream_t st)
{
    const int32_t chunk = chunk_of(in.n, in.F);
    const int64_t chunks = ((int64_t)in.n + chunk - 1) / chunk;
    const unsigned slices = (unsigned)((in.F + G * V - 1) / (G * V));
    CSGS_LAUNCH(K_EMBED_SUM, (chunk_sums_k<TG, TD, V, G>), dim3((unsigned)((chunks * G + 255) / 256), slices), dim3(256), st, (const TG *)in.g, in.ldg, in.F,
                in.key, in.pos, in.n, in.n_dev, in.rows, chunk, in.part, o);
    CSGS_LAUNCH(K_EMBED_JOIN, (chunk_join_k<TD, V, G>), dim3((unsigned)((chunks + JOIN_WAVES - 1) / JOIN_WAVES), slices), dim3(JOIN_WAVES * WAVE), st, in.F, in.key,
                in.n, in.n_dev, in.rows, chunk, in.part, o);
}
template <typename TG, typename TD>
static int embed_grad_sums(const SumIn &in, const SumOut &o, hipStream_t st)
{
    if (!o.rank && !o.accumulate) {
        CSGS_LAUNCH(K_EMBED_ZERO, rows_zero_k<TD>, dim3(wave_blocks(in.rows)), dim3(256), st, (TD *)o.d, o.ldd, (int64_t)in.rows, in.F);
        CSGS_LAUNCH_CHECK();
    }
    constexpr int V = sizeof(TG) == 4 ? 4 : 8;
    if (in.F < V) launch_sums<TG, TD, 1, 16>(in, o, st);
    else if (in.F <= 16 * V) launch_sums<TG, TD, V, 16>(in, o, st);
    else if (in.F <= 32 * V) launch_sums<TG, TD, V, 32>(in, o, st);
    else launch_sums<TG, TD, V, 64>(in, o, st);
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
    if (uniq) {
        CSGS_LAUNCH(K_EMBED_HEADS, heads_count_k, dim3((unsigned)tiles), dim3(SORT_BLOCK), st, s.key[last], (int32_t)n, n_dev, tile, (uint32_t)rows, s.heads);
        CSGS_LAUNCH(K_EMBED_HEADS, heads_place_k, dim3((unsigned)tiles), dim3(SORT_BLOCK), st, s.key[last], (int32_t)n, n_dev, tile, tiles, (uint32_t)rows, s.heads,
                    s.rank, uniq, n_uniq);
        CSGS_LAUNCH_CHECK();
    }
    const SumIn in{G, ldg, F, s.key[last], s.pos[last], (int32_t)n, n_dev, (uint32_t)rows, s.part};
    const SumOut o{uniq ? s.rank : nullptr, d, ldd, scale, accumulate};
    if (g_dtype == CSGS_F32) return d_dtype == CSGS_F32 ? embed_grad_sums<float, float>(in, o, st) : embed_grad_sums<float, uint16_t>(in, o, st);
    return d_dtype == CSGS_F32 ? embed_grad_sums<uint16_t, float>(in, o, st) : embed_grad_sums<uint16_t, uint16_t>(in, o, st);
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
