// csgs_embed: rows of a learned table by id, scaled, and the table's gradient by sorted ids.
//
// Forward: out[t] = s T[i_t].  Gradient: dT[v] = s sum_{t : i_t = v} G[t].  The positions t are sorted by id (stable), so that those of a row
// lie side by side, in order; rows of G are then summed where they lie, in chunks of a fixed number of positions, in double, and
// every row of the gradient is written once.  Nothing is added with atomics: two calls give the same bits.
//
// A lookup is bound by memory: the rows of T once, the output once.  So is the gradient of many wide rows (G once, the output once); of
// few or narrow ones it is bound by the latency of its launches (3 to 4 us each) and of the loads in a row in them.  Three forms, by the
// number of positions n (us for gradient rows of 100 floats, one launch / ranges / digits; hubs: half of the positions uniform over 2.4 M
// rows, half log-uniform; zipf: log-uniform over 50 K; one: a single id):
//     n = 300     hubs 9.7 / 19.1   zipf 8.9 / 19.2    one 12.6 / 17.3
//     n = 2048    hubs 13.1 / 21.2 / 39   zipf 12.0 / 20.6 / 32   one 39 / 21.2 / 32
//     n = 32768   hubs - / 30.8 / 53.6   zipf - / 27.6 / 42.2   one - / 42.7 / 42.7
//     n = 98304   hubs - / 50.2 / 71.1   zipf - / 47.0 / 55.7   one - / 83.8 / 62.6
//     n = 131072  hubs - / 58.6 / 77.9   zipf - / 72.4 / 59.6   one - / 104 / 70.1
#include "common.hpp"
#include "row_pieces.hpp"

namespace csgs {

// ---------------------------------------------------------------- lookup
// G lanes take a row in pieces of V columns, and four rows at a time: the rows are as far apart as the ids say, so what counts is how many
// are asked for before the first is needed.  The last piece of a width that V does not divide ends with the row and overlaps the one before.
// (131 K rows of 100 bfloat16 values out of 2.4 M to floats 19.5 us, 4.0 TB/s of what has to move, a row lying across three lines of 128 bytes; a
// value a lane and a row at a time 38.)
template <typename TI, typename TO, int V, int G>
__global__ __launch_bounds__(256) void embed_k(const TI *T, int64_t ld, int64_t rows, int32_t F, const int32_t *__restrict__ ids, int32_t n_cap,
                                               const int32_t *__restrict__ n_dev, float scale, TO *out, int64_t ldo)
{
    constexpr int R = 4;
    const int32_t n = resolve_count(n_cap, n_dev);
    const int32_t begin = (int32_t)(blockIdx.y * G + threadIdx.x % G) * V, col = begin > F - V ? F - V : begin;
    const int64_t groups = (int64_t)gridDim.x * (256 / G);
    for (int64_t t0 = (int64_t)blockIdx.x * (256 / G) + threadIdx.x / G; t0 < n; t0 += groups * R) {
        int32_t id[R];
#pragma unroll
        for (int k = 0; k < R; ++k) id[k] = ids[t0 + k * groups < n ? t0 + k * groups : t0];
        if (begin >= F) continue;
        RawPiece<TI, V> r[R];
        bool ok[R];
#pragma unroll
        for (int k = 0; k < R; ++k) {
            ok[k] = id[k] >= 0 && id[k] < rows;
            r[k].load(T + (ok[k] ? id[k] : 0) * ld + col);
        }
#pragma unroll
        for (int k = 0; k < R; ++k) {
            const int64_t t = t0 + k * groups;
            Vec<V> v;
#pragma unroll
            for (int i = 0; i < V; ++i) v.x[i] = ok[k] ? scale * r[k].value(i) : 0.0f;
            if (t < n) store_row<TO, V>(out + t * ldo + col, v);
        }
    }
}

// ---------------------------------------------------------------- positions sorted by id
// An entry is an id and its position, id << 32 | position.  A pass sorts by one digit of up to 8 bits.  At most SORT_TILES blocks
// take consecutive tiles of the entries: the first kernel counts a tile's digits, the second one adds up what lies before its own
// (the counts of all tiles, at most 64 K of them) and places its entries.  No block waits for another.  (1 M entries: 7 and 22 us a pass.)
constexpr int SORT_TILES = 256, SORT_BLOCK = 256, SORT_WAVES = SORT_BLOCK / WAVE, DIGITS = 256;
static_assert(DIGITS == SORT_BLOCK, "a thread per digit");
constexpr int SORT_ITEMS = 8;                              // entries that a thread places at a time
constexpr int32_t SORT_STEP = SORT_BLOCK * SORT_ITEMS;     // a tile is a number of these

// Sorted positions are summed in chunks of a fixed number, whatever ids they hold (see chunk_sums_k): a block takes a chunk, groups of G lanes
// take equal shares of it.  A share is as many positions as leave a million values of the sums at a time (1024 wavefronts of 16 bytes a lane), 8
// to 64, no more than the lanes that take a row.
constexpr int SUM_BLOCK = 256;
__host__ inline int32_t share_of(int64_t n, int32_t F)
{
    const int32_t most = F <= 128 ? 16 : (F <= 256 ? 32 : 64);
    int32_t c = 8;
    while (c < most && n / (2 * c) * F >= 1 << 20) c *= 2;
    return c;
}
// Lanes that take a row in pieces of V columns.
__host__ inline int sum_lanes(int32_t F, int V) { return F <= 16 * V ? 16 : (F <= 32 * V ? 32 : 64); }

struct EmbedScratch {
    uint64_t *entry[2];          // [n] entries, used in turn
    uint32_t *hist;              // [SORT_TILES][DIGITS] of a pass
    uint32_t *heads;             // [SORT_TILES] different ids that begin in a tile; of every range
    int32_t *n_valid;            // positions whose id is in the table
    uint32_t *rank;              // [n] of an entry's id among the different ones
    double *part;                // [chunks][2][F] sums of rows that go on across chunks
    size_t bytes;
};
// Room for the parts of n positions, [chunks][2][F] doubles, and of fewer or narrower ones: a buffer for the largest call serves the smaller ones, though
// these may have more chunks (a share doubles where there is enough to do).  F ceil(n / chunk) <= n F / chunk + F, and with the smallest lanes of all types
//     a chunk is never shorter than 8 positions times 256 / lanes,
//     one whose share is at its most never shorter than 128 positions,
//     any other share c has n F < 2 c (2^20 + F), which leaves n F / chunk < (2^20 + F) lanes / 128 <= (2^20 + F) / 2.
// Each bound grows with n and with F.
__host__ inline size_t part_doubles(int64_t n, int32_t F)
{
    const int64_t shortest = n * F / (8 * SUM_BLOCK / sum_lanes(F, 4)), at_most = n * F / 128, other = ((1 << 20) + (int64_t)F) / 2;
    const int64_t any = at_most > other ? at_most : other;
    return 2 * (size_t)((shortest < any ? shortest : any) + F + 1);
}
__host__ inline EmbedScratch carve_embed(void *base, int64_t n, int32_t F)
{
    EmbedScratch s;
    size_t off = 0;
    auto take = [&](size_t bytes) {
        const size_t o = off;
        off = align_up(off + bytes, 256);
        return (char *)base + o;
    };
    for (int i = 0; i < 2; ++i) s.entry[i] = (uint64_t *)take((size_t)n * 8);
    s.hist = (uint32_t *)take(sizeof(uint32_t) * DIGITS * SORT_TILES);
    s.heads = (uint32_t *)take(sizeof(uint32_t) * SORT_TILES);
    s.n_valid = (int32_t *)take(4);
    s.rank = (uint32_t *)take((size_t)n * 4);
    s.part = (double *)take(sizeof(double) * part_doubles(n, F));
    s.bytes = off;
    return s;
}

// Where the entries of a pass come from: the caller's ids in the first one (ids outside the table take the key `rows`, behind
// all others), the entries of the pass before in the others.
__device__ inline uint32_t key_of(uint64_t entry) { return (uint32_t)(entry >> 32); }
struct SortIn {
    const int32_t *ids;
    const uint64_t *entry;
    uint32_t rows;
    __device__ uint64_t get(int64_t i) const
    {
        if (!ids) return entry[i];
        const uint32_t id = (uint32_t)ids[i];
        return (uint64_t)(id < rows ? id : rows) << 32 | (uint32_t)i;
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
    for (int64_t i = beg + threadIdx.x; i < end; i += SORT_BLOCK) atomicAdd(&count[(key_of(in.get(i)) >> shift) & mask], 1u);
    __syncthreads();
    hist[blockIdx.x * DIGITS + threadIdx.x] = count[threadIdx.x];
}

// The lanes of the wavefront whose digit (of up to 8 bits) is this lane's own, among those that take part.
struct Lanes {
    uint32_t lo, hi;
    __device__ uint32_t count() const { return (uint32_t)(__popc(lo) + __popc(hi)); }
    __device__ uint32_t before() const { return (uint32_t)__builtin_amdgcn_mbcnt_hi(hi, __builtin_amdgcn_mbcnt_lo(lo, 0)); }   // lower lanes
};
__device__ inline Lanes same_digit(uint32_t digit, uint64_t active)
{
    Lanes p{(uint32_t)active, (uint32_t)(active >> 32)};
#pragma unroll
    for (int b = 0; b < 8; ++b) {
        const uint32_t all = (uint32_t)((int32_t)(digit << (31 - b)) >> 31);   // the bit, 32 times
        const uint64_t with = __ballot(all != 0);
        p.lo &= ~((uint32_t)with ^ all);
        p.hi &= ~((uint32_t)(with >> 32) ^ all);
    }
    return p;
}

__device__ inline uint32_t digit_of(uint64_t e, uint32_t least, int shift, int bits) { return ((key_of(e) - least) >> shift) & ((1u << bits) - 1u); }
__device__ inline int bits_of(uint32_t x) { return x ? 32 - __clz((int)x) : 0; }

// A wavefront's entries of a step: rank[u] = entries before that one with its digit in the wavefront's share, `count` [DIGITS] (zeros before) = how
// many there are of each.  Entries u * 64 + lane, of which those with `active` count.
// (The counts are read and written through a pointer that says that it is one to LDS: through a generic one they would be flat accesses, and volatile
// ones past all caches at that, 2 us a pass.)
typedef volatile __attribute__((address_space(3))) uint32_t *LdsCounts;
template <int ITEMS>
__device__ inline void rank_digits(const uint64_t (&e)[ITEMS], const bool (&active)[ITEMS], int shift, int bits, LdsCounts count, uint32_t (&rank)[ITEMS],
                                   uint32_t least = 0)
{
#pragma unroll
    for (int u = 0; u < ITEMS; ++u) {
        rank[u] = 0;
        const uint64_t some = __ballot(active[u]);
        if (some == 0) continue;
        const uint32_t digit = digit_of(e[u], least, shift, bits);
        const Lanes peers = same_digit(digit, some);
        const uint32_t before = peers.before();
        uint32_t seen = 0;
        if (active[u]) seen = count[digit];
        __builtin_amdgcn_wave_barrier();
        if (active[u] && before == 0) count[digit] = seen + peers.count();
        __builtin_amdgcn_wave_barrier();
        rank[u] = seen + before;
    }
}

__global__ __launch_bounds__(SORT_BLOCK) void sort_place_k(SortIn in, int32_t n_cap, const int32_t *__restrict__ n_dev, int32_t tile, int tiles,
                                                           int shift, int bits, const uint32_t *__restrict__ hist, uint64_t *__restrict__ out)
{
    __shared__ uint32_t at[SORT_WAVES][DIGITS];   // a wavefront's entries by digit, then the place of its first
    __shared__ uint32_t scan[17];
    const int32_t n = resolve_count(n_cap, n_dev);
    const int64_t beg = (int64_t)blockIdx.x * tile;
    const int64_t end = beg + tile < n ? beg + tile : n;
    if (beg >= end) return;
    const uint32_t mask = (1u << bits) - 1;
    const int tid = (int)threadIdx.x, wave = tid / WAVE;
    auto load = [&](int64_t i0, uint64_t (&e)[SORT_ITEMS], bool (&active)[SORT_ITEMS]) {
#pragma unroll
        for (int u = 0; u < SORT_ITEMS; ++u) {
            const int64_t i = i0 + wave * (SORT_ITEMS * WAVE) + u * WAVE + lane_id();
            active[u] = i < end;
            e[u] = in.get(active[u] ? i : end - 1);
        }
    };
    uint64_t e[SORT_ITEMS];
    bool active[SORT_ITEMS];
    load(beg, e, active);
    // entries with a smaller digit, and of this digit in earlier tiles
    uint32_t before = 0, all = 0, total;
#pragma unroll 8
    for (int t = 0; t < tiles; ++t) {
        const uint32_t c = hist[t * DIGITS + tid];
        before += t < (int)blockIdx.x ? c : 0u;
        all += c;
    }
    uint32_t next = block_exclusive_scan<uint32_t>(all, scan, &total) + before;   // of the thread's digit
    for (int64_t i0 = beg; i0 < end; i0 += SORT_STEP) {
        if (i0 > beg) load(i0, e, active);
        __syncthreads();
#pragma unroll
        for (int w = 0; w < SORT_WAVES; ++w) at[w][tid] = 0;
        __syncthreads();
        uint32_t rank[SORT_ITEMS];
        rank_digits(e, active, shift, bits, (LdsCounts)at[wave], rank);
        __syncthreads();
#pragma unroll
        for (int w = 0; w < SORT_WAVES; ++w) {
            const uint32_t c = at[w][tid];
            at[w][tid] = next;
            next += c;
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < SORT_ITEMS; ++u)
            if (active[u]) {
                const uint32_t dst = at[wave][(key_of(e[u]) >> shift) & mask] + rank[u];
                if (dst < (uint32_t)n) out[dst] = e[u];
            }
    }
}

// ---------------------------------------------------------------- a block's own sort
constexpr int WIDE = 1024, WIDE_WAVES = WIDE / WAVE, WIDE_ITEMS = 7;
constexpr int LDS_ENTRIES = WIDE * WIDE_ITEMS;   // most entries that a block sorts in LDS (two such blocks fit on a compute unit)
struct __attribute__((aligned(16))) SortLds {
    uint32_t at[WIDE_WAVES][DIGITS];   // a wavefront's entries by digit, then the place of its first
    uint32_t scan[17];
};

// Ranks of a step of at most WIDE * ITEMS entries among those of their wavefront and digit, which at[][] is left counting, for
// the first `waves` wavefronts (the others hold no entry).  The caller's entries are loaded when it returns, and nothing is stored yet.
template <int ITEMS>
__device__ inline void step_ranks(const uint64_t (&e)[ITEMS], const bool (&active)[ITEMS], uint32_t least, int shift, int bits, int waves, SortLds &l,
                                  uint32_t (&rank)[ITEMS])
{
    const int tid = (int)threadIdx.x;
    __syncthreads();
    for (int x = tid; x < waves * DIGITS; x += WIDE) (&l.at[0][0])[x] = 0;
    __syncthreads();
    rank_digits(e, active, shift, bits, (LdsCounts)l.at[tid / WAVE], rank, least);
    __syncthreads();
}
// Threads 0 .. 255, thread = digit: each wavefront's entries of it, then (places()) the place of each wavefront's first, from `next` on.
struct DigitCounts {
    uint32_t c[WIDE_WAVES], all;
    __device__ DigitCounts(const SortLds &l, int waves)
    {
        all = 0;
#pragma unroll
        for (int w = 0; w < WIDE_WAVES; ++w) c[w] = w < waves ? l.at[w][threadIdx.x % DIGITS] : 0u;
#pragma unroll
        for (int w = 0; w < WIDE_WAVES; ++w) all += c[w];
    }
    __device__ void places(SortLds &l, int waves, uint32_t next) const
    {
#pragma unroll
        for (int w = 0; w < WIDE_WAVES; ++w) {
            if (w < waves) l.at[w][threadIdx.x] = next;
            next += c[w];
        }
    }
};
// Exclusive sum over threads 0 .. 255 (a thread per digit); all threads call it.
__device__ inline uint32_t digits_scan(uint32_t v, uint32_t *lds /*[DIGITS / WAVE]*/)
{
    const int wave = (int)threadIdx.x / WAVE;
    uint32_t incl = 0;
    if (wave < DIGITS / WAVE) {
        incl = wave_inclusive_scan(v);
        if (lane_id() == WAVE - 1) lds[wave] = incl;
    }
    __syncthreads();
    uint32_t before = 0;
#pragma unroll
    for (int w = 0; w < DIGITS / WAVE; ++w) before += w < wave ? lds[w] : 0u;
    return before + incl - v;
}

// Sorts m <= WIDE * ITEMS entries in LDS by key, stable, where keys lie in [least, least + span].
template <int ITEMS>
__device__ inline void sort_in_lds(uint64_t *e, int m, uint32_t least, uint32_t span, SortLds &l)
{
    const int key_bits = bits_of(span), passes = (key_bits + 7) / 8, bits = passes ? (key_bits + passes - 1) / passes : 0;
    const int tid = (int)threadIdx.x, wave = tid / WAVE, steps = (m + WIDE - 1) / WIDE, waves = (m + steps * WAVE - 1) / (steps * WAVE);
    for (int p = 0; p < passes; ++p) {
        uint64_t v[ITEMS];
        bool active[ITEMS];
        uint32_t rank[ITEMS];
#pragma unroll
        for (int u = 0; u < ITEMS; ++u) {
            const int i = (wave * steps + u) * WAVE + lane_id();
            active[u] = u < steps && i < m;
            v[u] = active[u] ? e[i] : 0ull;
        }
        step_ranks(v, active, least, p * bits, bits, waves, l, rank);
        const DigitCounts dc(l, waves);   // (threads past the digits: not used)
        const uint32_t first = digits_scan(dc.all, l.scan);
        if (tid < DIGITS) dc.places(l, waves, first);
        __syncthreads();
#pragma unroll
        for (int u = 0; u < ITEMS; ++u)
            if (active[u]) e[l.at[wave][digit_of(v[u], least, p * bits, bits)] + rank[u]] = v[u];
        __syncthreads();
    }
}

// Sorts m <= COUNTED entries in LDS by key, stable, where keys lie less than COUNTED_SPAN above `least`, by the number of smaller ones: a power of
// two of threads for the entries, as many sets of them as there are threads, each looking at its share.
constexpr int COUNTED_BITS = 9, COUNTED = 1 << COUNTED_BITS;
constexpr uint32_t COUNTED_SPAN = 1u << (32 - COUNTED_BITS);
__device__ inline void sort_by_counting(uint64_t *e, int m, uint32_t least, SortLds &l)
{
    uint32_t *order = &l.at[0][0], *smaller = order + COUNTED;   // key and place of an entry in 32 bits; what is counted
    const int tid = (int)threadIdx.x;
    int width = WAVE;
    while (width < m) width *= 2;
    const int i = tid & (width - 1), sets = WIDE / width, share = ((m + sets - 1) / sets + 3) / 4 * 4;
    const int j0 = tid / width * share, j1 = j0 + share < m ? j0 + share : m;
    const uint64_t mine = i < m ? e[i] : 0ull;
    if (tid < COUNTED) {
        order[tid] = tid < m ? (key_of(e[tid]) - least) << COUNTED_BITS | (uint32_t)tid : 0xFFFFFFFFu;   // (none: no smaller than any)
        smaller[tid] = 0;
    }
    __syncthreads();
    const uint32_t own = order[i];
    uint32_t c = 0;
#pragma unroll 4
    for (int j = j0; j < j1; j += 4) {
        const uint4 q = *reinterpret_cast<const uint4 *>(order + j);
        c += (q.x < own ? 1u : 0u) + (q.y < own ? 1u : 0u) + (q.z < own ? 1u : 0u) + (q.w < own ? 1u : 0u);
    }
    if (c && i < m) atomicAdd(&smaller[i], c);
    __syncthreads();
    if (tid < m) e[smaller[tid]] = mine;
    __syncthreads();
}

// Order statistics of a sample, SAMPLES of whose keys a thread holds (has[i]: it does): found[t] = the one that target[t] others precede, by
// digits from the top.  A level counts the samples that share what is known of a target by their next digit; targets of which the same is
// known share the counts.  Keys of up to key_bits bits.
constexpr int TARGETS = 3;
struct SelectLds {
    uint32_t count[TARGETS][DIGITS];
    uint32_t key[TARGETS], left[TARGETS];
};
template <int SAMPLES>
__device__ inline void select_samples(const uint32_t (&sample)[SAMPLES], const bool (&has)[SAMPLES], int key_bits, const int (&target)[TARGETS], SelectLds &l,
                                      uint32_t (&found)[TARGETS])
{
    const int tid = (int)threadIdx.x, wave = tid / WAVE, lane = lane_id();
    uint32_t left[TARGETS];
#pragma unroll
    for (int t = 0; t < TARGETS; ++t) {
        found[t] = 0;
        left[t] = (uint32_t)target[t];
    }
    for (int v = (key_bits + 7) / 8 - 1; v >= 0; --v) {
        const uint64_t known = ~0ull << (8 * v + 8);
        int counts[TARGETS];   // whose counts a target uses
#pragma unroll
        for (int t = 0; t < TARGETS; ++t) counts[t] = t > 0 && ((found[t] ^ found[t - 1]) & known) == 0 ? counts[t - 1] : t;
        if (tid < DIGITS)
#pragma unroll
            for (int t = 0; t < TARGETS; ++t) l.count[t][tid] = 0;
        __syncthreads();
#pragma unroll
        for (int t = 0; t < TARGETS; ++t)
            if (counts[t] == t)
#pragma unroll
                for (int i = 0; i < SAMPLES; ++i)
                    if (has[i] && ((sample[i] ^ found[t]) & known) == 0) atomicAdd(&l.count[t][(sample[i] >> (8 * v)) & (DIGITS - 1)], 1u);
        __syncthreads();
        if (wave < TARGETS) {   // a wavefront a target, four digits a lane
            uint32_t want = left[0], key = found[0];
            int from = counts[0];
#pragma unroll
            for (int t = 1; t < TARGETS; ++t)
                if (wave == t) { want = left[t]; key = found[t]; from = counts[t]; }
            const uint4 c = *reinterpret_cast<const uint4 *>(&l.count[from][4 * lane]);
            const uint32_t sum = c.x + c.y + c.z + c.w, before = wave_inclusive_scan(sum) - sum;
            if (before <= want && want < before + sum) {   // one lane
                uint32_t r = want - before, d = 0;
                if (r >= c.x) { r -= c.x; d = 1;
                    if (r >= c.y) { r -= c.y; d = 2;
                        if (r >= c.z) { r -= c.z; d = 3; } } }
                l.key[wave] = key | (uint32_t)(4 * lane + (int)d) << (8 * v);
                l.left[wave] = r;
            }
        }
        __syncthreads();
#pragma unroll
        for (int t = 0; t < TARGETS; ++t) {
            found[t] = l.key[t];
            left[t] = l.left[t];
        }
    }
}

// The same for any number of entries in global memory, from a to b and back; returns where they are in the end (a or b).
__device__ inline uint64_t *sort_in_memory(uint64_t *a, uint64_t *b, int64_t m, uint32_t least, uint32_t span, SortLds &l)
{
    constexpr int ITEMS = 4;
    const int key_bits = bits_of(span), passes = (key_bits + 7) / 8, bits = passes ? (key_bits + passes - 1) / passes : 0;
    const int tid = (int)threadIdx.x, wave = tid / WAVE;
    for (int p = 0; p < passes; ++p) {
        __syncthreads();
        if (tid < DIGITS) l.at[0][tid] = 0;
        __syncthreads();
        for (int64_t i = tid; i < m; i += WIDE) atomicAdd(&l.at[0][digit_of(a[i], least, p * bits, bits)], 1u);
        __syncthreads();
        const uint32_t all = tid < DIGITS ? l.at[0][tid] : 0u;
        uint32_t total, next = block_exclusive_scan<uint32_t>(all, l.scan, &total);
        for (int64_t i0 = 0; i0 < m; i0 += WIDE * ITEMS) {
            uint64_t v[ITEMS];
            bool active[ITEMS];
            uint32_t rank[ITEMS];
#pragma unroll
            for (int u = 0; u < ITEMS; ++u) {
                const int64_t i = i0 + (wave * ITEMS + u) * WAVE + lane_id();
                active[u] = i < m;
                v[u] = active[u] ? a[i] : 0ull;
            }
            step_ranks(v, active, least, p * bits, bits, WIDE_WAVES, l, rank);
            if (tid < DIGITS) {
                const DigitCounts dc(l, WIDE_WAVES);
                dc.places(l, WIDE_WAVES, next);
                next += dc.all;
            }
            __syncthreads();
#pragma unroll
            for (int u = 0; u < ITEMS; ++u)
                if (active[u]) b[l.at[wave][digit_of(v[u], least, p * bits, bits)] + rank[u]] = v[u];
        }
        __syncthreads();
        uint64_t *t = a;
        a = b;
        b = t;
    }
    return a;
}

// ---------------------------------------------------------------- zeros
// Rows of `row` bytes (a multiple of 2), `ld` bytes apart, by worker `me` of `workers` wavefronts.
struct ZeroRows {
    void *d;
    int64_t rows, row, ld;   // rows = 0: none
};
__device__ inline void zero_rows(const ZeroRows &z, int64_t me, int64_t workers)
{
    const bool flat = z.row == z.ld;   // then one row of everything, in pieces of 16 KB
    const int64_t rows = flat ? (z.rows * z.row + 16383) / 16384 : z.rows, ld = flat ? 16384 : z.ld;
    for (int64_t r = me; r < rows; r += workers) {
        char *p = (char *)z.d + r * ld;
        const int64_t len = !flat ? z.row : (r + 1 < rows ? 16384 : z.rows * z.row - r * 16384);
        for (int64_t at = lane_id() * 16; at < len; at += WAVE * 16) {
            if (at + 16 <= len) store_global<u32x4, 2>(p + at, u32x4{0, 0, 0, 0});
            else
                for (int64_t b = at; b < len; b += 2) store_global<uint16_t>(p + b, (uint16_t)0);
        }
    }
}
__global__ __launch_bounds__(256) void rows_zero_k(ZeroRows z)
{
    zero_rows(z, ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) / WAVE, (int64_t)gridDim.x * blockDim.x / WAVE);
}

// ---------------------------------------------------------------- positions sorted by id, in one launch
// A block owns a range of ids, looks at all ids itself and lists those of its range in order of position; how many lie below the range
// says where its list belongs among the sorted entries, so that no block waits for another.  Ranges hold about as many positions
// each: every block selects its bounds from the same sample of the ids.  An id that fills bounds by itself has a
// range of its own, which needs no sorting however many positions it holds; a list that outgrows LDS all the same (a sample that misses) is
// sorted in memory.  Further blocks clear the gradient's rows meanwhile.  Bound by the instructions that look at every id in every block (13 us for
// 131 K) and by latency.  (us, 32 K positions: 13; of those 2 until the ids are there, 3 for the bounds, 2 for the lists, 1 to sort 120
// entries.  Bounds by sorting 1024 samples took 6; lists sorted by digits 4; the ids kept in registers between counting and listing is level.)
constexpr int RANGES = 256, SAMPLE = 4 * WIDE;
constexpr uint32_t OWN_LIST = LDS_ENTRIES / WIDE_WAVES;   // entries of its range that a wavefront lists in LDS
// Block b's ids are [lo, lo + width): bounds are, of the sorted samples, the (r samples / RANGES)-th.  All threads call it.
struct Range {
    uint32_t lo, width;
};
template <int SAMPLES>
__device__ inline Range range_of(int b, const uint32_t (&sample)[SAMPLES], const bool (&has)[SAMPLES], int samples, uint32_t rows, SelectLds &sel)
{
    auto target = [&](int r) { return (int)((int64_t)(r < 0 ? 0 : r < RANGES ? r : RANGES - 1) * samples / RANGES); };
    const int targets[TARGETS] = {target(b - 1), target(b), target(b + 1)};
    uint32_t bound[TARGETS];
    select_samples(sample, has, bits_of(rows), targets, sel, bound);
    uint32_t lo = b > 0 ? bound[1] : 0u, hi = b + 1 < RANGES ? bound[2] : rows;
    const bool again = b > 0 && (b > 1 ? bound[0] : 0u) == lo;   // the id `lo` is another block's
    if (lo == hi && !again) hi = lo + 1;                         // ... this one's, alone
    else if (again) ++lo;
    if (hi > rows) hi = rows;
    if (lo > hi) lo = hi;
    return Range{lo, hi - lo};
}
__global__ __launch_bounds__(WIDE) void sort_ranges_k(const int32_t *__restrict__ ids, int32_t n_cap, const int32_t *__restrict__ n_dev, uint32_t rows,
                                                      uint64_t *out, uint64_t *other, uint32_t *__restrict__ rank, uint32_t *__restrict__ distinct,
                                                      int32_t *__restrict__ n_valid, ZeroRows z)
{
    constexpr int U = 8;   // ids on their way per lane
    __shared__ uint64_t e[LDS_ENTRIES];
    __shared__ SortLds l;
    __shared__ __attribute__((aligned(16))) SelectLds sel;
    __shared__ uint32_t w_below[WIDE_WAVES], w_own[WIDE_WAVES];
    const int tid = (int)threadIdx.x, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(tid / WAVE), b = (int)blockIdx.x;
    if (b >= RANGES) return zero_rows(z, (int64_t)(b - RANGES) * WIDE_WAVES + wave, (int64_t)(gridDim.x - RANGES) * WIDE_WAVES);
    const int32_t n = resolve_count(n_cap, n_dev);
    if (n == 0) {
        if (tid == 0) {
            distinct[b] = 0;
            if (b == 0) *n_valid = 0;
        }
        return;
    }
    auto key_at = [&](int64_t i) {
        const uint32_t id = (uint32_t)ids[i];
        return id < rows ? id : rows;
    };
    const int32_t share = (n + WIDE - 1) / WIDE * WAVE;   // positions of a wavefront
    const int32_t w_beg = wave * share, w_end = w_beg + share < n ? w_beg + share : n;
    const int samples = n < SAMPLE ? n : SAMPLE;
    uint32_t sample[SAMPLE / WIDE];
    bool has[SAMPLE / WIDE];
#pragma unroll
    for (int i = 0; i < SAMPLE / WIDE; ++i) {
        const int k = i * WIDE + tid;
        has[i] = k < samples;
        sample[i] = key_at((int64_t)(has[i] ? k : 0) * n / samples);
    }
    // the ids from position i0 on, a wavefront's 64 at a time, and what lies past its share as none
    auto ask = [&](int32_t i0, uint32_t (&id)[U]) {
        if (i0 + U * WAVE <= w_end) {
#pragma unroll
            for (int u = 0; u < U; ++u) id[u] = (uint32_t)(ids + i0)[(uint32_t)(lane + u * WAVE)];
            return;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int32_t i = i0 + u * WAVE + lane;
            id[u] = (uint32_t)ids[i < n ? i : n - 1];
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (i0 + u * WAVE + lane >= w_end) id[u] = 0xFFFFFFFFu;
    };
    // f(ids, first position), over the wavefront's share
    auto each = [&](auto f) {
        for (int32_t i0 = w_beg; i0 < w_end; i0 += U * WAVE) {
            uint32_t id[U];
            ask(i0, id);
            f(id, i0);
        }
    };
    const Range range = range_of(b, sample, has, samples, rows, sel);
    const uint32_t lo = range.lo;
    const uint32_t width = range.width;
    // ids below the range, and those in it: each wavefront lists its own in its part of LDS as far as that goes
    const uint64_t lanes_below = (1ull << lane) - 1ull;
    uint32_t n_below = 0, n_own = 0;   // (n_below: the lane's)
    each([&](const uint32_t (&id)[U], int32_t i0) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            n_below += id[u] < lo ? 1u : 0u;
            const bool is = id[u] - lo < width;
            const uint64_t m = __ballot(is);
            if (m == 0) continue;
            const uint32_t dst = n_own + (uint32_t)__popcll(m & lanes_below);
            if (is && dst < OWN_LIST) e[wave * OWN_LIST + dst] = (uint64_t)id[u] << 32 | (uint32_t)(i0 + u * WAVE + lane);
            n_own += (uint32_t)__popcll(m);
        }
    });
    n_below = wave_sum(n_below);
    if (lane == 0) {
        w_below[wave] = n_below;
        w_own[wave] = n_own;
    }
    __syncthreads();
    uint32_t below = 0, own = 0, at = 0, most = 0;
    for (int w = 0; w < WIDE_WAVES; ++w) {
        const uint32_t c = w_own[w];
        below += w_below[w];
        if (w == wave) at = own;
        own += c;
        most = c > most ? c : most;
    }
    if (b == RANGES - 1 && tid == 0) *n_valid = (int32_t)(below + own);
    if (own == 0) {
        if (tid == 0) distinct[b] = 0;
        return;
    }
    const bool alone = width == 1, in_lds = most <= OWN_LIST;
    if (in_lds) {
        // the wavefronts' lists after each other
        uint64_t v[OWN_LIST / WAVE];
#pragma unroll
        for (int u = 0; u < OWN_LIST / WAVE; ++u)
            if (u * WAVE + lane < (int)n_own) v[u] = e[wave * OWN_LIST + u * WAVE + lane];
        __syncthreads();
#pragma unroll
        for (int u = 0; u < OWN_LIST / WAVE; ++u)
            if (u * WAVE + lane < (int)n_own) e[at + u * WAVE + lane] = v[u];
        __syncthreads();
        if (alone) {
        } else if (own <= COUNTED && width <= COUNTED_SPAN) sort_by_counting(e, (int)own, lo, l);
        else sort_in_lds<WIDE_ITEMS>(e, (int)own, lo, width - 1, l);
    } else {
        const int passes = (bits_of(width - 1) + 7) / 8;
        uint64_t *mine = passes % 2 == 0 ? out : other;   // the sorted list has to end in `out`
        each([&](const uint32_t (&id)[U], int32_t i0) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const bool is = id[u] - lo < width;
                const uint64_t m = __ballot(is);
                const uint32_t dst = below + at + (uint32_t)__popcll(m & lanes_below);
                if (is && dst < (uint32_t)n) mine[dst] = (uint64_t)id[u] << 32 | (uint32_t)(i0 + u * WAVE + lane);
                at += (uint32_t)__popcll(m);
            }
        });
        __syncthreads();
        sort_in_memory(mine + below, (mine == out ? other : out) + below, own, lo, width - 1, l);   // (an id alone: no pass)
    }
    // entries out, with their id's rank in the list
    uint32_t base = 0;
    for (uint32_t i0 = 0; i0 < own; i0 += WIDE) {
        const uint32_t i = i0 + (uint32_t)tid;
        if (in_lds && i < own) out[below + i] = e[i];
        if (!rank) continue;
        if (alone) {
            if (i < own) rank[below + i] = (uint32_t)b << 24;
            continue;
        }
        bool head = false;
        if (i < own) head = i == 0 || (in_lds ? key_of(e[i]) != key_of(e[i - 1]) : key_of(out[below + i]) != key_of(out[below + i - 1]));
        uint32_t total;
        const uint32_t before = base + block_exclusive_scan<uint32_t>(head ? 1u : 0u, l.scan, &total);
        base += total;
        if (i < own) rank[below + i] = (uint32_t)b << 24 | (before + (head ? 1u : 0u) - 1u);
    }
    if (tid == 0) distinct[b] = alone ? 1u : base;
}
constexpr int64_t RANGES_MAX = 3 << 15;   // most positions of this form
static_assert(RANGES_MAX <= 1 << 24 && RANGES <= 256, "a block and a rank in 32 bits");

// ---------------------------------------------------------------- the different ids
// The keys of sorted entries.
struct Keys {
    const uint64_t *entry;
    __device__ uint32_t operator[](int64_t i) const { return (uint32_t)(entry[i] >> 32); }
};
__device__ inline bool is_head(const Keys &key, int64_t i, uint32_t rows)
{
    const uint32_t k = key[i], before = key[i > 0 ? i - 1 : 0];
    return k < rows && (i == 0 || before != k);
}

__global__ __launch_bounds__(SORT_BLOCK) void heads_count_k(Keys key, int32_t n_cap, const int32_t *__restrict__ n_dev,
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

__global__ __launch_bounds__(SORT_BLOCK) void heads_place_k(Keys key, int32_t n_cap, const int32_t *__restrict__ n_dev,
                                                            int32_t tile, int tiles, uint32_t rows, const uint32_t *__restrict__ heads,
                                                            uint32_t *__restrict__ rank, int32_t *__restrict__ n_uniq)
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
        if (i < end) rank[i] = before + (head ? 1u : 0u) - 1u;
    }
}

// ---------------------------------------------------------------- sums
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
    const uint32_t *rank;       // null: dense
    const uint32_t *distinct;   // the different ids of every range (rank: range << 24 | rank in it); null: ranks are ranks
    int32_t *uniq, *n_uniq;
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
        for (int i = 0; i < V; ++i) v.x[i] = float_to_store<TD>(acc[i] * (double)o.scale + (double)v.x[i]);
        store_row<TD, V>(d, v);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i >= pc.skip) {
                const float old = o.accumulate ? load_row<TD, 1>(d + i).x[0] : 0.0f;
                store_row<TD, 1>(d + i, Vec<1>{{float_to_store<TD>(acc[i] * (double)o.scale + (double)old)}});
            }
    }
}
template <int V>
__device__ inline void write_part(double *part, const Piece1<V> &pc, const double (&acc)[V])
{
    if (!pc.active) return;
#pragma unroll
    for (int i = 0; i < V; ++i) part[pc.col + i] = acc[i];   // (values of two pieces: the same from both)
}

// Rows of the output before each range's.  All threads of a block of 256 or more.
__device__ inline void range_bases(const SumOut &o, uint32_t *base /*[RANGES]*/, uint32_t *scan /*[17]*/, uint32_t *total)
{
    const int tid = (int)threadIdx.x;
    const uint32_t first = block_exclusive_scan<uint32_t>(tid < RANGES ? o.distinct[tid] : 0u, scan, total);
    if (tid < RANGES) base[tid] = first;
    __syncthreads();
}
__device__ inline uint32_t row_of_rank(const SumOut &o, uint32_t rank, const uint32_t *base) { return o.distinct ? base[rank >> 24] + (rank & 0xFFFFFFu) : rank; }

// Value of lane `from` of the G lanes that work together.
template <int G>
__device__ inline uint32_t from_lane(uint32_t v, int from)
{
    if constexpr (G == WAVE) return (uint32_t)__builtin_amdgcn_readlane((int)v, from);
    return (uint32_t)__shfl((int)v, from, G);
}

// G lanes take a share of a chunk of sorted positions: the rows of G that they point to are added up in order, eight on their way at a time; a
// table row all of whose positions lie in the share is written at once.  Parts of rows that go on across shares are joined in LDS, in order, and written
// there as far as they lie in the chunk; parts of others go to `part`, slot 1 of a row that begins in the chunk and goes on, slot 0 of one that
// began before it.  The work per chunk does not depend on how often an id occurs.  Bound by memory.  (131 K rows of 250 floats 24 us, 5.4 TB/s; 65 K of
// 512 bfloat16 values into 50 K rows of floats 21.  Parts left in memory by every share instead: 131 K positions of 100 values 18 and 20 us to join them,
// 16 and 7 now.)
template <typename TG, typename TD, int V, int G>
__global__ __launch_bounds__(256) void chunk_sums_k(const TG *g, int64_t ldg, int32_t F, const uint64_t *__restrict__ entry,
                                                    int32_t n_cap, const int32_t *__restrict__ n_dev, uint32_t rows, int32_t share,
                                                    double *__restrict__ part, SumOut o)
{
    constexpr int U = 8, GROUPS = SUM_BLOCK / G;
    constexpr uint32_t OPEN = 1, GOES_ON = 2, ONE = 4;   // a share's first row began before it; its last one goes on after it; it holds one row
    __shared__ uint32_t base[RANGES], scan[17], kinds[GROUPS], first_row[GROUPS];
    __shared__ double slot[2][GROUPS][G * V];
    const int32_t n = resolve_count(n_cap, n_dev);
    if (o.distinct) {
        uint32_t total;
        range_bases(o, base, scan, &total);
        if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *o.n_uniq = (int32_t)total;
    }
    const int lane = (int)threadIdx.x % G;
    const int q = (int)threadIdx.x / G;
    const int64_t beg = ((int64_t)blockIdx.x * GROUPS + q) * share;
    const int64_t end = beg + share < n ? beg + share : n;
    const int len = end > beg ? (int)(end - beg) : 0;
    const uint32_t NONE = 0xFFFFFFFFu;
    uint32_t k = NONE, p = 0, rk = 0;
    if (lane < len) {
        const uint64_t e = entry[beg + lane];
        k = key_of(e);
        p = (uint32_t)e;
        if (o.rank) rk = row_of_rank(o, o.rank[beg + lane], base);
    }
    const uint32_t row = o.rank ? rk : k;
    const Keys key{entry};
    const uint32_t before = len > 0 && beg > 0 ? key[beg - 1] : NONE, after = len > 0 && end < n ? key[end] : NONE;
    const uint32_t prev = (uint32_t)__shfl_up((int)k, 1, G);
    const uint32_t next = (uint32_t)__shfl_down((int)k, 1, G);
    const bool valid = lane < len && k < rows;
    const bool last = valid && (lane == len - 1 ? after != k : next != k);      // the row's last position
    const bool first = valid && (lane == 0 ? before != k : prev != k);
    if (first && o.rank && blockIdx.y == 0) o.uniq[rk] = (int32_t)k;
    const int shift = (int)(threadIdx.x & (WAVE - 1)) / G * G;
    const uint64_t lanes = G == WAVE ? ~0ull : (1ull << (G % WAVE)) - 1ull;
    const uint64_t m_valid = (__ballot(valid) >> shift) & lanes, m_last = (__ballot(last) >> shift) & lanes, m_first = (__ballot(first) >> shift) & lanes;
    const int count = __popcll(m_valid);
    const Piece1<V> pc((int32_t)(blockIdx.y * G + lane), F);
    double acc[V];
#pragma unroll
    for (int i = 0; i < V; ++i) acc[i] = 0.0;
    bool inside = true;    // the row's sum began in this share
    for (int i0 = 0; i0 < share; i0 += U) {
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
                    else
#pragma unroll
                        for (int j = 0; j < V; ++j) slot[inside ? 1 : 0][q][lane * V + j] = acc[j];
#pragma unroll
                    for (int j = 0; j < V; ++j) acc[j] = 0.0;
                }
            }
        }
    }
    if (lane == 0) {
        const uint64_t own = m_first & ((2ull << (count > 0 ? count - 1 : 0)) - 1ull);   // where rows begin
        kinds[q] = count == 0 ? 0u : ((own & 1ull) ? 0u : OPEN) | ((m_last >> (count - 1)) & 1ull ? 0u : GOES_ON) | ((own & ~1ull) ? 0u : ONE);
        first_row[q] = row;
    }
    __syncthreads();
    // a row that goes on is followed by the group in whose share it begins, one that began before the chunk by the first group
    const uint32_t kind = kinds[q];
    auto follow = [&](int k, bool ends) {   // from share k on; returns the share it ends in, GROUPS if it goes on
        while (!ends && ++k < GROUPS) {
#pragma unroll
            for (int j = 0; j < V; ++j) acc[j] += slot[0][k][lane * V + j];
            ends = (kinds[k] & (GOES_ON | ONE)) != (GOES_ON | ONE);
        }
        return k;
    };
    if (q == 0 && (kind & OPEN)) {
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] = slot[0][0][lane * V + j];
        (void)follow(0, (kind & (GOES_ON | ONE)) != (GOES_ON | ONE));
        write_part<V>(part + 2 * (int64_t)blockIdx.x * F, pc, acc);
    }
    if ((kind & GOES_ON) && (kind & (OPEN | ONE)) != (OPEN | ONE)) {
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] = slot[1][q][lane * V + j];
        const int k = follow(q, false);
        if (k < GROUPS) write_sum<TD, V>(o, first_row[k], pc, acc);
        else write_part<V>(part + (2 * (int64_t)blockIdx.x + 1) * F, pc, acc);
    }
}

// Table rows that go on across chunks: a wavefront per chunk looks whether one begins in it, and adds up its parts in order; one
// of more than JOIN_LONG chunks is left to the whole block, whose groups of G lanes take consecutive shares of the parts.  Bound by the latency of
// four dependent loads (4 to 8 us).
constexpr int JOIN_WAVES = 16, JOIN_LONG = 16;
template <typename TD, int V, int G>
__global__ __launch_bounds__(JOIN_WAVES * WAVE) void chunk_join_k(int32_t F, Keys key, int32_t n_cap, const int32_t *__restrict__ n_dev, uint32_t rows,
                                                                  int32_t chunk, const double *__restrict__ part, SumOut o)
{
    constexpr int GROUPS = JOIN_WAVES * WAVE / G;
    __shared__ int64_t long_parts[JOIN_WAVES];
    __shared__ double lds[GROUPS][G * V];
    __shared__ uint32_t base[RANGES], scan[17];
    const int32_t n = resolve_count(n_cap, n_dev);
    const int lane = lane_id(), wave = (int)threadIdx.x / WAVE, sub = lane % G, group = (int)threadIdx.x / G;
    const Piece1<V> pc((int32_t)(blockIdx.y * G + sub), F);
    const int64_t c0 = (int64_t)blockIdx.x * JOIN_WAVES, c = c0 + wave;
    if (c0 * chunk >= n) return;
    const int64_t beg = c * chunk, end = beg + chunk;
    int64_t parts = 0;     // chunks after c that the row is in
    uint32_t k = 0;
    if (end < n) {
        // (all asked for at once; lane t: the first position of chunk c + 1 + t)
        const int64_t mine = (c + 1 + lane) * chunk;
        const uint32_t first = key[beg], before = key[beg > 0 ? beg - 1 : 0], here = key[mine < n ? mine : n - 1];
        k = key[end - 1];
        const bool begins = first != k || beg == 0 || before != k;
        if (k < rows && begins) {
            const uint64_t m = __ballot(mine < n && here == k);
            parts = m == ~0ull ? WAVE : __ffsll((unsigned long long)~m) - 1;
            // a long one: its end by sixty-fourths of what is left
            int64_t lo = c + 1 + parts, hi = ((int64_t)n + chunk - 1) / chunk;   // it is in the chunks before lo, and not in hi
            while (parts >= WAVE && lo < hi) {
                const int64_t step = (hi - lo + WAVE - 1) / WAVE, at = lo + (lane + 1) * step - 1;
                const uint64_t in = __ballot(at < hi && key[at * chunk] == k);   // ascending: the lower lanes
                const int full = in == ~0ull ? WAVE : __ffsll((unsigned long long)~in) - 1;
                lo += full * step;
                hi = lo + step - 1 < hi ? lo + step - 1 : hi;
            }
            if (parts >= WAVE) parts = lo - (c + 1);
        }
    }
    if (o.distinct) {
        if (!__syncthreads_or(parts > 0 ? 1 : 0)) return;
        uint32_t total;
        range_bases(o, base, scan, &total);
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
#pragma unroll 8
        for (int64_t t = 1; t <= parts; ++t) add(acc, part + 2 * (c + t) * F);
        write_sum<TD, V>(o, o.rank ? row_of_rank(o, o.rank[end - 1], base) : k, pc, acc);
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
#pragma unroll 8
        for (int64_t t = t0; t < t1; ++t) add(acc, part + 2 * (cw + t) * F);
#pragma unroll
        for (int i = 0; i < V; ++i) lds[group][sub * V + i] = acc[i];
        __syncthreads();
        if (group == 0) {
#pragma unroll 1
            for (int q = 1; q < GROUPS; ++q)
#pragma unroll
                for (int i = 0; i < V; ++i) acc[i] += lds[q][sub * V + i];
            const int64_t at = (cw + 1) * chunk - 1;
            write_sum<TD, V>(o, o.rank ? row_of_rank(o, o.rank[at], base) : key[at], pc, acc);
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------- few positions: everything in one launch
// Ranges as above, but a block also adds up the rows of its range: all positions of an id are in one block.  The block that an often repeated id falls
// to reads its rows alone, at 25 GB/s or so, so that the rows must be few and not wide.  Groups of G lanes take consecutive shares of the sorted list; a row within a share
// is written at once, parts of one that goes on across shares are joined in LDS.  The rank of a range's first id is the number of different ids
// below it, which every block counts with a hash table.  Rows without positions are cleared in even shares of the table.
constexpr int FEW = 2 * WIDE;
constexpr int64_t FEW_VALUES = 1 << 18;   // most values of G: 1 MB of floats, 40 us for one compute unit if all of them belong to one id, half of that otherwise lost
constexpr int FEW_TABLE = 2 * FEW, FEW_ROWS = 1 << 15;   // hash table; rows whose being met a block notes at a time
template <typename TG, typename TD, int V, int G>
__global__ __launch_bounds__(WIDE) void few_sums_k(const TG *g, int64_t ldg, int32_t F, const int32_t *__restrict__ ids, int32_t n_cap,
                                                   const int32_t *__restrict__ n_dev, uint32_t rows, ZeroRows z, SumOut o)
{
    constexpr int PER = FEW / WIDE, GROUPS = WIDE / G;
    __shared__ uint64_t e[FEW];
    __shared__ SortLds l;
    __shared__ __attribute__((aligned(16))) SelectLds sel;
    __shared__ double slot[2][GROUPS][G * V];
    __shared__ uint16_t local_rank[FEW];
    __shared__ uint32_t w_own[WIDE_WAVES], n_met, kinds[GROUPS], first_row[GROUPS];
    static_assert(sizeof(slot) >= FEW_TABLE * 4 && sizeof(slot) >= FEW_ROWS / 8, "what else is kept in its place");
    const int tid = (int)threadIdx.x, lane = lane_id(), wave = tid / WAVE, b = (int)blockIdx.x;
    const int32_t n = resolve_count(n_cap, n_dev);
    const int32_t steps = (n + WIDE - 1) / WIDE;   // of 64 positions of a wavefront
    uint32_t id[PER], sample[PER];
    bool has[PER];
#pragma unroll
    for (int u = 0; u < PER; ++u) {
        const int32_t i = (wave * steps + u) * WAVE + lane;
        has[u] = u < steps && i < n;
        id[u] = has[u] ? (uint32_t)ids[i] : 0xFFFFFFFFu;
        sample[u] = id[u] < rows ? id[u] : rows;
    }
    if (z.rows) {
        uint32_t *met = (uint32_t *)&slot[0][0][0];
        const int64_t r_beg = z.rows * b / RANGES, r_end = z.rows * (b + 1) / RANGES;
        for (int64_t r0 = r_beg; r0 < r_end; r0 += FEW_ROWS) {
            const int32_t len = (int32_t)(r_end - r0 < FEW_ROWS ? r_end - r0 : FEW_ROWS);
            for (int x = tid; x < FEW_ROWS / 32; x += WIDE) met[x] = 0;
            __syncthreads();
#pragma unroll
            for (int u = 0; u < PER; ++u) {
                const int64_t r = (int64_t)id[u] - r0;
                if (id[u] < rows && r >= 0 && r < len) atomicOr(&met[r >> 5], 1u << (r & 31));
            }
            __syncthreads();
            if (z.row == z.ld && z.row < 1024) {
                // narrow rows side by side: 16 bytes a lane across rows, two bytes at a time where one of those rows was met
                const uint32_t row = (uint32_t)z.row, bytes = (uint32_t)len * row;
                char *p = (char *)z.d + r0 * z.ld;
                for (uint32_t at = (uint32_t)tid * 16; at < bytes; at += WIDE * 16) {
                    const uint32_t first = at / row, to = at + 16 <= bytes ? at + 16 : bytes, last = (to - 1) / row;
                    bool any = to != at + 16;
                    for (uint32_t r = first; r <= last; ++r) any |= (met[r >> 5] >> (r & 31)) & 1u;
                    if (!any) store_global<u32x4, 2>(p + at, u32x4{0, 0, 0, 0});
                    else
                        for (uint32_t x = at; x < to; x += 2) {
                            const uint32_t r = x / row;
                            if (!((met[r >> 5] >> (r & 31)) & 1u)) store_global<uint16_t>(p + x, (uint16_t)0);
                        }
                }
            } else
            for (int32_t r = wave; r < len; r += WIDE_WAVES)
                if (!((met[r >> 5] >> (r & 31)) & 1u)) zero_rows(ZeroRows{(char *)z.d + (r0 + r) * z.ld, 1, z.row, z.ld + 2}, 0, 1);
            __syncthreads();
        }
    }
    if (n == 0) {
        if (o.rank && b == 0 && tid == 0) *o.n_uniq = 0;
        return;
    }
    const Range range = range_of(b, sample, has, n, rows, sel);
    const uint32_t lo = range.lo, width = range.width;
    uint32_t n_own = 0;
#pragma unroll
    for (int u = 0; u < PER; ++u) n_own += (uint32_t)__popcll(__ballot(id[u] - lo < width));
    if (lane == 0) w_own[wave] = n_own;
    uint32_t base = 0;
    if (o.rank) {
        uint32_t *table = (uint32_t *)&slot[0][0][0];
        for (int x = tid; x < FEW_TABLE; x += WIDE) table[x] = 0xFFFFFFFFu;
        if (tid == 0) n_met = 0;
        __syncthreads();
        uint32_t added = 0;
#pragma unroll
        for (int u = 0; u < PER; ++u)
            if (id[u] < lo) {
                for (uint32_t h = id[u] * 0x9E3779B1u >> 20;; h = (h + 1) & (FEW_TABLE - 1)) {   // at least half of the table stays free
                    const uint32_t old = atomicCAS(&table[h & (FEW_TABLE - 1)], 0xFFFFFFFFu, id[u]);
                    if (old == id[u]) break;
                    if (old == 0xFFFFFFFFu) { ++added; break; }
                }
            }
        if (added) atomicAdd(&n_met, added);
    }
    __syncthreads();
    if (o.rank) base = n_met;
    uint32_t own = 0, at = 0;
    for (int w = 0; w < WIDE_WAVES; ++w) {
        if (w == wave) at = own;
        own += w_own[w];
    }
#pragma unroll
    for (int u = 0; u < PER; ++u) {
        const bool is = id[u] - lo < width;
        const uint64_t m = __ballot(is);
        if (is) e[at + (uint32_t)__popcll(m & ((1ull << lane) - 1ull))] = (uint64_t)id[u] << 32 | (uint32_t)((wave * steps + u) * WAVE + lane);
        at += (uint32_t)__popcll(m);
    }
    __syncthreads();
    if (width > 1 && own > 1) {
        if (own <= COUNTED && width <= COUNTED_SPAN) sort_by_counting(e, (int)own, lo, l);
        else sort_in_lds<PER>(e, (int)own, lo, width - 1, l);
    }
    if (o.rank) {
        uint32_t met = 0;
        for (uint32_t i0 = 0; i0 < own; i0 += WIDE) {
            const uint32_t i = i0 + (uint32_t)tid;
            const bool head = i < own && (i == 0 || key_of(e[i]) != key_of(e[i - 1]));
            uint32_t total;
            const uint32_t before = met + block_exclusive_scan<uint32_t>(head ? 1u : 0u, l.scan, &total);
            met += total;
            if (head) o.uniq[base + before] = (int32_t)key_of(e[i]);
            if (i < own) local_rank[i] = (uint16_t)(before + (head ? 1u : 0u) - 1u);
        }
        if (b == RANGES - 1 && tid == 0) *o.n_uniq = (int32_t)(base + met);
    }
    __syncthreads();
    if (own == 0) return;
    auto row_of = [&](int i) { return o.rank ? base + local_rank[i] : key_of(e[i]); };
    constexpr int U = 8, LEAST = 4;   // rows on their way; fewest of a share (they take no longer than one, and there are fewer shares to join)
    const int even = ((int)own + GROUPS - 1) / GROUPS, share = even < LEAST ? LEAST : even, groups = ((int)own + share - 1) / share, q = tid / G, sub = tid % G;
    struct Share {
        int beg, end;
        bool open, goes_on, one;   // its first row began before it; its last one goes on after it; it holds one row
    };
    auto share_of = [&](int k) {
        Share s;
        s.beg = k * share;
        s.end = s.beg + share < (int)own ? s.beg + share : (int)own;
        const uint32_t first = key_of(e[s.beg]), last = key_of(e[s.end - 1]);
        s.open = s.beg > 0 && key_of(e[s.beg > 0 ? s.beg - 1 : 0]) == first;
        s.goes_on = s.end < (int)own && key_of(e[s.end < (int)own ? s.end : s.end - 1]) == last;
        s.one = first == last;
        return s;
    };
    for (int32_t slice = 0; slice * (G * V) < F; ++slice) {
        const Piece1<V> pc(slice * G + sub, F);
        if (q < groups) {
            const Share s = share_of(q);
            if (slice == 0 && sub == 0) {
                kinds[q] = (s.open ? 1u : 0u) | (s.goes_on ? 2u : 0u) | (s.one ? 4u : 0u);
                first_row[q] = row_of(s.beg);
            }
            double acc[V];
#pragma unroll
            for (int i = 0; i < V; ++i) acc[i] = 0.0;
            bool open = s.open;
            for (int i0 = s.beg; i0 < s.end; i0 += U) {
                RawPiece<TG, V> r[U];
                uint64_t en[U + 1];
#pragma unroll
                for (int u = 0; u <= U; ++u) en[u] = e[i0 + u < s.end ? i0 + u : s.end - 1];
#pragma unroll
                for (int u = 0; u < U; ++u) r[u].load(g + (int64_t)(uint32_t)en[u] * ldg + pc.col);
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int i = i0 + u;
                    if (i < s.end) {
#pragma unroll
                        for (int j = 0; j < V; ++j) acc[j] += (double)r[u].value(j);
                        const bool last = i == s.end - 1;
                        if (last || key_of(en[u + 1]) != key_of(en[u])) {
                            if (open || (last && s.goes_on))
#pragma unroll
                                for (int j = 0; j < V; ++j) slot[open ? 0 : 1][q][sub * V + j] = acc[j];
                            else write_sum<TD, V>(o, row_of(i), pc, acc);
#pragma unroll
                            for (int j = 0; j < V; ++j) acc[j] = 0.0;
                            open = false;
                        }
                    }
                }
            }
        }
        __syncthreads();
        if (q == 0 && groups > 1) {
            double acc[V];
#pragma unroll
            for (int i = 0; i < V; ++i) acc[i] = 0.0;
#pragma unroll 1
            for (int k = 0; k < groups; ++k) {
                const uint32_t kind = kinds[k];
                const bool open = kind & 1u, goes_on = kind & 2u, one = kind & 4u;
                if (open) {
#pragma unroll
                    for (int j = 0; j < V; ++j) acc[j] += slot[0][k][sub * V + j];
                    if (!(one && goes_on)) write_sum<TD, V>(o, first_row[k], pc, acc);
                }
                if (goes_on && !(open && one))
#pragma unroll
                    for (int j = 0; j < V; ++j) acc[j] = slot[1][k][sub * V + j];
            }
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
    const uint64_t *entry;
    int32_t n;
    const int32_t *n_dev;
    uint32_t rows;
    double *part;
};
template <typename TG, typename TD, int V, int G>
static void launch_sums(const SumIn &in, const SumOut &o, hipStream_t st)
{
    const int32_t share = share_of(in.n, in.F), chunk = share * (SUM_BLOCK / G);
    const unsigned slices = (unsigned)((in.F + G * V - 1) / (G * V));
    CSGS_LAUNCH(K_EMBED_SUM, (chunk_sums_k<TG, TD, V, G>), dim3((unsigned)(((int64_t)in.n + chunk - 1) / chunk), slices), dim3(SUM_BLOCK), st, (const TG *)in.g, in.ldg,
                in.F, in.entry, in.n, in.n_dev, in.rows, share, in.part, o);
}
template <typename TD, int V, int G>
static void launch_join(const SumIn &in, const SumOut &o, int32_t chunk, hipStream_t st)
{
    const int64_t chunks = ((int64_t)in.n + chunk - 1) / chunk;
    const unsigned slices = (unsigned)((in.F + G * V - 1) / (G * V));
    CSGS_LAUNCH(K_EMBED_JOIN, (chunk_join_k<TD, V, G>), dim3((unsigned)((chunks + JOIN_WAVES - 1) / JOIN_WAVES), slices), dim3(JOIN_WAVES * WAVE), st, in.F, Keys{in.entry},
                in.n, in.n_dev, in.rows, chunk, in.part, o);
}
template <typename TG, typename TD>
static int embed_grad_few(const SumIn &in, const int32_t *ids, const ZeroRows &z, const SumOut &o, hipStream_t st)
{
    auto launch = [&](auto pieces, auto lanes) {
        constexpr int V = decltype(pieces)::value, G = decltype(lanes)::value;
        CSGS_LAUNCH(K_EMBED_FEW, (few_sums_k<TG, TD, V, G>), dim3(RANGES), dim3(WIDE), st, (const TG *)in.g, in.ldg, in.F, ids, in.n, in.n_dev, in.rows, z, o);
    };
    using std::integral_constant;
    if (in.F < 4) launch(integral_constant<int, 1>{}, integral_constant<int, 16>{});
    else if (in.F <= 64) launch(integral_constant<int, 4>{}, integral_constant<int, 16>{});
    else launch(integral_constant<int, 4>{}, integral_constant<int, 64>{});
    CSGS_LAUNCH_CHECK();
    return CSGS_OK;
}

template <typename TG, typename TD>
static int embed_grad_sums(const SumIn &in, const SumOut &o, hipStream_t st)
{
    constexpr int V = sizeof(TG) == 4 ? 4 : 8;
    const int lanes = in.F < V ? 16 : sum_lanes(in.F, V);
    if (in.F < V) launch_sums<TG, TD, 1, 16>(in, o, st);
    else if (lanes == 16) launch_sums<TG, TD, V, 16>(in, o, st);
    else if (lanes == 32) launch_sums<TG, TD, V, 32>(in, o, st);
    else launch_sums<TG, TD, V, 64>(in, o, st);
    // (parts are doubles: pieces of two are 16 bytes)
    const int32_t chunk = share_of(in.n, in.F) * (SUM_BLOCK / lanes);
    if (in.n <= chunk) {   // nothing goes on
    } else if (in.F < 2) launch_join<TD, 1, 16>(in, o, chunk, st);
    else if (in.F <= 32) launch_join<TD, 2, 16>(in, o, chunk, st);
    else if (in.F <= 64) launch_join<TD, 2, 32>(in, o, chunk, st);
    else launch_join<TD, 2, 64>(in, o, chunk, st);
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
    const int64_t elt = d_dtype == CSGS_F32 ? 4 : 2;
    const ZeroRows z{d, uniq || accumulate ? 0 : rows, F * elt, ldd * elt};
    SumIn in{G, ldg, F, nullptr, (int32_t)n, n_dev, (uint32_t)rows, s.part};
    SumOut o{uniq ? s.rank : nullptr, nullptr, uniq, n_uniq, d, ldd, scale, accumulate};
    if (n <= FEW && n * F <= FEW_VALUES) {
        if (g_dtype == CSGS_F32) return d_dtype == CSGS_F32 ? embed_grad_few<float, float>(in, ids, z, o, st) : embed_grad_few<float, uint16_t>(in, ids, z, o, st);
        return d_dtype == CSGS_F32 ? embed_grad_few<uint16_t, float>(in, ids, z, o, st) : embed_grad_few<uint16_t, uint16_t>(in, ids, z, o, st);
    }
    if (n <= RANGES_MAX) {
        const dim3 grid(RANGES + (z.rows ? RANGES : 0)), block(WIDE);
        CSGS_LAUNCH(K_EMBED_RANGES, sort_ranges_k, grid, block, st, ids, (int32_t)n, n_dev, (uint32_t)rows, s.entry[0], s.entry[1], uniq ? s.rank : nullptr, s.heads,
                    s.n_valid, z);
        CSGS_LAUNCH_CHECK();
        in.entry = s.entry[0];
        in.n_dev = s.n_valid;
        if (uniq) o.distinct = s.heads;
    } else {
        const int32_t tile = (int32_t)(((n + SORT_TILES - 1) / SORT_TILES + SORT_STEP - 1) / SORT_STEP * SORT_STEP);
        const int tiles = (int)((n + tile - 1) / tile);
        int key_bits = 0;
        while ((rows >> key_bits) != 0) ++key_bits;   // the key `rows` too
        const int passes = (key_bits + 7) / 8, bits = (key_bits + passes - 1) / passes;
        if (z.rows) CSGS_LAUNCH(K_EMBED_ZERO, rows_zero_k, dim3(wave_blocks(z.rows)), dim3(256), st, z);
        for (int p = 0; p < passes; ++p) {
            const SortIn si{p == 0 ? ids : nullptr, p == 0 ? nullptr : s.entry[(p + 1) & 1], (uint32_t)rows};
            CSGS_LAUNCH(K_EMBED_COUNT, sort_count_k, dim3((unsigned)tiles), dim3(SORT_BLOCK), st, si, (int32_t)n, n_dev, tile, p * bits, (1u << bits) - 1, s.hist);
            CSGS_LAUNCH(K_EMBED_PLACE, sort_place_k, dim3((unsigned)tiles), dim3(SORT_BLOCK), st, si, (int32_t)n, n_dev, tile, tiles, p * bits, bits, s.hist, s.entry[p & 1]);
            CSGS_LAUNCH_CHECK();
        }
        in.entry = s.entry[(passes - 1) & 1];
        if (uniq) {
            CSGS_LAUNCH(K_EMBED_HEADS, heads_count_k, dim3((unsigned)tiles), dim3(SORT_BLOCK), st, Keys{in.entry}, (int32_t)n, n_dev, tile, (uint32_t)rows, s.heads);
            CSGS_LAUNCH(K_EMBED_HEADS, heads_place_k, dim3((unsigned)tiles), dim3(SORT_BLOCK), st, Keys{in.entry}, (int32_t)n, n_dev, tile, tiles, (uint32_t)rows, s.heads,
                        s.rank, n_uniq);
            CSGS_LAUNCH_CHECK();
        }
    }
    if (g_dtype == CSGS_F32) return d_dtype == CSGS_F32 ? embed_grad_sums<float, float>(in, o, st) : embed_grad_sums<float, uint16_t>(in, o, st);
    return d_dtype == CSGS_F32 ? embed_grad_sums<uint16_t, float>(in, o, st) : embed_grad_sums<uint16_t, uint16_t>(in, o, st);
}

template <typename TI, typename TO>
static void launch_embed(const void *T, int64_t ld, int64_t rows, int32_t F, const int32_t *ids, int32_t n, const int32_t *n_dev, float scale, void *out,
                         int64_t ldo, hipStream_t st)
{
    auto launch = [&](auto pieces, auto lanes) {
        constexpr int V = decltype(pieces)::value, G = decltype(lanes)::value;
        const int64_t blocks = ((int64_t)n + 256 / G - 1) / (256 / G);
        const dim3 grid((unsigned)(blocks < 2048 ? blocks : 2048), (unsigned)(((int64_t)F + G * V - 1) / (G * V)));
        CSGS_LAUNCH(K_EMBED, (embed_k<TI, TO, V, G>), grid, dim3(256), st, (const TI *)T, ld, rows, F, ids, n, n_dev, scale, (TO *)out, ldo);
    };
    using std::integral_constant;
    constexpr int V = sizeof(TI) == 2 && sizeof(TO) == 2 ? 8 : 4;
    if (F < V) launch(integral_constant<int, 1>{}, integral_constant<int, 8>{});
    else if (F <= 8 * V) launch(integral_constant<int, V>{}, integral_constant<int, 8>{});
    else if (F <= 16 * V) launch(integral_constant<int, V>{}, integral_constant<int, 16>{});
    else if (F <= 32 * V) launch(integral_constant<int, V>{}, integral_constant<int, 32>{});
    else launch(integral_constant<int, V>{}, integral_constant<int, 64>{});
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
