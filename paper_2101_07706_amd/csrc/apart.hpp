// Whether the memory of two matrices meets: host code, for calls that refuse outputs which lie on something else.
#pragma once
#include <stdint.h>
#include <algorithm>
#include <initializer_list>
#include <tuple>
#include <vector>

namespace csgs {

// `rows` pieces of `width` bytes, `step` bytes apart.  p null: none.
struct Memory {
    const void *p;
    int64_t rows, width, step;
};
// Bytes from the first to behind the last: nothing on a device spans MOST_MEMORY, and a call that says so is refused before the sums below could overflow.
constexpr int64_t MOST_MEMORY = 1ll << 40;
// A matrix of entries of `size` bytes.
inline Memory matrix_memory(const void *p, int64_t rows, int64_t cols, int64_t ld, int64_t size)
{
    const auto bytes = [&](int64_t n) { return n > MOST_MEMORY ? 2 * MOST_MEMORY : n * size; };
    return Memory{p, rows, bytes(cols), bytes(ld)};
}
inline bool spans_too_much(const Memory &m)
{
    return m.p && ((__int128)(m.rows - 1) * m.step + m.width > MOST_MEMORY || (uintptr_t)m.p > ~(uintptr_t)0 - (uintptr_t)MOST_MEMORY);
}
inline uintptr_t memory_end(const Memory &m) { return (uintptr_t)m.p + (uintptr_t)((m.rows - 1) * m.step + m.width); }

// Row i of a and row j of b meet where -b.width < d + n step < a.width, with d between the first rows and n = j - i.
inline bool rows_meet(const Memory &a, const Memory &b, int64_t step)
{
    const int64_t d = (int64_t)((uintptr_t)b.p - (uintptr_t)a.p), above = -b.width - d;       // n step > above
    int64_t n = above / step + (above % step < 0 ? 0 : 1);
    if (n < 1 - a.rows) n = 1 - a.rows;
    return n <= b.rows - 1 && d + n * step < a.width;
}
inline bool memory_meets(Memory a, Memory b)
{
    if (!a.p || !b.p || (uintptr_t)a.p >= memory_end(b) || (uintptr_t)b.p >= memory_end(a)) return false;
    if (a.rows == 1 && b.rows == 1) return true;
    if (a.rows == 1 || b.rows == 1 || a.step == b.step) return rows_meet(a, b, a.rows == 1 ? b.step : a.step);
    // rows of different steps: one after the other, of those that lie within the other matrix
    if (a.rows > b.rows) std::swap(a, b);
    const uintptr_t first = (uintptr_t)a.p, from = (uintptr_t)b.p;
    for (int64_t i = from < first + (uintptr_t)a.width ? 0 : (int64_t)((from - first - (uintptr_t)a.width) / (uintptr_t)a.step); i < a.rows; ++i) {
        const Memory row{(const char *)a.p + i * a.step, 1, a.width, a.step};
        if ((uintptr_t)row.p >= memory_end(b)) return false;
        if (rows_meet(row, b, b.step)) return true;
    }
    return false;
}

// Whether each output lies apart from the inputs and from the other outputs.
inline bool outputs_apart(const std::initializer_list<Memory> &in, const std::initializer_list<Memory> &out)
{
    for (const Memory *o = out.begin(); o != out.end(); ++o) {
        for (const Memory &i : in)
            if (memory_meets(*o, i)) return false;
        for (const Memory *other = out.begin(); other != o; ++other)
            if (memory_meets(*o, *other)) return false;
    }
    return true;
}
inline bool spans_too_much(const std::initializer_list<Memory> &all)
{
    for (const Memory &m : all)
        if (spans_too_much(m)) return true;
    return false;
}

// Memory of one of many tensors.
struct Held {
    Memory at;
    int32_t owner;
    bool written, beside;      // beside: not compared with its owner's other memory
};
enum class Lie { APART, MEET, TOO_MANY };
// Whether what is written lies apart from everything else; what is only read may be shared.  In the order of the first bytes, each is compared with those before it that have not ended: columns
// of one buffer are compared in pairs, MOST_PAIRS of them at most.
constexpr int64_t MOST_PAIRS = 1ll << 26;
inline Lie all_apart(std::vector<Held> &all)
{
    const auto key = [](const Held &h) { return std::make_tuple((uintptr_t)h.at.p, h.written, h.at.rows, h.at.width, h.at.step); };
    std::sort(all.begin(), all.end(), [&](const Held &a, const Held &b) { return key(a) < key(b); });
    std::vector<const Held *> open[2];       // read, written
    int64_t pairs = 0;
    for (size_t i = 0; i < all.size(); ++i) {
        const Held &h = all[i];
        if (!h.written && i > 0 && key(h) == key(all[i - 1])) continue;
        for (int w = h.written ? 0 : 1; w < 2; ++w) {
            size_t kept = 0;
            for (const Held *o : open[w]) {
                if (memory_end(o->at) <= (uintptr_t)h.at.p) continue;
                open[w][kept++] = o;
                if (o->owner == h.owner && (o->beside || h.beside)) continue;
                if (++pairs > MOST_PAIRS) return Lie::TOO_MANY;
                if (memory_meets(o->at, h.at)) return Lie::MEET;
            }
            open[w].resize(kept);
        }
        open[h.written].push_back(&h);
    }
    return Lie::APART;
}

}  // namespace csgs
