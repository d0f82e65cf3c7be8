// Whether what a call writes shares memory with what it reads.
#pragma once

#include <algorithm>
#include <cstdint>

namespace pictura {

// `rows` rows of `bytes` bytes, `apart` bytes from one to the next (0 or more).
struct Region {
    uintptr_t at;
    int64_t rows, bytes, apart;
};

inline Region region(const void* at, int64_t rows, int64_t bytes, int64_t apart)
{
    return Region{reinterpret_cast<uintptr_t>(at), rows, bytes, apart};
}

// The same rows at the same places.
inline bool same(const Region& a, const Region& b)
{
    return a.at == b.at && a.rows == b.rows && a.bytes == b.bytes && (a.rows < 2 || a.apart == b.apart);
}

inline int64_t floor_div(int64_t a, int64_t b) { return a / b - (a % b < 0); }   // (b above 0)

// Whether any byte is in both, exactly: rows that stand between one another's share none.  Rows at
// one distance are compared at once, others row by row.
inline bool overlap(const Region& a, const Region& b)
{
    if (!a.at || !b.at || a.rows < 1 || b.rows < 1 || a.bytes < 1 || b.bytes < 1) return false;
    const int64_t from = (int64_t)(b.at - a.at);   // b's first byte, a's being 0
    const int64_t a_end = (a.rows - 1) * a.apart + a.bytes, b_end = from + (b.rows - 1) * b.apart + b.bytes;
    if (from >= a_end || b_end <= 0) return false;
    // whether any of the rows [at + k s, at + k s + bytes), k = low..high, meets [0, length)
    auto meets = [](int64_t at, int64_t s, int64_t bytes, int64_t low, int64_t high, int64_t length) {
        if (s == 0) return low <= high && at < length && at + bytes > 0;
        return std::max(low, floor_div(-at - bytes, s) + 1) <= std::min(high, floor_div(length - at - 1, s));
    };
    if (a.apart == b.apart) return meets(from, a.apart, b.bytes, -(a.rows - 1), b.rows - 1, a.bytes);
    const int64_t first = a.apart == 0 ? 0 : std::max<int64_t>(0, floor_div(from - a.bytes, a.apart) + 1),
                  last = a.apart == 0 ? 0 : std::min(a.rows - 1, floor_div(b_end - 1, a.apart));
    for (int64_t i = first; i <= last; ++i)
        if (meets(from - i * a.apart, b.apart, b.bytes, 0, b.rows - 1, a.bytes)) return true;
    return false;
}

}  // namespace pictura
