// Where a token of a paged cache lives.  Plain C++: the same functions run in the kernels and in the host tests.
#pragma once

#include <stdint.h>

#if defined(__HIPCC__)
#define SPECGBV_HD __host__ __device__ __forceinline__
#else
#define SPECGBV_HD inline
#endif

namespace specgbv {

// n / d for 0 <= n < 2^31, 1 <= d < 2^31 by a multiplication: with s = ceil(log2 d) and m = ceil(2^(31+s) / d) the quotient is
// floor(n m / 2^(31+s)), since m d exceeds 2^(31+s) by less than 2^s and n times that stays below 2^(31+s).
struct Divider {
    uint32_t d, m;
    int32_t s;

    static Divider of(int32_t d)
    {
        int s = 0;
        while ((static_cast<int64_t>(1) << s) < d) ++s;
        const uint64_t top = static_cast<uint64_t>(1) << (31 + s);
        return {static_cast<uint32_t>(d), static_cast<uint32_t>((top + d - 1) / d), s};
    }
    SPECGBV_HD int32_t div(int32_t n) const
    {
        return static_cast<int32_t>((static_cast<uint64_t>(static_cast<uint32_t>(n)) * m) >> (31 + s));
    }
    SPECGBV_HD int32_t mod(int32_t n, int32_t q) const { return n - q * static_cast<int32_t>(d); }
};

struct PageMap {
    const int32_t *table;
    int64_t table_stride;
    Divider page;              // by the page's size
    int32_t pages, width;
};

struct Place {
    int32_t page, slot;        // page < 0: there is none
};

// First position that the table of a sequence cannot hold.
SPECGBV_HD int64_t capacity_of(const PageMap &m) { return static_cast<int64_t>(m.width) * m.page.d; }

// The place of position pos >= 0 of a sequence.  Nothing is read where the position lies behind the table's width.
SPECGBV_HD Place place_of(const PageMap &m, int32_t sequence, int32_t pos)
{
    const int32_t n = m.page.div(pos);
    if (pos < 0 || n >= m.width) return {-1, 0};
    const int32_t page = m.table[sequence * m.table_stride + n];
    return {static_cast<uint32_t>(page) < static_cast<uint32_t>(m.pages) ? page : -1, m.page.mod(pos, n)};
}

}  // namespace specgbv
