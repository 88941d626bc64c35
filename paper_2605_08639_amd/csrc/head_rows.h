// Tensors [T, H, d] of 16-bit values whose heads lie side by side and whose tokens lie `stride` values apart, so that the parts of a fused
// projection's output need no copy; what the entry points check of them.
#pragma once
#include "common.h"

#include <initializer_list>

namespace relibra {

constexpr int64_t kMaxHeadStride = 1 << 27;                   // eight rows' distance stays within 31 bits of bytes, a lane's offset

struct HeadRows {
    const void *p;
    int64_t stride;
    int width;                                                // H * d; 0: no such tensor
    bool usable() const { return width == 0 || (p && aligned16(p) && stride >= width && stride % 8 == 0 && stride <= kMaxHeadStride); }
    bool same(const HeadRows &o) const { return p == o.p && stride == o.stride && width == o.width; }
    // Whether one of T rows shares a byte with a piece of memory; what lies between the rows is not theirs.
    bool overlaps(const Piece &x, int64_t T) const
    {
        if (width == 0 || T < 1 || !x.p || !x.bytes) return false;
        const int64_t row = stride * 2, mine = (int64_t)width * 2, from = (int64_t)((intptr_t)x.p - (intptr_t)p);
        const int64_t n = from < mine ? 0 : (from - mine) / row + 1;      // the first row that ends behind the piece's first byte
        return n < T && n * row < from + (int64_t)x.bytes;
    }
    // Whether the two share a byte over T tokens.  Rows of one stride may interleave; of unlike strides only whole ranges are compared.
    bool overlaps(const HeadRows &o, int64_t T) const
    {
        if (width == 0 || o.width == 0 || T < 1) return false;
        const size_t mine = (size_t)((T - 1) * stride + width) * 2, theirs = (size_t)((T - 1) * o.stride + o.width) * 2;
        if (!overlap(p, mine, o.p, theirs)) return false;
        if (stride != o.stride || T == 1) return true;
        const int64_t row = stride * 2, diff = (int64_t)((intptr_t)p - (intptr_t)o.p), off = ((diff % row) + row) % row;     // where a row of mine starts in a row of theirs
        return off < o.width * 2 || off + width * 2 > row;
    }
};

// Whether what a call writes beside its rows (`written`: sums, tables, the workspace) shares no byte with anything else of the call, and its output
// rows none with what it reads beside rows.  Rows among themselves are the entry points' own checks: some may be in place.
inline bool pieces_apart(int64_t T, std::initializer_list<HeadRows> in, std::initializer_list<HeadRows> out, std::initializer_list<Piece> read, std::initializer_list<Piece> written)
{
    for (auto w = written.begin(); w != written.end(); ++w) {
        for (const HeadRows &x : in)
            if (x.overlaps(*w, T)) return false;
        for (const HeadRows &x : out)
            if (x.overlaps(*w, T)) return false;
        for (const Piece &x : read)
            if (overlap(*w, x)) return false;
        for (auto v = written.begin(); v != w; ++v)
            if (overlap(*w, *v)) return false;
    }
    for (const HeadRows &x : out)
        for (const Piece &r : read)
            if (x.overlaps(r, T)) return false;
    return true;
}

}  // namespace relibra
