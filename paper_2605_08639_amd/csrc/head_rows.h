// Tensors [T, H, d] of 16-bit values whose heads lie side by side and whose tokens lie `stride` values apart, so that the parts of a fused
// projection's output need no copy; what the entry points check of them.
#pragma once
#include "common.h"

namespace relibra {

constexpr int64_t kMaxHeadStride = 1 << 27;                   // eight rows' distance stays within 31 bits of bytes, a lane's offset

struct HeadRows {
    const void *p;
    int64_t stride;
    int width;                                                // H * d; 0: no such tensor
    bool usable() const { return width == 0 || (p && aligned16(p) && stride >= width && stride % 8 == 0 && stride <= kMaxHeadStride); }
    bool same(const HeadRows &o) const { return p == o.p && stride == o.stride && width == o.width; }
    bool overlaps(const void *other, size_t bytes, int64_t T) const { return width > 0 && T > 0 && overlap(p, (size_t)((T - 1) * stride + width) * 2, other, bytes); }
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

}  // namespace relibra
