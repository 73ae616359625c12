// Checks of the arguments that operators on their own share.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include "common.h"

namespace tmps {

inline bool known(int dtype) { return dtype == TMPS_F32 || dtype == TMPS_BF16_F32MASTER; }

inline bool aligned(const void* p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

// Memory of `bytes` bytes at p (null: none); with a pitch rows of `width` bytes, `pitch` bytes apart.
struct Range {
    const void* p;
    size_t bytes;
    size_t pitch = 0, width = 0;
    bool meets(const Range& o) const {
        const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(o.p);
        if (!(p && o.p && bytes && o.bytes && a < b + o.bytes && b < a + bytes)) return false;
        if (!pitch || pitch != o.pitch) return true;
        // (other columns of the same rows)
        const size_t d = b >= a ? (b - a) % pitch : (pitch - (a - b) % pitch) % pitch;
        return d < width || d + o.width > pitch;
    }
};

// Whether a result overlaps an operand or another result; `same`: operand that results[0] may be, whole.
template <int NO, int NR> bool overlaps(const Range (&operands)[NO], const Range (&results)[NR], const void* same = nullptr) {
    for (int i = 0; i < NR; ++i) {
        for (const Range& o : operands)
            if (results[i].meets(o) && !(i == 0 && same && o.p == same && results[i].p == same)) return true;
        for (int k = 0; k < i; ++k)
            if (results[i].meets(results[k])) return true;
    }
    return false;
}

// Elements that 63 bits of bytes count.
constexpr int64_t kMaxElems = int64_t(1) << 59;

}  // namespace tmps
