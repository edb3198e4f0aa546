// Checks of arguments that the training operators' entry points share (not installed): spans of arrays and whether they meet,
// element types, alignment, sizes.
#pragma once
#include <cstdint>

#include "decentlam.h"

namespace dlm {

// The bytes of a row-major array: rows of `width` bytes, `pitch` bytes apart.
struct Rows {
    uintptr_t lo;
    int64_t rows, width, pitch;
    uintptr_t hi() const { return lo + (uintptr_t)((rows - 1) * pitch + width); }
    bool same(const Rows& o) const { return lo == o.lo && pitch == o.pitch && width == o.width && rows == o.rows; }
};

inline Rows span(const void* p, int64_t rows, int64_t cols, int64_t ld, int64_t esz) {
    return {(uintptr_t)p, rows, cols * esz, rows > 1 ? ld * esz : cols * esz};
}

// Whether two arrays share a byte.  Column ranges of one array (equal pitch) may interleave without doing so.
inline bool meet(const Rows& a, const Rows& b) {
    if (a.lo == 0 || b.lo == 0 || a.rows <= 0 || b.rows <= 0) return false;
    if (a.hi() <= b.lo || b.hi() <= a.lo) return false;
    if (a.pitch == b.pitch && a.rows > 1 && b.rows > 1) {
        const int64_t off = (int64_t)((b.lo >= a.lo ? b.lo - a.lo : (uintptr_t)a.pitch - (a.lo - b.lo) % (uintptr_t)a.pitch) %
                                      (uintptr_t)a.pitch);  // b's place within a's rows
        if (off >= a.width && off + b.width <= a.pitch) return false;
    }
    return true;
}

inline int64_t element_bytes(int dtype) { return dtype == DLM_G_BF16 ? 2 : 4; }
inline bool known(int dtype) { return dtype == DLM_G_F32 || dtype == DLM_G_BF16; }
inline bool aligned(const void* p, int64_t esz) { return (uintptr_t)p % (uintptr_t)esz == 0; }

// Any array longer than this could not exist on the device; keeps the arithmetic of the checks in range.
constexpr int64_t kMaxElements = (int64_t)1 << 42;
inline bool fits(int64_t rows, int64_t ld) { return ld <= kMaxElements && rows <= kMaxElements && (rows == 0 || ld <= kMaxElements / rows); }

}  // namespace dlm
