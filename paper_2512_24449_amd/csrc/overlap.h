// Whether memory that a call writes is also memory that it reads: entry points refuse such calls, as which of the two
// comes first would be left to the workgroups.  Host only.
#pragma once
#include <algorithm>
#include <cstdint>
#include <initializer_list>

namespace packkv {

// `rows` runs of `bytes` bytes, the beginnings `stride` (at least bytes) apart; of a null pointer nothing.  128 bits: the sizes are the caller's.
struct Rows {
    using Wide = __int128;
    Wide at, bytes, stride, rows;
    Rows(const void *p, Wide bytes_, Wide stride_, Wide rows_)
        : at(Wide(reinterpret_cast<uintptr_t>(p))), bytes(bytes_), stride(stride_), rows(p && bytes_ > 0 ? std::max(rows_, Wide(0)) : 0) {
        if (rows > 1 && stride > bytes) return;
        bytes = std::max(rows - 1, Wide(0)) * stride + bytes, rows = std::min(rows, Wide(1));
    }
    // All of it without gaps: so many values of `size` bytes.
    Rows(const void *p, Wide values, int size) : Rows(p, values * size, 0, 1) {}
    Wide end() const { return at + (rows - 1) * stride + bytes; }
};

inline bool overlap(const Rows &a, const Rows &b) {
    using Wide = Rows::Wide;
    if (a.rows == 0 || b.rows == 0 || a.end() <= b.at || b.end() <= a.at) return false;
    // Whether the run [at, at + bytes) reaches one of `rows` runs of a's from `first` on: the first that does not end before it.
    const auto reached = [&a](Wide first, Wide rows, Wide at, Wide bytes) {
        const Wide i = at < first + a.bytes ? 0 : (at - first - a.bytes) / a.stride + 1;
        return i < rows && first + i * a.stride < at + bytes;
    };
    if (a.rows == 1 && b.rows == 1) return true;
    if (a.rows == 1) return overlap(b, a);
    if (b.rows == 1) return reached(a.at, a.rows, b.at, b.bytes);
    // Runs at the same distance: run j of b is to run i of a as run 0 is to run i - j, which may be one before the first.
    if (a.stride == b.stride) return reached(a.at - (b.rows - 1) * a.stride, a.rows + b.rows - 1, b.at, b.bytes);
    // Interleaved at two distances, with gaps in both: one by one, of the tensor with fewer.
    if (a.rows < b.rows) return overlap(b, a);
    for (Wide j = 0; j < b.rows; ++j)
        if (reached(a.at, a.rows, b.at + j * b.stride, b.bytes)) return true;
    return false;
}

inline bool overlap(const Rows &written, std::initializer_list<Rows> read) {
    for (const Rows &r : read)
        if (overlap(written, r)) return true;
    return false;
}

}  // namespace packkv
