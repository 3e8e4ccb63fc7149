// csrc/overlap.h on the host.
#include "overlap.h"

extern "C" int rows_overlap(uint64_t a, int64_t a_bytes, int64_t a_stride, int64_t a_rows, uint64_t b, int64_t b_bytes, int64_t b_stride,
                            int64_t b_rows) {
    using packkv::Rows;
    return packkv::overlap(Rows(reinterpret_cast<void *>(a), a_bytes, a_stride, a_rows), Rows(reinterpret_cast<void *>(b), b_bytes, b_stride, b_rows));
}
