// Rows of `width` neighbouring elements within a tensor: its last dimensions make up a row, the others count rows that lie evenly and apart.
#ifndef VECTOR_ROWS_H_
#define VECTOR_ROWS_H_

#include <cstdint>

namespace vec {

// The distance between neighbouring rows, in elements; false: the tensor is no such rows.  It holds a whole number of rows, one at the least.
inline bool row_distance(const int64_t* sizes, const int64_t* strides, int dims, int64_t width, int64_t* distance) {
    int64_t run = 1;
    int at = dims;
    while (run < width) {
        --at;
        if (sizes[at] == 1) continue;
        if (strides[at] != run || width % (run * sizes[at])) return false;
        run *= sizes[at];
    }
    *distance = width;                                  // one row
    bool known = false;                                 // whether a dimension of rows has been met: a distance of its own may be zero, as broadcast rows' is
    int64_t next = 0;                                   // the distance of the next dimension's steps
    while (--at >= 0) {
        if (sizes[at] == 1) continue;
        if (!known) *distance = strides[at];
        else if (strides[at] != next) return false;
        known = true;
        next = strides[at] * sizes[at];
    }
    return *distance >= width;
}

}  // namespace vec
#endif
