// Rows of layer values in 8-bit integers, as the int8 products read them.
#pragma once

#include "common.hpp"
#include "validate.hpp"

namespace moe {

// Bytes between quantised rows of n values: whole 16-byte vectors, the bytes
// behind the values zero, so that products may contract over the whole width.
inline int quantized_width(int n) { return (n + 15) / 16 * 16; }

// Quantises rows of n values (x, ldx elements apart) to q (quantized_width(n)
// apart) and scale.  offsets, region_rows (with E regions): only the rows
// [offsets[e], offsets[e] + region_rows[e]) below rows; the others keep what
// they held.
moe_status quantize_launch(hipStream_t s, moe_dtype dt, int64_t rows, int n, const void* x,
                           int64_t ldx, int8_t* q, float* scale, int E, const int32_t* offsets,
                           const int32_t* region_rows);

}  // namespace moe
