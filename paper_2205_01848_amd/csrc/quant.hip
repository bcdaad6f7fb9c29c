// Rows of layer values in 8-bit integers with one scale each:
//     scale = max_j |x_j| (1/127),   q_j = rint(x_j / scale)   (ties to even).
// The scale is the fp32 product with the fp32 nearest to 1/127, not the rounded
// quotient max |x| / 127, from which it is one unit in the last place away for 6
// of the 128 bf16 maxima and 4.7 % of the fp32 ones: a tensor's division by a
// constant is computed as that product on the device, so rows quantised here
// equal those of a program of tensor operations, integer for integer.  (By the
// quotient 36 of the 33.6 million integers of 8192 x 4096 bf16 values would
// be others.)  q is the integer nearest to the exact
// quotient of x_j and that scale, clamped to +-127.  A row of zeros (or of
// values so small that the scale rounds to zero) has scale 0 and q 0; a row
// that holds a NaN or an infinity has scale NaN and q 0, so every product
// with it is NaN.
//
// Bound by memory: n (es + 1) bytes a row, each value read once into registers,
// where the row's maximum is found before anything is written.

#include <algorithm>

#include "quant.hpp"

namespace moe {
namespace {

constexpr int kQuantThreads = 256;

// G threads take a row, in units of 8 values; the first kHeld G units stay in
// registers between the two passes, a longer row's others are read again (from
// the caches).  Rows are dealt round-robin.
template <typename T, int G, int kHeld>
__global__ __launch_bounds__(kQuantThreads) void quantize_kernel(
    const T* __restrict__ x, int64_t ldx, int64_t rows, int n, int8_t* __restrict__ q,
    float* __restrict__ scale, int E, const int32_t* __restrict__ offsets,
    const int32_t* __restrict__ region_rows) {
  constexpr int kPer = kQuantThreads / G;   // rows of a workgroup at a time
  const int t = threadIdx.x % G, lane = threadIdx.x & 63;
  const int units = n / 8, qunits = (n + 15) / 16 * 2;   // of values, of bytes written
  const int64_t ldq = qunits * 8;
  int64_t r0 = 0, r1 = 0;   // the lane's region of valid rows
  if (offsets && lane < E) {
    r0 = offsets[lane];
    r1 = min(static_cast<int64_t>(offsets[lane + 1]), r0 + region_rows[lane]);
  }
  __shared__ uint32_t part[2][kQuantThreads / kWave];
  int turn = 0;
  for (int64_t base = static_cast<int64_t>(blockIdx.x) * kPer; base < rows;
       base += static_cast<int64_t>(gridDim.x) * kPer) {
    const int64_t row = base + threadIdx.x / G;   // the same for a whole wavefront
    bool live = row < rows;
    if (offsets) live = live && __any(row >= r0 && row < r1);
    Unit<T> held[kHeld];
    uint32_t m = 0;
    const T* xr = x + row * ldx;
    if (live) {
#pragma unroll
      for (int i = 0; i < kHeld; ++i)
        if (t + i * G < units) held[i].load(xr + (t + i * G) * 8);
#pragma unroll
      for (int i = 0; i < kHeld; ++i)
        if (t + i * G < units) m = abs_bits_max<T>(held[i], m);
      for (int u = t + kHeld * G; u < units; u += G) {
        Unit<T> v;
        v.load(xr + u * 8);
        m = abs_bits_max<T>(v, m);
      }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), o, 64)));
    if constexpr (G > kWave) {
      // one row per workgroup: two sets of partial maxima in turn, so one
      // barrier a row suffices
      part[turn][threadIdx.x / kWave] = m;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < kQuantThreads / kWave; ++w) m = max(m, part[turn][w]);
      turn ^= 1;
    }
    if (!live) continue;
    float sc;
    const RowScale rs = row_scale(m, sc);
    if (t == 0) scale[row] = sc;
    int8_t* qr = q + row * ldq;
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      const int u = t + i * G;
      if (u < units) *reinterpret_cast<uint2*>(qr + u * 8) = quantize8<T>(held[i], rs);
      else if (u < qunits) *reinterpret_cast<uint2*>(qr + u * 8) = make_uint2(0, 0);
    }
    for (int u = t + kHeld * G; u < qunits; u += G) {
      uint2 b = make_uint2(0, 0);
      if (u < units) {
        Unit<T> v;
        v.load(xr + u * 8);
        b = quantize8<T>(v, rs);
      }
      *reinterpret_cast<uint2*>(qr + u * 8) = b;
    }
  }
}

struct QuantArgs {
  int64_t rows;
  int n;
  const void* x;
  int64_t ldx;
  int8_t* q;
  float* scale;
  int E;
  const int32_t *offsets, *region_rows;
};

template <typename T, int G, int kHeld>
moe_status launch(hipStream_t s, const QuantArgs& a) {
  constexpr int kPer = kQuantThreads / G;
  const int grid = static_cast<int>(std::min<int64_t>((a.rows + kPer - 1) / kPer, 16 * num_cus()));
  MOE_TIMED("quantize_rows", s);
  quantize_kernel<T, G, kHeld><<<grid, kQuantThreads, 0, s>>>(static_cast<const T*>(a.x), a.ldx, a.rows,
                                                               a.n, a.q, a.scale, a.E, a.offsets,
                                                               a.region_rows);
  MOE_LAUNCH_CHECK();
  return MOE_OK;
}

// A wavefront a row up to 2048 values, else a workgroup, and just the
// registers that hold the row (up to 16384 values), as fewer of them leave room for
// more rows in flight.
template <typename T>
moe_status launch_width(hipStream_t s, const QuantArgs& a) {
  const int units = a.n / 8;
  if (units <= kWave) return launch<T, kWave, 1>(s, a);
  if (units <= 2 * kWave) return launch<T, kWave, 2>(s, a);
  if (units <= 4 * kWave) return launch<T, kWave, 4>(s, a);
  if (units <= 2 * kQuantThreads) return launch<T, kQuantThreads, 2>(s, a);
  if (units <= 4 * kQuantThreads) return launch<T, kQuantThreads, 4>(s, a);
  return launch<T, kQuantThreads, 8>(s, a);
}

}  // namespace

moe_status quantize_launch(hipStream_t s, moe_dtype dt, int64_t rows, int n, const void* x,
                           int64_t ldx, int8_t* q, float* scale, int E, const int32_t* offsets,
                           const int32_t* region_rows) {
  if (rows == 0) return MOE_OK;
  const QuantArgs a = {rows, n, x, ldx, q, scale, E, offsets, region_rows};
  return dt == MOE_BF16 ? launch_width<uint16_t>(s, a) : launch_width<float>(s, a);
}

}  // namespace moe

using namespace moe;

extern "C" int moe_quantized_width(int n) { return n < 0 ? 0 : quantized_width(n); }

extern "C" moe_status moe_quantize_rows(void* stream, moe_dtype dt, int64_t rows, int n,
                                        const void* x, int64_t ldx, int8_t* q, float* scale) {
  if (!dtype_ok(dt) || rows < 0 || !width_ok(n) || n > kMaxQuant || ldx < n || ldx % 8 != 0)
    return MOE_EINVAL;
  if (rows == 0) return MOE_OK;
  if (!x || !q || !scale || !aligned16(x) || !aligned16(q)) return MOE_EINVAL;
  return quantize_launch(static_cast<hipStream_t>(stream), dt, rows, n, x, ldx, q, scale, 0,
                         nullptr, nullptr);
}
