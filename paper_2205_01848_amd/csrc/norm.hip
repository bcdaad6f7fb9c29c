// Root-mean-square norm of rows, with the addition that comes before it on a
// residual stream, forward and backward:
//     s = x + add (rounded to the layer dtype),  r = 1 / sqrt(mean_j s_j^2 + eps),
//     y_j = s_j r w_j
// and, for experts in 8-bit integers, the same rows quantised.  With a = s w (fp32),
//     q_j = rint(a_j / c),  c = max_j |a_j| (1/127),  scale = c r:
// the row's factor r cancels in the quotient, so q does not depend on the order in which
// the squares are summed, and both reductions, of the squares and of |a|, are one
// pass over values in registers.  (From the rounded y the integers of bf16 rows would
// carry y's rounding, half a step of 2^-8, beside their own.)
// Backward, with g = dy w:
//     dx = r (g - s r^2 mean_j(g s)) + dsum,   dw_j = sum_t dy_tj s_tj r_t;
// dx is the gradient of x and of add alike, dsum what reaches s from beside the norm.
//
// Bound by memory: every row is read once into registers.  G threads take a row, in
// units of 8 values, U units a thread: a wavefront up to 2048 values, so that most
// rows need no barrier, 256 threads up to 8192, 1024 up to 32768.  8192 x 4096 bf16 with
// the addition, y and 8-bit rows: 63 us, 4.8 TB/s; 16384 x 4096 with the addition and y 89 us,
// 6.0 TB/s, its backward 111 us, 4.8 TB/s, and dw's partial sums 4.6 us; one row 6 us.

#include <algorithm>
#include <utility>

#include "quant.hpp"

namespace moe {
namespace {

constexpr int kMaxNorm = 32768;       // values of a row that 1024 threads hold
constexpr int64_t kNormParts = 512;   // partial sums of dw, at most

struct NormArgs {
  const void *x, *add, *w;
  void *sum, *y;
  int64_t ldx, ldadd, ldsum, ldy, rows;
  int d;
  float eps;
  float* rstd;
  int8_t* q;
  float* scale;
};

// v summed over a row's G threads, m their largest, in all of them; `part`: LDS of one
// entry per wavefront, another set each turn, so that one barrier a row suffices.
struct SumMax {
  float v;
  uint32_t m;
};
template <int G, bool MAX>
__device__ __forceinline__ SumMax row_reduce(SumMax a, SumMax (*part)[G / kWave], int& turn) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    a.v += __shfl_xor(a.v, o, 64);
    if (MAX) a.m = max(a.m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(a.m), o, 64)));
  }
  if constexpr (G > kWave) {
    if ((threadIdx.x & 63) == 0) part[turn][threadIdx.x / kWave] = a;
    __syncthreads();
    a = part[turn][0];
#pragma unroll
    for (int w = 1; w < G / kWave; ++w) {
      a.v += part[turn][w].v;
      if (MAX) a.m = max(a.m, part[turn][w].m);
    }
    turn ^= 1;
  }
  return a;
}

template <int G> constexpr int kNormThreads = G < 256 ? 256 : G;

template <typename T, int G, int U, bool Q>
__global__ __launch_bounds__(kNormThreads<G>) void norm_fwd_kernel(const NormArgs a) {
  constexpr int kPer = kNormThreads<G> / G;   // rows of a workgroup at a time
  __shared__ SumMax part[2][G / kWave];
  int turn = 0;
  const int t = threadIdx.x % G, units = a.d / 8, qunits = (a.d + 15) / 16 * 2;
  const T* w = static_cast<const T*>(a.w);
  for (int64_t base = static_cast<int64_t>(blockIdx.x) * kPer; base < a.rows;
       base += static_cast<int64_t>(gridDim.x) * kPer) {
    const int64_t row = base + threadIdx.x / G;   // the same for a whole wavefront
    if (row >= a.rows) break;                     // (G > 64: the whole workgroup's row)
    const T* x = static_cast<const T*>(a.x) + row * a.ldx;
    Unit<T> s[U], b[U];
#pragma unroll
    for (int i = 0; i < U; ++i)
      if (t + i * G < units) s[i].load(x + (t + i * G) * 8);
    if (a.add) {
      const T* add = static_cast<const T*>(a.add) + row * a.ldadd;
#pragma unroll
      for (int i = 0; i < U; ++i)
        if (t + i * G < units) b[i].load(add + (t + i * G) * 8);
    }
    SumMax acc = {0.f, 0};
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int u = t + i * G;
      if (u >= units) continue;
      float f[8];
      if (a.add) {
        float g[8];
        s[i].get(f);
        b[i].get(g);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] += g[e];
        s[i].set(f);
        if (a.sum) s[i].store(static_cast<T*>(a.sum) + row * a.ldsum + u * 8);
      }
      s[i].get(f);
#pragma unroll
      for (int e = 0; e < 8; ++e) acc.v += f[e] * f[e];
      if constexpr (Q) {
        Unit<T> wu;
        wu.load(w + u * 8);
        float g[8];
        wu.get(g);
#pragma unroll
        for (int e = 0; e < 8; ++e) g[e] *= f[e];
        acc.m = abs_bits_max(g, acc.m);
      }
    }
    acc = row_reduce<G, Q>(acc, part, turn);
    const float r = 1.f / __builtin_sqrtf(acc.v / static_cast<float>(a.d) + a.eps);
    RowScale rs;
    if constexpr (Q) {
      float c;
      rs = row_scale(acc.m, c);
      if (t == 0) a.scale[row] = c * r;
    }
    if (a.rstd && t == 0) a.rstd[row] = r;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int u = t + i * G;
      if (u < units) {
        Unit<T> wu;
        wu.load(w + u * 8);
        float f[8], g[8];
        s[i].get(f);
        wu.get(g);
        if (a.y) {
          float v[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = f[e] * r * g[e];
          Unit<T> o;
          o.set(v);
          o.store(static_cast<T*>(a.y) + row * a.ldy + u * 8);
        }
        if constexpr (Q) {
#pragma unroll
          for (int e = 0; e < 8; ++e) f[e] *= g[e];
          *reinterpret_cast<uint2*>(a.q + row * qunits * 8 + u * 8) = quantize8(f, rs);
        }
      } else if (Q && u < qunits) {
        *reinterpret_cast<uint2*>(a.q + row * qunits * 8 + u * 8) = make_uint2(0, 0);
      }
    }
  }
}

struct NormBwdArgs {
  const void *s, *w, *dy, *dsum;
  void* dx;
  int64_t lds, lddy, lddsum, lddx, rows;
  int d;
  const float* rstd;
  float* parts;   // [gridDim, d]; NULL: no dw
};

template <typename T, int G, int U>
__global__ __launch_bounds__(kNormThreads<G>) void norm_bwd_kernel(const NormBwdArgs a) {
  constexpr int kPer = kNormThreads<G> / G;
  // dsum with the other rows' loads, but where 1024 threads hold 4 units of fp32 each: of
  // their 128 registers 63 would go to scratch memory, 9 this way (4096 x 32768: 595 and 463 us,
  // 4.6 TB/s).  bf16 rows of that width keep 19 there with dsum ahead: 302 us, 3.6 TB/s
  constexpr bool kAhead = sizeof(T) == 2 || G * U < 4096;
  __shared__ SumMax part[2][G / kWave];
  __shared__ float join[kPer > 1 ? kPer * U * G * 8 : 1];
  int turn = 0;
  const int t = threadIdx.x % G, units = a.d / 8;
  const T* w = static_cast<const T*>(a.w);
  float dw[U][8];
#pragma unroll
  for (int i = 0; i < U; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) dw[i][e] = 0.f;
  for (int64_t base = static_cast<int64_t>(blockIdx.x) * kPer; base < a.rows;
       base += static_cast<int64_t>(gridDim.x) * kPer) {
    const int64_t row = base + threadIdx.x / G;
    if (row >= a.rows) break;
    const T* s = static_cast<const T*>(a.s) + row * a.lds;
    const T* dy = static_cast<const T*>(a.dy) + row * a.lddy;
    const T* ds = a.dsum ? static_cast<const T*>(a.dsum) + row * a.lddsum : nullptr;
    Unit<T> su[U], gu[U], du[U];
#pragma unroll
    for (int i = 0; i < U; ++i)
      if (t + i * G < units) {
        su[i].load(s + (t + i * G) * 8);
        gu[i].load(dy + (t + i * G) * 8);
      }
    if (kAhead && ds) {
#pragma unroll
      for (int i = 0; i < U; ++i)
        if (t + i * G < units) du[i].load(ds + (t + i * G) * 8);
    }
    const float r = a.rstd[row];
    SumMax acc = {0.f, 0};
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if (t + i * G >= units) continue;
      Unit<T> wu;
      wu.load(w + (t + i * G) * 8);
      float f[8], g[8], v[8];
      su[i].get(f);
      gu[i].get(g);
      wu.get(v);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float p = f[e] * g[e];
        acc.v += p * v[e];
        dw[i][e] += p * r;
      }
    }
    acc = row_reduce<G, false>(acc, part, turn);
    const float c = acc.v / static_cast<float>(a.d) * r * r;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int u = t + i * G;
      if (u >= units) continue;
      Unit<T> wu;
      wu.load(w + u * 8);
      float f[8], g[8], v[8];
      su[i].get(f);
      gu[i].get(g);
      wu.get(v);
#pragma unroll
      for (int e = 0; e < 8; ++e) g[e] = r * (g[e] * v[e] - f[e] * c);
      if (ds) {
        if (!kAhead) du[i].load(ds + u * 8);
        du[i].get(f);
#pragma unroll
        for (int e = 0; e < 8; ++e) g[e] += f[e];
      }
      Unit<T> o;
      o.set(g);
      o.store(static_cast<T*>(a.dx) + row * a.lddx + u * 8);
    }
  }
  if (!a.parts) return;
  // the workgroup's rows, in order of its wavefronts
  float* to = a.parts + static_cast<int64_t>(blockIdx.x) * a.d;
  if constexpr (kPer > 1) {
    float* mine = join + (threadIdx.x / G) * (U * G * 8);
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) mine[(t + i * G) * 8 + e] = dw[i][e];
    __syncthreads();
    for (int j = threadIdx.x; j < a.d; j += kNormThreads<G>) {
      float v = join[j];
#pragma unroll
      for (int k = 1; k < kPer; ++k) v += join[k * (U * G * 8) + j];
      to[j] = v;
    }
  } else {
#pragma unroll
    for (int i = 0; i < U; ++i)
      if (t + i * G < units) {
        float4* p = reinterpret_cast<float4*>(to + (t + i * G) * 8);
        p[0] = make_float4(dw[i][0], dw[i][1], dw[i][2], dw[i][3]);
        p[1] = make_float4(dw[i][4], dw[i][5], dw[i][6], dw[i][7]);
      }
  }
}

// dw = the partial sums of `parts` workgroups, added in order: 16 columns a workgroup,
// 16 threads for each, every one its share of the sums.
constexpr int kDwCols = 16, kDwShares = 16;
template <typename T>
__global__ __launch_bounds__(kDwCols * kDwShares) void norm_dw_kernel(const float* __restrict__ parts,
                                                                      int n, int d, T* __restrict__ dw) {
  __shared__ float sums[kDwShares][kDwCols];
  const int c = threadIdx.x % kDwCols, k = threadIdx.x / kDwCols, col = blockIdx.x * kDwCols + c;
  const int per = (n + kDwShares - 1) / kDwShares, last = min(n, (k + 1) * per);
  float v = 0.f;
  if (col < d)
#pragma unroll 8
    for (int i = k * per; i < last; ++i) v += parts[static_cast<int64_t>(i) * d + col];
  sums[k][c] = v;
  __syncthreads();
  if (k > 0 || col >= d) return;
#pragma unroll
  for (int j = 1; j < kDwShares; ++j) v += sums[j][c];
  dw[col] = Elem<T>::from_f(v);
}

// Workgroups of the backward, and with it the partial sums, from the sizes alone:
// rows per workgroup at a time as the launch has them.
int norm_rows_at_once(int d) { return d <= 2048 ? 4 : 1; }
int64_t norm_parts(int64_t rows, int d) {
  const int per = norm_rows_at_once(d);
  return std::min(kNormParts, (rows + per - 1) / per);
}

// f(threads a row, units a thread) for rows of d values
template <typename F> moe_status by_width(int d, F&& f) {
  const int units = d / 8;
#define MOE_WIDTH(G, U) \
  if (units <= G * U) return f(std::integral_constant<int, G>{}, std::integral_constant<int, U>{});
  MOE_WIDTH(64, 1)
  MOE_WIDTH(64, 2)
  MOE_WIDTH(64, 4)
  MOE_WIDTH(256, 2)
  MOE_WIDTH(256, 4)
  MOE_WIDTH(1024, 2)
  MOE_WIDTH(1024, 4)
#undef MOE_WIDTH
  return MOE_EINVAL;
}

template <typename T> moe_status launch_fwd(hipStream_t s, const NormArgs& a) {
  return by_width(a.d, [&](auto g, auto u) -> moe_status {
    constexpr int G = decltype(g)::value, U = decltype(u)::value, kPer = kNormThreads<G> / G;
    const int grid = static_cast<int>(std::min<int64_t>((a.rows + kPer - 1) / kPer, 16 * num_cus()));
    MOE_TIMED("rms_norm", s);
    if (a.q) norm_fwd_kernel<T, G, U, true><<<grid, kNormThreads<G>, 0, s>>>(a);
    else norm_fwd_kernel<T, G, U, false><<<grid, kNormThreads<G>, 0, s>>>(a);
    MOE_LAUNCH_CHECK();
    return MOE_OK;
  });
}
template <typename T> moe_status launch_bwd(hipStream_t s, const NormBwdArgs& a) {
  return by_width(a.d, [&](auto g, auto u) -> moe_status {
    constexpr int G = decltype(g)::value, U = decltype(u)::value;
    MOE_TIMED("rms_norm_bwd", s);
    norm_bwd_kernel<T, G, U><<<static_cast<int>(norm_parts(a.rows, a.d)), kNormThreads<G>, 0, s>>>(a);
    MOE_LAUNCH_CHECK();
    return MOE_OK;
  });
}

bool norm_shape_ok(int64_t rows, int d) { return rows >= 0 && width_ok(d) && d <= kMaxNorm; }
bool norm_pitch_ok(int64_t ld, int d) { return ld >= d && ld % 8 == 0; }

// Rows written over an input's rows: the same ones, or a workgroup would overwrite another's.
bool in_place_ok(int64_t rows, const void* out, int64_t ldout, const void* in, int64_t ldin) {
  return out != in || ldout == ldin || rows <= 1;
}

}  // namespace
}  // namespace moe

using namespace moe;

extern "C" moe_status moe_rms_norm_fwd(void* stream, moe_dtype dt, int64_t rows, int d, const void* x,
                                       int64_t ldx, const void* add, int64_t ldadd, const void* weight,
                                       float eps, void* sum, int64_t ldsum, void* y, int64_t ldy,
                                       float* rstd, int8_t* q, float* scale) {
  if (!dtype_ok(dt) || !norm_shape_ok(rows, d) || !(eps > 0.f) || !(eps < INFINITY)) return MOE_EINVAL;
  if (!norm_pitch_ok(ldx, d) || (add && !norm_pitch_ok(ldadd, d)) || (sum && !norm_pitch_ok(ldsum, d)) ||
      (y && !norm_pitch_ok(ldy, d)))
    return MOE_EINVAL;
  if (rows == 0) return MOE_OK;
  if ((!y && !q) || !q != !scale || (sum && !add) || (y && y == sum)) return MOE_EINVAL;
  for (const auto& [out, ld] : {std::pair<const void*, int64_t>{sum, ldsum}, {y, ldy}})
    if (out && (!in_place_ok(rows, out, ld, x, ldx) || !in_place_ok(rows, out, ld, add, ldadd))) return MOE_EINVAL;
  if (!x || !weight || !aligned16(x) || !aligned16(add) || !aligned16(weight) || !aligned16(sum) ||
      !aligned16(y) || !aligned16(q))
    return MOE_EINVAL;
  const NormArgs a = {x, add, weight, sum, y, ldx, ldadd, ldsum, ldy, rows, d, eps, rstd, q, scale};
  hipStream_t s = static_cast<hipStream_t>(stream);
  return dt == MOE_BF16 ? launch_fwd<uint16_t>(s, a) : launch_fwd<float>(s, a);
}

extern "C" size_t moe_rms_norm_bwd_workspace_bytes(int64_t rows, int d) {
  if (!norm_shape_ok(rows, d)) return 0;
  return static_cast<size_t>(std::max<int64_t>(norm_parts(rows, d), 1)) * d * 4;
}

extern "C" moe_status moe_rms_norm_bwd(void* stream, moe_dtype dt, int64_t rows, int d, const void* s,
                                       int64_t lds, const void* weight, const float* rstd,
                                       const void* dy, int64_t lddy, const void* dsum, int64_t lddsum,
                                       void* dx, int64_t lddx, moe_dtype dw_dt, void* dw,
                                       void* workspace, size_t workspace_bytes) {
  if (!dtype_ok(dt) || !norm_shape_ok(rows, d)) return MOE_EINVAL;
  if (dw && dw_dt != dt && dw_dt != MOE_F32) return MOE_EINVAL;
  if (!norm_pitch_ok(lds, d) || !norm_pitch_ok(lddy, d) || (dsum && !norm_pitch_ok(lddsum, d)) ||
      !norm_pitch_ok(lddx, d))
    return MOE_EINVAL;
  if (rows > 0 && (!s || !weight || !rstd || !dy || !dx)) return MOE_EINVAL;
  if (!in_place_ok(rows, dx, lddx, s, lds) || !in_place_ok(rows, dx, lddx, dy, lddy) ||
      !in_place_ok(rows, dx, lddx, dsum, lddsum))
    return MOE_EINVAL;
  if (!aligned16(s) || !aligned16(weight) || !aligned16(dy) || !aligned16(dsum) || !aligned16(dx))
    return MOE_EINVAL;
  if (dw && (!workspace || !aligned16(workspace) ||
             workspace_bytes < moe_rms_norm_bwd_workspace_bytes(rows, d)))
    return MOE_EWORKSPACE;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (rows > 0) {
    const NormBwdArgs a = {s, weight, dy, dsum, dx, lds, lddy, lddsum, lddx, rows, d, rstd,
                           dw ? static_cast<float*>(workspace) : nullptr};
    const moe_status e = dt == MOE_BF16 ? launch_bwd<uint16_t>(st, a) : launch_bwd<float>(st, a);
    if (e != MOE_OK) return e;
  }
  if (!dw) return MOE_OK;
  MOE_TIMED("rms_norm_dw", st);
  const int grid = (d + kDwCols - 1) / kDwCols, n = static_cast<int>(rows > 0 ? norm_parts(rows, d) : 0);
  if (dw_dt == MOE_BF16)
    norm_dw_kernel<uint16_t><<<grid, kDwCols * kDwShares, 0, st>>>(static_cast<float*>(workspace), n, d,
                                                                  static_cast<uint16_t*>(dw));
  else
    norm_dw_kernel<float><<<grid, kDwCols * kDwShares, 0, st>>>(static_cast<float*>(workspace), n, d,
                                                               static_cast<float*>(dw));
  MOE_LAUNCH_CHECK();
  return MOE_OK;
}
