// Products of few rows (decoding): C[m, n] = sum_k A[m, k] B[n, k], both
// operands K-contiguous, for a handful of rows per expert.  Bound by the one read of
// the weights, so the kernel is built around that stream: a workgroup owns 16
// columns (16 hidden units of W1 and of W3 in a gated product), its W
// wavefronts take the K steps of 128 bytes in turn, and every wavefront loads
// the weight rows straight into MFMA layout (16x16 blocks; lane l = 16 G + c
// holds bytes 16 G .. of row c, each load touching 64 whole bytes of 16 rows)
// through a ring of D steps, with no LDS, no barrier and no address dependent on
// data inside the loop.  The tokens' rows come from the caches the same way.
// The W partial sums meet in LDS at the end, added in wavefront order.
//
// Against tiles of 32 rows and 128 columns, which stage both operands through
// LDS with a barrier per step, a wavefront keeps 4 KB of weights in flight (8 in a
// gated product) and waits for nobody: 16 KB a CU for 1024 columns, 32 for 4096, 110 for
// the 2 x 14336 of a gated product.
#pragma once

#include "deep.hpp"
#include "quant.hpp"

namespace moe {
namespace {

constexpr int kFewCols = 16;

template <int ES>
using FewAcc = std::conditional_t<ES == 1, intx4, floatx4>;

__device__ __forceinline__ void few_mma(intx4& c, const uint4& a, const uint4& b) {
  c = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(intx4, a), __builtin_bit_cast(intx4, b),
                                            c, 0, 0, 0);
}
template <int ES> __device__ __forceinline__ void few_mma(floatx4& c, const uint4& a, const uint4& b) {
  if constexpr (ES == 2) {
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  } else {
    // element j of every lane's four: k = 4 G + j, the same for both operands
    const floatx4 av = __builtin_bit_cast(floatx4, a), bv = __builtin_bit_cast(floatx4, b);
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(av[j], bv[j], c, 0, 0, 0);
  }
}

// LDS the quantised tokens of a product may take (with the partial sums of 16
// wavefronts, 56 KB of the 64 a launch may ask for).
constexpr int kFewQuant = 40960;
// Bytes between those rows: 16 more than a row, so that a fragment's 16 rows
// fall on different banks.
inline __host__ __device__ int few_pitch(int kbytes) { return kbytes + 16; }

// The rows of A (values of type T, K of them; K a multiple of 8, kb bytes once
// quantised) as int8 in LDS, with their scales: what quantize_kernel does, for
// the at most 16 rows of a workgroup.  Every thread takes units of 8
// values, first for the rows' maxima, then (read again, from the caches) for the
// integers.
template <typename T, int THREADS>
__device__ __forceinline__ void few_quantize(const char* a, int64_t lda, int rows, int K, int kb,
                                             char* q, uint32_t* amax, float* scales) {
  const int units = K / 8, all = kb / 8, pitch = few_pitch(kb);
  auto at = [&](int row, int u) { return reinterpret_cast<const T*>(a + row * lda) + u * 8; };
  if (threadIdx.x < 16) amax[threadIdx.x] = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < rows * units; i += THREADS) {
    const int row = i / units;
    Unit<T> v;
    v.load(at(row, i - row * units));
    atomicMax(&amax[row], abs_bits_max<T>(v, 0));   // a maximum: any order gives it
  }
  __syncthreads();
  for (int i = threadIdx.x; i < rows * all; i += THREADS) {
    const int row = i / all, u = i - row * all;
    float sc;
    const RowScale rs = row_scale(amax[row], sc);
    uint2 b = make_uint2(0, 0);
    if (u < units) {
      Unit<T> v;
      v.load(at(row, u));
      b = quantize8<T>(v, rs);
    }
    *reinterpret_cast<uint2*>(q + row * pitch + u * 8) = b;
    if (u == 0) scales[row] = sc;
  }
  __syncthreads();
}

// RB blocks of 16 rows, W wavefronts.  QUANT (int8, RB = 1): A holds values of
// the layer dtype, which every workgroup quantises for itself while its first
// weights are on their way.
template <int MODE, int ES, int RB, int W, bool QUANT = false>
__global__ __launch_bounds__(64 * W) void ffn_few_rows_kernel(const GroupParams fp) {
  constexpr bool GATED = is_gated(MODE), I8 = ES == 1;
  constexpr int NB = GATED ? 2 : 1;                     // weight matrices
  constexpr int D = 2;                                 // steps in flight per wavefront
  using Acc = FewAcc<ES>;
  static_assert(W >= RB, "a wavefront finishes each block of rows");
  static_assert(!QUANT || (I8 && RB == 1 && !GATED), "quantised in place: one int8 product");
  __shared__ Acc part[W][RB * NB][64];
  __shared__ uint32_t amax[QUANT ? 16 : 1];
  __shared__ float scales[QUANT ? 16 : 1];
  extern __shared__ __attribute__((aligned(16))) char quantised[];   // QUANT: kFewQuant at most
  const GemmParams& p = fp.p;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
  const int c16 = lane & 15, G = lane >> 4;
  const int ntiles = (p.N + kFewCols - 1) / kFewCols;

  // the experts that have rows; lane e keeps expert e's
  int my_first = 0, my_rows = 0;
  uint64_t live = 1;
  if (fp.E) {
    my_rows = group_rows(fp, lane, my_first);
    live = __ballot(my_rows > 0);
  }
  const int items = __popcll(live) * ntiles;
  const int kb = p.K * ES, steps = (kb + kRowBytes - 1) / kRowBytes;
  auto bad = [](bool b) { return static_cast<uint32_t>(b) << 31; };

  for (int item = blockIdx.x; item < items; item += gridDim.x) {
    const int which = item / ntiles, n0 = (item - which * ntiles) * kFewCols;
    int e = 0, m = p.dense.T;
    int64_t first = 0;
    if (fp.E) {
      uint64_t left = live;
      for (int i = 0; i < which; ++i) left &= left - 1;
      e = __builtin_ctzll(left);
      m = __builtin_amdgcn_readlane(my_rows, e);
      first = __builtin_amdgcn_readlane(my_first, e);
    }
    const char* b1 = p.B + e * p.b_gstride + n0 * p.ldb;
    const char* b2 = GATED ? p.B2 + e * p.b_gstride + n0 * p.ldb : b1;
    const __amdgpu_buffer_rsrc_t rb[2] = {tile_rsrc(b1), tile_rsrc(b2)};
    const uint32_t ob = static_cast<uint32_t>(c16 * static_cast<int>(p.ldb) + G * 16) |
                        bad(n0 + c16 >= p.N);
    // rows at a time (as many as LDS was asked for, where they are quantised)
    const int block = QUANT ? min(16, fp.quant_rows) : 16 * RB;
    for (int r0 = 0; r0 < m; r0 += block) {
      const __amdgpu_buffer_rsrc_t ra = tile_rsrc(p.A + (first + r0) * p.lda);
      uint32_t oa[RB];
#pragma unroll
      for (int i = 0; i < RB; ++i)
        oa[i] = static_cast<uint32_t>((16 * i + c16) * static_cast<int>(p.lda) + G * 16) |
                bad(r0 + 16 * i + c16 >= m);
      Acc acc[RB][NB];
#pragma unroll
      for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[i][j] = Acc{};
      uint4 fa[D][RB][2], fb[D][NB][2];
      // both halves of step kt; past K (and past the last step) everything
      // reads as zero
      const int turn = item * 5 % steps;
      auto load = [&](int d, int s) {
        const int kt = s >= steps ? s : s + turn >= steps ? s + turn - steps : s + turn;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t kbad = bad(kt * kRowBytes + h * 64 + G * 16 >= kb);
          const int soff = kt * kRowBytes + h * 64;
#pragma unroll
          for (int j = 0; j < NB; ++j)
            fb[d][j][h] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(rb[j], ob | kbad, soff, 0));
#pragma unroll
          for (int i = 0; i < RB; ++i)
            if constexpr (!QUANT)
              fa[d][i][h] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(ra, oa[i] | kbad, soff, 0));
        }
      };
      // (the scheduling barriers keep the ring in order: a step's products wait
      // for its own loads alone)
#pragma unroll
      for (int d = 0; d < D; ++d) {
        load(d, wave + d * W);
        __builtin_amdgcn_sched_barrier(0);
      }
      if constexpr (QUANT) {
        const int rows = min(block, m - r0);
        const char* a = p.A + (first + r0) * p.lda;
        if (p.out_f32) few_quantize<float, 64 * W>(a, p.lda, rows, fp.k_values, kb, quantised, amax, scales);
        else few_quantize<uint16_t, 64 * W>(a, p.lda, rows, fp.k_values, kb, quantised, amax, scales);
      }
      // this lane's 16 bytes of the quantised rows at half h of K step s, zeros outside
      auto quant_frag = [&](int s, int h) {
        const int kt = s + turn >= steps ? s + turn - steps : s + turn, o = kt * kRowBytes + h * 64 + G * 16;
        const bool ok = s < steps && o < kb && c16 < block && r0 + c16 < m;
        const uint4 v = *reinterpret_cast<const uint4*>(quantised + (ok ? c16 * few_pitch(kb) + o : 0));
        return ok ? v : make_uint4(0, 0, 0, 0);
      };
      for (int kt = wave; kt < steps; kt += D * W) {
#pragma unroll
        for (int d = 0; d < D; ++d) {
          if constexpr (QUANT) {
#pragma unroll
            for (int h = 0; h < 2; ++h) fa[d][0][h] = quant_frag(kt + d * W, h);
          }
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < RB; ++i)
#pragma unroll
              for (int j = 0; j < NB; ++j) {
                if constexpr (I8) few_mma(acc[i][j], fa[d][i][h], fb[d][j][h]);
                else few_mma<ES>(acc[i][j], fa[d][i][h], fb[d][j][h]);
              }
          load(d, kt + (d + D) * W);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      __syncthreads();   // the last tile's sums have been read
#pragma unroll
      for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) part[wave][i * NB + j][lane] = acc[i][j];
      __syncthreads();
      if (wave < RB) {
        Acc sum[NB];
#pragma unroll
        for (int j = 0; j < NB; ++j) {
          sum[j] = part[0][wave * NB + j][lane];
#pragma unroll
          for (int w = 1; w < W; ++w) sum[j] += part[w][wave * NB + j][lane];
        }
        // element q: row 4 G + q of the block, column c16
        const int col = n0 + c16;
        if (col < p.N) {
          float s1 = 1.f, s3 = 1.f;
          if constexpr (I8) {
            s1 = p.b_scale[e * p.s_gstride + col];
            if constexpr (GATED) s3 = p.b2_scale[e * p.s_gstride + col];
          }
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const int lr = r0 + 16 * wave + 4 * G + q;
            if (lr >= m || (QUANT && lr >= r0 + block)) continue;
            const int64_t row = first + lr;
            float v = static_cast<float>(sum[0][q]), v3 = GATED ? static_cast<float>(sum[NB - 1][q]) : 0.f;
            if constexpr (I8) {
              const float as = QUANT ? scales[lr - r0] : row_scale_at(p.a_scale, row);
              v = v * as * s1;
              v3 = v3 * as * s3;
            }
            constexpr int OS = ES == 4 ? 4 : 2;   // bytes of the dense block's values
            if constexpr (MODE == M_GATED_FWD) {
              float g, dg;
              gate_f(v, p.act, g, dg);
              if (p.H1) {   // the backward's factors
                char *h1 = p.H1 + row * p.ldh + static_cast<int64_t>(col) * OS,
                     *h3 = p.H3 + row * p.ldh + static_cast<int64_t>(col) * OS;
                if constexpr (ES == 4) {
                  *reinterpret_cast<float*>(h1) = v3 * dg;
                  *reinterpret_cast<float*>(h3) = g;
                } else {
                  *reinterpret_cast<uint16_t*>(h1) = f2bf(v3 * dg);
                  *reinterpret_cast<uint16_t*>(h3) = f2bf(g);
                }
              }
              v = g * v3;
            } else if constexpr (MODE == M_I8_FWD1_SWIGLU) {
              v = v * sigm(v) * v3;
            } else if constexpr (MODE == M_I8_FWD1) {
              v = act_i8(v, p.act);
            } else if constexpr (MODE == M_ADD_STORE) {
              if (p.add) {
                const char* b = p.add + row * p.ldadd + static_cast<int64_t>(col) * OS;
                v += ES == 4 ? *reinterpret_cast<const float*>(b) : bf2f(*reinterpret_cast<const uint16_t*>(b));
              }
            }
            const bool wide = I8 ? p.out_f32 != 0 : ES == 4;
            char* c = p.C + row * p.ldc + static_cast<int64_t>(col) * (wide ? 4 : 2);
            if (wide) *reinterpret_cast<float*>(c) = v;
            else *reinterpret_cast<uint16_t*>(c) = f2bf(v);
          }
        }
      }
    }
  }
}

// Wavefronts per workgroup: 16, halved while they are more than 8 a CU or more
// than there are K steps, but not below 4.
inline int few_waves(int64_t items, int steps) {
  const int64_t want = 8 * static_cast<int64_t>(num_cus());
  int w = 16;
  while (w > 4 && (items * w > want || w > steps)) w /= 2;
  return w;
}

// Launches a product of few rows: most_rows rows in one expert at the most,
// most_groups experts with rows.
// quantise: A holds values of the layer dtype.  That saves a launch (32 experts of
// 1024 -> 2048, 16 rows: 31.8 -> 28.6 us a call) while the rows are short; two
// passes over a long one in every workgroup cost more (2 rows of 14336 values: 67.5
// -> 70.3 us).
inline bool few_fits_quant(int64_t most_rows, int kbytes) {
  return kbytes <= 8192 && most_rows <= 16 && most_rows * few_pitch(kbytes) <= kFewQuant;
}
template <int MODE, int ES>
moe_status launch_few(hipStream_t s, const char* name, const GroupParams& fp, int64_t most_rows,
                      int most_groups, bool quantise = false) {
  const int64_t items = static_cast<int64_t>(most_groups) * cdiv(fp.p.N, kFewCols);
  const int steps = cdiv(static_cast<int64_t>(fp.p.K) * ES, kRowBytes), w = few_waves(items, steps);
  const int grid = static_cast<int>(std::min<int64_t>(items, 16 * num_cus()));
  MOE_TIMED(name, s);
  auto go = [&](auto rb_c, auto w_c) {
    constexpr int RB = decltype(rb_c)::value, W = decltype(w_c)::value;
    if constexpr (MODE == M_I8_STORE && RB == 1) {
      if (quantise) {
        ffn_few_rows_kernel<MODE, ES, RB, W, true>
            <<<grid, 64 * W, most_rows * few_pitch(fp.p.K), s>>>(fp);
        return;
      }
    }
    ffn_few_rows_kernel<MODE, ES, RB, W><<<grid, 64 * W, 0, s>>>(fp);
  };
  auto rows = [&](auto w_c) {
    if constexpr (ES == 4) {   // only the fp32 block takes it for more than 16 rows
      if (most_rows > 16) return go(std::integral_constant<int, 2>{}, w_c);
    }
    go(std::integral_constant<int, 1>{}, w_c);
  };
  if (w == 16) rows(std::integral_constant<int, 16>{});
  else if (w == 8) rows(std::integral_constant<int, 8>{});
  else rows(std::integral_constant<int, 4>{});
  MOE_LAUNCH_CHECK();
  return MOE_OK;
}

}  // namespace
}  // namespace moe
