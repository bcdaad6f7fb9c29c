// Products on tiles of 32 RB rows and 128 columns with NS stages in flight.
//
// The two-stage kernels of gemm.hpp issue a K step's loads about one step ahead
// of their use.  Where a CU holds only one workgroup, or a step is short
// because the tile has few rows, that is less than the memory latency: a step
// takes about 0.6 us whatever its height.  Here a step's loads are issued NS - 1 steps
// ahead (one barrier per step): four stages of 20 KB for tiles of 32 rows and three of
// 24 KB for 64 rows, two workgroups per CU, so 64 to 96 KB of weights are in
// flight per CU; four stages of 32 KB for 128 rows, one workgroup per CU, for
// products with no more tiles than CUs.
//
// Grouped products need no schedule: every workgroup numbers the experts' tiles
// itself, from their rows, by a prefix sum over its lanes.
#pragma once

#include "gemm.hpp"

namespace moe {
namespace {

// A product over the regions of E experts (E = 0: dense, p.dense).
struct GroupParams {
  GemmParams p;
  int E;
  const int32_t* rows;
  int64_t rows_alloc;
  // few rows, quantised in place: the values of a row (K counts the quantised
  // bytes) and the rows that LDS holds at a time
  int k_values = 0, quant_rows = 0;
};

// The rows of expert `lane`, clamped to its region and to rows_alloc, and
// where they start.
__device__ __forceinline__ int group_rows(const GroupParams& gp, int lane, int& first) {
  if (lane >= gp.E) return 0;
  const int64_t off = gp.p.offsets[lane];
  first = static_cast<int>(off);
  int64_t r = gp.rows[lane];
  if (off < 0 || off >= gp.rows_alloc) r = 0;
  r = min(r, static_cast<int64_t>(gp.p.offsets[lane + 1]) - off);
  r = min(r, gp.rows_alloc - off);
  return static_cast<int>(max(r, int64_t(0)));
}

// One block's product by the compiler's MFMA (its hazards are the compiler's).
template <int ES>
__device__ __forceinline__ void mma16(floatx4& c, const uint4& a, const uint4& b) {
  if constexpr (ES == 1)
    c = __builtin_bit_cast(floatx4, __builtin_amdgcn_mfma_i32_16x16x64_i8(
                                        __builtin_bit_cast(intx4, a), __builtin_bit_cast(intx4, b),
                                        __builtin_bit_cast(intx4, c), 0, 0, 0));
  else
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// acc += A_tile * B_tile^T: wave w owns tile rows 16 RB (w >> 1) .. and columns
// 64 (w & 1) .. +63, over the nk K steps from k_first on.  LDS tiles, swizzles, loads and fragments are those of the
// mid kernel (gemm.hpp): K-contiguous tiles as rows of 128 bytes, K-major ones as k-rows
// of 128 elements (K-major A: RB = 4).
// K-major k-rows r with r & 8 also have the two 16-element halves of every 32-element
// segment swapped: a transpose read takes half a segment of k-rows r .. r + 3 and of
// r + 8 .. r + 11 at once, which would otherwise lie on the same banks (2048 tokens,
// 1024 -> 2816: the backward's dX, then on one group of wavefronts, 9 % shorter.  The mid and the 256x256 kernels,
// bound by other things, gain 0 to 1 % by it and do without.)
template <int RB, int NS, int ALAY, int BLAY, bool GATED, int ES>
__device__ __forceinline__ void mainloop_deep(const TileOps& op, int wave, int k_first, int nk,
                                              char* const (&sa)[NS], char* const (&sb)[NS],
                                              floatx4 (&acc)[RB][4]) {
  static_assert(ALAY == L_KC || RB == 4, "K-major A tiles are 128 columns wide");
  static_assert(ES == 2 || (ALAY == L_KC && BLAY == L_KC), "int8 operands are K-contiguous");
  constexpr int KSTEP = kRowBytes / ES, KMROW = 256;
  const int lane = static_cast<int>(threadIdx.x) & 63;
  const int wm = wave >> 1, wn = wave & 1;
#pragma unroll
  for (int i = 0; i < RB; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
  const int K = op.K;

  // ---- loads: of every stage, wave w loads the 1 KB blocks 4i + w of A
  // (i < RB) and of B (i < 4); a lane's offset has bit 31 set where it would
  // read past the valid rows, columns or k (it then reads zeros)
  const int l3 = lane >> 3;
  const int co = ((lane & 7) ^ swz(l3 + (wave & 1) * 8)) * 16;
  const int kr = lane >> 4, pe = (lane & 15) * 8;
  const int km_col = ((((pe >> 5) ^ kr) << 5) + (pe & 31)) ^ (wave & 2 ? 16 : 0);
  const int lda = static_cast<int>(op.a.ld), ldb = static_cast<int>(op.b.ld);
  auto bad = [](bool b) { return static_cast<uint32_t>(b) << 31; };
  auto brow = [&](int i) { return GATED ? (i >> 1) * 32 + wave * 8 : (4 * i + wave) * 8; };
  const __amdgpu_buffer_rsrc_t ra = tile_rsrc(op.a.base), rb = tile_rsrc(op.b.base);
  const __amdgpu_buffer_rsrc_t rb3 = tile_rsrc(GATED ? op.b.base2 : op.b.base);
  uint32_t offa[ALAY == L_KC ? RB : 1], offb[BLAY == L_KC ? 4 : 1];
  if constexpr (ALAY == L_KC) {
#pragma unroll
    for (int i = 0; i < RB; ++i)
      offa[i] = static_cast<uint32_t>(l3 * lda + co) | bad((4 * i + wave) * 8 + l3 >= op.a.rows);
  } else {
    offa[0] = static_cast<uint32_t>(kr * lda + km_col * 2) | bad(km_col >= op.a.rows);
  }
  if constexpr (BLAY == L_KC) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      offb[i] = static_cast<uint32_t>(l3 * ldb + co) | bad(brow(i) + l3 >= op.b.rows);
  } else {
    offb[0] = static_cast<uint32_t>(kr * ldb + km_col * 2) | bad(km_col >= op.b.rows);
  }
  auto km_rsrc = [&](const Operand& o, int kt, bool second) {
    const int64_t k = static_cast<int64_t>(kt) * KSTEP - (second ? o.split : 0);
    return tile_rsrc((second ? o.base2 : o.base) + k * o.ld);
  };
  auto issue = [&](const __amdgpu_buffer_rsrc_t& rs, char* dst, uint32_t off, int soff) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, MOE_LDS(dst), 16, off, soff, 0, 0);
  };
  auto load = [&](int kt, char* da, char* db) {
    kt += k_first;
    const uint32_t kbad = bad(kt * kRowBytes + co >= K * ES);
    if constexpr (ALAY == L_KC) {
#pragma unroll
      for (int i = 0; i < RB; ++i)
        issue(ra, da + (4 * i + wave) * 1024, offa[i] | kbad, (4 * i + wave) * 8 * lda + kt * kRowBytes);
    } else {
      const __amdgpu_buffer_rsrc_t rs = km_rsrc(op.a, kt, false);
#pragma unroll
      for (int i = 0; i < RB; ++i) {
        const int blk = 4 * i + wave;
        issue(rs, da + blk * 1024, offa[0] | bad(kt * KSTEP + 4 * blk + kr >= K), 4 * blk * lda);
      }
    }
    if constexpr (BLAY == L_KC) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        issue(GATED && (i & 1) ? rb3 : rb, db + (4 * i + wave) * 1024, offb[i] | kbad,
              brow(i) * ldb + kt * kRowBytes);
    } else {
      const __amdgpu_buffer_rsrc_t rs = km_rsrc(op.b, kt, false);
      const __amdgpu_buffer_rsrc_t rs2 = op.b.base2 ? km_rsrc(op.b, kt, true) : rs;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int blk = 4 * i + wave, kabs = kt * KSTEP + 4 * blk;   // split: a multiple of 8
        issue(kabs >= op.b.split ? rs2 : rs, db + blk * 1024, offb[0] | bad(kabs + kr >= K), 4 * blk * ldb);
      }
    }
  };

  // ---- fragments, as in the mid kernel
  const int c16 = lane & 15, G = lane >> 4;
  const int fa_kc = (wm * 16 * RB + c16) * kRowBytes, fb_kc = (wn * 64 + c16) * kRowBytes;
  auto km_frag = [&](const char* st, int cb, int h) -> uint4 {
    const int phys = (((cb >> 5) ^ (c16 >> 2)) << 5) + ((cb & 31) ^ (16 * (G & 1))) + 4 * (c16 & 3);
    const char* p0 = st + (32 * h + 8 * G + (c16 >> 2)) * KMROW + phys * 2;
    const uint2 lo = read_tr(p0), hi = read_tr(p0 + 4 * KMROW);
    return make_uint4(lo.x, lo.y, hi.x, hi.y);
  };
  auto compute = [&](const char* ca, const char* cb) {
    uint4 fa[2][RB], fb[2][4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int sw = ((4 * h + G) ^ (c16 >> 1)) << 4;
#pragma unroll
      for (int i = 0; i < RB; ++i) {
        if constexpr (ALAY == L_KC) fa[h][i] = *reinterpret_cast<const uint4*>(ca + fa_kc + i * 16 * kRowBytes + sw);
        else fa[h][i] = km_frag(ca, wm * 64 + i * 16, h);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (BLAY == L_KC) fb[h][j] = *reinterpret_cast<const uint4*>(cb + fb_kc + j * 16 * kRowBytes + sw);
        else fb[h][j] = km_frag(cb, wn * 64 + j * 16, h);
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) mma16<ES>(acc[i][j], fa[h][i], fb[h][j]);
  };

  ring_steps<NS, RB + 4>(nk, sa, sb, load, compute);
}

// KG = 2 (64 rows, dense): a second group of four wavefronts takes the second half of
// the K steps into stages of its own, and its sums are added through LDS at the end.
// A wavefront alone on its SIMD waits for its fragments between the matrix
// instructions; two overlap.  For tiles that leave every CU one workgroup (2048
// tokens, 2816 -> 1024, operands in the last-level cache: Y 18.8 -> 17.2, dX 38.0 ->
// 31.9 us; six stages for one group instead left Y as it was and made dX 7 %
// longer).  The plan (plan.hpp) knows the time of one group only.
template <int MODE, int PASS, int RB, int NS, int KG>
__global__ __launch_bounds__(KG * kThreads16, RB <= 2 ? 2 : 1) void ffn_gemm16_deep_kernel(const GroupParams gp) {
  constexpr bool GATED = is_gated(MODE), DENSE = is_dense(MODE), VARK = is_dw(MODE);
  constexpr int ES = op_bytes(MODE), TM = 32 * RB, TN = kMidN;
  constexpr int kA = TM * kRowBytes, kB = TN * kRowBytes;
  using C = Tile16<RB, 4>;
  // one object per stage, so that the compiler can tell the loads into one
  // from the reads of another
  __shared__ __attribute__((aligned(16))) char a0[KG * kA], b0[KG * kB], a1[KG * kA], b1[KG * kB],
      a2[KG * kA], b2[KG * kB];
  __shared__ __attribute__((aligned(16))) char a3[NS > 3 ? kA : 16], b3[NS > 3 ? kB : 16];
  const GemmParams& p = gp.p;
  const int lane = threadIdx.x & 63;
  const int wave8 = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
  const int wave = wave8 & 3, kg = wave8 >> 2, ga = KG > 1 ? kg * kA : 0, gb = KG > 1 ? kg * kB : 0;
  const int wm = wave >> 1, wn = wave & 1;
  int my_first = 0, my_rows = 0, my_end = 0, n_mt = 0;
  if constexpr (!DENSE) {
    my_rows = group_rows(gp, lane, my_first);
    my_end = wave_incl_scan((my_rows + TM - 1) / TM);
    n_mt = __builtin_amdgcn_readlane(my_end, 63);
  }
  const int n_items = DENSE ? dense_items<MODE>(p) : n_mt * p.ntiles;
  for (int round = 0;; ++round) {
    const int L = round_item(round, n_items);
    if (L < 0) break;
    TileOps op;
    int g = 0, row0, m_valid, n0, slot = -1, mt, nt;
    if constexpr (DENSE) {
      const int si = dense_tile<MODE>(p, L, mt, nt);
      row0 = mt * TM;
      n0 = nt * (GATED ? TN / 2 : TN);
      m_valid = min(TM, (VARK ? p.M_out : p.dense.T) - row0);
      slot = p.dense.splits > 1 ? si : -1;
      op = dense_ops<MODE, PASS, ES>(p, row0, m_valid, n0, TN, si);
    } else {
      decode_banded(L, n_mt, p.ntiles, mt, nt);
      g = __builtin_popcountll(__ballot(my_end <= mt));
      const int rows = __builtin_amdgcn_readlane(my_rows, g);
      const int m0 = (mt - (__builtin_amdgcn_readlane(my_end, g) - (rows + TM - 1) / TM)) * TM;
      row0 = __builtin_amdgcn_readlane(my_first, g) + m0;
      m_valid = min(TM, rows - m0);
      n0 = nt * (GATED ? TN / 2 : TN);
      const int64_t o = g * p.b_gstride + n0 * p.ldb;
      op.a = {p.A + row0 * p.lda, nullptr, p.lda, m_valid, 0};
      op.b = {p.B + o, GATED ? p.B2 + o : nullptr, p.ldb, min(GATED ? TN / 2 : TN, p.N - n0), 0};
      op.K = p.K;
    }
    std::conditional_t<is_i8(MODE), ScalesI8<MODE, C>, int> sc;   // read beside the first stages
    if constexpr (is_i8(MODE)) sc.load(p, lane, wm, wn, g, row0, m_valid, n0);
    floatx4 acc[RB][4];
    const int steps = ((op.K * ES + kRowBytes - 1) / kRowBytes + KG - 1) / KG;
    if constexpr (NS == 3) {
      char *const sa[3] = {a0 + ga, a1 + ga, a2 + ga}, *const sb[3] = {b0 + gb, b1 + gb, b2 + gb};
      mainloop_deep<RB, NS, a_layout(PASS), b_layout(PASS), GATED, ES>(op, wave, kg * steps, steps, sa, sb, acc);
    } else {
      char *const sa[4] = {a0, a1, a2, a3}, *const sb[4] = {b0, b1, b2, b3};
      mainloop_deep<RB, NS, a_layout(PASS), b_layout(PASS), GATED, ES>(op, wave, 0, steps, sa, sb, acc);
    }
    if constexpr (KG > 1) {
      static_assert(DENSE && NS == 3 && RB * 4 * 16 * kThreads16 <= KG * kB, "the sums fit a stage of B");
      floatx4* sums = reinterpret_cast<floatx4*>(b2) + (threadIdx.x & (kThreads16 - 1));
      if (kg) {
#pragma unroll
        for (int i = 0; i < RB; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) sums[(i * 4 + j) * kThreads16] = acc[i][j];
      }
      __syncthreads();
      if (!kg) {
#pragma unroll
        for (int i = 0; i < RB; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[i][j] += sums[(i * 4 + j) * kThreads16];
      }
    }
    if (KG == 1 || !kg) {
      float* strip = reinterpret_cast<float*>((wave < 2 ? b0 : b1) + (wave & 1) * strip_bytes<MODE, C>());
      if constexpr (is_i8(MODE))
        epilogue_i8<MODE, C>(p, acc, sc, strip, row_scales<C>(b0, b1, wave), lane, wm, wn, g, row0, m_valid, n0);
      else
        epilogue16<MODE, C>(p, acc, strip, lane, wm, wn, g, slot, row0, m_valid, n0, false);
    }
    __syncthreads();   // strips are free before the next tile's loads
  }
}

// The same for fp32 (dense products): K steps of 32, tiles and fragments of the
// two-stage fp32 kernel.  Its matrix instructions keep a step of a full CU busy (96 %
// of their peak in a product of whole rounds), so it gains a little where a CU has one
// workgroup (777 tokens, 1384 -> 512: Y 23.0 -> 20.6 us, dW2 24.8 -> 21.3).
template <int MODE, int PASS, int RB, int NS>
__global__ __launch_bounds__(kThreads16, RB <= 2 ? 2 : 1) void ffn_gemm_f32_deep_kernel(const GemmParams p) {
  constexpr bool GATED = is_gated(MODE), VARK = is_dw(MODE);
  constexpr int kA = 32 * RB * kRowBytes, kB = kMidN * kRowBytes, NB = GATED ? (RB + 1) / 2 : RB;
  __shared__ __attribute__((aligned(16))) char a0[kA], b0[kB], a1[kA], b1[kB], a2[kA], b2[kB];
  __shared__ __attribute__((aligned(16))) char a3[NS > 3 ? kA : 16], b3[NS > 3 ? kB : 16];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
  const int n_items = dense_items<MODE>(p);
  for (int round = 0;; ++round) {
    const int L = round_item(round, n_items);
    if (L < 0) break;
    MidTile t;
    int mt, nt;
    const int si = dense_tile<MODE>(p, L, mt, nt);
    t.g = 0;
    t.h = RB;
    t.row0 = mt * 32 * RB;
    t.m_valid = min(32 * RB, (VARK ? p.M_out : p.dense.T) - t.row0);
    t.n0 = nt * (GATED ? kMidN / 2 : kMidN);
    t.slot = p.dense.splits > 1 ? si : -1;
    t.op = dense_ops<MODE, PASS, 4>(p, t.row0, t.m_valid, t.n0, kMidN, si);
    AccF32<NB> c1, c3;
    if constexpr (NS == 3) {
      char *const sa[3] = {a0, a1, a2}, *const sb[3] = {b0, b1, b2};
      mainloop_f32<RB, PASS, GATED, NB, NS>(t.op, sa, sb, c1, c3);
    } else {
      char *const sa[4] = {a0, a1, a2, a3}, *const sb[4] = {b0, b1, b2, b3};
      mainloop_f32<RB, PASS, GATED, NB, NS>(t.op, sa, sb, c1, c3);
    }
    epilogue_f32<MODE, RB, NB>(p, t, c1, c3, lane, wave);
  }
}

// RB and NS of the three tiles, workgroups per CU.
template <int RB> constexpr int kDeepStages = RB == 2 ? 3 : 4;
template <int RB> constexpr int kDeepPerCu = RB <= 2 ? 2 : 1;

template <int MODE, int PASS, int RB>
moe_status launch_deep(hipStream_t s, moe_dtype dt, const GroupParams& gp, int64_t most_items) {
  const int64_t full = kDeepPerCu<RB> * static_cast<int64_t>(persistent_grid());
  const int grid = static_cast<int>(std::min(full, (most_items + kXcds - 1) / kXcds * kXcds));
  MOE_TIMED(pass_name(PASS), s);
  if constexpr (is_dense(MODE) && PASS != P_BWD_DX_T) {
    if (dt == MOE_F32) {
      ffn_gemm_f32_deep_kernel<MODE, PASS, RB, kDeepStages<RB>><<<grid, kThreads16, 0, s>>>(gp.p);
      MOE_LAUNCH_CHECK();
      return MOE_OK;
    }
  }
  if constexpr (RB == 2 && is_dense(MODE) && !is_dw(MODE)) {
    if (most_items <= persistent_grid()) {
      ffn_gemm16_deep_kernel<MODE, PASS, RB, 3, 2><<<grid, 2 * kThreads16, 0, s>>>(gp);
      MOE_LAUNCH_CHECK();
      return MOE_OK;
    }
  }
  if constexpr (!is_dw(MODE) || RB == 4)
    ffn_gemm16_deep_kernel<MODE, PASS, RB, kDeepStages<RB>, 1><<<grid, kThreads16, 0, s>>>(gp);
  MOE_LAUNCH_CHECK();
  return MOE_OK;
}

}  // namespace
}  // namespace moe
