// Dense products: one group of rows, sizes known on the host.  Plan (kernel,
// tile height, K ranges) and launch.
#pragma once

#include "deep.hpp"

namespace moe {
namespace {

enum DenseKernel { K_BIG, K_MID, K_DEEP };
struct DensePlan {
  DenseKernel kernel;
  int h;          // units of rows per tile (mid, deep)
  int n_mt, nt;   // tiles along M and N
  int splits, klen;
};

// Time of a round of tiles on all places of the persistent grid: `step` ns per K
// step (64 bf16 or 32 fp32 values) and `fix` ns of launch, prologue and
// epilogue; a last round that leaves one of the two places of every CU empty takes
// `half` percent of that.  Fitted on 10,388 bf16 and 6165 fp32 measurements of
// the block's six products (32 to 4096 tokens, d from 512 to 4096, f from 1384 to
// 14336, every kernel, height and 1 to 8 K ranges): residual 3 to 19 % a product;
// the plan's choice takes 1.6 % (bf16) and 2.1 % (fp32) more than the best
// measured one on average (of 168 bf16 products, 79 on the mid kernel, 69 deep,
// 20 on 256x256 tiles).
// Examples, us: 1021 tokens, 5632 -> 2048, 64-row tiles two-stage / deep 58 /
// 34; 2048 tokens, 2816 -> 1024 26 / 20; 32 tokens, 28672 -> 4096, whole K / six
// ranges 173 / 50; 4096 tokens, 4096 -> 2 x 14336, 256x256 / mid 677 / 832.
struct TileTime {
  int step, fix, half;
};
enum DenseClass { D_KC, D_KM, D_DW, D_GATED };   // B K-contiguous, B K-major, both K-major, gated fp32
inline TileTime tile_time(bool f32, DenseKernel k, int h, DenseClass c) {
  if (f32) {   // the gated kernel gives a wavefront every other block of rows: odd heights idle half
    static const TileTime kc[] = {{1000, 6100, 68}, {1795, 10300, 60}, {2610, 11300, 60},
                                  {3425, 18000, 58}, {4230, 20000, 58}, {5230, 20000, 58}};
    static const TileTime km[] = {{1365, 7700, 71}, {2060, 14100, 62}, {2830, 16500, 62},
                                  {3750, 20000, 60}, {4605, 20000, 60}, {5575, 20000, 60}};
    static const TileTime dw[] = {{1070, 4100, 90}, {1810, 7000, 75}, {}, {3390, 12500, 73}};
    static const TileTime gated[] = {{1825, 8500, 59}, {1875, 9400, 61}, {3570, 16300, 57},
                                     {3635, 16300, 58}, {5075, 20000, 59}, {5665, 20000, 59}};
    static const TileTime deep[4][4] = {{{925, 5900, 63}, {1775, 8700, 57}, {}, {1910, 9100, 100}},
                                        {{1225, 8800, 62}, {2060, 13000, 58}, {}, {2050, 13400, 100}},
                                        {{1025, 4300, 80}, {1800, 6900, 71}, {}, {1940, 9300, 100}},
                                        {{1770, 7600, 58}, {1775, 9500, 57}, {}, {1915, 9100, 100}}};
    if (k == K_DEEP) return deep[c][h - 1];
    return (c == D_KC ? kc : c == D_KM ? km : c == D_DW ? dw : gated)[h - 1];
  }
  if (c == D_DW) return k == K_BIG ? TileTime{1390, 21000, 100} : k == K_MID ? TileTime{800, 10000, 55} : TileTime{600, 7500, 100};
  if (k == K_BIG) return c == D_KC ? TileTime{1310, 12500, 100} : TileTime{1430, 17500, 100};
  static const TileTime mid_kc[] = {{630, 4800, 80}, {720, 6200, 73}, {750, 7300, 71},
                                    {955, 9500, 63}, {1000, 10400, 60}, {1045, 12600, 59}};
  static const TileTime mid_km[] = {{590, 5200, 84}, {680, 6700, 75}, {760, 8300, 69},
                                    {965, 10200, 60}, {1035, 11000, 57}, {1135, 13300, 56}};
  static const TileTime deep_kc[] = {{550, 4900, 55}, {720, 5700, 56}, {}, {525, 6200, 100}};
  static const TileTime deep_km[] = {{540, 6100, 69}, {690, 6400, 58}, {}, {560, 7500, 100}};
  if (k == K_MID) return (c == D_KC ? mid_kc : mid_km)[h - 1];
  return (c == D_KC ? deep_kc : deep_km)[h - 1];
}

// The kernel, tile height and number of K ranges of a dense product: the host
// knows every size, so it compares the estimated times of them all.  Splitting K
// gives a product of few tiles to more CUs and costs the write and the read of
// the partial sums (about 4700 bytes per ns) and a launch.  Row pitches that are no
// multiple of 128 bytes make a K step of the smaller tiles as long as its cache
// lines (step16, big_step16).
template <int MODE, int PASS>
DensePlan dense_plan(moe_dtype dt, int M, int N, int K, int64_t lda, int64_t ldb) {
  constexpr bool VARK = is_dw(MODE), GATED = is_gated(MODE), BKM = b_layout(PASS) == L_KM;
  constexpr bool ACTIVE = MODE == M_GATED_FWD || MODE == M_GATED_DA;
  const bool f32 = dt == MOE_F32;
  const DenseClass cl = VARK ? D_DW : BKM ? D_KM : GATED && f32 ? D_GATED : D_KC;
  const int ks = f32 ? kF32Step : 64, steps = cdiv(K, ks), cus = persistent_grid();
  const StepCost lines = VARK ? StepCost{0, 0, (lda % 128 ? 600 : 400) + (ldb % 128 ? 600 : 400), 0}
                              : step16(lda, ldb, BKM);
  DensePlan best{};
  int64_t t_best = -1;
  // an activation needs the whole sum
  const int most = ACTIVE ? 1 : std::max(1, std::min(16, steps / 4));
  for (int want = 1; want <= most; ++want) {
    const int per = cdiv(steps, want), splits = cdiv(steps, per);   // K steps of a range
    if (splits != want) continue;
    const int64_t join = splits == 1 ? 0 : static_cast<int64_t>(M) * N * (8 * splits + (f32 ? 4 : 2)) / 4700 + 3000;
    auto take = [&](DenseKernel k, int h, int n_mt, int nt, int per_cu) {
      TileTime t = tile_time(f32, k, h, cl);
      if (!f32) {
        const int both = lines.lines_fixed + lines.lines_per_unit * h;
        const int least = k == K_BIG ? (VARK ? 0 : big_step16(lda, ldb, BKM, false) - (BKM ? 270 : 90))
                                     : per_cu == 2 ? both : both / 2;
        t.step = std::max(t.step, least);
        // operands beyond the last-level cache (256 MB) cost the smaller
        // tiles, which read them more often (8192 tokens, dW2 of 4096 x 14336: 854 us
        // on 256x256 tiles, 931 on the others; 4096 tokens 461 / 456)
        if (k != K_BIG && (static_cast<int64_t>(M) + N) * K * 2 > (int64_t(256) << 20)) t.step += t.step / 8;
      }
      const int64_t tiles = static_cast<int64_t>(n_mt) * nt * splits, places = static_cast<int64_t>(per_cu) * cus;
      const int64_t full = tiles / places, rem = tiles % places;
      const int64_t part = rem == 0 ? 0 : per_cu == 2 && 2 * rem <= places ? t.half : 100;
      const int64_t time = (100 * full + part) * (static_cast<int64_t>(t.step) * per + t.fix) / 100 + join;
      if (t_best >= 0 && time >= t_best) return;
      t_best = time;
      best = {k, h, n_mt, nt, splits, per * ks};
    };
    const int units = cdiv(M, kMidUnit), nt = cdiv(N, GATED ? kMidN / 2 : kMidN);
    if (!f32 && g_tile_mode != 2) take(K_BIG, 0, cdiv(M, BM), cdiv(N, GATED ? BN / 2 : BN), 1);
    for (int h = 1; h <= kMidMaxH && (f32 || g_tile_mode != 1); ++h) {
      if (VARK && (f32 ? h > 4 || h == 3 : h != kMidDwH)) continue;
      // the rows spread evenly over the tiles may need a lower one
      const int n = cdiv(units, h);
      take(K_MID, VARK ? h : cdiv(units, n), n, nt, 2);
    }
    for (int h = VARK && !f32 ? 4 : 1; h <= 4 && g_tile_mode == 0; h *= 2)
      take(K_DEEP, h, cdiv(units, h), nt, h <= 2 ? 2 : 1);
  }
  return best;
}

// Sums the `splits` slots of an [M, N] product in order, adds the addend and
// writes rows [0, split_row) to c1 and the others to c2, ldc elements apart.
struct JoinArgs {
  const float* partial;
  int64_t slot_elems;
  int splits, M, N;
  const char* add; int64_t ldadd;   // bytes
  char *c1, *c2; int64_t ldc;       // bytes
  int split_row;
};
template <typename T>
__global__ __launch_bounds__(256) void dense_join_kernel(const JoinArgs a) {
  const int per_row = a.N / 4;
  const int64_t total = static_cast<int64_t>(a.M) * per_row;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < total;
       i += static_cast<int64_t>(gridDim.x) * 256) {
    const int row = static_cast<int>(i / per_row), col = static_cast<int>(i - static_cast<int64_t>(row) * per_row) * 4;
    const float* p = a.partial + i * 4;
    float4 v = *reinterpret_cast<const float4*>(p);
    for (int s = 1; s < a.splits; ++s) {
      const float4 u = *reinterpret_cast<const float4*>(p + s * a.slot_elems);
      v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w;
    }
    if (a.add) {
      const T* b = reinterpret_cast<const T*>(a.add + row * a.ldadd) + col;
      if constexpr (sizeof(T) == 4) {
        const float4 u = *reinterpret_cast<const float4*>(b);
        v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w;
      } else {
        const uint2 u = *reinterpret_cast<const uint2*>(b);
        v.x += __uint_as_float(u.x << 16); v.y += __uint_as_float(u.x & 0xFFFF0000u);
        v.z += __uint_as_float(u.y << 16); v.w += __uint_as_float(u.y & 0xFFFF0000u);
      }
    }
    T* c = reinterpret_cast<T*>(row < a.split_row ? a.c1 + row * a.ldc : a.c2 + (row - a.split_row) * a.ldc) + col;
    if constexpr (sizeof(T) == 4) *reinterpret_cast<float4*>(c) = v;
    else *reinterpret_cast<uint2*>(c) = make_uint2(pack2bf(v.x, v.y), pack2bf(v.z, v.w));
  }
}

// Bytes of partial sums of a planned product.
inline size_t dense_partial_bytes(const DensePlan& d, int M, int N) {
  return d.splits > 1 ? align_up(static_cast<size_t>(d.splits) * M * N * 4, 256) : 0;
}

// Launches one dense product of M x N results by plan d, its partial sums in p.partial.
template <int MODE, int PASS>
moe_status launch_dense(hipStream_t s, moe_dtype dt, const DensePlan& d, int T, int M, GemmParams p) {
  constexpr bool VARK = is_dw(MODE);
  p.ntiles = d.nt;
  p.dense = {T, d.n_mt, d.splits, d.klen};
  p.mtiles_out = d.n_mt;
  p.dw_h = d.h;
  p.slot_elems = static_cast<int64_t>(M) * p.N;
  const int64_t items = static_cast<int64_t>(d.splits) * d.n_mt * d.nt;
  const int64_t full = (d.kernel == K_MID ? 2 : 1) * static_cast<int64_t>(persistent_grid());
  const int grid = static_cast<int>(std::min(full, (items + kXcds - 1) / kXcds * kXcds));
  if (d.kernel == K_DEEP) {
    const GroupParams gp{p, 0, nullptr, 0};
    // (bf16 weight gradients: 128 rows only, see mainloop_deep)
    if (d.h == 1) MOE_TRY(launch_deep<MODE, PASS, 1>(s, dt, gp, items));
    else if (d.h == 2) MOE_TRY(launch_deep<MODE, PASS, 2>(s, dt, gp, items));
    else MOE_TRY(launch_deep<MODE, PASS, 4>(s, dt, gp, items));
  } else {
    MOE_TIMED(pass_name(PASS), s);
    if (dt == MOE_F32) {
      if constexpr (PASS != P_BWD_DX_T) ffn_gemm_f32_kernel<MODE, PASS><<<grid, kThreads16, 0, s>>>(p);
    } else if (d.kernel == K_MID) {
      ffn_gemm16_mid_kernel<MODE, PASS><<<grid, kThreads16, 0, s>>>(p);
    } else {
      ffn_gemm16_kernel<MODE, PASS><<<grid, kThreads16, 0, s>>>(p);
    }
    MOE_LAUNCH_CHECK();
  }
  if (d.splits == 1) return MOE_OK;
  const bool f32 = VARK ? p.out_f32 : dt == MOE_F32;
  JoinArgs j{p.partial, p.slot_elems, d.splits, M, p.N, p.add, p.ldadd, p.C, p.C, p.ldc, M};
  if (VARK) {
    j.c1 = reinterpret_cast<char*>(p.dwA);
    j.c2 = reinterpret_cast<char*>(p.dwB);
    j.ldc = static_cast<int64_t>(p.N) * (f32 ? 4 : 2);
    j.split_row = p.split_row;
  }
  const int jgrid = static_cast<int>(std::min<int64_t>(8 * num_cus(), (p.slot_elems / 4 + 255) / 256));
  MOE_TIMED("split_reduce", s);
  if (f32) dense_join_kernel<float><<<jgrid, 256, 0, s>>>(j);
  else dense_join_kernel<uint16_t><<<jgrid, 256, 0, s>>>(j);
  MOE_LAUNCH_CHECK();
  return MOE_OK;
}

}  // namespace
}  // namespace moe
