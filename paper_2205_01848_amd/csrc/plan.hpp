// Which kernel runs a product of the dense block or of the int8 experts, on which
// tiles.  Plain C++: the host compares estimated times, fitted on measurements.
#pragma once

#include <algorithm>
#include <cmath>

#include "tiles.hpp"

namespace moe {

inline int cdiv(int64_t a, int64_t b) { return static_cast<int>((a + b - 1) / b); }

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
// 14336, every kernel, height and 1 to 8 K ranges): residual 3 to 19 % a product.
// The fit is of the kernels before their epilogues read ahead and before 64-row
// deep tiles, where a CU has at most one, shared K between two groups of
// wavefronts (deep.hpp), so those are estimated up to a fifth too long.  With the
// kernels as they are the choice takes 1.7 % (bf16, 168 products) and 2.8 % (fp32,
// 90) more than the best measured one on average, 27 and 41 % at the worst (512
// tokens, dX of 4096 x 14336; 100 tokens, dX of 1024 x 2816); of the bf16 ones 79
// are on the mid kernel, 68 deep, 21 on 256x256 tiles.
// Examples, us (operands in the last-level cache): 1021 tokens, 5632 -> 2048,
// 64-row tiles two-stage / deep 45 / 31; 2048 tokens, 2816 -> 1024 24.4 / 17.2; 32
// tokens, 28672 -> 4096 (weights K-major), whole K / six ranges 221 / 76 with their
// join; 4096 tokens, 4096 -> 2 x 14336, 256x256 / mid 695 / 832.
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

// One dense product: M x N results over K.
struct DenseProduct {
  bool f32;
  bool gated;       // W1 and W3 share a tile
  bool active;      // an activation or its factors in the epilogue: K stays whole
  bool b_km, dw;    // B K-major; both operands K-major (weight gradients)
  int M, N, K;
  int64_t lda, ldb; // row pitches, bytes
};

// The kernel, tile height and number of K ranges of a dense product: the host
// knows every size, so it compares the estimated times of them all.  Splitting K
// gives a product of few tiles to more CUs and costs the write and the read of
// the partial sums (about 4700 bytes per ns) and a launch.  Row pitches that are no
// multiple of 128 bytes make a K step of the smaller tiles as long as its cache
// lines (step16, big_step16).  tile_mode: moe_set_gemm_tiles.
inline DensePlan plan_dense(const DenseProduct& p, int cus, int tile_mode) {
  const bool f32 = p.f32, gated = p.gated, dw = p.dw;
  const int M = p.M, N = p.N;
  const DenseClass cl = dw ? D_DW : p.b_km ? D_KM : gated && f32 ? D_GATED : D_KC;
  const int ks = f32 ? 32 : 64, steps = cdiv(p.K, ks);
  const StepCost lines = dw ? StepCost{0, 0, (p.lda % 128 ? 600 : 400) + (p.ldb % 128 ? 600 : 400), 0}
                              : step16(p.lda, p.ldb, p.b_km);
  DensePlan best{};
  int64_t t_best = -1;
  // an activation needs the whole sum
  const int most = p.active ? 1 : std::max(1, std::min(16, steps / 4));
  for (int want = 1; want <= most; ++want) {
    const int per = cdiv(steps, want), splits = cdiv(steps, per);   // K steps of a range
    if (splits != want) continue;
    const int64_t join = splits == 1 ? 0 : static_cast<int64_t>(M) * N * (8 * splits + (f32 ? 4 : 2)) / 4700 + 3000;
    auto take = [&](DenseKernel k, int h, int n_mt, int nt, int per_cu) {
      TileTime t = tile_time(f32, k, h, cl);
      if (!f32) {
        const int both = lines.lines_fixed + lines.lines_per_unit * h;
        const int least = k == K_BIG ? (dw ? 0 : big_step16(p.lda, p.ldb, p.b_km, false) - (p.b_km ? 270 : 90))
                                     : per_cu == 2 ? both : both / 2;
        t.step = std::max(t.step, least);
        // operands beyond the last-level cache (256 MB) cost the smaller
        // tiles, which read them more often (8192 tokens, dW2 of 4096 x 14336: 854 us
        // on 256x256 tiles, 931 on the others; 4096 tokens 461 / 456)
        if (k != K_BIG && (static_cast<int64_t>(M) + N) * p.K * 2 > (int64_t(256) << 20)) t.step += t.step / 8;
      }
      const int64_t tiles = static_cast<int64_t>(n_mt) * nt * splits, places = static_cast<int64_t>(per_cu) * cus;
      const int64_t full = tiles / places, rem = tiles % places;
      const int64_t part = rem == 0 ? 0 : per_cu == 2 && 2 * rem <= places ? t.half : 100;
      const int64_t time = (100 * full + part) * (static_cast<int64_t>(t.step) * per + t.fix) / 100 + join;
      if (t_best >= 0 && time >= t_best) return;
      t_best = time;
      best = {k, h, n_mt, nt, splits, per * ks};
    };
    const int units = cdiv(M, kMidUnit), nt = cdiv(N, gated ? kMidN / 2 : kMidN);
    if (!f32 && tile_mode != 2) take(K_BIG, 0, cdiv(M, BM), cdiv(N, gated ? BN / 2 : BN), 1);
    for (int h = 1; h <= kMidMaxH && (f32 || tile_mode != 1); ++h) {
      if (dw && (f32 ? h > 4 || h == 3 : h != kMidDwH)) continue;
      // the rows spread evenly over the tiles may need a lower one
      const int n = cdiv(units, h);
      take(K_MID, dw ? h : cdiv(units, n), n, nt, 2);
    }
    for (int h = dw && !f32 ? 4 : 1; h <= 4 && tile_mode == 0; h *= 2)
      take(K_DEEP, h, cdiv(units, h), nt, h <= 2 ? 2 : 1);
  }
  return best;
}

// The kernel of one product: the one for few rows, deep tiles of 32, 64 or 128
// rows, or, with a schedule, the tiles of gemm.hpp (128 columns and up to 192
// rows, or 256 x 256).
enum KernelI8 { I8_FEW, I8_DEEP32, I8_DEEP64, I8_DEEP128, I8_MID, I8_BIG };
inline bool scheduled(KernelI8 k) { return k >= I8_MID; }

// The host knows the rows at most and their mean over the experts, not the
// loads: it compares the estimated times for experts of the mean, half a tile
// more for raggedness.  A product is as long as its rounds of tiles (tile_time; a K
// step is 128 bytes, as in bf16) or as the read of its live experts' weights, at
// 5600 bytes per ns, a tenth more for every further tile of an expert.  Few rows:
// up to 16, bound by that read.  Over 47 calls (1 to 64 experts, 1 to 6000
// rows, K from 1000 to 14336) the choice takes 0.3 % more than the best kernel.
// Examples, us a call, few / deep 32 / deep 64 / deep 128 / tiles: FFN 4096,
// 14336 of 8 experts, 8 rows 176 / 182 / 192 / 197 / 231, 256 rows 685 / 324 / 282
// / 295 / 326, 1024 rows 2224 / 625 / 473 / 441 / 381; 64 experts 2048, 1408,
// 512 rows 132 / 90 / 91 / 101 / 103; one product 14336 -> 4096, 16 rows 18 / 28
// / 38 / 53 / 58.  The two tiles, us, 256 x 256 / 128 columns: 8192 rows on 8
// experts, 4096 -> 2 x 14336 897 / 1000, 14336 -> 4096 506 / 468.
inline KernelI8 plan_i8(int E, int64_t rows_most, int K, int N, bool gated, int cus, int tile_mode) {
  if (tile_mode != 0) return tile_mode == 1 ? I8_BIG : I8_MID;
  const int groups = static_cast<int>(std::min<int64_t>(E, rows_most));
  const double mean = std::max(1., static_cast<double>(rows_most) / E);
  const int steps = cdiv(K, 128);
  const double read = static_cast<double>(groups) * N * (gated ? 2 : 1) * K / 5600;
  auto tiles = [&](int unit) {   // of all experts, along M
    return groups > 1 ? groups * std::max(1., mean / unit + 0.5) : static_cast<double>(cdiv(rows_most, unit));
  };
  auto rounds = [&](double n, int per_cu, int half) {
    const int places = per_cu * cus;
    return n > places ? n / places + 0.25 : per_cu == 2 && 2 * n <= places ? half / 100. : 1.;
  };
  auto tile = [&](DenseKernel k, int h, int unit, int cols, int per_cu, int slower) {
    const TileTime t = tile_time(false, k, h, D_KC);
    const double n = tiles(unit) * cdiv(N, gated ? cols / 2 : cols);
    // the tiles of gemm.hpp are for many rows: whole rounds
    const double r = k != K_DEEP && n > per_cu * cus ? std::ceil(n / (per_cu * cus)) : rounds(n, per_cu, t.half);
    return r * (static_cast<double>(t.step) * slower / 100 * steps + t.fix);
  };
  // the int8 matrix instructions draw more power than the bf16 ones: a step of
  // the large tiles takes 7 to 10 % longer
  const double big = tile(K_BIG, 0, BM, BN, 1, 107);
  double mid = 0;
  for (int h = 1; h <= kMidMaxH; ++h) {
    const double t = tile(K_MID, h, kMidUnit * h, kMidN, 2, 110);
    if (h == 1 || t < mid) mid = t;
  }
  KernelI8 best = big <= mid ? I8_BIG : I8_MID;
  double t_best = std::max(std::min(big, mid), 1.15 * read + 3000) + 7000;   // and the schedule's launch
  auto take = [&](KernelI8 k, double t) {
    if (t < t_best) { t_best = t; best = k; }
  };
  for (int h = 1; h <= 4; h *= 2)
    take(h == 1 ? I8_DEEP32 : h == 2 ? I8_DEEP64 : I8_DEEP128,
         std::max(tile(K_DEEP, h, kMidUnit * h, kMidN, h <= 2 ? 2 : 1, 100),
                  read * (0.9 + 0.1 * tiles(kMidUnit * h) / groups) + 3000));
  if (rows_most <= 16) take(I8_FEW, read + 2500);
  return best;
}

}  // namespace moe
