// The experts on 8-bit integers (serving): the grouped product
//     y[r, n] = xs[r] ws[e, n] sum_k xq[r, k] wq[e, n, k]
// over the rows r of every expert e, and the expert FFN made of it: H = X W1^T
// (and H3 = X W3^T), A = act(H) (SwiGLU: silu(H1) H3) rounded to the layer
// dtype, A quantised row by row, Y = A W2^T.  The sums are exact (int32).
//
// The products run on the tiles, schedule and K loop of the bf16 ones (gemm.hpp)
// with v_mfma_i32_16x16x64_i8: a K step is 128 bytes of a row, 128 values
// instead of 64, at the same number of matrix instructions, so the same loop
// does twice the products per second, and the same bytes.

#include "dense.hpp"
#include "few_rows.hpp"
#include "quant.hpp"

namespace moe {
namespace {

// Buffers of the int8 FFN behind the schedule: A in the layer dtype, then
// its quantised rows and their scales.
struct PlanI8 {
  FfnPlan pl;
  size_t o_a, o_aq, o_as, total;
};

bool layout_i8(moe_dtype dt, moe_act act, int E, int d, int f, int64_t rows_alloc, PlanI8& q) {
  if (!dtype_ok(dt) || d > kMaxQuant || f > kMaxQuant) return false;
  if (!make_plan(MOE_BF16, act, E, d, f, rows_alloc, q.pl)) return false;
  q.pl.es = 1;
  size_t o = q.pl.o_end_sched;
  q.o_a = o;  o = align_up(o + static_cast<size_t>(rows_alloc) * f * esize(dt), 256);
  q.o_aq = o; o = align_up(o + static_cast<size_t>(rows_alloc) * quantized_width(f), 256);
  q.o_as = o; o = align_up(o + static_cast<size_t>(rows_alloc) * 4, 256);
  q.total = o;
  return true;
}

KernelI8 kernel_i8(const FfnPlan& pl, int K, int N, bool gated) {
  return plan_i8(pl.E, pl.rows_most, K, N, gated, persistent_grid(), g_tile_mode);
}

// One product by kernel k.
template <int MODE, int PASS>
moe_status launch_i8(hipStream_t s, KernelI8 k, const FfnPlan& pl, char* ws, const int32_t* rows,
                     const GemmParams& p) {
  if (scheduled(k)) return launch_gemm<MODE, PASS>(s, MOE_BF16, pl, ws, p, k == I8_MID);
  GroupParams gp{p, pl.E, rows, pl.rows_alloc};
  const int groups = static_cast<int>(std::min<int64_t>(pl.E, pl.rows_most));
  if (k == I8_FEW) return launch_few<MODE, 1>(s, pass_name(PASS), gp, pl.rows_most, groups);
  gp.p.ntiles = cdiv(p.N, is_gated(MODE) ? kMidN / 2 : kMidN);
  const int unit = k == I8_DEEP32 ? 32 : k == I8_DEEP64 ? 64 : 128;
  const int64_t most = (pl.rows_most / unit + groups) * gp.p.ntiles;
  if (k == I8_DEEP32) return launch_deep<MODE, PASS, 1>(s, MOE_BF16, gp, most);
  if (k == I8_DEEP64) return launch_deep<MODE, PASS, 2>(s, MOE_BF16, gp, most);
  return launch_deep<MODE, PASS, 4>(s, MOE_BF16, gp, most);
}

bool scales_ok(const float* x_scale, const int32_t* src, int T, int k) {
  return src ? T >= 0 && k > 0 && (x_scale || T == 0) : x_scale != nullptr;
}

// The product of one expert region's rows xq (K bytes each) with wq, wq3.
GemmParams params_i8(const FfnPlan& pl, const int32_t* offsets, char* ws, int K, int N,
                     const int8_t* xq, const RowScales& xs, const int8_t* wq, const float* wscale,
                     moe_dtype dt, void* out) {
  GemmParams p = base_params(pl, offsets, ws);
  p.A = reinterpret_cast<const char*>(xq);
  p.lda = K;
  p.B = reinterpret_cast<const char*>(wq);
  p.ldb = K;
  p.b_gstride = static_cast<int64_t>(N) * K;
  p.K = K;
  p.N = N;
  p.a_scale = xs;
  p.b_scale = wscale;
  p.s_gstride = N;
  p.C = static_cast<char*>(out);
  p.ldc = N * static_cast<int64_t>(esize(dt));
  p.out_f32 = dt == MOE_F32;
  return p;
}

}  // namespace
}  // namespace moe

using namespace moe;

extern "C" size_t moe_expert_matmul_i8_workspace_bytes(int E, int N, int64_t rows_alloc) {
  FfnPlan pl;
  return make_plan(MOE_BF16, MOE_RELU, E, 8, N, rows_alloc, pl) ? pl.o_end_sched : 0;
}

extern "C" moe_status moe_expert_matmul_i8(void* stream, moe_dtype dt, int E, int K, int N,
                                           const int32_t* offsets, const int32_t* rows,
                                           int64_t rows_alloc, const int8_t* xq,
                                           const float* x_scale, const int32_t* src, int T, int k,
                                           const int8_t* wq, const float* w_scale, void* y,
                                           void* workspace, size_t workspace_bytes) {
  FfnPlan pl;
  if (!dtype_ok(dt) || K < 16 || K % 16 != 0 || K > kMaxQuant) return MOE_EINVAL;
  if (!make_plan(MOE_BF16, MOE_RELU, E, 8, N, rows_alloc, pl)) return MOE_EINVAL;
  if (!offsets || !rows || !wq || !w_scale || !aligned16(wq)) return MOE_EINVAL;
  if (rows_alloc == 0) return MOE_OK;
  if (!xq || !scales_ok(x_scale, src, T, k) || !y || !aligned16(xq) || !aligned16(y)) return MOE_EINVAL;
  if (!workspace || workspace_bytes < pl.o_end_sched || !aligned16(workspace)) return MOE_EWORKSPACE;
  if (src && T == 0) return MOE_OK;   // no tokens, so no rows
  pl.es = 1;
  pl.d = K;
  if (src) pl.rows_most = std::min<int64_t>(rows_alloc, static_cast<int64_t>(T) * k);
  hipStream_t s = static_cast<hipStream_t>(stream);
  char* ws = static_cast<char*>(workspace);
  const StepCost c = step16(K, K, false);
  const KernelI8 kernel = kernel_i8(pl, K, N, false);
  if (scheduled(kernel))
    MOE_TRY(launch_schedule(s, sched_args(pl, cdiv(N, kMidN), cdiv(N, kMidN), K, c, c, ws), offsets,
                            rows));
  return launch_i8<M_I8_STORE, P_FWD_Y>(
      s, kernel, pl, ws, rows,
      params_i8(pl, offsets, ws, K, N, xq, {x_scale, src, T, k}, wq, w_scale, dt, y));
}

extern "C" size_t moe_ffn_fwd_i8_workspace_bytes(moe_dtype dt, moe_act act, int E, int d, int f,
                                                 int64_t rows_alloc) {
  PlanI8 q;
  return layout_i8(dt, act, E, d, f, rows_alloc, q) ? q.total : 0;
}

extern "C" moe_status moe_expert_ffn_fwd_i8(void* stream, moe_dtype dt, moe_act act, int E, int d,
                                            int f, const int32_t* offsets, const int32_t* rows,
                                            int64_t rows_alloc, const int8_t* xq,
                                            const float* x_scale, const int32_t* src, int T, int k,
                                            const int8_t* w1q, const float* w1_scale,
                                            const int8_t* w3q, const float* w3_scale,
                                            const int8_t* w2q, const float* w2_scale, void* y_disp,
                                            void* workspace, size_t workspace_bytes) {
  PlanI8 q;
  if (!layout_i8(dt, act, E, d, f, rows_alloc, q)) return MOE_EINVAL;
  const bool sw = act == MOE_SWIGLU;
  if (!offsets || !rows || !w1q || !w1_scale || !w2q || !w2_scale) return MOE_EINVAL;
  if (sw && (!w3q || !w3_scale || !aligned16(w3q))) return MOE_EINVAL;
  if (!aligned16(w1q) || !aligned16(w2q)) return MOE_EINVAL;
  if (rows_alloc == 0) return MOE_OK;
  if (!xq || !scales_ok(x_scale, src, T, k) || !y_disp || !aligned16(xq) || !aligned16(y_disp)) return MOE_EINVAL;
  if (!workspace || workspace_bytes < q.total || !aligned16(workspace)) return MOE_EWORKSPACE;
  if (src && T == 0) return MOE_OK;   // no tokens, so no rows
  hipStream_t s = static_cast<hipStream_t>(stream);
  char* ws = static_cast<char*>(workspace);
  FfnPlan& pl = q.pl;
  if (src) pl.rows_most = std::min<int64_t>(rows_alloc, static_cast<int64_t>(T) * k);
  const int kd = quantized_width(d), kf = quantized_width(f);
  const KernelI8 up = kernel_i8(pl, kd, f, sw), down = kernel_i8(pl, kf, d, false);
  if (scheduled(up) || scheduled(down))
    MOE_TRY(launch_schedule(s, sched_args(pl, cdiv(f, sw ? kMidN / 2 : kMidN), cdiv(d, kMidN), kf,
                                          step16(kd, kd, false), step16(kf, kf, false), ws),
                            offsets, rows));
  char* a = ws + q.o_a;
  int8_t* aq = reinterpret_cast<int8_t*>(ws + q.o_aq);
  float* as = reinterpret_cast<float*>(ws + q.o_as);
  GemmParams p = params_i8(pl, offsets, ws, kd, f, xq, {x_scale, src, T, k}, w1q, w1_scale, dt,
                           a);
  p.act = act == MOE_RELU ? ACT_RELU : ACT_GELU;
  if (sw) {
    p.B2 = reinterpret_cast<const char*>(w3q);
    p.b2_scale = w3_scale;
    MOE_TRY(launch_i8<M_I8_FWD1_SWIGLU, P_FWD_H>(s, up, pl, ws, rows, p));
  } else {
    MOE_TRY(launch_i8<M_I8_FWD1, P_FWD_H>(s, up, pl, ws, rows, p));
  }
  if (down == I8_FEW && few_fits_quant(pl.rows_most, kf)) {
    // A straight into the second product, quantised there
    GroupParams gp{params_i8(pl, offsets, ws, kf, d, nullptr, {}, w2q, w2_scale, dt, y_disp), E, rows,
                   rows_alloc, f, static_cast<int>(pl.rows_most)};
    gp.p.A = a;
    gp.p.lda = f * static_cast<int64_t>(esize(dt));
    return launch_few<M_I8_STORE, 1>(s, pass_name(P_FWD_Y), gp, pl.rows_most,
                                     static_cast<int>(std::min<int64_t>(E, pl.rows_most)), true);
  }
  MOE_TRY(quantize_launch(s, dt, rows_alloc, f, a, f, aq, as, E, offsets, rows));
  return launch_i8<M_I8_STORE, P_FWD_Y>(
      s, down, pl, ws, rows, params_i8(pl, offsets, ws, kf, d, aq, {as, nullptr, 0, 0}, w2q, w2_scale, dt,
                                     y_disp));
}
