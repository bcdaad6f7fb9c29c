// Entry points of the expert FFN of the MoE layer (the expert modules E_e of
// Algorithm 1) on dynamically sized per-expert tensors (Section 4.1), forward
// and backward: which products run, in which order, on which buffers.  The
// products themselves are in gemm.hpp.

#include "gemm.hpp"

namespace moe {

int g_tile_mode = 0;
int g_wt_mode = 0;

}  // namespace moe

using namespace moe;

extern "C" moe_status moe_set_gemm_tiles(int mode) {
  if (mode < 0 || mode > 2) return MOE_EINVAL;
  g_tile_mode = mode;
  return MOE_OK;
}

extern "C" size_t moe_ffn_fwd_workspace_bytes(moe_dtype dt, moe_act act, int E, int d, int f,
                                              int64_t rows_alloc) {
  FfnPlan pl;
  return make_plan(dt, act, E, d, f, rows_alloc, pl) ? pl.total_fwd : 0;
}

extern "C" size_t moe_ffn_bwd_workspace_bytes(moe_dtype dt, moe_act act, int E, int d, int f,
                                              int64_t rows_alloc) {
  FfnPlan pl;
  if (!make_plan(dt, act, E, d, f, rows_alloc, pl)) return 0;
  return use_wt13(pl, dt) ? pl.total_bwd_wt : pl.total_bwd;
}

extern "C" moe_status moe_set_dx_weight_copy(int mode) {
  if (mode < 0 || mode > 2) return MOE_EINVAL;
  g_wt_mode = mode;
  return MOE_OK;
}

namespace moe {

moe_status ffn_fwd_check(const FfnFwd& a, size_t workspace_bytes) {
  FfnPlan pl;
  if (!make_plan(a.dt, a.act, a.E, a.d, a.f, a.rows_alloc, pl)) return MOE_EINVAL;
  if (!a.offsets || !a.rows || !a.w1 || !a.w2) return MOE_EINVAL;
  if (a.act == MOE_SWIGLU && !a.w3) return MOE_EINVAL;
  if (a.rows_alloc > 0 && (!a.x_disp || !a.y_disp)) return MOE_EINVAL;
  if (!aligned16(a.w1) || !aligned16(a.w2) || (a.w3 && !aligned16(a.w3)) ||
      (a.x_disp && !aligned16(a.x_disp)) || (a.y_disp && !aligned16(a.y_disp)) ||
      (a.h_save && !aligned16(a.h_save)))
    return MOE_EINVAL;
  if (a.rows_alloc == 0) return MOE_OK;
  if (!a.workspace || workspace_bytes < pl.total_fwd || !aligned16(a.workspace)) return MOE_EWORKSPACE;
  return MOE_OK;
}

SchedArgs ffn_fwd_sched(const FfnFwd& a) {
  FfnPlan pl;
  make_plan(a.dt, a.act, a.E, a.d, a.f, a.rows_alloc, pl);
  return sched_args(pl, cdiv(a.f, a.act == MOE_SWIGLU ? kMidN / 2 : kMidN), cdiv(a.d, kMidN), a.f,
                    step16(a.d * 2ll, a.d * 2ll, false), step16(a.f * 2ll, a.f * 2ll, false),
                    static_cast<char*>(a.workspace));
}

moe_status ffn_fwd_launch(hipStream_t s, const FfnFwd& a, bool scheduled) {
  if (a.rows_alloc == 0) return MOE_OK;
  FfnPlan pl;
  make_plan(a.dt, a.act, a.E, a.d, a.f, a.rows_alloc, pl);
  pl.rows_most = a.rows_most;
  if (!scheduled) MOE_TRY(launch_schedule(s, ffn_fwd_sched(a), a.offsets, a.rows));
  char* ws = static_cast<char*>(a.workspace);
  const moe_dtype dt = a.dt;
  const moe_act act = a.act;
  const int d = a.d, f = a.f;
  const int32_t* offsets = a.offsets;
  const int64_t rows_alloc = a.rows_alloc;
  const void *x_disp = a.x_disp, *w1 = a.w1, *w3 = a.w3, *w2 = a.w2;
  void *h_save = a.h_save, *y_disp = a.y_disp;
  const int64_t es = static_cast<int64_t>(pl.es);
  const int64_t plane = rows_alloc * f * es;   // one [rows_alloc, f] plane of h_save
  const bool sw = act == MOE_SWIGLU;
  // A = act(H): the last plane of h_save when the caller keeps activations.
  // ReLU keeps A alone (relu'(H) = [A > 0]), so H is never written there.
  const int h_planes = h_save_planes(act) - 1;
  char* abuf = h_save ? static_cast<char*>(h_save) + h_planes * plane : ws + pl.o_abuf;

  GemmParams p = base_params(pl, offsets, ws);
  p.A = static_cast<const char*>(x_disp);
  p.lda = d * es;
  p.B = static_cast<const char*>(w1);
  p.B2 = static_cast<const char*>(w3);
  p.ldb = d * es;
  p.b_gstride = static_cast<int64_t>(f) * d * es;
  p.K = d;
  p.N = f;
  p.act = act == MOE_RELU ? ACT_RELU : (act == MOE_GELU_TANH ? ACT_GELU : ACT_SWIGLU);
  p.C = abuf;
  p.ldc = f * es;
  p.H1 = h_planes > 0 ? static_cast<char*>(h_save) : nullptr;
  p.H3 = h_save && sw ? static_cast<char*>(h_save) + plane : nullptr;
  p.ldh = f * es;
  if (sw) MOE_TRY(launch_gemm<M_FWD1_SWIGLU, P_FWD_H>(s, dt, pl, ws, p));
  else MOE_TRY(launch_gemm<M_FWD1, P_FWD_H>(s, dt, pl, ws, p));

  GemmParams q = base_params(pl, offsets, ws);
  q.A = abuf;
  q.lda = f * es;
  q.B = static_cast<const char*>(w2);
  q.ldb = f * es;
  q.b_gstride = static_cast<int64_t>(d) * f * es;
  q.K = f;
  q.N = d;
  q.C = static_cast<char*>(y_disp);
  q.ldc = d * es;
  MOE_TRY(launch_gemm<M_STORE, P_FWD_Y>(s, dt, pl, ws, q));
  return MOE_OK;
}

}  // namespace moe

extern "C" moe_status moe_expert_ffn_fwd(void* stream, moe_dtype dt, moe_act act, int E, int d,
                                         int f, const int32_t* offsets, const int32_t* rows,
                                         int64_t rows_alloc, const void* x_disp, const void* w1,
                                         const void* w3, const void* w2, void* h_save,
                                         void* y_disp, void* workspace, size_t workspace_bytes) {
  const FfnFwd a = {dt, act, E, d, f, offsets, rows, rows_alloc, x_disp, w1, w3, w2, h_save,
                    y_disp, workspace, rows_alloc};
  MOE_TRY(ffn_fwd_check(a, workspace_bytes));
  return ffn_fwd_launch(static_cast<hipStream_t>(stream), a, false);
}

extern "C" moe_status moe_expert_ffn_bwd(void* stream, moe_dtype dt, moe_act act, int E, int d,
                                         int f, const int32_t* offsets, const int32_t* rows,
                                         int64_t rows_alloc, const void* x_disp,
                                         const void* h_save, const void* w1, const void* w3,
                                         const void* w2, const void* dy_disp, void* dx_disp,
                                         float* dw1, float* dw3, float* dw2, void* workspace,
                                         size_t workspace_bytes) {
  FfnPlan pl;
  if (!make_plan(dt, act, E, d, f, rows_alloc, pl)) return MOE_EINVAL;
  if (!offsets || !rows || !w1 || !w2 || !dw1 || !dw2) return MOE_EINVAL;
  if (act == MOE_SWIGLU && (!w3 || !dw3)) return MOE_EINVAL;
  if (rows_alloc > 0 && (!x_disp || !h_save || !dy_disp || !dx_disp)) return MOE_EINVAL;
  if (!aligned16(w1) || !aligned16(w2) || (w3 && !aligned16(w3)) || !aligned16(dw1) ||
      !aligned16(dw2) || (dw3 && !aligned16(dw3)) || (x_disp && !aligned16(x_disp)) ||
      (h_save && !aligned16(h_save)) || (dy_disp && !aligned16(dy_disp)) ||
      (dx_disp && !aligned16(dx_disp)))
    return MOE_EINVAL;
  if (!workspace || workspace_bytes < pl.total_bwd || !aligned16(workspace)) return MOE_EWORKSPACE;
  hipStream_t s = static_cast<hipStream_t>(stream);
  char* ws = static_cast<char*>(workspace);
  // dX reads [W1; W3] from a transposed copy (K-contiguous) when the rule
  // or the caller's setting asks for it and the workspace has room for it
  const bool wt = use_wt13(pl, dt) && workspace_bytes >= pl.total_bwd_wt;
  MOE_TRY(launch_schedule(s, sched_args(pl, cdiv(f, kMidN), cdiv(d, kMidN), pl.F,
                                        step16(d * 2ll, f * 2ll, true),
                                        step16(pl.F * 2ll, (wt ? pl.F : d) * 2ll, !wt), ws),
                          offsets, rows));
  const int64_t es = static_cast<int64_t>(pl.es);
  const bool sw = act == MOE_SWIGLU;
  const int F = pl.F;
  char* dh = ws + pl.o_dh;      // [rows_alloc, F]: dH, or [dH1 | dH3]
  const int actc = act == MOE_RELU ? ACT_RELU : (act == MOE_GELU_TANH ? ACT_GELU : ACT_SWIGLU);
  const int64_t plane = rows_alloc * f * es;
  // A = act(H), saved by the forward after H (or H1, H3); ReLU saves A alone
  // and its derivative reads A: relu'(H) = [H > 0] = [A > 0]
  const char* abuf = static_cast<const char*>(h_save) + (h_save_planes(act) - 1) * plane;
  const char* h1 = act == MOE_RELU ? abuf : static_cast<const char*>(h_save);
  const char* h3 = sw ? h1 + plane : nullptr;

  char* wt13 = ws + pl.o_wt13;
  if (wt) MOE_TRY(launch_transpose_w(s, E, w1, sw ? w3 : nullptr, f, sw ? f : 0, d, wt13));

  // dx_disp = [dH1 | dH3] [W1; W3]: from the transposed copy, or W1, W3 read
  // K-major (W3 from k = f on)
  auto launch_dx = [&]() -> moe_status {
    if (wt) {
      GemmParams q = base_params(pl, offsets, ws);
      q.A = dh;
      q.lda = F * es;
      q.B = wt13;
      q.ldb = F * es;
      q.b_gstride = static_cast<int64_t>(d) * F * es;
      q.K = F;
      q.N = d;
      q.C = static_cast<char*>(dx_disp);
      q.ldc = d * es;
      return launch_gemm<M_STORE, P_BWD_DX_T>(s, dt, pl, ws, q);
    }
    GemmParams q = base_params(pl, offsets, ws);
    q.A = dh;
    q.lda = F * es;
    q.B = static_cast<const char*>(w1);
    q.B2 = sw ? static_cast<const char*>(w3) : nullptr;
    q.kmsplit = sw ? f : 0x7FFFFFFF;
    q.ldb = d * es;
    q.b_gstride = static_cast<int64_t>(f) * d * es;
    q.K = F;
    q.N = d;
    q.C = static_cast<char*>(dx_disp);
    q.ldc = d * es;
    return launch_gemm<M_STORE, P_BWD_DX>(s, dt, pl, ws, q);
  };
  // Order of the four products: dA first (it writes dH), dX right after it,
  // except when dx_disp is small enough to stay in the last-level cache: then
  // dX goes last, so the dispatch backward that follows reads dx_disp from
  // that cache rather than from HBM.
  const bool dx_last = rows_alloc * d * es <= kDxLastBytes;

  // dA = dY W2 (W2 read K-major: its rows are the d inputs) -> dH
  GemmParams p = base_params(pl, offsets, ws);
  p.A = static_cast<const char*>(dy_disp);
  p.lda = d * es;
  p.B = static_cast<const char*>(w2);
  p.ldb = f * es;
  p.b_gstride = static_cast<int64_t>(d) * f * es;
  p.K = d;
  p.N = f;
  p.act = actc;
  p.C = dh;
  p.ldc = F * es;
  p.H1 = const_cast<char*>(h1);
  p.H3 = const_cast<char*>(h3);
  p.ldh = f * es;
  p.f = f;
  if (sw) MOE_TRY(launch_gemm<M_BWD_DA_SWIGLU, P_BWD_DA>(s, dt, pl, ws, p));
  else MOE_TRY(launch_gemm<M_BWD_DA, P_BWD_DA>(s, dt, pl, ws, p));
  if (!dx_last) MOE_TRY(launch_dx());

  // dW2 [d, f] = dY^T A, contracting over each expert's dispatched rows
  GemmParams r = base_params(pl, offsets, ws);
  r.A = static_cast<const char*>(dy_disp);
  r.lda = d * es;
  r.M_out = d;
  r.B = abuf;
  r.ldb = f * es;
  r.N = f;
  r.dwA = dw2;
  r.dwB = dw2;
  r.dw_gstride = static_cast<int64_t>(d) * f;
  r.split_row = d;
  r.partial = reinterpret_cast<float*>(ws + pl.o_part);
  r.slot_elems = static_cast<int64_t>(d) * f;
  MOE_TRY(launch_gemm<M_DW, P_BWD_DW2>(s, dt, pl, ws, r));
  MOE_TRY(launch_split_reduce(s, pl, ws, d, f, dw2, dw2, d, r.dw_gstride));

  // [dW1; dW3] [F, d] = [dH1 dH3]^T X
  GemmParams u = base_params(pl, offsets, ws);
  u.A = dh;
  u.lda = F * es;
  u.M_out = F;
  u.B = static_cast<const char*>(x_disp);
  u.ldb = d * es;
  u.N = d;
  u.dwA = dw1;
  u.dwB = sw ? dw3 : dw1;
  u.dw_gstride = static_cast<int64_t>(f) * d;
  u.split_row = f;
  u.partial = reinterpret_cast<float*>(ws + pl.o_part);
  u.slot_elems = static_cast<int64_t>(F) * d;
  MOE_TRY(launch_gemm<M_DW, P_BWD_DW13>(s, dt, pl, ws, u));
  MOE_TRY(launch_split_reduce(s, pl, ws, F, d, dw1, sw ? dw3 : dw1, f, u.dw_gstride));

  // dx_disp last when it fits the last-level cache (see kDxLastBytes)
  if (dx_last) MOE_TRY(launch_dx());
  return MOE_OK;
}
