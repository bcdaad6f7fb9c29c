// The dense gated feed-forward block: the expert every token passes (a shared
// expert), on plain row-major tensors without routing arrays:
//     H1 = X W1^T, H3 = X W3^T, A = act(H1) * H3, Y = add + A W2^T
// with act silu (SwiGLU), GELU (tanh form) or ReLU, and its backward
//     dA = dY W2, dH1 = dA * H3 * act'(H1), dH3 = dA * act(H1),
//     dX = add + dH1 W1 + dH3 W3,
//     dW1 = dH1^T X, dW3 = dH3^T X, dW2 = dY^T A.
// Both projections, the activation and the product are one kernel, and the
// addend (the routed experts' output, or their gradient) goes into the
// epilogue of the last product, so y and dx are written once.
//
// The products are those of the experts (gemm.hpp) with one expert of T rows.

#include "gemm.hpp"

namespace moe {
namespace {

// The schedule of one expert of T rows, and the row layout the products read.
__global__ __launch_bounds__(64 * kSchedTasks) void schedule_dense_kernel(int T, int32_t* offsets,
                                                                          const SchedArgs A) {
  if (threadIdx.x < 2) offsets[threadIdx.x] = threadIdx.x ? T : 0;
  build_schedule<kSchedTasks>((threadIdx.x & 63) == 0 ? T : 0, A);
}

// Workspace: the products' schedule and buffers as for E = 1, then the row
// layout (two int32).
struct GatedPlan {
  FfnPlan pl;
  size_t o_off, total_fwd, total_bwd, total_bwd_wt;
};

bool plan_gated(moe_dtype dt, int T, int d, int f, GatedPlan& g) {
  if (T < 0 || !make_plan(dt, MOE_SWIGLU, 1, d, f, T, g.pl)) return false;
  g.o_off = g.pl.o_end_sched;
  // every buffer behind the schedule moves by the layout's 256 bytes
  FfnPlan& pl = g.pl;
  pl.o_abuf += 256; pl.o_dh += 256; pl.o_part += 256; pl.o_wt13 += 256;
  g.total_fwd = pl.total_fwd + 256;
  g.total_bwd = pl.total_bwd + 256;
  g.total_bwd_wt = pl.total_bwd_wt + 256;
  return true;
}

int gate_act(moe_act act) {
  return act == MOE_RELU ? ACT_RELU : act == MOE_GELU_TANH ? ACT_GELU : ACT_SWIGLU;
}

bool act_ok(moe_act act) { return act == MOE_RELU || act == MOE_GELU_TANH || act == MOE_SWIGLU; }

// Rows ld elements apart: whole 16-byte vectors, 256 rows within 2^31 bytes.
bool pitch_ok(int64_t ld, int d, size_t es) {
  return ld >= d && ld % 8 == 0 && ld * static_cast<int64_t>(es) <= kMaxOperandRowBytes;
}

moe_status schedule_dense(hipStream_t s, int T, const SchedArgs& a, int32_t* offsets) {
  MOE_TIMED("ffn_schedule", s);
  schedule_dense_kernel<<<1, 64 * kSchedTasks, 0, s>>>(T, offsets, a);
  MOE_LAUNCH_CHECK();
  return MOE_OK;
}

}  // namespace
}  // namespace moe

using namespace moe;

extern "C" size_t moe_gated_ffn_fwd_workspace_bytes(moe_dtype dt, int T, int d, int f) {
  GatedPlan g;
  return plan_gated(dt, T, d, f, g) ? g.total_fwd : 0;
}

extern "C" size_t moe_gated_ffn_bwd_workspace_bytes(moe_dtype dt, int T, int d, int f) {
  GatedPlan g;
  if (!plan_gated(dt, T, d, f, g)) return 0;
  return use_wt13(g.pl, dt) ? g.total_bwd_wt : g.total_bwd;
}

extern "C" moe_status moe_gated_ffn_fwd(void* stream, moe_dtype dt, moe_act act, int T, int d,
                                        int f, const void* x, int64_t ldx, const void* w1,
                                        const void* w3, const void* w2, const void* add,
                                        int64_t ldadd, void* h_save, void* y, int64_t ldy,
                                        void* workspace, size_t workspace_bytes) {
  GatedPlan g;
  if (!act_ok(act) || !plan_gated(dt, T, d, f, g)) return MOE_EINVAL;
  const size_t e = g.pl.es;
  if (!pitch_ok(ldx, d, e) || !pitch_ok(ldy, d, e) || (add && !pitch_ok(ldadd, d, e)))
    return MOE_EINVAL;
  if (T == 0) return MOE_OK;
  if (!x || !w1 || !w3 || !w2 || !y) return MOE_EINVAL;
  if (!aligned16(x) || !aligned16(w1) || !aligned16(w3) || !aligned16(w2) || !aligned16(y) ||
      !aligned16(add) || !aligned16(h_save))
    return MOE_EINVAL;
  if (!workspace || workspace_bytes < g.total_fwd || !aligned16(workspace)) return MOE_EWORKSPACE;
  hipStream_t s = static_cast<hipStream_t>(stream);
  char* ws = static_cast<char*>(workspace);
  const FfnPlan& pl = g.pl;
  const int64_t es = static_cast<int64_t>(e), plane = static_cast<int64_t>(T) * f * es;
  int32_t* offsets = reinterpret_cast<int32_t*>(ws + g.o_off);
  MOE_TRY(schedule_dense(s, T, sched_args(pl, cdiv(f, kMidN / 2), cdiv(d, kMidN), f,
                                          step16(ldx * es, d * es, false),
                                          step16(f * es, f * es, false), ws), offsets));
  char* a = h_save ? static_cast<char*>(h_save) + 2 * plane : ws + pl.o_abuf;
  GemmParams p = base_params(pl, offsets, ws);
  p.A = static_cast<const char*>(x);
  p.lda = ldx * es;
  p.B = static_cast<const char*>(w1);
  p.B2 = static_cast<const char*>(w3);
  p.ldb = d * es;
  p.K = d;
  p.N = f;
  p.act = gate_act(act);
  p.C = a;
  p.ldc = f * es;
  p.H1 = static_cast<char*>(h_save);
  p.H3 = h_save ? static_cast<char*>(h_save) + plane : nullptr;
  p.ldh = f * es;
  MOE_TRY(launch_gemm<M_GATED_FWD, P_FWD_H>(s, dt, pl, ws, p));
  GemmParams q = base_params(pl, offsets, ws);
  q.A = a;
  q.lda = f * es;
  q.B = static_cast<const char*>(w2);
  q.ldb = f * es;
  q.K = f;
  q.N = d;
  q.C = static_cast<char*>(y);
  q.ldc = ldy * es;
  q.add = static_cast<const char*>(add);
  q.ldadd = ldadd * es;
  return launch_gemm<M_ADD_STORE, P_FWD_Y>(s, dt, pl, ws, q);
}

extern "C" moe_status moe_gated_ffn_bwd(void* stream, moe_dtype dt, moe_act act, int T, int d,
                                        int f, const void* x, int64_t ldx, const void* h_save,
                                        const void* w1, const void* w3, const void* w2,
                                        const void* dy, int64_t lddy, const void* add,
                                        int64_t ldadd, void* dx, int64_t lddx, moe_dtype dw_dt,
                                        void* dw1, void* dw3, void* dw2, void* workspace,
                                        size_t workspace_bytes) {
  GatedPlan g;
  if (!act_ok(act) || !plan_gated(dt, T, d, f, g)) return MOE_EINVAL;
  if (dw_dt != dt && dw_dt != MOE_F32) return MOE_EINVAL;
  const size_t e = g.pl.es;
  if (!pitch_ok(ldx, d, e) || !pitch_ok(lddy, d, e) || !pitch_ok(lddx, d, e) ||
      (add && !pitch_ok(ldadd, d, e)))
    return MOE_EINVAL;
  if (!w1 || !w3 || !w2 || !dw1 || !dw3 || !dw2) return MOE_EINVAL;
  if (T > 0 && (!x || !h_save || !dy || !dx)) return MOE_EINVAL;
  if (!aligned16(x) || !aligned16(h_save) || !aligned16(w1) || !aligned16(w3) || !aligned16(w2) ||
      !aligned16(dy) || !aligned16(add) || !aligned16(dx) || !aligned16(dw1) || !aligned16(dw3) ||
      !aligned16(dw2))
    return MOE_EINVAL;
  if (!workspace || workspace_bytes < g.total_bwd || !aligned16(workspace)) return MOE_EWORKSPACE;
  hipStream_t s = static_cast<hipStream_t>(stream);
  char* ws = static_cast<char*>(workspace);
  const FfnPlan& pl = g.pl;
  const int64_t es = static_cast<int64_t>(e), plane = static_cast<int64_t>(T) * f * es;
  const int F = 2 * f;
  const bool wt = use_wt13(pl, dt) && workspace_bytes >= g.total_bwd_wt;
  int32_t* offsets = reinterpret_cast<int32_t*>(ws + g.o_off);
  MOE_TRY(schedule_dense(s, T, sched_args(pl, cdiv(f, kMidN), cdiv(d, kMidN), F,
                                          step16(lddy * es, f * es, true),
                                          step16(F * es, (wt ? F : d) * es, !wt), ws), offsets));
  const char* h1 = static_cast<const char*>(h_save);
  const char* a = h1 + 2 * plane;
  char* dh = ws + pl.o_dh;      // [T, 2f]: dH1 | dH3
  char* wt13 = ws + pl.o_wt13;
  if (wt) MOE_TRY(launch_transpose_w(s, 1, w1, w3, f, f, d, wt13));

  // dH from dA = dY W2 (W2 read K-major)
  GemmParams p = base_params(pl, offsets, ws);
  p.A = static_cast<const char*>(dy);
  p.lda = lddy * es;
  p.B = static_cast<const char*>(w2);
  p.ldb = f * es;
  p.K = d;
  p.N = f;
  p.act = gate_act(act);
  p.C = dh;
  p.ldc = F * es;
  p.H1 = const_cast<char*>(h1);
  p.H3 = const_cast<char*>(h1) + plane;
  p.ldh = f * es;
  p.f = f;
  MOE_TRY(launch_gemm<M_GATED_DA, P_BWD_DA>(s, dt, pl, ws, p));

  // dX = add + [dH1 | dH3] [W1; W3]
  GemmParams q = base_params(pl, offsets, ws);
  q.A = dh;
  q.lda = F * es;
  q.K = F;
  q.N = d;
  q.C = static_cast<char*>(dx);
  q.ldc = lddx * es;
  q.add = static_cast<const char*>(add);
  q.ldadd = ldadd * es;
  if (wt) {
    q.B = wt13;
    q.ldb = F * es;
    MOE_TRY(launch_gemm<M_ADD_STORE, P_BWD_DX_T>(s, dt, pl, ws, q));
  } else {
    q.B = static_cast<const char*>(w1);
    q.B2 = static_cast<const char*>(w3);
    q.kmsplit = f;
    q.ldb = d * es;
    MOE_TRY(launch_gemm<M_ADD_STORE, P_BWD_DX>(s, dt, pl, ws, q));
  }

  // dW2 [d, f] = dY^T A, then [dW1; dW3] [2f, d] = [dH1 dH3]^T X
  const bool layer_dw = dw_dt == MOE_BF16;
  auto launch_dw = [&](auto pass, const void* l, int64_t ldl, const void* r, int64_t ldr, int m,
                       int n, void* to1, void* to2, int split) -> moe_status {
    constexpr int PASS = decltype(pass)::value;
    GemmParams u = base_params(pl, offsets, ws);
    u.A = static_cast<const char*>(l);
    u.lda = ldl * es;
    u.M_out = m;
    u.B = static_cast<const char*>(r);
    u.ldb = ldr * es;
    u.N = n;
    u.dwA = static_cast<float*>(to1);
    u.dwB = static_cast<float*>(to2);
    u.split_row = split;
    u.partial = reinterpret_cast<float*>(ws + pl.o_part);
    u.slot_elems = static_cast<int64_t>(m) * n;
    if (layer_dw) MOE_TRY(launch_gemm<M_DW_LAYER, PASS>(s, dt, pl, ws, u));
    else MOE_TRY(launch_gemm<M_DW, PASS>(s, dt, pl, ws, u));
    return launch_split_reduce(s, pl, ws, m, n, u.dwA, u.dwB, split, 0, layer_dw);
  };
  MOE_TRY(launch_dw(std::integral_constant<int, P_BWD_DW2>{}, dy, lddy, a, f, d, f, dw2, dw2, d));
  return launch_dw(std::integral_constant<int, P_BWD_DW13>{}, dh, F, x, ldx, F, d, dw1, dw3, f);
}
