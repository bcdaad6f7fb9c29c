// The dense gated feed-forward block: the expert every token passes (a shared
// expert), on plain row-major tensors without routing arrays:
//     H1 = X W1^T, H3 = X W3^T, A = act(H1) * H3, Y = add + A W2^T
// with act silu (SwiGLU), GELU (tanh form) or ReLU, and its backward
//     dA = dY W2, dH1 = dA * (H3 * act'(H1)), dH3 = dA * act(H1),
//     dX = add + dH1 W1 + dH3 W3,
//     dW1 = dH1^T X, dW3 = dH3^T X, dW2 = dY^T A.
// The forward saves the two factors of dA and A.  Against saving H1 and H3 the
// backward evaluates no activation (dA of 8192 tokens, 4096 x 14336, 907 -> 880 us) and each
// factor is rounded to bf16 once, from the unrounded H (relative error of
// dW1 0.0035 -> 0.0029; factors of 32 bits would give 0.0024 and take 0.9 GB more
// traffic in that step, about 3 % of it).
//
// Both projections, the activation and the product are one kernel, and the
// addend (the routed experts' output, or their gradient) goes into the
// epilogue of the last product, so y and dx are written once.
//
// The products are those of the experts (gemm.hpp) on one expert of T rows.  The
// host knows T, so it plans them itself (dense_plan) and no schedule kernel runs.

#include "dense.hpp"
#include "few_rows.hpp"

namespace moe {
namespace {

// The block's products, planned from the sizes alone (rows as if contiguous, so
// that the workspace query and the calls agree), and the workspace: forward,
// A (where h_save does not hold it) and Y's partial sums; backward, dH, the
// partial sums of the product that has most, and the transposed weights.
struct GatedPlan {
  DensePlan h, y, da, dx, dw2, dw13;
  bool few;                // the forward's products by the kernel for few rows
  bool wt;                 // dX reads a transposed copy of [W1; W3]
  size_t o_part_fwd, total_fwd;
  size_t o_part, o_wt, total_bwd;
};

// Rows up to which the forward streams its weights through the kernel for few rows
// (a forced tile mode, moe_set_gemm_tiles, has its tiles run instead).
constexpr int kFewDense = 16;

bool plan_gated(moe_dtype dt, int T, int d, int f, GatedPlan& g) {
  FfnPlan pl;   // its limits on the sizes
  if (T < 0 || !make_plan(dt, MOE_SWIGLU, 1, d, f, T, pl)) return false;
  const int F = 2 * f;
  const int64_t es = static_cast<int64_t>(pl.es), rd = d * es, rf = f * es, rF = F * es;
  g = {};
  g.total_fwd = g.total_bwd = 256;
  if (T == 0) return true;
  g.few = g_tile_mode == 0 && T <= (dt == MOE_F32 ? 2 : 1) * kFewDense;
  g.wt = use_wt13(pl, dt);
  g.h = dense_plan<M_GATED_FWD, P_FWD_H>(dt, T, f, d, rd, rd);
  g.y = dense_plan<M_ADD_STORE, P_FWD_Y>(dt, T, d, f, rf, rf);
  g.da = dense_plan<M_GATED_DA, P_BWD_DA>(dt, T, f, d, rd, rf);
  g.dx = g.wt ? dense_plan<M_ADD_STORE, P_BWD_DX_T>(dt, T, d, F, rF, rF)
              : dense_plan<M_ADD_STORE, P_BWD_DX>(dt, T, d, F, rF, rd);
  g.dw2 = dense_plan<M_DENSE_DW, P_BWD_DW2>(dt, d, f, T, rd, rf);
  g.dw13 = dense_plan<M_DENSE_DW, P_BWD_DW13>(dt, F, d, T, rF, rd);
  const size_t rows = static_cast<size_t>(T);
  g.o_part_fwd = align_up(rows * f * pl.es, 256);
  g.total_fwd = g.o_part_fwd + (g.few ? 0 : dense_partial_bytes(g.y, T, d)) + 256;
  g.o_part = align_up(rows * F * pl.es, 256);
  g.o_wt = g.o_part + std::max({dense_partial_bytes(g.dx, T, d), dense_partial_bytes(g.dw2, d, f),
                                dense_partial_bytes(g.dw13, F, d)});
  g.total_bwd = g.o_wt + (g.wt ? align_up(static_cast<size_t>(d) * F * pl.es, 256) : 0) + 256;
  return true;
}

int gate_act(moe_act act) {
  return act == MOE_RELU ? ACT_RELU : act == MOE_GELU_TANH ? ACT_GELU : ACT_SWIGLU;
}

template <int MODE, int PASS>
moe_status launch_few_dense(hipStream_t s, moe_dtype dt, int T, const GemmParams& p) {
  GroupParams fp{p, 0, nullptr, 0};
  fp.p.dense.T = T;
  if (dt == MOE_F32) return launch_few<MODE, 4>(s, pass_name(PASS), fp, T, 1);
  return launch_few<MODE, 2>(s, pass_name(PASS), fp, T, 1);
}

bool act_ok(moe_act act) { return act == MOE_RELU || act == MOE_GELU_TANH || act == MOE_SWIGLU; }

// Rows ld elements apart: whole 16-byte vectors, 256 rows within 2^31 bytes.
bool pitch_ok(int64_t ld, int d, size_t es) {
  return ld >= d && ld % 8 == 0 && ld * static_cast<int64_t>(es) <= kMaxOperandRowBytes;
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
  return plan_gated(dt, T, d, f, g) ? g.total_bwd : 0;
}

extern "C" moe_status moe_gated_ffn_fwd(void* stream, moe_dtype dt, moe_act act, int T, int d,
                                        int f, const void* x, int64_t ldx, const void* w1,
                                        const void* w3, const void* w2, const void* add,
                                        int64_t ldadd, void* h_save, void* y, int64_t ldy,
                                        void* workspace, size_t workspace_bytes) {
  GatedPlan g;
  if (!act_ok(act) || !plan_gated(dt, T, d, f, g)) return MOE_EINVAL;
  const size_t e = esize(dt);
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
  const int64_t es = static_cast<int64_t>(e), plane = static_cast<int64_t>(T) * f * es;
  char* a = h_save ? static_cast<char*>(h_save) + 2 * plane : ws;
  GemmParams p{};
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
  if (g.few) MOE_TRY(launch_few_dense<M_GATED_FWD, P_FWD_H>(s, dt, T, p));
  else MOE_TRY(launch_dense<M_GATED_FWD, P_FWD_H>(s, dt, g.h, T, T, p));
  GemmParams q{};
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
  q.partial = reinterpret_cast<float*>(ws + g.o_part_fwd);
  if (g.few) return launch_few_dense<M_ADD_STORE, P_FWD_Y>(s, dt, T, q);
  return launch_dense<M_ADD_STORE, P_FWD_Y>(s, dt, g.y, T, T, q);
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
  const size_t e = esize(dt);
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
  const int64_t es = static_cast<int64_t>(e), plane = static_cast<int64_t>(T) * f * es;
  const int F = 2 * f;
  float* partial = reinterpret_cast<float*>(ws + g.o_part);
  const char* h1 = static_cast<const char*>(h_save);
  const char* a = h1 + 2 * plane;
  char* dh = ws;   // [T, 2f]: dH1 | dH3
  char* wt13 = ws + g.o_wt;
  if (T == 0) {
    // nothing to contract over: the weight gradients are zero
    const size_t bytes = static_cast<size_t>(d) * f * esize(dw_dt);
    for (void* w : {dw1, dw3, dw2}) MOE_TRY(launch_zero(s, w, bytes));
    return MOE_OK;
  }
  // dH from dA = dY W2 (W2 read K-major)
  GemmParams p{};
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
  MOE_TRY(launch_dense<M_GATED_DA, P_BWD_DA>(s, dt, g.da, T, T, p));

  // dW2 [d, f] = dY^T A, then [dW1; dW3] [2f, d] = [dH1 dH3]^T X
  auto weights = [&](const void* l, int64_t ldl, const void* r, int64_t ldr, int m, int n, void* to1,
                     void* to2, int split) {
    GemmParams u{};
    u.A = static_cast<const char*>(l);
    u.lda = ldl * es;
    u.M_out = m;
    u.B = static_cast<const char*>(r);
    u.ldb = ldr * es;
    u.N = n;
    u.out_f32 = dw_dt == MOE_F32;
    u.dwA = static_cast<float*>(to1);
    u.dwB = static_cast<float*>(to2);
    u.split_row = split;
    u.partial = partial;
    return u;
  };
  MOE_TRY(launch_dense<M_DENSE_DW, P_BWD_DW2>(s, dt, g.dw2, T, d,
                                              weights(dy, lddy, a, f, d, f, dw2, dw2, d)));
  MOE_TRY(launch_dense<M_DENSE_DW, P_BWD_DW13>(s, dt, g.dw13, T, F,
                                               weights(dh, F, x, ldx, F, d, dw1, dw3, f)));

  // dX = add + [dH1 | dH3] [W1; W3], last: it may be written over dY or X
  GemmParams q{};
  q.A = dh;
  q.lda = F * es;
  q.K = F;
  q.N = d;
  q.C = static_cast<char*>(dx);
  q.ldc = lddx * es;
  q.add = static_cast<const char*>(add);
  q.ldadd = ldadd * es;
  q.partial = partial;
  if (g.wt) {
    MOE_TRY(launch_transpose_w(s, 1, w1, w3, f, f, d, wt13));
    q.B = wt13;
    q.ldb = F * es;
    return launch_dense<M_ADD_STORE, P_BWD_DX_T>(s, dt, g.dx, T, T, q);
  }
  q.B = static_cast<const char*>(w1);
  q.B2 = static_cast<const char*>(w3);
  q.kmsplit = f;
  q.ldb = d * es;
  return launch_dense<M_ADD_STORE, P_BWD_DX>(s, dt, g.dx, T, T, q);
}
