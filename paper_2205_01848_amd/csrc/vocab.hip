// The loss of a vocabulary projection, and its gradients, in pieces of rows:
//     l = x W^T,  lse_t = log sum_v exp l_tv,  loss_t = lse_t - l_t,target
//     dl_tv = weight_t (exp(l_tv - lse_t) - [v = target_t]),
//     dx = scale dl W,  dW = scale dl^T x.
//
// The logits' product leaves, for every row and block of 16 to 128 columns, their maximum m
// and sum of exp(l - m), and the target's logit; a pass over those forms lse and
// loss = log sum + (maximum - l_target), in which the size of the logits cancels: a small loss is
// off by a few 2^-24 (beside the logits' own errors), not by lse 2^-24.  The sum holds the maximum's
// own 1, so a target with more than 1 - 2^-24 of the probability has loss 0, and 0 in dl, while the
// other words keep theirs.  Without gradients no logit is ever written.
//
// With gradients the product also writes exp(l - m) of its piece, in 16 bits (11 of
// mantissa), and one pass turns them into dl in place: weight exp(m - lse) times that, and
// weight (exp(-loss) - 1) at the target.  Then dl W and dl^T x.  So nothing is computed twice:
// 6 T V d operations and 6 bytes of traffic a logit, against 8 T V d for a second product of
// the logits (8192 tokens, 4096 x 131072: the second product would take 6.3 ms, the
// two passes over 2.1 GB of exponentials take 1 ms).  Kept as bf16 the exponentials would
// round twice, and dx be off by sqrt(3) roundings for sqrt(2).  scale joins the fp32 sums at
// the end: in dl it would round every token's largest entry, near -scale, the same way, by up
// to 2^-8 (1 / 509 by 0.0019).  Without weights the targets' entries, near -1, are nearly exact, and dx and
// dw are off by 0.0017 to 0.0019 of themselves, 0.0016 of it their own rounding; tokens' weights stay
// in dl (dw sums over the tokens), whose largest entries then round too: 0.0024, sqrt(2) roundings.
//
// dW's product reads a copy of x that the pass makes, with zeros in the rows of ignored
// tokens, so that nothing they contain reaches it.
//
// A piece holds at most kPieceBytes of exponentials; dW of further pieces is added to the
// fp32 sums of those before, in order.

#include "dense.hpp"
#include "few_rows.hpp"

namespace moe {
namespace {

constexpr int64_t kPieceBytes = int64_t(1) << 31;    // of exponentials
constexpr int64_t kStatBytes = int64_t(1) << 28;     // of maxima and sums, without gradients

struct VocabPiece {
  DensePlan l, dx, dw;
  int stats, width;            // blocks of columns in a row, their width
};
struct VocabPlan {
  int rows, pieces;            // of a piece (the last may hold fewer)
  int64_t pitch;               // bytes of a row of exponentials: whole cache lines
  bool few;
  VocabPiece full, last;
  int64_t o_x, o_stat, o_target, o_part, o_sum, total;
};

bool plan_vocab(moe_dtype dt, int T, int d, int V, bool grad, moe_dtype dw_dt, VocabPlan& g) {
  if (!dtype_ok(dt) || T < 0 || !width_ok(d) || V < 1) return false;
  if (grad && dw_dt != dt && dw_dt != MOE_F32) return false;
  const int64_t es = static_cast<int64_t>(esize(dt)), rd = d * es, line = 128 / es;
  const int64_t pitch = (V + line - 1) / line * line * es;
  if (rd > kMaxOperandRowBytes || pitch > kMaxOperandRowBytes) return false;
  g = {};
  g.total = 256;
  g.pitch = pitch;
  if (T == 0) return true;
  const int64_t least = dt == MOE_F32 ? 32 : 64;   // columns of a block, of the kernels for many rows
  const int64_t row = grad ? pitch : (V + least - 1) / least * 8, cap = grad ? kPieceBytes : kStatBytes;
  const int64_t most = std::max<int64_t>(cap / row / BM * BM, BM);
  g.pieces = cdiv(T, most);
  g.rows = g.pieces == 1 ? T : std::min<int64_t>(T, (cdiv(T, g.pieces) + BM - 1) / BM * BM);
  g.pieces = cdiv(T, g.rows);
  auto piece = [&](int rows) {
    VocabPiece p{};
    p.l = dense_plan<M_VOCAB, P_VOCAB>(dt, rows, V, d, rd, rd);
    g.few = g_tile_mode == 0 && vocab_few(dt == MOE_F32, T, V, d, p.l);   // (of all rows: then one piece)
    p.width = g.few ? kFewCols : dt == MOE_F32 ? 32 : p.l.kernel == K_BIG ? TileBig::WC : kMidN / 2;
    p.stats = g.few ? cdiv(V, kFewCols) : p.l.nt * (dt == MOE_F32 ? 4 : 2);
    if (grad) {
      p.dx = dense_plan<M_VOCAB_DX, P_VOCAB_DX>(dt, rows, d, V, pitch, rd);
      p.dw = dense_plan<M_VOCAB_DW, P_VOCAB_DW>(dt, V, d, rows, pitch, rd);
    }
    return p;
  };
  const int left = T - (g.pieces - 1) * g.rows;
  g.full = piece(g.rows);
  g.last = left == g.rows ? g.full : piece(left);
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    const int64_t o = at;
    at += (bytes + 255) / 256 * 256;
    return o;
  };
  if (grad) take(g.rows * pitch);
  g.o_x = grad ? take(g.rows * rd) : 0;
  g.o_stat = take(std::max(static_cast<int64_t>(g.rows) * g.full.stats, static_cast<int64_t>(left) * g.last.stats) * 8);
  g.o_target = take(static_cast<int64_t>(g.rows) * 4);
  if (grad) {
    g.o_part = take(std::max({dense_partial_bytes(g.full.dx, g.rows, d), dense_partial_bytes(g.full.dw, V, d),
                              dense_partial_bytes(g.last.dx, left, d), dense_partial_bytes(g.last.dw, V, d)}));
    g.o_sum = take(g.pieces > 1 && dw_dt != MOE_F32 ? static_cast<int64_t>(V) * d * 4 : 0);
  }
  g.total = at;
  return true;
}

// Maxima and sums of exponentials joined: {m, s} stands for s e^m.
__device__ __forceinline__ float2 join(float2 a, float2 b) {
  const float m = fmaxf(a.x, b.x);
  if (m == -INFINITY) return make_float2(m, a.y + b.y);
  return make_float2(m, a.y * exp_fast(a.x - m) + b.y * exp_fast(b.x - m));
}

struct VocabRows {
  const float2* stat;
  const int32_t* target;
  const float *target_logit, *weights;
  float *loss, *lse;
  int32_t* status;
  int rows, V, stats, width, parts;
  char* z;             // exponentials in, dl out; NULL: no gradients
  int64_t pitch;
  const char* x;       // and x, copied to x_live with zeros in the rows of ignored tokens
  int64_t ldx;         // bytes
  char* x_live;
  int x_units;         // vectors of a row
};

// A workgroup takes one of `parts` ranges of a row: the row's sum from its blocks', the loss,
// and (GRAD) its range of dl.  Bound by memory: 4 bytes a logit (8 in fp32), 8192 x 131072 in 0.88
// ms, 4.9 TB/s.  The row of one token has 8192 blocks: 6 us with 1024 threads and eight
// loads in flight, 15 with 256 and one.
template <typename T, bool GRAD, int THREADS>
__global__ __launch_bounds__(THREADS) void vocab_rows_kernel(const VocabRows a) {
  __shared__ float2 sums[THREADS / 64];
  const int64_t items = static_cast<int64_t>(a.rows) * a.parts;
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const int row = static_cast<int>(item / a.parts), part = static_cast<int>(item - static_cast<int64_t>(row) * a.parts);
    const float2* stat = a.stat + static_cast<int64_t>(row) * a.stats;
    float2 s = make_float2(-INFINITY, 0.f);
    // (eight at a time, so that a long row waits for few loads)
    for (int i = threadIdx.x; i < a.stats; i += 8 * THREADS) {
      float2 b[8];
#pragma unroll
      for (int k = 0; k < 8; ++k)
        b[k] = i + k * THREADS < a.stats ? stat[i + k * THREADS] : make_float2(-INFINITY, 0.f);
#pragma unroll
      for (int o = 4; o > 0; o >>= 1)
#pragma unroll
        for (int k = 0; k < o; ++k) b[k] = join(b[k], b[k + o]);
      s = join(s, b[0]);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1)
      s = join(s, make_float2(__shfl_xor(s.x, o, 64), __shfl_xor(s.y, o, 64)));
    __syncthreads();   // the last row's sums have been read
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = s;
    __syncthreads();
    s = sums[0];
#pragma unroll
    for (int k = 1; k < THREADS / 64; ++k) s = join(s, sums[k]);
    const int target = a.target[row];
    const bool live = target >= 0 && target < a.V;
    const float logs = logf(s.y);
    const float loss = live ? logs + (s.x - a.target_logit[row]) : 0.f;
    if (part == 0 && threadIdx.x == 0) {
      a.loss[row] = loss;
      if (a.lse) a.lse[row] = live ? s.x + logs : 0.f;
      if (target >= a.V) atomicOr(a.status, MOE_STATUS_BAD_TARGET);
    }
    if constexpr (GRAD) {
      if (part == 0) {
        const uint4* from = reinterpret_cast<const uint4*>(a.x + row * a.ldx);
        uint4* to = reinterpret_cast<uint4*>(a.x_live) + static_cast<int64_t>(row) * a.x_units;
        for (int u = threadIdx.x; u < a.x_units; u += THREADS) to[u] = live ? from[u] : make_uint4(0, 0, 0, 0);
      }
      constexpr int kVec = Elem<T>::kVec;   // 16 bytes of exponentials and of dl
      const float c = a.weights ? a.weights[row] : 1.f;
      const float at = c * expm1f(-loss), f = c / s.y * (sizeof(T) == 2 ? 1.f / (1 << kVocabLift) : 1.f);
      const int units = (a.V + kVec - 1) / kVec, per = (units + a.parts - 1) / a.parts;
      uint4* z = reinterpret_cast<uint4*>(a.z + row * a.pitch);
      for (int u = part * per + threadIdx.x; u < min(units, (part + 1) * per); u += THREADS) {
        const int col = u * kVec;
        float v[kVec];
        if constexpr (sizeof(T) == 2) {
          typedef _Float16 half8 __attribute__((ext_vector_type(8)));
          const half8 h = __builtin_bit_cast(half8, z[u]);
#pragma unroll
          for (int e = 0; e < kVec; ++e) v[e] = static_cast<float>(h[e]);
        } else {
          Elem<T>::load(z[u], v);
        }
        const float g = f * exp_fast(stat[col / a.width].x - s.x);
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
          v[e] *= g;
          if (col + e == target) v[e] = at;
          if (!live || col + e >= a.V) v[e] = 0.f;
        }
        z[u] = Elem<T>::store(v);
      }
    }
  }
}

template <typename T>
moe_status launch_rows(hipStream_t s, VocabRows a) {
  // enough workgroups for the chip, ranges of no less than 512 vectors
  const int units = cdiv(static_cast<int64_t>(a.V) * sizeof(T), 16);
  a.parts = a.z ? static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(cdiv(4 * num_cus(), a.rows), units / 512))) : 1;
  const int grid = static_cast<int>(std::min<int64_t>(static_cast<int64_t>(a.rows) * a.parts, 16 * num_cus()));
  MOE_TIMED(a.z ? "vocab_dlogits" : "vocab_rows", s);
  if (a.z) vocab_rows_kernel<T, true, 256><<<grid, 256, 0, s>>>(a);
  else if (a.stats > 2048) vocab_rows_kernel<T, false, 1024><<<grid, 1024, 0, s>>>(a);
  else vocab_rows_kernel<T, false, 256><<<grid, 256, 0, s>>>(a);
  MOE_LAUNCH_CHECK();
  return MOE_OK;
}

}  // namespace
}  // namespace moe

using namespace moe;

extern "C" size_t moe_vocab_loss_workspace_bytes(moe_dtype dt, int T, int d, int V, int grad, moe_dtype dw_dt) {
  VocabPlan g;
  return plan_vocab(dt, T, d, V, grad != 0, dw_dt, g) ? static_cast<size_t>(g.total) : 0;
}

extern "C" moe_status moe_vocab_loss(void* stream, moe_dtype dt, int T, int d, int V, const void* x, int64_t ldx,
                                     const void* w, const int32_t* targets, float scale, const float* weights,
                                     float* loss, float* lse, void* dx, int64_t lddx, moe_dtype dw_dt, void* dw,
                                     int32_t* status, void* workspace, size_t workspace_bytes) {
  const bool grad = dx || dw;
  VocabPlan g;
  if (!plan_vocab(dt, T, d, V, grad, dw_dt, g)) return MOE_EINVAL;
  const int64_t es = static_cast<int64_t>(esize(dt));
  auto pitch_ok = [&](int64_t ld) { return ld >= d && ld % 8 == 0 && ld * es <= kMaxOperandRowBytes; };
  if (!pitch_ok(ldx) || (grad && !pitch_ok(lddx)) || !(scale > -INFINITY && scale < INFINITY)) return MOE_EINVAL;
  if (grad && (!dw || (T > 0 && !dx))) return MOE_EINVAL;   // both
  if (!w || !aligned16(w) || !aligned16(x) || !aligned16(dx) || !aligned16(dw)) return MOE_EINVAL;
  if (T > 0 && (!x || !targets || !loss || !status)) return MOE_EINVAL;
  if (T > 1 && dx == x && lddx != ldx) return MOE_EINVAL;   // rows of one piece over those of the next
  if (!workspace || workspace_bytes < static_cast<size_t>(g.total) || !aligned16(workspace)) return MOE_EWORKSPACE;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (T == 0) return grad ? launch_zero(s, dw, static_cast<size_t>(V) * d * esize(dw_dt)) : MOE_OK;
  char* ws = static_cast<char*>(workspace);
  float2* stat = reinterpret_cast<float2*>(ws + g.o_stat);
  float* target_logit = reinterpret_cast<float*>(ws + g.o_target);
  float* sums = dw_dt == MOE_F32 ? static_cast<float*>(dw) : reinterpret_cast<float*>(ws + g.o_sum);
  for (int piece = 0; piece < g.pieces; ++piece) {
    const int t0 = piece * g.rows, rows = std::min(g.rows, T - t0);
    const bool last = piece + 1 == g.pieces;
    const VocabPiece& plan = last ? g.last : g.full;
    const char* xp = static_cast<const char*>(x) + t0 * ldx * es;
    GemmParams p{};
    p.A = xp;
    p.lda = ldx * es;
    p.B = static_cast<const char*>(w);
    p.ldb = d * es;
    p.K = d;
    p.N = V;
    p.C = grad ? ws : nullptr;
    p.ldc = g.pitch;
    p.stat = stat;
    p.n_stat = plan.stats;
    p.target = targets + t0;
    p.target_logit = target_logit;
    if (g.few) {
      GroupParams fp{p, 0, nullptr, 0};
      fp.p.dense.T = rows;
      if (dt == MOE_F32) MOE_TRY((launch_few<M_VOCAB, 4>(s, pass_name(P_VOCAB), fp, rows, 1)));
      else MOE_TRY((launch_few<M_VOCAB, 2>(s, pass_name(P_VOCAB), fp, rows, 1)));
    } else {
      MOE_TRY(launch_dense<M_VOCAB, P_VOCAB>(s, dt, plan.l, rows, rows, p));
    }
    VocabRows r{stat, targets + t0, target_logit, weights ? weights + t0 : nullptr, loss + t0,
                lse ? lse + t0 : nullptr, status, rows, V, plan.stats, plan.width, 1, grad ? ws : nullptr, g.pitch,
                xp, ldx * es, ws + g.o_x, static_cast<int>(d * es / 16)};
    if (dt == MOE_BF16) MOE_TRY(launch_rows<uint16_t>(s, r));
    else MOE_TRY(launch_rows<float>(s, r));
    if (!grad) continue;
    GemmParams q{};
    q.A = ws;
    q.lda = g.pitch;
    q.B = static_cast<const char*>(w);
    q.ldb = d * es;
    q.K = V;
    q.N = d;
    q.C = static_cast<char*>(dx) + t0 * lddx * es;
    q.ldc = lddx * es;
    q.alpha = scale;
    q.partial = reinterpret_cast<float*>(ws + g.o_part);
    MOE_TRY(launch_dense<M_VOCAB_DX, P_VOCAB_DX>(s, dt, plan.dx, rows, rows, q));
    GemmParams u{};
    u.A = ws;
    u.lda = g.pitch;
    u.M_out = V;
    u.B = ws + g.o_x;
    u.ldb = d * es;
    u.N = d;
    u.out_f32 = !last || dw_dt == MOE_F32;
    u.dwA = u.dwB = u.out_f32 ? sums : static_cast<float*>(dw);
    u.split_row = V;
    u.alpha = scale;
    u.acc = piece > 0 ? sums : nullptr;
    u.partial = q.partial;
    MOE_TRY(launch_dense<M_VOCAB_DW, P_VOCAB_DW>(s, dt, plan.dw, rows, V, u));
  }
  return MOE_OK;
}
