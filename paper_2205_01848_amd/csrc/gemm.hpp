// The products of the feed-forward blocks: device kernels, the tile choice and
// the host functions that launch them.  Of the experts (the modules E_e of
// Algorithm 1, on the dynamically sized tensors of Section 4.1) in ffn.hip.
//
// Every product is one persistent grouped GEMM kernel in "NT" form,
//     C[m, n] = sum_k A[m, k] * B[n, k]     (both operands K-contiguous),
// K tiles of 128 bytes, operand tiles loaded HBM -> LDS by buffer loads,
// double-buffered, with an XOR swizzle that keeps the MFMA fragment reads
// bank-conflict free.
//  * bf16 layers: 4 wavefronts on v_mfma_f32_16x16x32_bf16, two barriers
//    per K step, loads and fragment reads issued one at a time between the
//    MFMAs: on 256x256 tiles (waves of 128x128, one workgroup per CU;
//    ffn_gemm16_kernel) or, for products with few tiles per CU, on tiles of
//    32 to 192 rows and 128 columns (two workgroups per CU;
//    ffn_gemm16_mid_kernel), whose heights the schedule chooses; both add
//    every output's products in the same order.
//  * fp32 layers: v_mfma_f32_32x32x2f32 on tiles of 32 to 192 rows and 128
//    columns, two workgroups per CU (ffn_gemm_f32_kernel).
//  * var-M products (forward H, Y; backward dA, dX): the M dimension of
//    expert e is its row count, read on the device; tiles are listed by a
//    one-workgroup schedule kernel, so no host synchronisation is needed.
//  * var-K products (dW): K of expert e is its row count; the K range is
//    split into chunks only when few experts carry most rows, and split
//    partial sums are added in a fixed order (deterministic).
//  * operands whose contraction index is their row index (the weights in dA
//    and dX, both operands of dW) are read K-major through transposing LDS
//    reads; on large experts dX instead reads a transposed copy of [W1; W3]
//    that the backward writes first.
// The persistent grid maps workgroup b to XCD b % 8 and hands each XCD a
// contiguous run of tiles arranged as 4 M-tiles x 8 N-tiles, so tiles that
// share operand panels share that XCD's L2.
// Epilogues (activation, SwiGLU, activation backward, transposed stores) run
// per wavefront on its fp32 accumulators, staged 16 rows at a time through a
// private LDS strip, and write 16-byte vectors.
#pragma once

#include <algorithm>
#include <type_traits>

#include "common.hpp"
#include "ffn.hpp"
#include "plan.hpp"
#include "sched.hpp"
#include "validate.hpp"

namespace moe {

extern int g_tile_mode, g_wt_mode;   // see use_mid_tiles, use_wt13 (ffn.hip sets them)

namespace {

constexpr int kRowBytes = 128;                    // one K tile of one operand row
constexpr int kTileBytes = BM * kRowBytes;        // 32 KB
constexpr int kGroupM = 4;      // M tiles per scheduling group
constexpr int kXcds = 8;
constexpr int64_t kMaxOperandRowBytes = (int64_t(1) << 23) - 64;  // 256 rows < 2^31 bytes
// dx_disp up to this size is produced last in the backward (MI355X has a
// 256 MB last-level cache; measured on a 268 MB dx_disp, T = 32768 tokens of
// d = 2048, k = 2: the dispatch backward reads it in 0.077 ms instead of
// 0.126 ms; on a 1.1 GB one the dX product was 2% slower when run last)
constexpr int64_t kDxLastBytes = int64_t(512) << 20;

enum Act { ACT_RELU = 0, ACT_GELU = 1, ACT_SWIGLU = 2 };

// ---------------------------------------------------------------------------
// activations (shared by forward epilogue, backward epilogue and transposes)
// ---------------------------------------------------------------------------
// The epilogues evaluate these once per output element, so they use the
// hardware base-2 exponential and reciprocal (relative error about 1e-6,
// far below the bf16 rounding of the stored results):
//   e^x = 2^(x log2 e),  sigmoid(h) = 1 / (1 + e^-h),
//   tanh(u) = 1 - 2 / (1 + e^(2u))  (both limits exact: e^(2u) -> inf or 0),
//   and GELU as h sigmoid(2u) (limits: -0 for large negative h, where the
//   exponential overflows to inf, and h for large positive h).
__device__ __forceinline__ float exp_fast(float x) {
  return __builtin_amdgcn_exp2f(x * 1.4426950408889634f);
}
__device__ __forceinline__ float rcp_fast(float x) { return __builtin_amdgcn_rcpf(x); }
__device__ __forceinline__ float tanh_fast(float u) {
  return 1.f - 2.f * rcp_fast(1.f + exp_fast(2.f * u));
}
constexpr float kGelu1 = -2.f * 0.7978845608028654f * 1.4426950408889634f;
constexpr float kGelu3 = kGelu1 * 0.044715f;
__device__ __forceinline__ float act_f(float h, int act) {
  if (act == ACT_RELU) return fmaxf(h, 0.f);
  // GELU, tanh form: 0.5 h (1 + tanh(u)) = h sigmoid(2u) = h / (1 + e^(-2u)),
  // u = sqrt(2/pi) (h + 0.044715 h^3); -2u log2(e) = h (kGelu1 + kGelu3 h^2)
  return h * rcp_fast(1.f + __builtin_amdgcn_exp2f(h * __builtin_fmaf(kGelu3, h * h, kGelu1)));
}
__device__ __forceinline__ float act_grad_f(float h, int act) {
  if (act == ACT_RELU) return h > 0.f ? 1.f : 0.f;
  const float u = 0.7978845608028654f * (h + 0.044715f * h * h * h);
  const float th = tanh_fast(u);
  const float du = 0.7978845608028654f * (1.f + 3.f * 0.044715f * h * h);
  return 0.5f * (1.f + th) + 0.5f * h * (1.f - th * th) * du;
}
__device__ __forceinline__ float sigm(float h) { return rcp_fast(1.f + exp_fast(-h)); }
// ReLU that keeps a NaN (a maximum with 0 would hide it).
__device__ __forceinline__ float relu_nan(float h) { return h <= 0.f ? 0.f : h; }

// The gate half of the dense block: g = act(h), silu (act SWIGLU), GELU or ReLU,
// and its derivative dg.  The forward saves h3 dg and g, the factors of dA in
// dH1 = dA (h3 dg) and dH3 = dA g, so the backward evaluates no activation.
__device__ __forceinline__ void gate_f(float h, int act, float& g, float& dg) {
  if (act == ACT_SWIGLU) {
    const float sg = sigm(h);
    g = h * sg;
    dg = __builtin_fmaf(g, 1.f - sg, sg);
  } else if (act == ACT_RELU) {
    g = relu_nan(h);
    dg = h <= 0.f ? 0.f : h == h ? 1.f : h;
  } else {
    // GELU = h s with s = sigmoid(2u): s + h s (1 - s) 2u'.  Past |h| = 10 the
    // derivative is 1 or 0 to the last bit of a float; there u', whose h^2
    // grows without bound, is taken at 10
    g = act_f(h, ACT_GELU);
    const float hc = fminf(fmaxf(h, -10.f), 10.f);
    const float sg = rcp_fast(1.f + __builtin_amdgcn_exp2f(
                                        hc * __builtin_fmaf(kGelu3, hc * hc, kGelu1)));
    const float du = 1.5957691216057308f * __builtin_fmaf(3.f * 0.044715f, hc * hc, 1.f);
    dg = h == h ? __builtin_fmaf(hc * du, sg * (1.f - sg), sg) : h;
  }
}
// The activation of an int8 expert: a token that holds a NaN has scale NaN,
// and its output has to show it.
__device__ __forceinline__ float act_i8(float h, int act) {
  return act == ACT_RELU ? relu_nan(h) : act_f(h, act);
}

// ---------------------------------------------------------------------------
// schedule
// ---------------------------------------------------------------------------
// Every expert's rows are clamped to its region and to rows_alloc, and the
// tile counts to the host bounds the workspace was sized for, so no later
// kernel can index out of bounds.
__global__ __launch_bounds__(64 * kSchedTasks) void schedule_kernel(
    const int32_t* __restrict__ offsets, const int32_t* __restrict__ rows, const SchedArgs A) {
  const int g = threadIdx.x & 63, E = A.E;
  int m = 0;
  if (g < E) {
    const int64_t off = offsets[g];
    int64_t r = rows[g];
    if (off < 0 || off >= A.rows_alloc) r = 0;
    r = min(r, static_cast<int64_t>(offsets[g + 1]) - off);
    r = min(r, A.rows_alloc - off);
    m = static_cast<int>(max(r, int64_t(0)));
  }
  build_schedule<kSchedTasks>(m, A);
}

// ---------------------------------------------------------------------------
// GEMM core
// ---------------------------------------------------------------------------
// c += a * b over four k values: one 32x32 fp32 block, k = 4 consecutive
// values per lane (one 32-bit element of each of the four words)
__device__ __forceinline__ void mma_f32(floatx16& c, const uint4& a, const uint4& b) {
  c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.x), __uint_as_float(b.x), c, 0, 0, 0);
  c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.y), __uint_as_float(b.y), c, 0, 0, 0);
  c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.z), __uint_as_float(b.z), c, 0, 0, 0);
  c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.w), __uint_as_float(b.w), c, 0, 0, 0);
}

// Operand layouts.  Every product is C[m, n] = sum_k A[m, k] B[n, k]; an
// operand is stored either K-contiguous (rows are m (or n), k along each
// row: activations in the forward, weights as out x in) or K-major (rows are
// k, m along each row: the weights in the data-gradient products, and both
// operands of the weight-gradient products, which contract over the
// dispatched rows).
enum Layout { L_KC = 0, L_KM = 1 };

// One operand of one tile (byte pointers, byte strides).
//  KC: base = tile row 0 at k = 0; rows = valid tile rows.
//  KM: base = k-row 0 at tile column 0; rows = valid tile columns; k-rows at
//      or past `split` come from base2 (k counted from split), else base.
//  Gated forward (KC B only): base holds the W1 rows, base2 the W3 rows.
struct Operand {
  const char* base;
  const char* base2;
  int64_t ld;         // bytes between consecutive rows
  int rows;
  int split;
};
struct TileOps {
  Operand a, b;
  int K;              // valid k values; rows / columns / k past the valid ones read as 0
};

// KC LDS tile: row r (0..255) of 128 bytes, its 16-byte chunk c stored at
// r*128 + ((c ^ ((r >> 1) & 7)) << 4).  gfx950 LDS serves 16 lanes of a
// 16-byte access per cycle from 64 banks (256 bytes): the MFMA fragment reads
// touch 16 consecutive rows at one logical chunk; rows alternate bank halves
// and (r >> 1) & 7 spreads each half's 8 rows over its 8 slots.
__device__ __forceinline__ int swz(int row) { return (row >> 1) & 7; }
// KM LDS tile: k-row r of 256 elements, its 32-element segment g stored at
// segment g ^ (r & 3).  A transpose read takes, per 32-lane half, 4
// consecutive k-rows of one 32-element segment (64 bytes of bf16 each); the
// XOR puts those rows in 4 different quarters of the 256-byte bank space.

// Buffer resource over an operand.  Every offset used is below 2^31 (host
// limits; K-major resources are re-based every K step), so 0x80000000 is
// always out of range: a lane given that offset loads zeros, which is how
// ragged rows, columns and K tails are filled.
constexpr uint32_t kOob = 0x80000000u;
__device__ __forceinline__ __amdgpu_buffer_rsrc_t tile_rsrc(const char* base) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base), static_cast<short>(0),
                                           0x7FFFFFFF, 0x00020000);
}
#define MOE_LDS(p) ((__attribute__((address_space(3))) void*)(p))

typedef short v4s __attribute__((ext_vector_type(4)));
// 4 bf16 of one k-row run, transposed across each 16-lane group (gfx950
// ds_read_b64_tr_b16): lane i = 4a + b of a group gets element b of the run
// addressed by lanes 4r + a, for r = 0..3.
__device__ __forceinline__ uint2 read_tr(const char* p) {
  const v4s v = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (__attribute__((address_space(3))) v4s*)(p));
  return __builtin_bit_cast(uint2, v);
}

// ---------------------------------------------------------------------------
// kernel parameters
// ---------------------------------------------------------------------------
enum Mode {
  M_FWD1 = 0,        // H = X W1^T -> A = act(H) [, H saved]
  M_FWD1_SWIGLU = 1, // H1, H3 -> A = silu(H1) H3 [, H1 H3 saved]
  M_STORE = 2,       // plain store (Y, dX)
  M_BWD_DA = 3,      // dA = dY W2 -> dH = dA act'(H)
  M_BWD_DA_SWIGLU = 4,
  M_DW = 5,          // var-K weight gradient, fp32
  // on int8 operands with a scale per row of A and per row of B (ffn_i8.hip)
  M_I8_STORE = 6,          // plain store in the layer dtype
  M_I8_FWD1 = 7,           // A = act(H)
  M_I8_FWD1_SWIGLU = 8,    // A = silu(H1) H3
  // the dense gated block (gated.hip): no routing arrays, see Dense; the gate
  // half's activation at run time
  M_GATED_FWD = 9,         // H1, H3 -> A = act(H1) H3 [, H3 act'(H1) and act(H1) saved]
  M_GATED_DA = 10,         // dA = dY W2 -> dH1, dH3: dA times the saved factors
  M_ADD_STORE = 11,        // store with an addend (Y, dX), or partial sums
  M_DENSE_DW = 12,         // weight gradient in fp32 or bf16, or partial sums
  // the loss of a vocabulary projection (vocab.hip)
  M_VOCAB = 13,            // logits: each block of columns' maximum and sum of exponentials
                           // [, the exponentials saved]
  M_VOCAB_DW = 14,         // M_DENSE_DW times alpha, added to the fp32 sums of earlier pieces
  M_VOCAB_DX = 15          // store of alpha times the product, or partial sums
};
constexpr bool is_dense(int mode) { return mode >= M_GATED_FWD; }
constexpr bool is_i8(int mode) { return mode >= M_I8_STORE && mode <= M_I8_FWD1_SWIGLU; }
// W1 and W3 share a tile
constexpr bool is_gated(int mode) {
  return mode == M_FWD1_SWIGLU || mode == M_I8_FWD1_SWIGLU || mode == M_GATED_FWD;
}
constexpr bool is_dense_dw(int mode) { return mode == M_DENSE_DW || mode == M_VOCAB_DW; }
constexpr bool is_dw(int mode) { return mode == M_DW || is_dense_dw(mode); }
// bytes per operand element of the 16x16 kernels
constexpr int op_bytes(int mode) { return is_i8(mode) ? 1 : 2; }

// Scales of the rows of int8 tokens: one per row, or, with moe_dispatch's src,
// one per token (row r holds token src[r] / k of T).
struct RowScales {
  const float* scale;
  const int32_t* src;
  int T, k;
};
__device__ __forceinline__ float row_scale_at(const RowScales& s, int64_t row) {
  if (!s.src) return s.scale[row];
  return s.scale[min(max(s.src[row] / s.k, 0), s.T - 1)];
}

// A dense product: the host knows its rows, so it needs no device schedule.  Its
// tiles are those of one expert of T rows; K (the weight gradients': T) is
// split into `splits` ranges of klen, whose partial sums go to slots.
struct Dense {
  int T;        // rows of the tokens' operands
  int n_mt;     // tiles along M
  int splits, klen;
};

struct GemmParams {
  // operands (bytes).  var-M: A rows of the dispatched buffer, B the
  // expert's weights (B2: W3 of the gated forward, or the k-rows from split
  // on of a K-major B).  var-K: A and B dispatched buffers read K-major.
  const char* A; int64_t lda;
  const char* B; const char* B2; int64_t ldb; int64_t b_gstride;
  int K;              // var-M: k values
  int kmsplit;        // var-M, K-major B: first k-row taken from B2
  int N;              // output columns
  int M_out;          // var-K: output rows
  int ntiles;         // tiles along N
  int mtiles_out;     // var-K: tiles along M
  int act;
  // outputs
  char* C; int64_t ldc;           // row-major output (bytes per row)
  char* H1; char* H3; int64_t ldh; // saved / read pre-activations (bytes per row)
  int f;                           // SwiGLU: width of one half
  float* dwA; float* dwB; int64_t dw_gstride; int split_row;
  float* partial; int64_t slot_elems;
  const int32_t* offsets;
  const Sched* sched;
  const int2* mtile;
  const int4* seg;
  int mid_list;       // two-workgroups-per-CU kernels: the tile list
  int dw_h;           // and the units of a weight-gradient tile
  const char* add; int64_t ldadd;  // M_ADD_STORE: addend (NULL: none), bytes per row
  // int8 operands: scales of A's rows and of the rows of B and B2 (per expert
  // s_gstride apart); fp32 outputs
  RowScales a_scale; const float* b_scale; const float* b2_scale; int64_t s_gstride;
  int out_f32;
  Dense dense;
  // M_VOCAB: per row n_stat blocks of columns {maximum, sum of exp(l - maximum)}, the
  // tokens' targets and their logits; C: the exponentials, or NULL.
  // M_VOCAB_DW: the earlier pieces' sums (NULL: none)
  float alpha;
  float2* stat; int n_stat;
  const int32_t* target; float* target_logit;
  const float* acc;
};

// The exponentials of M_VOCAB in 16 bits: fp16 of 2^15 exp(l - maximum), so that their 11
// bits hold down to 2^-29.
constexpr int kVocabLift = 15;

// Tile order, two levels above each XCD's kGroupM x 8 block of tiles.
// Tiles come in bands of kBandM M-tiles; inside a band, in N-blocks of 8
// columns, and inside an N-block, in M-blocks of kGroupM rows whose tiles
// run M fastest.  The blocks of one N-block follow each other, so the 8
// blocks in flight at once (one per XCD) are 2 N-blocks x 4 M-blocks: 16 x
// 16 tiles that read 16 + 16 operand panels, against 4 + 64 when the XCDs
// take 8 N-blocks of the same 4 M-tiles, and a band's A panels stay in the
// last-level cache while its weight panels stream past.  Partial bands and
// blocks at the edges keep the same order with fewer rows or columns.
constexpr int kBandM = 4 * kGroupM;
__device__ __forceinline__ void decode_banded(int L, int n_mt, int n_nt, int& mt, int& nt) {
  const int full_bands = n_mt / kBandM;
  int r, m0, bh;
  if (L < full_bands * kBandM * n_nt) {
    const int band = L / (kBandM * n_nt);
    r = L - band * kBandM * n_nt;
    m0 = band * kBandM;
    bh = kBandM;
  } else {
    r = L - full_bands * kBandM * n_nt;
    m0 = full_bands * kBandM;
    bh = n_mt - m0;
  }
  const int full_nb = n_nt / 8;
  int n0, w;
  if (r < full_nb * 8 * bh) {
    const int nb = r / (8 * bh);
    r -= nb * 8 * bh;
    n0 = nb * 8;
    w = 8;
  } else {
    r -= full_nb * 8 * bh;
    n0 = full_nb * 8;
    w = n_nt - n0;
  }
  const int full_mb = bh / kGroupM;
  int h;
  if (r < full_mb * kGroupM * w) {
    const int mb = r / (kGroupM * w);
    r -= mb * kGroupM * w;
    m0 += mb * kGroupM;
    h = kGroupM;
  } else {
    r -= full_mb * kGroupM * w;
    m0 += full_mb * kGroupM;
    h = bh - full_mb * kGroupM;
  }
  mt = m0 + r % h;
  nt = n0 + r / h;
}

// The products: PASS names the instance (so each is its own kernel in
// traces) and fixes the operand layouts.
// P_BWD_DX_T is dX with the weights read from a transposed copy,
// K-contiguous like the forward's operands.
enum Pass {
  P_FWD_H = 0, P_FWD_Y = 1, P_BWD_DA = 2, P_BWD_DX = 3, P_BWD_DW2 = 4, P_BWD_DW13 = 5,
  P_BWD_DX_T = 6, P_VOCAB = 7, P_VOCAB_DX = 8, P_VOCAB_DW = 9
};
__host__ __device__ constexpr int a_layout(int pass) {
  return pass == P_BWD_DW2 || pass == P_BWD_DW13 || pass == P_VOCAB_DW ? L_KM : L_KC;
}
__host__ __device__ constexpr int b_layout(int pass) {
  return pass == P_BWD_DA || pass == P_BWD_DX || pass == P_BWD_DW2 || pass == P_BWD_DW13 ||
                 pass == P_VOCAB_DX || pass == P_VOCAB_DW
             ? L_KM
             : L_KC;
}

// ---------------------------------------------------------------------------
// bf16 products: four wavefronts of 128x128
// ---------------------------------------------------------------------------
// bf16 layers run every product on 4 wavefronts, one per SIMD, each holding a
// 128x128 block of the 256x256 tile as 64 blocks of 16x16 fp32 accumulators
// (v_mfma_f32_16x16x32_bf16, 256 accumulation registers).  Per K step of 64
// there are two barriers, one after the A and one after the B fragment reads
// of the step's stage.  Between the MFMAs each wave issues, one at a time,
// the fragment reads of the next half step and, once a barrier has freed its
// part of the stage, its share of the direct-to-LDS loads of the step after
// next, so the memory pipeline sees a steady stream of requests while the
// matrix core stays busy.  A 128x128 block reads a third less LDS per MFMA
// than a 128x64 one.
constexpr int kThreads16 = 256;

typedef int intx4 __attribute__((ext_vector_type(4)));

// c += a * b for one 16x16 block.  Lane l = 16 G + c16 supplies row c16 of
// the A and B sub-blocks at k = 8 G .. 8 G + 7 and holds rows 4 G .. 4 G + 3,
// column c16 of the result.  Inline assembly keeps each accumulator in place
// in its accumulation registers through the K loop (compiled MFMAs get their
// accumulators shuffled between loop iterations).  The compiler inserts no
// wait states around it, and none are needed inside the loops:
//  * an accumulator updated again, 64 MFMAs later on 256x256 tiles and 4 RB
//    later on the others (4 at the least), is read as the very registers the
//    earlier MFMA writes, which the hardware forwards without wait states;
//  * an MFMA has read its A and B registers before an LDS read issued after it
//    can return into them (on the smallest tile the next stage's first A
//    fragment is requested right behind the last MFMA that used the registers);
//  * fragments read from LDS are waited for by the compiler, as operands.
// The epilogue waits before it reads the accumulators.
__device__ __forceinline__ void mfma16(floatx4& c, const uint4& a, const uint4& b) {
  asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0"
               : "+a"(c)
               : "v"(__builtin_bit_cast(intx4, a)), "v"(__builtin_bit_cast(intx4, b)));
}

// The same on int8: 64 products of whole numbers per lane pair, four int32
// sums, which the floatx4 carries as bits (0.f is 0).  A fragment is the same
// 16 bytes per lane (k = 16 G .. 16 G + 15), so tiles, loads and fragment
// reads are those of bf16 with twice the k values per 128-byte row.
__device__ __forceinline__ void mfma16_i8(floatx4& c, const uint4& a, const uint4& b) {
  asm volatile("v_mfma_i32_16x16x64_i8 %0, %1, %2, %0"
               : "+a"(c)
               : "v"(__builtin_bit_cast(intx4, a)), "v"(__builtin_bit_cast(intx4, b)));
}
template <int ES>
__device__ __forceinline__ void mfma_es(floatx4& c, const uint4& a, const uint4& b) {
  if constexpr (ES == 1) mfma16_i8(c, a, b);
  else mfma16(c, a, b);
}

// acc += A_tile * B_tile^T over the whole K extent (see above).  Wave w owns
// tile rows 128 (w >> 1) .. +127 and columns 128 (w & 1) .. +127 (gated
// forward: hidden units 64 (w & 1) .. +63 of W1, then the same units of W3).
// The four stage objects are distinct, and the loop is unrolled by two so
// every LDS access names its object statically: the compiler can then tell
// the loads into one stage from the reads of the other.
template <int ALAY, int BLAY, bool GATED, bool FULL, int ES>
__device__ __forceinline__ void mainloop16(const TileOps& op, char* la0, char* lb0, char* la1,
                                           char* lb1, floatx4 (&acc)[8][8], int zt) {
  static_assert(ES == 2 || (ALAY == L_KC && BLAY == L_KC), "int8 operands are K-contiguous");
  constexpr int KSTEP = kRowBytes / ES;
  const int lane = (static_cast<int>(threadIdx.x) & 63) + zt;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
  const int wm = wave >> 1, wn = wave & 1;
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
  const int K = op.K;
  const int nk = (K + KSTEP - 1) / KSTEP;
  if (nk <= 0) return;
  const int nk2 = (nk + 1) & ~1;   // odd counts load one all-zero step

  // ---- loads: 1 KB blocks (8 rows of a KC tile: lane l -> row l >> 3,
  // physical chunk l & 7; or 2 k-rows of a KM tile: lane l -> k-row l >> 5,
  // physical elements 8 (l & 31) .. +7); wave w loads blocks 8w .. 8w+7 of
  // A (g = 0..7) and of B (g = 8..15) of every stage.
  const int l3 = lane >> 3;
  const int co0 = ((lane & 7) ^ swz(l3)) * 16, co1 = ((lane & 7) ^ swz(l3 + 8)) * 16;
  const int kr = lane >> 5;            // KM: k-row within the block
  const int pe = (lane & 31) * 8;      // KM: physical element within the k-row
  auto km_col = [&](int q) { return (((pe >> 5) ^ q) << 5) + (pe & 31); };
  const __amdgpu_buffer_rsrc_t ra_t = tile_rsrc(op.a.base);
  const __amdgpu_buffer_rsrc_t rb_t = tile_rsrc(op.b.base);
  const __amdgpu_buffer_rsrc_t rb3_t = tile_rsrc(GATED ? op.b.base2 : op.b.base);
  auto km_rsrc = [&](const Operand& o, int kt, bool second) {
    const int64_t k = static_cast<int64_t>(kt) * KSTEP - (second ? o.split : 0);
    return tile_rsrc((second ? o.base2 : o.base) + k * o.ld);
  };
  // the resources and flags of one K step, set once per step
  struct StepLd {
    __amdgpu_buffer_rsrc_t ra, ra2, rb, rb2;
    int kt;
    bool kfull, kany;
  };
  auto step_ld = [&](int kt) {
    StepLd s;
    s.kt = kt;
    s.kfull = (kt + 1) * KSTEP <= K;
    s.kany = kt * KSTEP < K;
    s.ra = ra_t; s.ra2 = ra_t; s.rb = rb_t; s.rb2 = rb3_t;
    if constexpr (ALAY == L_KM) {
      s.ra = km_rsrc(op.a, kt, false);
      s.ra2 = op.a.base2 ? km_rsrc(op.a, kt, true) : s.ra;
    }
    if constexpr (BLAY == L_KM) {
      s.rb = km_rsrc(op.b, kt, false);
      s.rb2 = op.b.base2 ? km_rsrc(op.b, kt, true) : s.rb;
    }
    return s;
  };
  // block blk of operand o (layout LAY) of step s.kt into dst
  auto load_blk = [&](auto lay, const Operand& o, const __amdgpu_buffer_rsrc_t& rs,
                      const __amdgpu_buffer_rsrc_t& rs2, char* dst, int blk, const StepLd& s,
                      bool gated) {
    constexpr int LAY = decltype(lay)::value;
    const int ld = static_cast<int>(o.ld);
    uint32_t off;
    int soff;
    bool second = false;
    if constexpr (LAY == L_KC) {
      const int co = (blk & 1) ? co1 : co0;
      // gated forward: 64-row groups alternate W1 / W3 rows of 64 hidden units
      const int row0 = gated ? (blk >> 4) * 64 + (blk & 7) * 8 : blk * 8;
      second = gated && ((blk >> 3) & 1);
      off = static_cast<uint32_t>(l3 * ld) + co;
      soff = row0 * ld + s.kt * kRowBytes;
      if (!FULL || !s.kfull) {
        const bool ok = (FULL || row0 + l3 < o.rows) && (s.kfull || s.kt * kRowBytes + co < K * ES);
        if (!ok) off = kOob;
      }
    } else {
      const int krel = 2 * blk;                  // first k-row of the block in the step
      const int kabs = s.kt * KSTEP + krel;
      const int q = (krel + kr) & 3;
      const int col = km_col(q);
      second = kabs >= o.split;
      off = static_cast<uint32_t>(kr * ld + col * 2);
      soff = krel * ld;
      if (!FULL || !s.kfull) {
        const bool ok = (FULL || col < o.rows) && (s.kfull || kabs + kr < K);
        if (!ok) off = kOob;
      }
    }
    if (!s.kany) off = kOob;
    if (second)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs2, MOE_LDS(dst + blk * 1024), 16, off, soff, 0, 0);
    else
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, MOE_LDS(dst + blk * 1024), 16, off, soff, 0, 0);
  };
  using KC_ = std::integral_constant<int, L_KC>;
  using KM_ = std::integral_constant<int, L_KM>;
  // one of the wave's 16 loads of a stage
  auto load1 = [&](const StepLd& s, char* sa, char* sb, int g) {
    const int blk = wave * 8 + (g & 7);
    if (g < 8) {
      if constexpr (ALAY == L_KC) load_blk(KC_{}, op.a, s.ra, s.ra2, sa, blk, s, false);
      else load_blk(KM_{}, op.a, s.ra, s.ra2, sa, blk, s, false);
    } else {
      if constexpr (BLAY == L_KC) load_blk(KC_{}, op.b, s.rb, s.rb2, sb, blk, s, GATED);
      else load_blk(KM_{}, op.b, s.rb, s.rb2, sb, blk, s, false);
    }
  };

  // ---- fragments.  KC: lane l = 16 G + c16 reads row c16 of a 16-row block,
  // logical chunk 4h + G (k = 32h + 8G .. +7) of the 128-byte row; the row's
  // swizzle is (c16 >> 1) since blocks start at multiples of 16.
  const int c16 = lane & 15, G = lane >> 4;
  const int fa_kc = (wm * 128 + c16) * kRowBytes, fb_kc = (wn * 128 + c16) * kRowBytes;
  // KM: two transpose reads, k-rows 32h + 8G + (c16 >> 2) and 4 below, columns
  // cb + 4 (c16 & 3) .. +3 (lane 4a + b of a 16-lane group then holds column
  // cb + 4a + b at 4 consecutive k); segment swizzle by k & 3 = c16 >> 2
  auto km_frag = [&](const char* st, int cb, int h) -> uint4 {
    const int phys = (((cb >> 5) ^ (c16 >> 2)) << 5) + (cb & 31) + 4 * (c16 & 3);
    const char* p0 = st + (32 * h + 8 * G + (c16 >> 2)) * 512 + phys * 2;
    const uint2 lo = read_tr(p0);
    const uint2 hi = read_tr(p0 + 4 * 512);
    return make_uint4(lo.x, lo.y, hi.x, hi.y);
  };
  // fragment g of half h: A sub-block g (g < 8) or B sub-block g - 8
  auto read1 = [&](const char* sa, const char* sb, int h, uint4 (&fa)[8], uint4 (&fb)[8], int g) {
    const int sw = ((4 * h + G) ^ (c16 >> 1)) << 4;
    if (g < 8) {
      if constexpr (ALAY == L_KC)
        fa[g] = *reinterpret_cast<const uint4*>(sa + fa_kc + g * 16 * kRowBytes + sw);
      else
        fa[g] = km_frag(sa, wm * 128 + g * 16, h);
    } else {
      if constexpr (BLAY == L_KC)
        fb[g - 8] = *reinterpret_cast<const uint4*>(sb + fb_kc + (g - 8) * 16 * kRowBytes + sw);
      else
        fb[g - 8] = km_frag(sb, wn * 128 + (g - 8) * 16, h);
    }
  };
  uint4 f0a[8], f0b[8], f1a[8], f1b[8];   // fragments of k-half 0 / 1 of a stage

  // Every wave runs the same instruction stream on every tile: rows, columns
  // and K past the valid ones were loaded as zeros, so a wave with no valid
  // rows or columns multiplies zeros, and the epilogue stores none of them.
  // (Skipping such a wave's reads and MFMAs with a branch per group broke
  // the interleaving for the whole tile: a partial tile then took several
  // times as long as a full one.)

  // One K step from stage (ca, cb), the next stage in (na, nb); the loads of
  // step kt + 2 go into (ca, cb): its A part once every wave has read the A
  // fragments of k-half 1, its B part once every wave has read the B ones.
  // Two barriers per step let the 16 loads spread over the last three
  // quarters of the step (one per 6 MFMAs) instead of crowding into the
  // second half.
  auto step = [&](int kt, char* ca, char* cb, const char* na, const char* nb) {
    const StepLd s = step_ld(kt + 2);
    // first quarter: MFMAs 0..31 of k-half 0, reads of the A fragments of k-half 1
#pragma unroll
    for (int g = 0; g < 8; ++g) {
      read1(ca, cb, 1, f1a, f1b, g);
#pragma unroll
      for (int m = 4 * g; m < 4 * g + 4; ++m) mfma_es<ES>(acc[m >> 3][m & 7], f0a[m >> 3], f0b[m & 7]);
      __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    // second quarter: MFMAs 32..63 of k-half 0, reads of the B fragments of
    // k-half 1, the A loads of step kt + 2
#pragma unroll
    for (int g = 8; g < 16; ++g) {
      // A loads 0..5 at groups 8, 9, 11, 12, 14, 15
      if (g % 3 != 1) load1(s, ca, cb, g - 8 - (g - 8) / 3);
      read1(ca, cb, 1, f1a, f1b, g);
#pragma unroll
      for (int m = 4 * g; m < 4 * g + 4; ++m) mfma_es<ES>(acc[m >> 3][m & 7], f0a[m >> 3], f0b[m & 7]);
      __builtin_amdgcn_sched_barrier(0);
    }
    // stage kt + 1 has landed (only the 6 A loads just issued may be pending)
    __builtin_amdgcn_s_waitcnt(0x0076);   // vmcnt(6) lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    // second half: MFMAs of k-half 1, reads of the next stage's k-half 0, the
    // B loads of step kt + 2
#pragma unroll
    for (int g = 0; g < 16; ++g) {
      // A loads 6, 7 and the B loads at groups 0, 2, 3, 5, 6, 8, 9, 11, 12, 14
      if (g % 3 != 1 && g < 15) load1(s, ca, cb, 6 + g - (g + 1) / 3);
      read1(na, nb, 0, f0a, f0b, g);
#pragma unroll
      for (int m = 4 * g; m < 4 * g + 4; ++m) mfma_es<ES>(acc[m >> 3][m & 7], f1a[m >> 3], f1b[m & 7]);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  {
    const StepLd s0 = step_ld(0), s1 = step_ld(1);
#pragma unroll
    for (int g = 0; g < 16; ++g) load1(s0, la0, lb0, g);
#pragma unroll
    for (int g = 0; g < 16; ++g) load1(s1, la1, lb1, g);
  }
  __builtin_amdgcn_s_waitcnt(0x4F70);   // vmcnt(16): this wave's stage-0 loads landed
  __builtin_amdgcn_s_barrier();
#pragma unroll
  for (int g = 0; g < 16; ++g) read1(la0, lb0, 0, f0a, f0b, g);
  for (int kt = 0; kt < nk2; kt += 2) {
    step(kt, la0, lb0, la1, lb1);
    step(kt + 1, la1, lb1, la0, lb0);
  }
  __builtin_amdgcn_s_waitcnt(0x0070);
  __builtin_amdgcn_s_barrier();   // every load landed, every read done: stages are free
  // the epilogue reads the accumulators with ordinary instructions
  asm volatile("s_nop 7\n\ts_nop 7\n\ts_nop 7" ::: "memory");
}

// ---------------------------------------------------------------------------
// bf16 products on tiles of 32 to 192 rows, two workgroups per CU
// ---------------------------------------------------------------------------
// The 256x256 kernel holds one wavefront per SIMD (256 accumulation
// registers), so a tile's prologue and epilogue leave the matrix cores idle,
// and its tiles are so large that the last round of them often leaves many
// CUs idle: on short K, few tiles per CU, or an epilogue heavy in VALU work
// that idle time is a large share.  This kernel computes tiles of 128
// columns and RB units of 32 rows (RB = 1 .. 6, per tile) with 4 wavefronts
// of 16 RB x 64 (16 RB accumulation registers, under 256 registers in all)
// and 80 KB of LDS, so two workgroups share each CU and one's epilogue
// overlaps the other's MFMAs.  The heights let the schedule spread an
// expert's rows evenly over just as many tiles as fill whole rounds.  It
// reads more operand bytes per flop than the 256x256 tile, which is why
// large products keep the big tile.  The K loop has the same structure: two
// stages of K 64, two barriers per step, loads and fragment reads issued one
// at a time between the MFMAs.
//
// Wave w owns tile rows 16 RB (w >> 1) .. and columns 64 (w & 1) .. +63
// (gated forward: hidden units 32 (w & 1) .. +31 of W1, then the same units
// of W3).  KC LDS tiles are rows of 128 bytes with the swizzle of the big
// tile; KM tiles are 64 k-rows of 128 elements (256 bytes) with the same XOR
// of 32-element segments by k mod 4 (KM A operands: RB = 4 only).
constexpr int wait_vm_lgkm0(int vm) { return (vm & 15) | ((vm >> 4) << 14) | 0x70; }
constexpr int wait_vm(int vm) { return (vm & 15) | ((vm >> 4) << 14) | 0xF70; }

template <int RB, int ALAY, int BLAY, bool GATED, int ES>
__device__ __forceinline__ void mainloop_mid(const TileOps& op, char* la0, char* lb0, char* la1,
                                             char* lb1, floatx4 (&acc)[RB][4], int zt) {
  static_assert(ALAY == L_KC || RB == 4, "K-major A tiles are 128 columns wide");
  static_assert(ES == 2 || (ALAY == L_KC && BLAY == L_KC), "int8 operands are K-contiguous");
  constexpr int KSTEP = kRowBytes / ES;
  constexpr int KMROW = 256;           // bytes per k-row of a KM tile
  constexpr int NM = 4 * RB;           // MFMAs per k-half: one per accumulator
  static_assert(NM >= 4, "updates of one accumulator are at least 4 MFMAs apart");
  const int lane = (static_cast<int>(threadIdx.x) & 63) + zt;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
  const int wm = wave >> 1, wn = wave & 1;
#pragma unroll
  for (int i = 0; i < RB; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
  const int K = op.K;
  const int nk = (K + KSTEP - 1) / KSTEP;
  if (nk <= 0) return;
  const int nk2 = (nk + 1) & ~1;   // odd counts load one all-zero step

  // ---- loads: 1 KB blocks (8 rows of a KC tile: lane l -> row l >> 3,
  // physical chunk l & 7; or 4 k-rows of a KM tile: lane l -> k-row l >> 4,
  // physical elements 8 (l & 15) .. +7); of every stage, wave w loads blocks
  // 4i + w of A (i < RB) and of B (i < 4).  A lane's offset within a block
  // has bit 31 set (out of range, reads zeros) where the block's row or
  // column is past the valid ones; past K and past the last step the bit is
  // or-ed in per step.
  const int l3 = lane >> 3;
  const int co = ((lane & 7) ^ swz(l3 + (wave & 1) * 8)) * 16;   // block 4i + w: rows 8(4i + w) + l3
  const int kr = lane >> 4;            // KM: k-row within the block (= k mod 4)
  const int pe = (lane & 15) * 8;      // KM: physical element within the k-row
  const int km_col = (((pe >> 5) ^ kr) << 5) + (pe & 31);
  const __amdgpu_buffer_rsrc_t ra_t = tile_rsrc(op.a.base);
  const __amdgpu_buffer_rsrc_t rb_t = tile_rsrc(op.b.base);
  const __amdgpu_buffer_rsrc_t rb3_t = tile_rsrc(GATED ? op.b.base2 : op.b.base);
  const int lda = static_cast<int>(op.a.ld), ldb = static_cast<int>(op.b.ld);
  auto bad = [](bool b) { return static_cast<uint32_t>(b) << 31; };
  uint32_t offa[ALAY == L_KC ? RB : 1], offb[BLAY == L_KC ? 4 : 1];
  if constexpr (ALAY == L_KC) {
#pragma unroll
    for (int i = 0; i < RB; ++i)
      offa[i] = static_cast<uint32_t>(l3 * lda + co) | bad((4 * i + wave) * 8 + l3 >= op.a.rows);
  } else {
    offa[0] = static_cast<uint32_t>(kr * lda + km_col * 2) | bad(km_col >= op.a.rows);
  }
  // gated: block 4i + w holds rows (hidden units) 32 (i >> 1) + 8w .. +7 of
  // W1 (i even) or W3 (i odd)
  auto brow = [&](int i) { return GATED ? (i >> 1) * 32 + wave * 8 : (4 * i + wave) * 8; };
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
  // what the loads of one K step share: resources of K-major operands, and
  // for K-contiguous ones the lane's K-tail bit
  struct StepLd {
    __amdgpu_buffer_rsrc_t ra, rb, rb2;
    uint32_t kbad;
    int kt;
  };
  auto step_ld = [&](int kt) {
    StepLd s;
    s.kt = kt;
    s.ra = ra_t; s.rb = rb_t; s.rb2 = rb3_t;
    s.kbad = bad(kt * kRowBytes + co >= K * ES);
    if constexpr (ALAY == L_KM) s.ra = km_rsrc(op.a, kt, false);
    if constexpr (BLAY == L_KM) {
      s.rb = km_rsrc(op.b, kt, false);
      s.rb2 = op.b.base2 ? km_rsrc(op.b, kt, true) : s.rb;
    }
    return s;
  };
  auto issue = [&](const __amdgpu_buffer_rsrc_t& rs, char* dst, uint32_t off, int soff) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, MOE_LDS(dst), 16, off, soff, 0, 0);
  };
  auto load_a = [&](const StepLd& s, char* sa, int i) {
    const int blk = 4 * i + wave;
    if constexpr (ALAY == L_KC)
      issue(s.ra, sa + blk * 1024, offa[i] | s.kbad, blk * 8 * lda + s.kt * kRowBytes);
    else
      issue(s.ra, sa + blk * 1024, offa[0] | bad(s.kt * KSTEP + 4 * blk + kr >= K), 4 * blk * lda);
  };
  auto load_b = [&](const StepLd& s, char* sb, int i) {
    const int blk = 4 * i + wave;
    if constexpr (BLAY == L_KC) {
      if (GATED && (i & 1))
        issue(s.rb2, sb + blk * 1024, offb[i] | s.kbad, brow(i) * ldb + s.kt * kRowBytes);
      else
        issue(s.rb, sb + blk * 1024, offb[i] | s.kbad, brow(i) * ldb + s.kt * kRowBytes);
    } else {
      const int kabs = s.kt * KSTEP + 4 * blk;   // split is a multiple of 8: no block straddles it
      const uint32_t off = offb[0] | bad(kabs + kr >= K);
      if (kabs >= op.b.split) issue(s.rb2, sb + blk * 1024, off, 4 * blk * ldb);
      else issue(s.rb, sb + blk * 1024, off, 4 * blk * ldb);
    }
  };

  // ---- fragments (as in the 256x256 kernel; KM k-rows are 256 bytes)
  const int c16 = lane & 15, G = lane >> 4;
  const int fa_kc = (wm * 16 * RB + c16) * kRowBytes, fb_kc = (wn * 64 + c16) * kRowBytes;
  auto km_frag = [&](const char* st, int cb, int h) -> uint4 {
    const int phys = (((cb >> 5) ^ (c16 >> 2)) << 5) + (cb & 31) + 4 * (c16 & 3);
    const char* p0 = st + (32 * h + 8 * G + (c16 >> 2)) * KMROW + phys * 2;
    const uint2 lo = read_tr(p0);
    const uint2 hi = read_tr(p0 + 4 * KMROW);
    return make_uint4(lo.x, lo.y, hi.x, hi.y);
  };
  auto read_a = [&](const char* sa, int h, uint4 (&fa)[RB], int i) {
    const int sw = ((4 * h + G) ^ (c16 >> 1)) << 4;
    if constexpr (ALAY == L_KC)
      fa[i] = *reinterpret_cast<const uint4*>(sa + fa_kc + i * 16 * kRowBytes + sw);
    else
      fa[i] = km_frag(sa, wm * 64 + i * 16, h);
  };
  auto read_b = [&](const char* sb, int h, uint4 (&fb)[4], int j) {
    const int sw = ((4 * h + G) ^ (c16 >> 1)) << 4;
    if constexpr (BLAY == L_KC)
      fb[j] = *reinterpret_cast<const uint4*>(sb + fb_kc + j * 16 * kRowBytes + sw);
    else
      fb[j] = km_frag(sb, wn * 64 + j * 16, h);
  };
  uint4 f0a[RB], f0b[4], f1a[RB], f1b[4];

  // One K step from stage (ca, cb), the next stage in (na, nb); the loads of
  // step kt + 2 go into (ca, cb).  MFMA m is block (m >> 2, m & 3).  The
  // first quarter reads the A fragments of k-half 1, the second the B
  // fragments and issues the A loads, the second half reads the next stage's
  // k-half 0 and issues the B loads.
  auto step = [&](int kt, char* ca, char* cb, const char* na, const char* nb) {
    const StepLd s = step_ld(kt + 2);
#pragma unroll
    for (int i = 0; i < RB; ++i) {
      read_a(ca, 1, f1a, i);
#pragma unroll
      for (int m = 2 * i; m < 2 * i + 2; ++m) mfma_es<ES>(acc[m >> 2][m & 3], f0a[m >> 2], f0b[m & 3]);
      __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int q = 0; q < 2 * RB; ++q) {
      if ((q & 1) == 0) load_a(s, ca, q >> 1);
      // B fragments spread over the quarter (RB = 1: two per MFMA)
#pragma unroll
      for (int j = 4 * q / (2 * RB); j < 4 * (q + 1) / (2 * RB); ++j) read_b(cb, 1, f1b, j);
      const int m = 2 * RB + q;
      mfma_es<ES>(acc[m >> 2][m & 3], f0a[m >> 2], f0b[m & 3]);
      __builtin_amdgcn_sched_barrier(0);
    }
    // stage kt + 1 has landed (only the RB A loads just issued may be pending)
    __builtin_amdgcn_s_waitcnt(wait_vm_lgkm0(RB));
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int m = 0; m < NM; ++m) {
      if (m % RB == 0) load_b(s, cb, m / RB);
#pragma unroll
      for (int r = (RB + 4) * m / NM; r < (RB + 4) * (m + 1) / NM; ++r) {
        if (r < RB) read_a(na, 0, f0a, r);
        else read_b(nb, 0, f0b, r - RB);
      }
      mfma_es<ES>(acc[m >> 2][m & 3], f1a[m >> 2], f1b[m & 3]);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  {
    const StepLd s0 = step_ld(0), s1 = step_ld(1);
#pragma unroll
    for (int i = 0; i < RB; ++i) load_a(s0, la0, i);
#pragma unroll
    for (int i = 0; i < 4; ++i) load_b(s0, lb0, i);
#pragma unroll
    for (int i = 0; i < RB; ++i) load_a(s1, la1, i);
#pragma unroll
    for (int i = 0; i < 4; ++i) load_b(s1, lb1, i);
  }
  __builtin_amdgcn_s_waitcnt(wait_vm(RB + 4));   // this wave's stage-0 loads landed
  __builtin_amdgcn_s_barrier();
#pragma unroll
  for (int i = 0; i < RB; ++i) read_a(la0, 0, f0a, i);
#pragma unroll
  for (int j = 0; j < 4; ++j) read_b(lb0, 0, f0b, j);
  for (int kt = 0; kt < nk2; kt += 2) {
    step(kt, la0, lb0, la1, lb1);
    step(kt + 1, la1, lb1, la0, lb0);
  }
  __builtin_amdgcn_s_waitcnt(0x0070);
  __builtin_amdgcn_s_barrier();   // every load landed, every read done: stages are free
  asm volatile("s_nop 7\n\ts_nop 7\n\ts_nop 7" ::: "memory");
}

// A wave's block of RB x CB blocks of 16x16, 2 x 2 waves per workgroup.
template <int RB_, int CB_> struct Tile16 {
  static constexpr int RB = RB_, CB = CB_;
  static constexpr int WR = 16 * RB, WC = 16 * CB;      // wave block
  static constexpr int TM = 2 * WR, TN = 2 * WC;        // workgroup tile
  static constexpr int kP = WC + 4;                     // strip pitch (floats): rows 4 apart
                                                        // fall 16 banks apart
  static constexpr int kStripBytes = 16 * kP * 4;
};
using TileBig = Tile16<8, 8>;
static_assert(TileBig::TM == BM && TileBig::TN == BN, "tile size");
static_assert(2 * TileBig::kStripBytes <= kTileBytes, "two staging strips per operand buffer");
static_assert(2 * Tile16<1, 4>::kStripBytes <= kMidN * kRowBytes, "two staging strips per buffer");
static_assert(Tile16<1, 4>::TN == kMidN && Tile16<1, 4>::TM == kMidUnit, "mid tile size");

// LDS of a wave's strip: 16 padded rows; M_VOCAB 32 rows of WC.
template <int MODE, typename C> constexpr int strip_bytes() {
  static_assert(2 * 32 * Tile16<1, 4>::WC * 4 <= kMidN * kRowBytes && 2 * 32 * TileBig::WC * 4 <= kTileBytes, "fits");
  return MODE == M_VOCAB ? 32 * C::WC * 4 : C::kStripBytes;
}
// Stage rows 16i .. 16i+15 of the wave's accumulators as fp32, row pitch C::kP.
template <typename C>
__device__ __forceinline__ void stage16(float* strip, const floatx4 (&acc)[C::RB][C::CB], int i,
                                        int lane) {
  const int c16 = lane & 15, G = lane >> 4;
#pragma unroll
  for (int j = 0; j < C::CB; ++j)
#pragma unroll
    for (int q = 0; q < 4; ++q) strip[(4 * G + q) * C::kP + 16 * j + c16] = acc[i][j][q];
}

// M_VOCAB: N neighbouring lanes hold a block of columns of row `row`, CN logits v each (-inf
// for none): their maximum m and the sum of exp(l - m), written by the lane `lead`; v becomes
// 2^LIFT exp(l - m).
template <int N, int CN, int LIFT>
__device__ __forceinline__ void vocab_row(const GemmParams& p, float (&v)[CN], int row, bool ok, int block,
                                          bool lead) {
  float m = v[0];
#pragma unroll
  for (int e = 1; e < CN; ++e) m = fmaxf(m, v[e]);
  m = group_max<N>(m);
  const float from = m == -INFINITY ? 0.f : m;   // (no column, or all of them -inf: zeros)
  float s = 0.f;
#pragma unroll
  for (int e = 0; e < CN; ++e) {
    v[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(v[e] - from, 1.4426950408889634f, LIFT));
    s += v[e];
  }
  s = group_sum<N>(s);
  if (ok && lead)
    p.stat[static_cast<int64_t>(row) * p.n_stat + block] = make_float2(m, s * (1.f / (1 << LIFT)));
}

// Epilogue of one wave's block (RB x CB blocks of C): 16 accumulator rows at
// a time go through the wave's LDS strip; a lane then finishes 8 consecutive
// columns of a row and writes them as one vector (bf16) or two (fp32 weight
// gradients).  el: the lane index, derived like the strip address from an
// opaque zero the caller produces after its K loop, so nothing the epilogue
// computes per lane is hoisted and held in registers across the K loop.
// empty: a weight-gradient tile with no rows to contract over.
template <int MODE, typename C>
__device__ __forceinline__ void epilogue16(const GemmParams& p,
                                           const floatx4 (&acc)[C::RB][C::CB], float* strip,
                                           int el, int wm, int wn, int g, int slot, int row0,
                                           int m_valid, int n0, bool empty) {
  constexpr int WR = C::WR, WC = C::WC, kP = C::kP;
  using T = uint16_t;
  constexpr int ES = 2;
  const int wr0 = wm * WR;                      // the wave's first tile row
  // weight gradients: where the fp32 result of tile row orow, column gc goes
  // (a split partial-sum slot, or the first or second gradient array)
  auto dw_dst = [&](int orow, int gc) -> float* {
    if (slot >= 0)
      return p.partial + static_cast<int64_t>(slot) * p.slot_elems +
             static_cast<int64_t>(orow) * p.N + gc;
    if (orow < p.split_row)
      return p.dwA + static_cast<int64_t>(g) * p.dw_gstride + static_cast<int64_t>(orow) * p.N + gc;
    return p.dwB + static_cast<int64_t>(g) * p.dw_gstride +
           static_cast<int64_t>(orow - p.split_row) * p.N + gc;
  };
  // M_DENSE_DW, no partial sums: one expert, results in bf16
  auto dw_dst16 = [&](int orow, int gc) -> uint16_t* {
    return orow < p.split_row
               ? reinterpret_cast<uint16_t*>(p.dwA) + static_cast<int64_t>(orow) * p.N + gc
               : reinterpret_cast<uint16_t*>(p.dwB) + static_cast<int64_t>(orow - p.split_row) * p.N + gc;
  };
  if constexpr (is_dw(MODE)) {
    if (empty) {
      // no rows to contract over (a split expert's last segment may be
      // empty): the tile is zero; each lane stores 8 zeros per row pass straight to memory,
      // with no staging, so the tile costs only its stores.  Every wave
      // of the workgroup takes this path, and none touched the LDS.
      constexpr int LR = WC / 8, RG = 64 / LR;
      const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
      for (int r = 0; r < WR; r += RG) {
        const int lm = wr0 + r + el / LR, gc = n0 + wn * WC + (el % LR) * 8;
        if (lm < m_valid && gc < p.N) {
          if (is_dense_dw(MODE) && slot < 0 && !p.out_f32) {
            *reinterpret_cast<uint4*>(dw_dst16(row0 + lm, gc)) = make_uint4(0, 0, 0, 0);
            continue;
          }
          float* dst = dw_dst(row0 + lm, gc);
          *reinterpret_cast<float4*>(dst) = zero;
          *reinterpret_cast<float4*>(dst + 4) = zero;
        }
      }
      return;
    }
  }
  // ReLU / GELU layers: the epilogue is specialised on the activation, one
  // uniform branch per tile instead of one per element
  auto epilogue = [&](auto act_c) {
  constexpr int ACT = decltype(act_c)::value;
  if constexpr (MODE == M_FWD1_SWIGLU || MODE == M_GATED_FWD) {
    // strip columns [0,U): H1, [U,2U): H3 of hidden units n0 + U wn + u, U =
    // WC / 2; LU lanes cover a row's U units, 8 each
    constexpr int U = WC / 2, LU = U / 8, RU = 64 / LU;
#pragma unroll
    for (int i = 0; i < C::RB; ++i) {
      stage16<C>(strip, acc, i, el);
#pragma unroll
      for (int it = 0; it < 16 / RU; ++it) {
        const int r = it * RU + el / LU, u8 = (el % LU) * 8;
        const int lm = wr0 + 16 * i + r;
        const int gc = n0 + wn * U + u8;
        if (lm < m_valid && gc < p.N) {
          // H1 and H3 rounded to bf16 once: the packed bits are stored and
          // their values feed the activation
          float h1[8], h3[8], a[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            h1[e] = strip[r * kP + u8 + e];
            h3[e] = strip[r * kP + U + u8 + e];
          }
          uint4 b1, b3;
          if constexpr (MODE == M_GATED_FWD) {
            // A from the unrounded H; what is saved are the backward's factors
            // (in the places of H1 and H3), rounded once
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              float g, dg;
              gate_f(h1[e], ACT, g, dg);
              a[e] = g * h3[e];
              h1[e] = h3[e] * dg;
              h3[e] = g;
            }
            b1 = pack8(h1);
            b3 = pack8(h3);
          } else {
            b1 = pack8(h1);
            b3 = pack8(h3);
            unpack8(b1, h1);
            unpack8(b3, h3);
#pragma unroll
            for (int e = 0; e < 8; ++e) a[e] = h1[e] * sigm(h1[e]) * h3[e];
          }
          const int64_t grow = row0 + lm;
          if (p.H1) {
            *reinterpret_cast<uint4*>(p.H1 + grow * p.ldh + static_cast<int64_t>(gc) * ES) = b1;
            *reinterpret_cast<uint4*>(p.H3 + grow * p.ldh + static_cast<int64_t>(gc) * ES) = b3;
          }
          *reinterpret_cast<uint4*>(p.C + grow * p.ldc + static_cast<int64_t>(gc) * ES) = pack8(a);
        }
      }
    }
  } else if constexpr (MODE == M_BWD_DA || MODE == M_BWD_DA_SWIGLU || MODE == M_GATED_DA) {
    // dH = dA act'(H): (row block, row group) iterations, each reading 8
    // saved pre-activations (two planes for SwiGLU) per lane, issued kPf
    // iterations ahead of their use into a ring of kPf + 1 registers.  LR
    // lanes cover a row of the wave block, RG rows form a group, GB groups
    // a 16-row block.
    constexpr bool SW = MODE != M_BWD_DA;
    constexpr int LR = WC / 8, RG = 64 / LR, GB = 16 / RG;
    constexpr int kIt = C::RB * GB, kPf = 4, kRing = kPf + 1;
    uint4 q1[kRing], q3[kRing];
    auto pos = [&](int n, int& lm, int& gc) {
      lm = wr0 + 16 * (n / GB) + RG * (n % GB) + el / LR;
      gc = n0 + wn * WC + (el % LR) * 8;
    };
    auto issue = [&](int n) {
      int lm, gc;
      pos(n, lm, gc);
      const bool ok = lm < m_valid && gc < p.N;
      // out-of-tile lanes read the tile's first valid element instead
      const int64_t o = static_cast<int64_t>(row0 + (ok ? lm : 0)) * p.ldh +
                        static_cast<int64_t>(ok ? gc : n0) * ES;
      q1[n % kRing] = *reinterpret_cast<const uint4*>(p.H1 + o);
      if constexpr (SW) q3[n % kRing] = *reinterpret_cast<const uint4*>(p.H3 + o);
    };
#pragma unroll
    for (int n = 0; n < kPf; ++n) issue(n);
#pragma unroll
    for (int n = 0; n < kIt; ++n) {
      if (n + kPf < kIt) issue(n + kPf);
      if (n % GB == 0) stage16<C>(strip, acc, n / GB, el);
      int lm, gc;
      pos(n, lm, gc);
      if (lm < m_valid && gc < p.N) {
        const int r = RG * (n % GB) + el / LR, c8 = (el % LR) * 8;
        const int64_t grow = row0 + lm;
        float h1[8], g1[8];
        unpack8(q1[n % kRing], h1);
        if constexpr (SW) {
          float h3[8], g3[8];
          unpack8(q3[n % kRing], h3);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            // d silu(h1) h3 / dh1 = h3 sg (1 + h1 (1 - sg)), d / dh3 = h1 sg
            const float da = strip[r * kP + c8 + e];
            if constexpr (MODE == M_GATED_DA) {
              g1[e] = da * h1[e];
              g3[e] = da * h3[e];
              continue;
            }
            const float sg = sigm(h1[e]);
            const float t = da * sg, u = t * h3[e];
            g1[e] = __builtin_fmaf(u, __builtin_fmaf(-h1[e], sg, h1[e]), u);
            g3[e] = t * h1[e];
          }
          *reinterpret_cast<uint4*>(p.C + grow * p.ldc + static_cast<int64_t>(gc) * ES) = pack8(g1);
          *reinterpret_cast<uint4*>(p.C + grow * p.ldc + static_cast<int64_t>(p.f + gc) * ES) = pack8(g3);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            g1[e] = strip[r * kP + c8 + e] * act_grad_f(h1[e], ACT);
          *reinterpret_cast<uint4*>(p.C + grow * p.ldc + static_cast<int64_t>(gc) * ES) = pack8(g1);
        }
      }
    }
  } else if constexpr (MODE == M_VOCAB) {
    // 32 rows at a time through LDS (pitch WC, 16-column groups swapped by the row's place
    // among 16, so that neither the stores of 4 rows nor the reads meet), then a loop whose
    // code is that of two passes: LR lanes hold a row's WC columns, 8 each.  Its 100 issue
    // slots a pass (32 of them the 8 exponentials) take as long as a plain store's traffic
    // (2048 rows, 1024 -> 32768, 256x256 tiles: 153 us, 158 with the exponentials
    // stored, 154 for the logits in bf16; all of it unrolled, straight from the
    // accumulators, 174 / 172 us in the loss's sequence)
    constexpr int LR = WC / 8, RG = 64 / LR;
    const int block = 2 * (n0 / C::TN) + wn, col0 = n0 + wn * WC;
    auto place = [](int r, int c) { return r * WC + (c ^ ((r >> 2 & 3) << 4)); };
#pragma unroll
    for (int i = 0; i < C::RB; i += 2) {
      constexpr int kLast = C::RB;
      const int rows = 16 * (i + 1 < kLast ? 2 : 1), r0 = wr0 + 16 * i;
      // the rows' targets, one a lane
      const int mine = el & 31;
      const int t = el < rows && r0 + mine < m_valid ? p.target[row0 + r0 + mine] - col0 : -1;
#pragma unroll
      for (int h = 0; h < 2; ++h)
        if (i + h < kLast) {
#pragma unroll
          for (int j = 0; j < C::CB; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q)
              strip[place(16 * h + 4 * (el >> 4) + q, 16 * j + (el & 15))] = acc[i + h < kLast ? i + h : 0][j][q];
        }
      if (t >= 0 && t < WC) p.target_logit[row0 + r0 + mine] = strip[place(mine, t)];
#pragma unroll 2
      for (int r1 = 0; r1 < rows; r1 += RG) {
        const int r = r1 + el / LR, c8 = (el % LR) * 8, lm = r0 + r, gc = col0 + c8;
        const float* sp = strip + place(r, c8);
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = sp[e];
        if (col0 + WC > p.N) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (gc + e >= p.N) v[e] = -INFINITY;
        }
        vocab_row<LR, 8, kVocabLift>(p, v, row0 + lm, lm < m_valid, block, el % LR == 0);
        if (lm < m_valid && p.C && gc < p.N) {
          typedef _Float16 half8 __attribute__((ext_vector_type(8)));
          half8 o;
#pragma unroll
          for (int e = 0; e < 8; ++e) o[e] = static_cast<_Float16>(v[e]);
          *reinterpret_cast<half8*>(p.C + (row0 + lm) * p.ldc + 2 * gc) = o;
        }
      }
    }
  } else {
    constexpr int LR = WC / 8, RG = 64 / LR;   // lanes per row, rows per pass
    // the addend's rows, kPf passes ahead of their use, as the factors above
    constexpr int GB = 16 / RG, kIt = C::RB * GB, kPf = kIt < 4 ? kIt : 4, kRing = kPf + 1;
    uint4 qa[kRing];
    const bool adds = MODE == M_ADD_STORE && p.add && slot < 0;
    auto issue = [&](int n) {
      const int lm = wr0 + 16 * (n / GB) + RG * (n % GB) + el / LR, gc = n0 + wn * WC + (el % LR) * 8;
      const bool ok = lm < m_valid && gc < p.N;
      qa[n % kRing] = *reinterpret_cast<const uint4*>(
          p.add + static_cast<int64_t>(row0 + (ok ? lm : 0)) * p.ldadd +
          static_cast<int64_t>(ok ? gc : n0) * ES);
    };
    if constexpr (MODE == M_ADD_STORE) {
      if (adds) {
#pragma unroll
        for (int n = 0; n < kPf; ++n) issue(n);
      }
    }
#pragma unroll
    for (int i = 0; i < C::RB; ++i) {
      stage16<C>(strip, acc, i, el);
#pragma unroll
      for (int it = 0; it < 16 / RG; ++it) {
        const int r = RG * it + el / LR, c8 = (el % LR) * 8;
        const int lm = wr0 + 16 * i + r;
        const int gc = n0 + wn * WC + c8;
        if constexpr (MODE == M_ADD_STORE) {
          if (adds && GB * i + it + kPf < kIt) issue(GB * i + it + kPf);
        }
        if (lm < m_valid && gc < p.N) {
          const float* sp = strip + r * kP + c8;
          if constexpr (is_dw(MODE)) {
            if constexpr (MODE == M_VOCAB_DW) {
              if (slot < 0) {
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = p.alpha * sp[e];
                if (p.acc) {
                  const float* q = p.acc + static_cast<int64_t>(row0 + lm) * p.N + gc;
                  float o[8];
                  Elem<float>::load(reinterpret_cast<const uint4*>(q)[0], o);
                  Elem<float>::load(reinterpret_cast<const uint4*>(q)[1], o + 4);
#pragma unroll
                  for (int e = 0; e < 8; ++e) v[e] += o[e];
                }
                if (!p.out_f32) {
                  *reinterpret_cast<uint4*>(dw_dst16(row0 + lm, gc)) = pack8(v);
                } else {
                  uint4* dst = reinterpret_cast<uint4*>(dw_dst(row0 + lm, gc));
                  dst[0] = Elem<float>::store(v);
                  dst[1] = Elem<float>::store(v + 4);
                }
                continue;
              }
            }
            if (is_dense_dw(MODE) && slot < 0 && !p.out_f32) {
              *reinterpret_cast<uint4*>(dw_dst16(row0 + lm, gc)) = pack8(sp);
              continue;
            }
            float* dst = dw_dst(row0 + lm, gc);
            *reinterpret_cast<float4*>(dst) = make_float4(sp[0], sp[1], sp[2], sp[3]);
            *reinterpret_cast<float4*>(dst + 4) = make_float4(sp[4], sp[5], sp[6], sp[7]);
          } else {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = sp[e];
            const int64_t grow = row0 + lm;
            if constexpr (MODE == M_ADD_STORE || MODE == M_VOCAB_DX) {
              if (slot >= 0) {
                float* dst = p.partial + slot * p.slot_elems + grow * p.N + gc;
                *reinterpret_cast<float4*>(dst) = make_float4(v[0], v[1], v[2], v[3]);
                *reinterpret_cast<float4*>(dst + 4) = make_float4(v[4], v[5], v[6], v[7]);
                continue;
              }
              if (adds) {
                float b[8];
                unpack8(qa[(GB * i + it) % kRing], b);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] += b[e];
              }
              if constexpr (MODE == M_VOCAB_DX) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] *= p.alpha;
              }
            }
            if constexpr (MODE == M_FWD1) {
              if constexpr (ACT == ACT_RELU) {
                // ReLU commutes with the rounding to bf16 (round(max(h, 0)) =
                // max(round(h), 0)), and ReLU layers keep A alone
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = fmaxf(v[e], 0.f);
              } else {
                // H rounded to bf16 once: the packed bits are stored and
                // their values feed the activation
                const uint4 hb = pack8(v);
                float hh[8];
                unpack8(hb, hh);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = act_f(hh[e], ACT);
                if (p.H1)
                  *reinterpret_cast<uint4*>(p.H1 + grow * p.ldh + static_cast<int64_t>(gc) * ES) = hb;
              }
            }
            *reinterpret_cast<uint4*>(p.C + grow * p.ldc + static_cast<int64_t>(gc) * ES) = pack8(v);
          }
        }
      }
    }
  }
  };
  if constexpr (MODE == M_FWD1 || MODE == M_BWD_DA) {
    if (p.act == ACT_RELU) epilogue(std::integral_constant<int, ACT_RELU>{});
    else epilogue(std::integral_constant<int, ACT_GELU>{});
  } else if constexpr (MODE == M_GATED_FWD) {
    if (p.act == ACT_RELU) epilogue(std::integral_constant<int, ACT_RELU>{});
    else if (p.act == ACT_GELU) epilogue(std::integral_constant<int, ACT_GELU>{});
    else epilogue(std::integral_constant<int, ACT_SWIGLU>{});
  } else {
    epilogue(std::integral_constant<int, ACT_SWIGLU>{});
  }
}

// Row scales of a wave's rows, behind the two strips of its operand buffer.
template <typename C>
__device__ __forceinline__ float* row_scales(char* buf01, char* buf23, int wave) {
  static_assert(2 * C::kStripBytes + 2 * C::WR * 4 <= kMidN * kRowBytes || C::WR == 128, "fits");
  static_assert(2 * C::kStripBytes + 2 * C::WR * 4 <= kTileBytes, "fits");
  return reinterpret_cast<float*>((wave < 2 ? buf01 : buf23) + 2 * C::kStripBytes) + (wave & 1) * C::WR;
}

// Epilogue of the int8 products: int32 sums, times the scale of their row of A,
// times the scale of their row of B, in that order, all in fp32 (an int32 sum
// is rounded to 24 bits once).  A lane's eight columns are the same for every
// row, so the B scales are read once per tile; the A scales of the wave's rows
// go through rs, WR floats of LDS behind the strips, so that their memory
// latency is paid once; the deep kernel, with registers to spare, reads both
// beside its first stages (3001 rows on 29 experts, 1008 -> 2504: 39.4 -> 38.0 us).
template <int MODE, typename C>
struct ScalesI8 {   // a lane's
  static constexpr int U = is_gated(MODE) ? C::WC / 2 : C::WC, LR = U / 8;
  float row[C::WR / 64 + (C::WR % 64 != 0)], s1[8], s3[is_gated(MODE) ? 8 : 1];
  __device__ __forceinline__ void load(const GemmParams& p, int el, int wm, int wn, int g, int row0,
                                       int m_valid, int n0) {
    const int wr0 = wm * C::WR, gc = n0 + wn * U + (el % LR) * 8;
#pragma unroll
    for (int r = el, i = 0; i < (C::WR + 63) / 64; r += 64, ++i)
      row[i] = r < C::WR && wr0 + r < m_valid ? row_scale_at(p.a_scale, row0 + wr0 + r) : 0.f;
    if (gc < p.N) {
      const int64_t o = static_cast<int64_t>(g) * p.s_gstride + gc;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        s1[e] = p.b_scale[o + e];
        if constexpr (is_gated(MODE)) s3[e] = p.b2_scale[o + e];
      }
    }
  }
};
template <int MODE, typename C>
__device__ __forceinline__ void epilogue_i8(const GemmParams& p, const floatx4 (&acc)[C::RB][C::CB],
                                            const ScalesI8<MODE, C>& sc, float* strip, float* rs, int el,
                                            int wm, int wn, int g, int row0, int m_valid, int n0) {
  constexpr int WR = C::WR, WC = C::WC, kP = C::kP;
  constexpr bool GATED = is_gated(MODE);
  constexpr int U = GATED ? WC / 2 : WC, LR = U / 8, RG = 64 / LR;
  const int wr0 = wm * WR, c8 = (el % LR) * 8, gc = n0 + wn * U + c8;
#pragma unroll
  for (int r = el, i = 0; i < (WR + 63) / 64; r += 64, ++i)
    if (r < WR) rs[r] = sc.row[i];
  const auto& s1 = sc.s1;
  const auto& s3 = sc.s3;
  auto run = [&](auto act_c) {
    constexpr int ACT = decltype(act_c)::value;
#pragma unroll
    for (int i = 0; i < C::RB; ++i) {
      const int c16 = el & 15, G = el >> 4;
#pragma unroll
      for (int j = 0; j < C::CB; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          strip[(4 * G + q) * kP + 16 * j + c16] = static_cast<float>(__float_as_int(acc[i][j][q]));
#pragma unroll
      for (int it = 0; it < 16 / RG; ++it) {
        const int r = it * RG + el / LR, lr = 16 * i + r, lm = wr0 + lr;
        if (lm < m_valid && gc < p.N) {
          const float* sp = strip + r * kP + c8;
          const float as = rs[lr];
          float v[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            v[e] = sp[e] * as * s1[e];
            if constexpr (GATED) v[e] = v[e] * sigm(v[e]) * (sp[U + e] * as * s3[e]);
            else if constexpr (MODE == M_I8_FWD1) v[e] = act_i8(v[e], ACT);
          }
          char* dst = p.C + static_cast<int64_t>(row0 + lm) * p.ldc;
          if (p.out_f32) {
            float4* d4 = reinterpret_cast<float4*>(dst + static_cast<int64_t>(gc) * 4);
            d4[0] = make_float4(v[0], v[1], v[2], v[3]);
            d4[1] = make_float4(v[4], v[5], v[6], v[7]);
          } else {
            *reinterpret_cast<uint4*>(dst + static_cast<int64_t>(gc) * 2) = pack8(v);
          }
        }
      }
    }
  };
  if constexpr (MODE == M_I8_FWD1) {
    if (p.act == ACT_RELU) run(std::integral_constant<int, ACT_RELU>{});
    else run(std::integral_constant<int, ACT_GELU>{});
  } else {
    run(std::integral_constant<int, ACT_SWIGLU>{});
  }
}
template <int MODE, typename C>
__device__ __forceinline__ void epilogue_i8(const GemmParams& p, const floatx4 (&acc)[C::RB][C::CB],
                                            float* strip, float* rs, int el, int wm, int wn, int g,
                                            int row0, int m_valid, int n0) {
  ScalesI8<MODE, C> sc;
  sc.load(p, el, wm, wn, g, row0, m_valid, n0);
  epilogue_i8<MODE, C>(p, acc, sc, strip, rs, el, wm, wn, g, row0, m_valid, n0);
}

// Items of a dense product: its tiles, once for every range of K.
template <int MODE>
__device__ __forceinline__ int dense_items(const GemmParams& p) {
  return p.dense.splits * (is_dw(MODE) ? p.mtiles_out : p.dense.n_mt) * p.ntiles;
}
// Tile of item L; returns its K range.
template <int MODE>
__device__ __forceinline__ int dense_tile(const GemmParams& p, int L, int& mt, int& nt) {
  const int n_mt = is_dw(MODE) ? p.mtiles_out : p.dense.n_mt, tiles = n_mt * p.ntiles;
  const int si = L / tiles;
  decode_banded(L - si * tiles, n_mt, p.ntiles, mt, nt);
  return si;
}
// Operands of K range si of the tile at row0, n0 (tn columns, the gated forward's
// half of W1 and half of W3); ES: bytes per element.
template <int MODE, int PASS, int ES>
__device__ __forceinline__ TileOps dense_ops(const GemmParams& p, int row0, int m_valid, int n0,
                                             int tn, int si) {
  TileOps op;
  const int k0 = si * p.dense.klen;
  if constexpr (is_dw(MODE)) {
    op.K = min(p.dense.klen, p.dense.T - k0);
    op.a = {p.A + k0 * p.lda + static_cast<int64_t>(row0) * ES, nullptr, p.lda, m_valid, 0x7FFFFFFF};
    op.b = {p.B + k0 * p.ldb + static_cast<int64_t>(n0) * ES, nullptr, p.ldb, min(tn, p.N - n0),
            0x7FFFFFFF};
  } else {
    op.K = min(p.dense.klen, p.K - k0);
    op.a = {p.A + row0 * p.lda + static_cast<int64_t>(k0) * ES, nullptr, p.lda, m_valid, 0};
    if constexpr (is_gated(MODE)) {
      op.b = {p.B + n0 * p.ldb, p.B2 + n0 * p.ldb, p.ldb, min(tn / 2, p.N - n0), 0};
    } else if constexpr (b_layout(PASS) == L_KC) {
      op.b = {p.B + n0 * p.ldb + static_cast<int64_t>(k0) * ES, nullptr, p.ldb, min(tn, p.N - n0), 0};
    } else {
      // k-rows below kmsplit come from B, the others from B2; this range starts at k0
      const int64_t o = static_cast<int64_t>(n0) * ES;
      op.b = {p.B + o + k0 * p.ldb,
              p.B2 ? p.B2 + o + max(k0 - p.kmsplit, 0) * p.ldb : nullptr, p.ldb,
              min(tn, p.N - n0), p.B2 ? max(p.kmsplit - k0, 0) : 0x7FFFFFFF};
    }
  }
  return op;
}

template <int MODE, int PASS>
__global__ __launch_bounds__(kThreads16, 1) void ffn_gemm16_kernel(const GemmParams p) {
  __shared__ __attribute__((aligned(16))) char la0[kTileBytes];
  __shared__ __attribute__((aligned(16))) char lb0[kTileBytes];
  __shared__ __attribute__((aligned(16))) char la1[kTileBytes];
  __shared__ __attribute__((aligned(16))) char lb1[kTileBytes];
  using C = TileBig;
  constexpr int TM = C::TM, TN = C::TN;
  constexpr int ES = op_bytes(MODE);
  constexpr bool VARK = is_dw(MODE);
  constexpr bool GATED = is_gated(MODE);
  constexpr int ALAY = a_layout(PASS), BLAY = b_layout(PASS);
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  constexpr bool DENSE = is_dense(MODE);
  const Sched& sc = *p.sched;   // not read by dense products
  const int n_mt = DENSE ? p.dense.n_mt : sc.n_mtiles;
  const int n_items = DENSE ? dense_items<MODE>(p)
                            : VARK ? sc.n_segs * p.mtiles_out * p.ntiles : n_mt * p.ntiles;
  const int G = gridDim.x;
  const int lbase = (blockIdx.x % kXcds) * (G / kXcds) + blockIdx.x / kXcds;

  for (int round = 0;; ++round) {
    const int L = round * G + lbase;
    if (L >= n_items) break;
    TileOps op;
    int g, row0, m_valid, n0;
    int slot = -1, mt, nt;
    if constexpr (DENSE) {
      const int si = dense_tile<MODE>(p, L, mt, nt);
      g = 0;
      row0 = mt * TM;
      n0 = nt * (GATED ? TN / 2 : TN);
      m_valid = min(TM, (VARK ? p.M_out : p.dense.T) - row0);
      slot = p.dense.splits > 1 ? si : -1;
      op = dense_ops<MODE, PASS, ES>(p, row0, m_valid, n0, TN, si);
    } else if constexpr (!VARK) {
      int mti;
      decode_banded(L, n_mt, p.ntiles, mti, nt);
      const int2 tm = p.mtile[mti];
      g = tm.x;
      row0 = p.offsets[g] + tm.y;
      m_valid = min(TM, sc.rows[g] - tm.y);
      op.a = {p.A + static_cast<int64_t>(row0) * p.lda, nullptr, p.lda, m_valid, 0};
      op.K = p.K;
      const char* bg = p.B + static_cast<int64_t>(g) * p.b_gstride;
      if constexpr (GATED) {
        n0 = nt * (TN / 2);
        op.b = {bg + static_cast<int64_t>(n0) * p.ldb,
                p.B2 + static_cast<int64_t>(g) * p.b_gstride + static_cast<int64_t>(n0) * p.ldb,
                p.ldb, min(TN / 2, p.N - n0), 0};
      } else if constexpr (BLAY == L_KC) {
        n0 = nt * TN;
        op.b = {bg + static_cast<int64_t>(n0) * p.ldb, nullptr, p.ldb, min(TN, p.N - n0), 0};
      } else {
        n0 = nt * TN;
        op.b = {bg + static_cast<int64_t>(n0) * ES,
                p.B2 ? p.B2 + static_cast<int64_t>(g) * p.b_gstride + static_cast<int64_t>(n0) * ES
                     : nullptr,
                p.ldb, min(TN, p.N - n0), p.B2 ? p.kmsplit : 0x7FFFFFFF};
      }
    } else {
      const int tmn = p.mtiles_out * p.ntiles;
      const int si = L / tmn;
      decode_banded(L - si * tmn, p.mtiles_out, p.ntiles, mt, nt);
      const int4 sg = p.seg[si];
      g = sg.x;
      slot = sg.w;
      const int k1 = min(sg.z, sc.rows[g]);
      const int64_t krow = static_cast<int64_t>(p.offsets[g]) + sg.y;
      row0 = mt * TM;
      n0 = nt * TN;
      m_valid = min(TM, p.M_out - row0);
      op.a = {p.A + krow * p.lda + static_cast<int64_t>(row0) * ES, nullptr, p.lda, m_valid,
              0x7FFFFFFF};
      op.b = {p.B + krow * p.ldb + static_cast<int64_t>(n0) * ES, nullptr, p.ldb,
              min(TN, p.N - n0), 0x7FFFFFFF};
      op.K = max(0, k1 - sg.y);
    }

    // the main loop derives its per-lane constants from an opaque zero made
    // per tile, so they are recomputed per tile instead of being hoisted out
    // of the tile loop and spilled (their reloads would wait on the loads)
    int zt;
    asm volatile("s_mov_b32 %0, 0" : "=s"(zt));
    floatx4 acc[C::RB][C::CB];
    const bool full = op.a.rows >= TM && op.b.rows >= (GATED ? TN / 2 : TN);
    if (full) mainloop16<ALAY, BLAY, GATED, true, ES>(op, la0, lb0, la1, lb1, acc, zt);
    else mainloop16<ALAY, BLAY, GATED, false, ES>(op, la0, lb0, la1, lb1, acc, zt);

    int z;
    asm volatile("s_mov_b32 %0, 0" : "=s"(z));
    float* strip = reinterpret_cast<float*>((wave < 2 ? la0 : lb0) + (wave & 1) * strip_bytes<MODE, C>() + z);
    if constexpr (is_i8(MODE))
      epilogue_i8<MODE, C>(p, acc, strip, row_scales<C>(la0, lb0, wave) + z, lane + z, wm, wn, g,
                           row0, m_valid, n0);
    else
      epilogue16<MODE, C>(p, acc, strip, lane + z, wm, wn, g, slot, row0, m_valid, n0,
                          VARK && op.K == 0);
    __syncthreads();   // strips are free before the next tile's loads
  }
}

// Item of this workgroup in a round of the two-workgroups-per-CU kernels'
// persistent grid, or -1 when it has none left.  Whole rounds give XCD b % 8 a
// contiguous run of items; the last, partial one is spread over all XCDs the
// same way, on as many workgroups as it has items, so it takes a CU each as
// far as they go.  (The grid follows the most tiles the schedule could list;
// with the runs of a whole round the items of a short one would all fall to
// the first XCDs: 4 experts of 306 rows, K = 2504, N = 1000, 112 tiles on two of
// the eight 44 us, now 29; of 1021 rows, 192 tiles of 192 rows 65 / 38.)
__device__ __forceinline__ int round_item(int round, int n_items) {
  const int b = blockIdx.x, first = round * static_cast<int>(gridDim.x), left = n_items - first;
  const int G = min(static_cast<int>(gridDim.x), (left + kXcds - 1) / kXcds * kXcds);
  if (left <= 0 || b >= G) return -1;
  const int L = first + (b % kXcds) * (G / kXcds) + b / kXcds;
  return L < n_items ? L : -1;
}

// One tile of the two-workgroups-per-CU kernels: var-M tiles of the heights
// the schedule chose, weight-gradient tiles of p.dw_h units of rows.
struct MidTile {
  TileOps op;
  int g, h;                // expert (or its segment's), units of rows
  int row0, m_valid, n0;   // first output row, valid rows, first column
  int slot;                // partial-sum slot, or -1
};

template <int MODE>
__device__ __forceinline__ int mid_items(const GemmParams& p) {
  if constexpr (is_dense(MODE)) return dense_items<MODE>(p);
  const Sched& sc = *p.sched;
  return (is_dw(MODE) ? sc.n_segs * p.mtiles_out : sc.n_mid[p.mid_list]) * p.ntiles;
}

// Tile L of the launch; ES: bytes per element.
template <int MODE, int PASS, int ES>
__device__ __forceinline__ void mid_operands(const GemmParams& p, int L, MidTile& t) {
  constexpr bool GATED = is_gated(MODE);
  constexpr int BLAY = b_layout(PASS), TN = kMidN;
  const Sched& sc = *p.sched;   // not read by dense products
  int mt, nt;
  t.slot = -1;
  if constexpr (is_dense(MODE)) {
    constexpr bool VARK = is_dw(MODE);
    const int si = dense_tile<MODE>(p, L, mt, nt);
    t.g = 0;
    if constexpr (VARK) {
      t.h = p.dw_h;
      t.row0 = mt * t.h * kMidUnit;
    } else {
      const int2 tm = mid_tile(p.dense.T, p.dense.n_mt, mt, 0);
      t.h = tm.x >> 8;
      t.row0 = tm.y;
    }
    t.m_valid = min(t.h * kMidUnit, (VARK ? p.M_out : p.dense.T) - t.row0);
    t.n0 = nt * (GATED ? TN / 2 : TN);
    t.slot = p.dense.splits > 1 ? si : -1;
    t.op = dense_ops<MODE, PASS, ES>(p, t.row0, t.m_valid, t.n0, TN, si);
  } else if constexpr (!is_dw(MODE)) {
    decode_banded(L, sc.n_mid[p.mid_list], p.ntiles, mt, nt);
    const int2 tm = p.mtile[mt];
    const int g = t.g = tm.x & 255;
    t.h = tm.x >> 8;
    t.row0 = p.offsets[g] + tm.y;
    t.m_valid = min(t.h * kMidUnit, sc.rows[g] - tm.y);
    t.op.a = {p.A + static_cast<int64_t>(t.row0) * p.lda, nullptr, p.lda, t.m_valid, 0};
    t.op.K = p.K;
    const char* bg = p.B + static_cast<int64_t>(g) * p.b_gstride;
    const char* bg2 = p.B2 + static_cast<int64_t>(g) * p.b_gstride;
    t.n0 = nt * (GATED ? TN / 2 : TN);
    if constexpr (GATED) {
      t.op.b = {bg + static_cast<int64_t>(t.n0) * p.ldb, bg2 + static_cast<int64_t>(t.n0) * p.ldb,
                p.ldb, min(TN / 2, p.N - t.n0), 0};
    } else if constexpr (BLAY == L_KC) {
      t.op.b = {bg + static_cast<int64_t>(t.n0) * p.ldb, nullptr, p.ldb, min(TN, p.N - t.n0), 0};
    } else {
      const int64_t o = static_cast<int64_t>(t.n0) * ES;
      t.op.b = {bg + o, p.B2 ? bg2 + o : nullptr, p.ldb, min(TN, p.N - t.n0),
                p.B2 ? p.kmsplit : 0x7FFFFFFF};
    }
  } else {
    const int tmn = p.mtiles_out * p.ntiles;
    const int si = L / tmn;
    decode_banded(L - si * tmn, p.mtiles_out, p.ntiles, mt, nt);
    const int4 sg = p.seg[si];
    t.g = sg.x;
    t.h = p.dw_h;
    t.slot = sg.w;
    const int k1 = min(sg.z, sc.rows[t.g]);
    const int64_t krow = static_cast<int64_t>(p.offsets[t.g]) + sg.y;
    t.row0 = mt * t.h * kMidUnit;
    t.n0 = nt * TN;
    t.m_valid = min(t.h * kMidUnit, p.M_out - t.row0);
    t.op.a = {p.A + krow * p.lda + static_cast<int64_t>(t.row0) * ES, nullptr, p.lda, t.m_valid,
              0x7FFFFFFF};
    t.op.b = {p.B + krow * p.ldb + static_cast<int64_t>(t.n0) * ES, nullptr, p.ldb,
              min(TN, p.N - t.n0), 0x7FFFFFFF};
    t.op.K = max(0, k1 - sg.y);
  }
}

template <int MODE, int PASS>
__global__ __launch_bounds__(kThreads16, 2) void ffn_gemm16_mid_kernel(const GemmParams p) {
  constexpr bool VARK = is_dw(MODE);
  constexpr int ES = op_bytes(MODE);
  constexpr int kRowsA = (VARK ? kMidDwH : kMidMaxH) * kMidUnit;
  __shared__ __attribute__((aligned(16))) char la0[kRowsA * kRowBytes];
  __shared__ __attribute__((aligned(16))) char lb0[kMidN * kRowBytes];
  __shared__ __attribute__((aligned(16))) char la1[kRowsA * kRowBytes];
  __shared__ __attribute__((aligned(16))) char lb1[kMidN * kRowBytes];
  constexpr bool GATED = is_gated(MODE);
  constexpr int ALAY = a_layout(PASS), BLAY = b_layout(PASS);
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  const int n_items = mid_items<MODE>(p);
  for (int round = 0;; ++round) {
    const int L = round_item(round, n_items);
    if (L < 0) break;
    MidTile t;
    mid_operands<MODE, PASS, ES>(p, L, t);
    auto run = [&](auto hc) {
      constexpr int RB = decltype(hc)::value;
      using C = Tile16<RB, 4>;
      int zt, z;   // opaque zeros: see ffn_gemm16_kernel
      asm volatile("s_mov_b32 %0, 0" : "=s"(zt));
      floatx4 acc[RB][4];
      mainloop_mid<RB, ALAY, BLAY, GATED, ES>(t.op, la0, lb0, la1, lb1, acc, zt);
      asm volatile("s_mov_b32 %0, 0" : "=s"(z));
      float* strip = reinterpret_cast<float*>((wave < 2 ? lb0 : lb1) + (wave & 1) * strip_bytes<MODE, C>() + z);
      if constexpr (is_i8(MODE))
        epilogue_i8<MODE, C>(p, acc, strip, row_scales<C>(lb0, lb1, wave) + z, lane + z, wm, wn, t.g,
                             t.row0, t.m_valid, t.n0);
      else
        epilogue16<MODE, C>(p, acc, strip, lane + z, wm, wn, t.g, t.slot, t.row0, t.m_valid, t.n0,
                            VARK && t.op.K == 0);
    };
    if constexpr (VARK) {
      run(std::integral_constant<int, kMidDwH>{});
    } else {
      switch (t.h) {
        case 1: run(std::integral_constant<int, 1>{}); break;
        case 2: run(std::integral_constant<int, 2>{}); break;
        case 3: run(std::integral_constant<int, 3>{}); break;
        case 4: run(std::integral_constant<int, 4>{}); break;
        case 5: run(std::integral_constant<int, 5>{}); break;
        default: run(std::integral_constant<int, 6>{}); break;
      }
    }
    __syncthreads();   // strips are free before the next tile's loads
  }
}

// The K loop with NS stages: step kt computes on stage kt mod NS while the
// loads of step kt + NS - 1 (LOADS a wavefront) go into the stage that step
// kt - 1 has read.
template <int NS, int LOADS, typename Load, typename Compute>
__device__ __forceinline__ void ring_steps(int nk, char* const (&sa)[NS], char* const (&sb)[NS],
                                           Load&& load, Compute&& compute) {
#pragma unroll
  for (int s = 0; s < NS - 1; ++s) load(s, sa[s], sb[s]);
  auto step = [&](int kt, auto slot) {
    constexpr int S = decltype(slot)::value, T = (S + NS - 1) % NS;
    // stage kt has landed when only the NS - 2 stages after it may be pending;
    // past the barrier that holds for every wave's part of it, and every wave
    // has read stage kt - 1, whose place step kt + NS - 1 takes over
    __builtin_amdgcn_s_waitcnt(wait_vm_lgkm0((NS - 2) * LOADS));
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    load(kt + NS - 1, sa[T], sb[T]);
    compute(sa[S], sb[S]);
    __builtin_amdgcn_sched_barrier(0);
  };
  using std::integral_constant;
  // whole groups without a branch between the steps: the compiler then knows
  // which loads are pending at each read and adds no wait of its own
  int k0 = 0;
  for (; k0 + NS <= nk; k0 += NS) {
    step(k0, integral_constant<int, 0>{});
    step(k0 + 1, integral_constant<int, 1>{});
    step(k0 + 2, integral_constant<int, 2>{});
    if constexpr (NS > 3) step(k0 + 3, integral_constant<int, 3>{});
  }
  if (k0 < nk) step(k0, integral_constant<int, 0>{});
  if (k0 + 1 < nk) step(k0 + 1, integral_constant<int, 1>{});
  if constexpr (NS > 3)
    if (k0 + 2 < nk) step(k0 + 2, integral_constant<int, 2>{});
  __builtin_amdgcn_s_waitcnt(0x0070);
  __builtin_amdgcn_s_barrier();   // every load landed, every read done: stages are free
}

// ---------------------------------------------------------------------------
// fp32 products
// ---------------------------------------------------------------------------
// fp32 matrix cores run at a sixteenth of the bf16 rate, so any tile keeps
// them fed from LDS and the caches; what costs time is tiles that leave
// wavefronts idle.  Every fp32 product therefore runs on tiles of 128 columns
// and RB units of 32 rows, RB chosen per tile by the schedule (weight
// gradients: per product by the host), two workgroups per CU, with
// v_mfma_f32_32x32x2f32.  (8 experts of about 512 rows, d = 256, f = 1024: the
// six products of a step took 991 us on 256x256 tiles and take 249 us; 8 of 4096 rows, 1024 x 4096 SwiGLU: step 25.9 -> 20.8 ms;
// 4 of 64 rows, 64 -> 128 -> 64: 31 -> 13 us against one wavefront per 32x32
// block reading memory directly.)  Wave w of four owns columns 32w .. +31 of the tile
// and all its rows (RB blocks of 32x32); of a gated forward tile (64 hidden
// units of W1 and of W3) units 32 (w & 1) .. +31 of both and row blocks
// w >> 1, (w >> 1) + 2, ..  K steps of 32 go HBM -> LDS by buffer loads, two
// stages, the next step's loads issued before the step's MFMAs.
constexpr int kF32Step = 32;

// LDS tiles.  K-contiguous: rows of 128 bytes with the swizzle of the bf16
// tiles.  K-major: 32 k-rows of SEG segments of 32 elements (SEG = RB for A,
// 4 for B), segment s of k-row k stored at s ^ (k & (SEG - 1)).
template <int NB> struct AccF32 { floatx16 v[NB]; };   // row blocks of a wave

// sa, sb: the operands' NS stages (NS = 2 here; more in deep.hpp).
template <int RB, int PASS, bool GATED, int NB, int NS>
__device__ __forceinline__ void mainloop_f32(const TileOps& op, char* const (&stage_a)[NS],
                                             char* const (&stage_b)[NS], AccF32<NB>& acc_,
                                             AccF32<NB>& acc3_) {
  static_assert(NB == (GATED ? (RB + 1) / 2 : RB), "row blocks per wave");
  constexpr int ALAY = a_layout(PASS), BLAY = b_layout(PASS);
  floatx16(&acc)[NB] = acc_.v;
  floatx16(&acc3)[NB] = acc3_.v;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int q = 0; q < 16; ++q) {
      acc[i][q] = 0.f;
      if constexpr (GATED) acc3[i][q] = 0.f;
    }
  const int K = op.K;
  const int nk = (K + kF32Step - 1) / kF32Step;
  if (nk <= 0) return;
  // ---- loads: 1 KB blocks 4i + w of A (i < RB) and of B (i < 4)
  const int l3 = lane >> 3;
  const int co = ((lane & 7) ^ swz(l3 + (wave & 1) * 8)) * 16;   // KC: block rows 8(4i + w) + l3
  const int lda = static_cast<int>(op.a.ld), ldb = static_cast<int>(op.b.ld);
  auto bad = [](bool b) { return static_cast<uint32_t>(b) << 31; };
  // KM: a block is 8 / SEG k-rows of SEG segments; the lane's k-row within
  // it and physical element
  auto km_row = [&](int seg) { return lane / (8 * seg); };
  auto km_elem = [&](int seg) { return (lane % (8 * seg)) * 4; };
  auto brow = [&](int i) { return GATED ? (i >> 1) * 32 + wave * 8 : (4 * i + wave) * 8; };
  const __amdgpu_buffer_rsrc_t ra_t = tile_rsrc(op.a.base);
  const __amdgpu_buffer_rsrc_t rb_t = tile_rsrc(op.b.base);
  const __amdgpu_buffer_rsrc_t rb3_t = tile_rsrc(GATED ? op.b.base2 : op.b.base);
  auto load_km = [&](auto seg_c, const Operand& o, char* dst, int i, int kt, int ld) {
    constexpr int SEG = decltype(seg_c)::value;
    const int blk = 4 * i + wave;
    const int k0 = blk * (8 / SEG), kr = km_row(SEG);      // first k-row of the block, the lane's
    const int pe = km_elem(SEG);
    const int col = (((pe >> 5) ^ ((k0 + kr) & (SEG - 1))) << 5) + (pe & 31);
    const int kabs = kt * kF32Step + k0;
    const bool second = kabs >= o.split;                   // a multiple of 8
    const int64_t kb = static_cast<int64_t>(kt) * kF32Step - (second ? o.split : 0);
    const __amdgpu_buffer_rsrc_t rs = tile_rsrc((second ? o.base2 : o.base) + kb * o.ld);
    const uint32_t off = static_cast<uint32_t>(kr * ld + col * 4) | bad(col >= o.rows || kabs + kr >= K);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, MOE_LDS(dst + blk * 1024), 16, off, k0 * ld, 0, 0);
  };
  auto load = [&](int kt, char* sa, char* sb) {
    const uint32_t kbad = bad(kt * kRowBytes + co >= K * 4);
#pragma unroll
    for (int i = 0; i < RB; ++i) {
      if constexpr (ALAY == L_KC) {
        const int blk = 4 * i + wave;
        const uint32_t off = static_cast<uint32_t>(l3 * lda + co) | bad(blk * 8 + l3 >= op.a.rows) | kbad;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(ra_t, MOE_LDS(sa + blk * 1024), 16, off,
                                                 blk * 8 * lda + kt * kRowBytes, 0, 0);
      } else {
        load_km(std::integral_constant<int, RB>{}, op.a, sa, i, kt, lda);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (BLAY == L_KC) {
        const int blk = 4 * i + wave;
        const uint32_t off = static_cast<uint32_t>(l3 * ldb + co) | bad(brow(i) + l3 >= op.b.rows) | kbad;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(GATED && (i & 1) ? rb3_t : rb_t,
                                                 MOE_LDS(sb + blk * 1024), 16, off,
                                                 brow(i) * ldb + kt * kRowBytes, 0, 0);
      } else {
        load_km(std::integral_constant<int, 4>{}, op.b, sb, i, kt, ldb);
      }
    }
  };
  // ---- fragments.  MFMA operand of lane l: row/column l % 32 of the block,
  // k values 8 s + 4 (l / 32) .. +3 of sub-step s
  const int r32 = lane & 31, kh = lane >> 5;
  auto frag_kc = [&](const char* st, int blk, int s) {
    const int row = blk * 32 + r32;
    return *reinterpret_cast<const uint4*>(st + row * kRowBytes + (((2 * s + kh) ^ swz(row)) << 4));
  };
  auto frag_km = [&](auto seg_c, const char* st, int blk, int s) {
    constexpr int SEG = decltype(seg_c)::value;
    uint32_t v[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int k = 8 * s + 4 * kh + c;
      v[c] = *reinterpret_cast<const uint32_t*>(
          st + (k * SEG + (blk ^ (c & (SEG - 1)))) * 128 + r32 * 4);   // k & (SEG - 1) = c & (SEG - 1)
    }
    return make_uint4(v[0], v[1], v[2], v[3]);
  };
  auto compute = [&](const char* sa, const char* sb) {
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      uint4 b, b3;
      if constexpr (GATED) {
        b = frag_kc(sb, 2 * (wave & 1), s);
        b3 = frag_kc(sb, 2 * (wave & 1) + 1, s);
      } else if constexpr (BLAY == L_KC) {
        b = frag_kc(sb, wave, s);
      } else {
        b = frag_km(std::integral_constant<int, 4>{}, sb, wave, s);
      }
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        const int blk = GATED ? min(2 * i + (wave >> 1), RB - 1) : i;
        uint4 a;
        if constexpr (ALAY == L_KC) a = frag_kc(sa, blk, s);
        else a = frag_km(std::integral_constant<int, RB>{}, sa, blk, s);
        mma_f32(acc[i], a, b);
        if constexpr (GATED) mma_f32(acc3[i], a, b3);
      }
    }
  };
  if constexpr (NS == 2) {
    char *const la0 = stage_a[0], *const lb0 = stage_b[0], *const la1 = stage_a[1], *const lb1 = stage_b[1];
    load(0, la0, lb0);
    __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0)
    __builtin_amdgcn_s_barrier();
    auto step = [&](int kt, char* ca, char* cb, char* na, char* nb) {
      if (kt + 1 < nk) load(kt + 1, na, nb);
      __builtin_amdgcn_sched_barrier(0);
      compute(ca, cb);
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_waitcnt(0x0070);   // vmcnt(0) lgkmcnt(0)
      __builtin_amdgcn_s_barrier();
    };
    for (int kt = 0; kt < nk; kt += 2) {
      step(kt, la0, lb0, la1, lb1);
      if (kt + 1 < nk) step(kt + 1, la1, lb1, la0, lb0);
    }
  } else {
    ring_steps<NS, RB + 4>(nk, stage_a, stage_b, load, compute);
  }
}

// Epilogue of an fp32 tile, straight from the accumulators.
template <int MODE, int RB, int NB>
__device__ __forceinline__ void epilogue_f32(const GemmParams& p, const MidTile& t, AccF32<NB>& c1,
                                             const AccF32<NB>& c3, int lane, int wave) {
  constexpr bool GATED = is_gated(MODE), VARK = is_dw(MODE);
  std::conditional_t<MODE == M_VOCAB_DW, floatx16, const floatx16>(&acc)[NB] = c1.v;
  const floatx16(&acc3)[NB] = c3.v;
  // accumulator q of lane l: column l % 32, row 8 (q / 4) + 4 (l / 32) + q % 4
  const int col = t.n0 + (GATED ? wave & 1 : wave) * 32 + (lane & 31);
  if (MODE != M_VOCAB && col >= p.N) return;
#pragma unroll
  for (int i = 0; i < NB; ++i) {
    const int blk = GATED ? 2 * i + (wave >> 1) : i;
    if (GATED && blk >= RB) continue;
    auto row_of = [&](int q) { return blk * 32 + 8 * (q >> 2) + 4 * (lane >> 5) + (q & 3); };
    // what the dense block's epilogues read, the whole block's before its first store
    // (rows behind the last one: the last one again)
    float u1[16], u3[16];
    if constexpr (MODE == M_GATED_DA || MODE == M_ADD_STORE) {
#pragma unroll
      for (int q = 0; q < 16; ++q) {
        const int64_t row = t.row0 + min(row_of(q), t.m_valid - 1);
        if constexpr (MODE == M_GATED_DA) {
          u1[q] = reinterpret_cast<const float*>(p.H1 + row * p.ldh)[col];
          u3[q] = reinterpret_cast<const float*>(p.H3 + row * p.ldh)[col];
        } else {
          u1[q] = p.add && t.slot < 0 ? reinterpret_cast<const float*>(p.add + row * p.ldadd)[col] : 0.f;
        }
      }
    }
    if constexpr (MODE == M_VOCAB) {
      int tg[16];
#pragma unroll
      for (int q = 0; q < 16; ++q) tg[q] = p.target[t.row0 + min(row_of(q), t.m_valid - 1)];
#pragma unroll
      for (int q = 0; q < 16; ++q) {
        const int row = t.row0 + row_of(q);
        const bool ok = row_of(q) < t.m_valid;
        if (ok && tg[q] == col) p.target_logit[row] = acc[i][q];
        float v[1] = {col < p.N ? acc[i][q] : -INFINITY};
        vocab_row<32, 1, 0>(p, v, row, ok, 4 * (t.n0 / kMidN) + wave, (lane & 31) == 0);
        if (ok && p.C && col < p.N) reinterpret_cast<float*>(p.C + row * p.ldc)[col] = v[0];
      }
      continue;
    }
#pragma unroll
    for (int q = 0; q < 16; ++q) {
      const int lm = row_of(q);
      if (lm >= t.m_valid) continue;
      const int64_t row = t.row0 + lm;
      if constexpr (VARK) {
        if constexpr (MODE == M_VOCAB_DW) {
          if (t.slot < 0) acc[i][q] = p.alpha * acc[i][q] + (p.acc ? p.acc[row * p.N + col] : 0.f);
        }
        float* dst;
        if (t.slot >= 0) dst = p.partial + static_cast<int64_t>(t.slot) * p.slot_elems + row * p.N;
        else if (row < p.split_row) dst = p.dwA + static_cast<int64_t>(t.g) * p.dw_gstride + row * p.N;
        else dst = p.dwB + static_cast<int64_t>(t.g) * p.dw_gstride + (row - p.split_row) * p.N;
        dst[col] = acc[i][q];
      } else {
        float* c = reinterpret_cast<float*>(p.C + row * p.ldc) + col;
        if constexpr (MODE == M_FWD1_SWIGLU) {
          const float h1 = acc[i][q], h3 = acc3[i][q];
          if (p.H1) {
            reinterpret_cast<float*>(p.H1 + row * p.ldh)[col] = h1;
            reinterpret_cast<float*>(p.H3 + row * p.ldh)[col] = h3;
          }
          *c = h1 * sigm(h1) * h3;
        } else if constexpr (MODE == M_GATED_FWD) {
          const float h3 = acc3[i][q];
          float g, dg;
          gate_f(acc[i][q], p.act, g, dg);
          if (p.H1) {
            reinterpret_cast<float*>(p.H1 + row * p.ldh)[col] = h3 * dg;
            reinterpret_cast<float*>(p.H3 + row * p.ldh)[col] = g;
          }
          *c = g * h3;
        } else if constexpr (MODE == M_GATED_DA) {
          *c = acc[i][q] * u1[q];
          c[p.f] = acc[i][q] * u3[q];
        } else if constexpr (MODE == M_VOCAB_DX) {
          if (t.slot >= 0) p.partial[t.slot * p.slot_elems + row * p.N + col] = acc[i][q];
          else *c = p.alpha * acc[i][q];
        } else if constexpr (MODE == M_ADD_STORE) {
          if (t.slot >= 0) {
            p.partial[t.slot * p.slot_elems + row * p.N + col] = acc[i][q];
            continue;
          }
          *c = acc[i][q] + u1[q];
        } else if constexpr (MODE == M_FWD1) {
          if (p.H1) reinterpret_cast<float*>(p.H1 + row * p.ldh)[col] = acc[i][q];
          *c = act_f(acc[i][q], p.act);
        } else if constexpr (MODE == M_BWD_DA_SWIGLU) {
          const float h1 = reinterpret_cast<const float*>(p.H1 + row * p.ldh)[col];
          const float h3 = reinterpret_cast<const float*>(p.H3 + row * p.ldh)[col];
          // d silu(h1) h3 / dh1 = h3 sg (1 + h1 (1 - sg)), d / dh3 = h1 sg
          const float sg = sigm(h1), x = acc[i][q] * sg, u = x * h3;
          *c = __builtin_fmaf(u, __builtin_fmaf(-h1, sg, h1), u);
          c[p.f] = x * h1;
        } else if constexpr (MODE == M_BWD_DA) {
          *c = acc[i][q] * act_grad_f(reinterpret_cast<const float*>(p.H1 + row * p.ldh)[col], p.act);
        } else {
          *c = acc[i][q];
        }
      }
    }
  }
}

template <int MODE, int PASS>
__global__ __launch_bounds__(kThreads16, 2) void ffn_gemm_f32_kernel(const GemmParams p) {
  constexpr bool VARK = is_dw(MODE);
  constexpr int kRowsA = (VARK ? 4 : kMidMaxH) * kMidUnit;
  __shared__ __attribute__((aligned(16))) char la0[kRowsA * kRowBytes];
  __shared__ __attribute__((aligned(16))) char lb0[kMidN * kRowBytes];
  __shared__ __attribute__((aligned(16))) char la1[kRowsA * kRowBytes];
  __shared__ __attribute__((aligned(16))) char lb1[kMidN * kRowBytes];
  constexpr bool GATED = is_gated(MODE);
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
  const int n_items = mid_items<MODE>(p);
  for (int round = 0;; ++round) {
    const int L = round_item(round, n_items);
    if (L < 0) break;
    MidTile t;
    mid_operands<MODE, PASS, 4>(p, L, t);
    auto run = [&](auto hc) {
      constexpr int RB = decltype(hc)::value;
      constexpr int NB = GATED ? (RB + 1) / 2 : RB;
      AccF32<NB> c1, c3;   // c3: the W3 half of a gated tile
      char *const sa[2] = {la0, la1}, *const sb[2] = {lb0, lb1};
      mainloop_f32<RB, PASS, GATED, NB, 2>(t.op, sa, sb, c1, c3);
      epilogue_f32<MODE, RB, NB>(p, t, c1, c3, lane, wave);
    };
    if constexpr (VARK) {
      switch (t.h) {
        case 1: run(std::integral_constant<int, 1>{}); break;
        case 2: run(std::integral_constant<int, 2>{}); break;
        default: run(std::integral_constant<int, 4>{}); break;
      }
    } else {
      switch (t.h) {
        case 1: run(std::integral_constant<int, 1>{}); break;
        case 2: run(std::integral_constant<int, 2>{}); break;
        case 3: run(std::integral_constant<int, 3>{}); break;
        case 4: run(std::integral_constant<int, 4>{}); break;
        case 5: run(std::integral_constant<int, 5>{}); break;
        default: run(std::integral_constant<int, 6>{}); break;
      }
    }
  }
}

// ---------------------------------------------------------------------------
// transposed weights
// ---------------------------------------------------------------------------
// Transposed copy of expert weights (bf16), so that dX reads them
// K-contiguous: dst[g][n][k] = src1[g][k][n] for k < K1 and src2[g][k - K1][n]
// for K1 <= k < K1 + K2 (dst rows of K1 + K2 elements).  A workgroup moves a
// 64 (k) x 64 (n) block through LDS: 16-byte loads along n, 16-byte stores
// along k.  K1, K2 and N are multiples of 8, so no vector straddles an edge
// or the seam between the two sources.
constexpr int kTr = 64;
__global__ __launch_bounds__(256) void transpose_w_kernel(const uint16_t* __restrict__ src1,
                                                          const uint16_t* __restrict__ src2,
                                                          int K1, int K2, int N,
                                                          uint16_t* __restrict__ dst) {
  __shared__ __attribute__((aligned(16))) uint16_t tile[kTr][kTr + 8];
  const int g = blockIdx.z;
  const int n0 = blockIdx.x * kTr;
  const int K = K1 + K2;
  const int64_t s1 = static_cast<int64_t>(g) * K1 * N, s2 = static_cast<int64_t>(g) * K2 * N;
  for (int k0 = blockIdx.y * kTr; k0 < K; k0 += gridDim.y * kTr) {
    __syncthreads();   // the previous block's reads of the tile are done
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int c = threadIdx.x + 256 * i;
      const int kk = c >> 3, nn = (c & 7) * 8;
      const int k = k0 + kk, n = n0 + nn;
      uint4 v = make_uint4(0, 0, 0, 0);
      if (k < K && n < N) {
        const uint16_t* src = k < K1 ? src1 + s1 + static_cast<int64_t>(k) * N + n
                                     : src2 + s2 + static_cast<int64_t>(k - K1) * N + n;
        v = *reinterpret_cast<const uint4*>(src);
      }
      *reinterpret_cast<uint4*>(&tile[kk][nn]) = v;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int c = threadIdx.x + 256 * i;
      const int nn = c >> 3, kk = (c & 7) * 8;
      const int n = n0 + nn, k = k0 + kk;
      if (n < N && k < K) {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
          w[j] = static_cast<uint32_t>(tile[kk + 2 * j][nn]) |
                 (static_cast<uint32_t>(tile[kk + 2 * j + 1][nn]) << 16);
        *reinterpret_cast<uint4*>(dst + (static_cast<int64_t>(g) * N + n) * K + k) =
            make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
  }
}

// ---------------------------------------------------------------------------
// split-K reduction
// ---------------------------------------------------------------------------
// dW[g] = sum over the expert's split slots, in slot order, or zeros for an
// expert without rows.  A bounded grid strides over the elements (blockIdx.y =
// expert), so experts with one segment cost one early exit per block rather
// than a launch per 1024 elements.  The zeros are written here and not by the
// products' tiles: streamed, the 1 GB of 61 of 64 experts at 4096 x 1024 takes
// 154 us beside the sums, after the products of the others, where tiles of
// zeros among the products took about 190 us more (the product 325 -> 156 us,
// this kernel 29 -> 154 us).
constexpr int kReduceBlocks = 1024;   // blocks per expert

// The slots are added in slot order; their loads are issued four at a time
// ahead of the adds, so a thread waits out one memory latency per four slots.
__global__ __launch_bounds__(256) void split_reduce_kernel(
    const float* __restrict__ partial, int64_t slot_elems, const Sched* __restrict__ sc,
    float* __restrict__ dwA, float* __restrict__ dwB, int64_t dw_gstride, int split_row,
    int N) {
  const int g = blockIdx.y;
  const int ns = sc->nsplit[g];
  if (ns == 1) return;
  if (ns == 0) {
    const int64_t na = static_cast<int64_t>(split_row) * N;   // elements in dwA, the rest in dwB
    for (int64_t i = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) * 4; i < slot_elems;
         i += static_cast<int64_t>(gridDim.x) * 1024) {
      float* dst = i < na ? dwA + static_cast<int64_t>(g) * dw_gstride + i
                          : dwB + static_cast<int64_t>(g) * dw_gstride + (i - na);
      *reinterpret_cast<float4*>(dst) = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    return;
  }
  const float* base = partial + static_cast<int64_t>(sc->slot0[g]) * slot_elems;
  auto add = [](float4& a, const float4& v) { a.x += v.x; a.y += v.y; a.z += v.z; a.w += v.w; };
  for (int64_t i = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) * 4; i < slot_elems;
       i += static_cast<int64_t>(gridDim.x) * 1024) {
    const float* p0 = base + i;
    float4 acc = *reinterpret_cast<const float4*>(p0);
    int sl = 1;
    for (; sl + 3 < ns; sl += 4) {
      float4 v[4];
#pragma unroll
      for (int u = 0; u < 4; ++u)
        v[u] = *reinterpret_cast<const float4*>(p0 + static_cast<int64_t>(sl + u) * slot_elems);
#pragma unroll
      for (int u = 0; u < 4; ++u) add(acc, v[u]);
    }
    for (; sl < ns; ++sl) add(acc, *reinterpret_cast<const float4*>(p0 + static_cast<int64_t>(sl) * slot_elems));
    int64_t row, col;
    if (slot_elems < (int64_t(1) << 31)) {   // the usual case: 32-bit division
      const uint32_t ii = static_cast<uint32_t>(i);
      row = ii / static_cast<uint32_t>(N);
      col = ii % static_cast<uint32_t>(N);
    } else {
      row = i / N;
      col = i % N;
    }
    float* dst = row < split_row
                     ? dwA + static_cast<int64_t>(g) * dw_gstride + row * N + col
                     : dwB + static_cast<int64_t>(g) * dw_gstride + (row - split_row) * N + col;
    *reinterpret_cast<float4*>(dst) = acc;
  }
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
int persistent_grid() {
  const int n = num_cus();
  return (n + kXcds - 1) / kXcds * kXcds;
}

// [rows_alloc, f] planes of h_save: A (ReLU), H and A (GELU), H1, H3 and A
// (SwiGLU).
int h_save_planes(moe_act act) { return act == MOE_SWIGLU ? 3 : act == MOE_GELU_TANH ? 2 : 1; }

// Sizes of the schedule and of every workspace buffer.
struct FfnPlan {
  int E, d, f, F;            // F = f (relu/gelu) or 2f (swiglu)
  int64_t rows_alloc;
  int64_t rows_most;         // rows_alloc, or fewer (FfnFwd)
  size_t es;
  int max_mtiles, max_mid, max_segs, max_slots, tmn_min;
  int64_t slot_elems;
  // byte offsets inside the workspace
  size_t o_sched, o_mtile, o_mid, o_seg, o_end_sched;
  size_t o_abuf, o_dh, o_part, o_wt13, total_fwd, total_bwd, total_bwd_wt;
};

bool make_plan(moe_dtype dt, moe_act act, int E, int d, int f, int64_t rows_alloc, FfnPlan& pl) {
  if (!dtype_ok(dt) || E < 1 || E > kMaxE || !width_ok(d) || !width_ok(f) || !rows_ok(rows_alloc))
    return false;
  if (act != MOE_RELU && act != MOE_GELU_TANH && act != MOE_SWIGLU) return false;
  pl.E = E; pl.d = d; pl.f = f; pl.F = act == MOE_SWIGLU ? 2 * f : f;
  pl.rows_alloc = pl.rows_most = rows_alloc;
  pl.es = esize(dt);
  // every operand offset inside a 256-row tile (K-contiguous operands) or a
  // K step (K-major ones) stays below 2^31 bytes: buffer loads take 32-bit
  // offsets
  const int64_t max_ld = static_cast<int64_t>(pl.es) * (2 * static_cast<int64_t>(f) > d ? 2 * static_cast<int64_t>(f) : d);
  if (max_ld > kMaxOperandRowBytes) return false;
  pl.max_mtiles = cdiv(rows_alloc, BM) + E;
  pl.max_mid = cdiv(rows_alloc, kMidUnit) + E;
  const int tmn2 = cdiv(d, BM) * cdiv(f, BN);
  const int tmn13 = cdiv(pl.F, BM) * cdiv(d, BN);
  pl.tmn_min = tmn2 < tmn13 ? tmn2 : tmn13;
  const int64_t kcap = (rows_alloc + kKc - 1) / kKc * kKc + static_cast<int64_t>(kKc) * E;
  const int64_t slots_a = 1024 / pl.tmn_min;
  const int64_t slots_b = 2 * kcap / kSplitFloor;
  pl.max_slots = static_cast<int>(slots_a < slots_b ? slots_a : slots_b) + 1;
  pl.max_segs = E + pl.max_slots;
  pl.slot_elems = static_cast<int64_t>(pl.F) * d > static_cast<int64_t>(d) * f
                      ? static_cast<int64_t>(pl.F) * d : static_cast<int64_t>(d) * f;
  size_t o = 0;
  pl.o_sched = o; o = align_up(o + sizeof(Sched), 256);
  pl.o_mtile = o; o = align_up(o + sizeof(int2) * pl.max_mtiles, 256);
  pl.o_mid = o; o = align_up(o + 2 * sizeof(int2) * pl.max_mid, 256);
  pl.o_seg = o;   o = align_up(o + sizeof(int4) * pl.max_segs, 256);
  pl.o_end_sched = o;
  const size_t es = pl.es;
  // forward: the activation buffer A [rows_alloc, f] when no h_save is given
  pl.o_abuf = o;
  pl.total_fwd = align_up(o + static_cast<size_t>(rows_alloc) * f * es, 256);
  // backward: dH [rows_alloc, F] and the split partial sums
  o = pl.o_end_sched;
  pl.o_dh = o;   o = align_up(o + static_cast<size_t>(rows_alloc) * pl.F * es, 256);
  pl.o_part = o; o = align_up(o + static_cast<size_t>(pl.max_slots) * pl.slot_elems * 4, 256);
  pl.total_bwd = o;
  // bf16: room for the transposed copy of [W1; W3] that dX may read
  // ([E, d, F]: row n of expert e = [W1_e[:, n]; W3_e[:, n]])
  pl.o_wt13 = o;
  pl.total_bwd_wt = dt == MOE_BF16 ? align_up(o + static_cast<size_t>(E) * d * pl.F * es, 256) : o;
  return true;
}

// nt0, nt1: column tiles (of kMidN columns) of the call's products with N = f
// (K = d) and with N = d (K = k1), c0, c1: their K steps' times, for the
// heights of the two mid tile lists.
SchedArgs sched_args(const FfnPlan& pl, int nt0, int nt1, int k1, const StepCost& c0,
                     const StepCost& c1, char* ws) {
  const bool f32 = pl.es == 4;
  const int ks = f32 ? kF32Step : kRowBytes / static_cast<int>(pl.es);
  return {pl.E, pl.rows_alloc, pl.max_mtiles, pl.max_mid, pl.max_segs, pl.tmn_min, pl.max_slots,
          {nt0, nt1}, {cdiv(pl.d, ks), cdiv(k1, ks)}, 2 * persistent_grid(),
          {f32 ? kStepF32 : c0, f32 ? kStepF32 : c1}, reinterpret_cast<Sched*>(ws + pl.o_sched),
          reinterpret_cast<int2*>(ws + pl.o_mtile), reinterpret_cast<int2*>(ws + pl.o_mid),
          reinterpret_cast<int4*>(ws + pl.o_seg)};
}

moe_status launch_schedule(hipStream_t s, const SchedArgs& a, const int32_t* offsets,
                           const int32_t* rows) {
  MOE_TIMED("ffn_schedule", s);
  schedule_kernel<<<1, 64 * kSchedTasks, 0, s>>>(offsets, rows, a);
  MOE_LAUNCH_CHECK();
  return MOE_OK;
}

GemmParams base_params(const FfnPlan& pl, const int32_t* offsets, char* ws) {
  GemmParams p{};
  p.offsets = offsets;
  p.sched = reinterpret_cast<const Sched*>(ws + pl.o_sched);
  p.mtile = reinterpret_cast<const int2*>(ws + pl.o_mtile);
  p.seg = reinterpret_cast<const int4*>(ws + pl.o_seg);
  p.kmsplit = 0x7FFFFFFF;
  return p;
}

// Tile choice of the bf16 products (moe_set_gemm_tiles: 0 automatic, 1 the
// 256x256 kernel only, 2 the two-workgroups-per-CU kernel only) is g_tile_mode:
// mid_pays (tiles.hpp) for the forward and the data gradients; the weight
// gradients (K not known on the host) compare rounds, a round of 128x128 tiles
// taking 0.65 of one of 256x256 tiles.
bool use_mid_tiles(const FfnPlan& pl, moe_dtype dt, bool vark, bool gated, bool act, bool b_km,
                   const GemmParams& p) {
  if (dt == MOE_F32) return true;
  if (g_tile_mode == 1) return false;
  if (g_tile_mode == 2) return true;
  const int G = persistent_grid();
  if (vark) {
    const int64_t big = static_cast<int64_t>(pl.E) * cdiv(p.M_out, BM) * cdiv(p.N, BN);
    const int64_t mid = static_cast<int64_t>(pl.E) * cdiv(p.M_out, kMidDwH * kMidUnit) * cdiv(p.N, kMidN);
    return 13 * ((mid + 2 * G - 1) / (2 * G)) < 20 * ((big + G - 1) / G);
  }
  return mid_pays({pl.E, pl.rows_alloc, pl.rows_most, p.N, p.K, gated, act, b_km, p.lda, p.ldb}, G);
}

// dX with a transposed copy of [W1; W3] (moe_set_dx_weight_copy, g_wt_mode: 0
// automatic, 1 never, 2 always; bf16 only).  Read K-major, the weights need
// two transpose reads per MFMA fragment; read K-contiguous, dX ran 8-9%
// faster on 16384-row experts (same box, c5 and c4 shapes), and the copy
// moves 4 E d F bytes at about 5 TB/s.  The copy pays for itself from about
// 6000 rows per expert; the rule takes it from 8192 (rows_alloc / E: the
// row budget, as the host knows no fills).
constexpr int64_t kWtRowsPerExpert = 8192;

bool use_wt13(const FfnPlan& pl, moe_dtype dt) {
  if (dt != MOE_BF16 || g_wt_mode == 1) return false;
  return g_wt_mode == 2 || pl.rows_alloc >= kWtRowsPerExpert * pl.E;
}

const char* pass_name(int pass) {
  static const char* names[] = {"gemm_fwd_h", "gemm_fwd_y", "gemm_bwd_da", "gemm_bwd_dx",
                                "gemm_bwd_dw2", "gemm_bwd_dw13", "gemm_bwd_dx",
                                "gemm_logits", "gemm_vocab_dx", "gemm_vocab_dw"};
  return names[pass];
}

// Launches one product; sets the tile counts along N (and M for the weight
// gradients) for the kernel it picks (int8: for the one the caller picked).
template <int MODE, int PASS>
moe_status launch_gemm(hipStream_t s, moe_dtype dt, const FfnPlan& pl, char* ws, GemmParams p,
                       bool mid_i8 = false) {
  constexpr bool VARK = is_dw(MODE), GATED = is_gated(MODE);
  constexpr bool ACTIVE = MODE != M_STORE && MODE != M_ADD_STORE && MODE != M_I8_STORE && !VARK;
  const bool mid = is_i8(MODE) ? mid_i8 : use_mid_tiles(pl, dt, VARK, GATED, ACTIVE, b_layout(PASS) == L_KM, p);
  const int tn = mid ? kMidN : BN;
  p.ntiles = cdiv(p.N, GATED ? tn / 2 : tn);
  p.dw_h = kMidDwH;
  if constexpr (VARK) {
    // fp32 weight gradients: the highest tile that still gives every place of
    // the persistent grid one
    if (dt == MOE_F32)
      while (p.dw_h > 1 && static_cast<int64_t>(pl.E) * cdiv(p.M_out, p.dw_h * kMidUnit) * p.ntiles <
                               2 * persistent_grid())
        p.dw_h /= 2;
    p.mtiles_out = cdiv(p.M_out, mid ? p.dw_h * kMidUnit : BM);
  }
  // tile list 0: the products with N = f (H, dA); list 1: N = d (Y, dX)
  p.mid_list = PASS == P_FWD_H || PASS == P_BWD_DA ? 0 : 1;
  if (mid) p.mtile = reinterpret_cast<const int2*>(ws + pl.o_mid) + p.mid_list * static_cast<int64_t>(pl.max_mid);
  // the persistent grid, or fewer workgroups (a multiple of 8, for the XCD
  // mapping) when even the most tiles the schedule can list are fewer
  const int64_t max_items = VARK ? static_cast<int64_t>(pl.max_segs) * p.mtiles_out * p.ntiles
                                 : static_cast<int64_t>(mid ? pl.max_mid : pl.max_mtiles) *
                                       p.ntiles;
  const int64_t full = (mid ? 2 : 1) * static_cast<int64_t>(persistent_grid());
  const int grid = static_cast<int>(std::min(full, std::max<int64_t>(kXcds, (max_items + kXcds - 1) / kXcds * kXcds)));
  MOE_TIMED(pass_name(PASS), s);
  if (dt == MOE_F32) {
    if constexpr (PASS != P_BWD_DX_T && !is_i8(MODE)) ffn_gemm_f32_kernel<MODE, PASS><<<grid, kThreads16, 0, s>>>(p);
  } else if (mid) {
    ffn_gemm16_mid_kernel<MODE, PASS><<<grid, kThreads16, 0, s>>>(p);
  } else {
    ffn_gemm16_kernel<MODE, PASS><<<grid, kThreads16, 0, s>>>(p);
  }
  MOE_LAUNCH_CHECK();
  return MOE_OK;
}

#define MOE_TRY(...)                       \
  do {                                     \
    moe_status st_ = (__VA_ARGS__);        \
    if (st_ != MOE_OK) return st_;         \
  } while (0)

// dW[g] = sum of expert g's split slots: rows [0, split_row) of the [M_out, N]
// result go to dwA, the rest to dwB; dw_gstride is the per-expert stride of
// dwA and dwB (f x d for [dW1; dW3], whose M_out is 2f under SwiGLU).
moe_status launch_split_reduce(hipStream_t s, const FfnPlan& pl, char* ws, int M_out, int N,
                               float* dwA, float* dwB, int split_row, int64_t dw_gstride) {
  const int64_t elems = static_cast<int64_t>(M_out) * N;
  const int64_t bx = cdiv(elems, 1024);
  dim3 grid(static_cast<unsigned>(bx < kReduceBlocks ? bx : kReduceBlocks), pl.E);
  MOE_TIMED("split_reduce", s);
  split_reduce_kernel<<<grid, 256, 0, s>>>(
      reinterpret_cast<const float*>(ws + pl.o_part), elems,
      reinterpret_cast<const Sched*>(ws + pl.o_sched), dwA, dwB, dw_gstride, split_row, N);
  MOE_LAUNCH_CHECK();
  return MOE_OK;
}

// dst[g] = [src1[g]; src2[g]]^T for g < E (src1 [K1, N], src2 [K2, N] per expert).
moe_status launch_transpose_w(hipStream_t s, int E, const void* src1, const void* src2, int K1,
                              int K2, int N, void* dst) {
  const dim3 grid(cdiv(N, kTr), std::min(cdiv(K1 + K2, kTr), 32768), E);
  MOE_TIMED("transpose_w", s);
  transpose_w_kernel<<<grid, 256, 0, s>>>(static_cast<const uint16_t*>(src1),
                                          static_cast<const uint16_t*>(src2), K1, K2, N,
                                          static_cast<uint16_t*>(dst));
  MOE_LAUNCH_CHECK();
  return MOE_OK;
}

}  // namespace
}  // namespace moe
