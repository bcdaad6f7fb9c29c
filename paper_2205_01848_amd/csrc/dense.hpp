// Dense products: one group of rows, sizes known on the host: their launch, by the
// plan of plan.hpp.
#pragma once

#include "deep.hpp"
#include "plan.hpp"

namespace moe {
namespace {

// The product's sizes as plan_dense (plan.hpp) takes them.
template <int MODE, int PASS>
DensePlan dense_plan(moe_dtype dt, int M, int N, int K, int64_t lda, int64_t ldb) {
  return plan_dense({dt == MOE_F32, is_gated(MODE), MODE == M_GATED_FWD || MODE == M_GATED_DA,
                     b_layout(PASS) == L_KM, is_dw(MODE), M, N, K, lda, ldb}, persistent_grid(), g_tile_mode);
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
