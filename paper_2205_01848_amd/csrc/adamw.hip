// AdamW over many tensors in one launch (40 a launch), with states in 32 or in 8 bits:
//     m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2   (g times an optional device scale)
//     p = p (1 - lr wd) - lr m / (1 - b1^t) / (sqrt(v / (1 - b2^t)) + eps)
// p taken from, and kept in, a 32-bit original where the tensor has one.
//
// States in 8 bits.  A block of 128 values shares one exponent e, that of its largest,
// kept in a byte; a value keeps the leading bits of its 32-bit number, counted down from
// the block's top octave: code c stands for the float with the bits
//     (c + ((e - 15) << k)) << (23 - k),     0 for c = 0,
// k = 3 bits of mantissa for m beside its sign, k = 4 for v, so both span 16 octaves.
// Encoding and decoding are integer additions and shifts, and a block whose values
// all shrink alike keeps its codes and lowers e.
//
// The bits that are dropped round up with the probability that they are worth.  Rounded
// to nearest, a step of b2 = 0.999 could not move v, whose codes lie 1/32 to 1/16 apart: its
// change of at most a thousandth a step is lost unless g^2 is more than 30 v, so v
// would climb with outliers and never come down.  Rounded at random the codes are right on
// average.  A v above 0 never becomes 0, where the next step would divide m by eps.  A v
// beyond float32 (a gradient of 1e21) is kept as its block's largest, and its m as 0: beside
// a v that has come down to its neighbours' size the next step would divide an m of 1e20 by it.
// Counted into the block's exponent instead it would hold up every neighbour's v.
// The random bits are a function of (seed, tensor, element), so a step can be repeated.
//
// So that a value's code does not depend on how its sums were rounded, the moments of
// 8-bit states are formed in float64, whose operations run at the rate of those of
// float32 here, and the code is taken from its high word (20 of the 52 bits of
// mantissa, 17 or 16 of them behind the code's, are all that the random bits reach).
// Every product is rounded by itself: with decimal betas sums like (9 m + g) / 10 lie
// exactly on the borders that the random bits draw often enough (2 of 40 million) for a
// fused multiply-add to give other codes than the formula written out.
//
// Bound by memory: bf16 weights, fp32 gradients and 8-bit states take 12 bytes a value,
// 32-bit states and originals beside them 32.  A thread takes 8 neighbouring values, so a
// block of 128 is a row of 16 lanes, whose maximum four DPP steps find.  277 million
// values of the first kind: 740 us, 4.5 TB/s (902 with a division by the compiler's exact sequence
// and guards on every access, as its vector units bound it); unpacking them 502 us,
// 5.5 TB/s (703 with 32 bytes a lane and array, half a line a store); 33.6 million of the second:
// 196 us, 5.5 TB/s.

#include <algorithm>
#include <cmath>

#include "common.hpp"
#include "validate.hpp"

namespace moe {
namespace {

constexpr int kList = 40;              // tensors of a launch (kernel arguments: at most 4 KB)
constexpr int kAdamThreads = 256;
constexpr int kTile = kAdamThreads * 8;
constexpr int kBlock = 128;            // values that share an exponent

struct AdamTensor {
  void* p;
  const void* g;
  float* master;
  void *m, *v;
  uint8_t *m_exp, *v_exp;
  int64_t n;
  float decay;
  uint32_t key;        // of its random bits, but for the seed
  int first;           // its first chunk
  int p16, g16;        // bf16
};
struct AdamArgs {
  AdamTensor t[kList];
  int count, chunks, tiles;   // tiles a chunk
  float lr, c1, c2, eps;      // c1 = 1 / (1 - b1^t), c2 = 1 / sqrt(1 - b2^t)
  double b1, b2, a1, a2;      // a = 1 - b
  uint32_t seed;
  const float* grad_scale;
  const moe_adamw_schedule* schedule;
};
static_assert(sizeof(AdamArgs) <= 4096, "kernel arguments");

// The tensor of a chunk: the last one that starts at or before it (empty tensors have no
// chunk).  All on scalars.
__device__ __forceinline__ int find_tensor(const AdamArgs& a, int chunk) {
  int lo = 0, hi = a.count;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (a.t[mid].first <= chunk) lo = mid;
    else hi = mid;
  }
  return lo;
}

// 8 values from p + i on, `left` of them there (FULL: all).
template <bool FULL>
__device__ __forceinline__ void load8(const void* p, bool b16, int64_t i, int64_t left, float (&f)[8]) {
  if (FULL || left >= 8) {
    if (b16) {
      unpack8(*reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + i), f);
    } else {
      const uint4* q = reinterpret_cast<const uint4*>(static_cast<const float*>(p) + i);
      const uint4 a = q[0], b = q[1];
      Elem<float>::load(a, f);
      Elem<float>::load(b, f + 4);
    }
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e)
    f[e] = e >= left ? 0.f : b16 ? bf2f(static_cast<const uint16_t*>(p)[i + e]) : static_cast<const float*>(p)[i + e];
}
template <bool FULL>
__device__ __forceinline__ void store8(void* p, bool b16, int64_t i, int64_t left, const float (&f)[8]) {
  if (FULL || left >= 8) {
    if (b16) {
      *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p) + i) = pack8(f);
    } else {
      uint4* q = reinterpret_cast<uint4*>(static_cast<float*>(p) + i);
      q[0] = Elem<float>::store(f);
      q[1] = Elem<float>::store(f + 4);
    }
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (e < left) {
      if (b16) static_cast<uint16_t*>(p)[i + e] = f2bf(f[e]);
      else static_cast<float*>(p)[i + e] = f[e];
    }
}
template <bool FULL> __device__ __forceinline__ uint2 load_codes(const void* p, int64_t i, int64_t left) {
  const uint8_t* q = static_cast<const uint8_t*>(p) + i;
  if (FULL || left >= 8) return *reinterpret_cast<const uint2*>(q);
  uint32_t w[2] = {0, 0};
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (e < left) w[e / 4] |= static_cast<uint32_t>(q[e]) << (e % 4 * 8);
  return make_uint2(w[0], w[1]);
}
template <bool FULL>
__device__ __forceinline__ void store_codes(void* p, int64_t i, int64_t left, const uint32_t (&c)[8]) {
  uint8_t* q = static_cast<uint8_t*>(p) + i;
  if (FULL || left >= 8) {
    *reinterpret_cast<uint2*>(q) = make_uint2(c[0] | c[1] << 8 | c[2] << 16 | c[3] << 24,
                                              c[4] | c[5] << 8 | c[6] << 16 | c[7] << 24);
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (e < left) q[e] = static_cast<uint8_t>(c[e]);
}
__device__ __forceinline__ uint32_t code_of(const uint2& c, int e) { return (e < 4 ? c.x : c.y) >> (e % 4 * 8) & 255; }

// What code c of a block with exponent e stands for, base = 8 (e - 15) for m, 16 (e - 15) for v.
__device__ __forceinline__ float decode_m(uint32_t c, int base) {
  const uint32_t size = c & 127;
  const float x = __uint_as_float(((size + base) << 20) | (c & 128) << 24);
  return size ? x : c ? NAN : 0.f;
}
__device__ __forceinline__ float decode_v(uint32_t c, int base) {
  return c ? __uint_as_float((c + base) << 19) : 0.f;
}

// The largest of a row of 16 lanes, in all of them.
template <int CTRL> __device__ __forceinline__ int dpp_max(int v) {
  return max(v, __builtin_amdgcn_update_dpp(v, v, CTRL, 0xF, 0xF, false));
}
__device__ __forceinline__ int row16_max(int v) {
  v = dpp_max<0xB1>(v);    // lanes 1 apart, then 2, then the other half of 8, of 16
  v = dpp_max<0x4E>(v);
  v = dpp_max<0x141>(v);
  return dpp_max<0x140>(v);
}

// The element's random bits: 16 low ones for m, 16 high ones for v.
__device__ __forceinline__ uint32_t random_bits(uint32_t x) {
  x = (x ^ x >> 16) * 0x9E3779B1u;
  x = (x ^ x >> 15) * 0x85157AF5u;
  return x ^ x >> 16;
}

// b x + a y in float64, three roundings.
__device__ __forceinline__ double mix(double b, double x, double a, double y) {
#pragma clang fp contract(off)
  const double p = b * x, q = a * y;
  return p + q;
}

struct AdamStep {
  float lr, c1, c2, scale;
  uint32_t seed;
};

// sqrt(v) by the hardware's root, within one unit in the last place (of a v that is tiny as
// of one 2^64 times its size: the hardware takes subnormal numbers for zero).
__device__ __forceinline__ float root(float v) {
  const bool tiny = v < 0x1p-96f;
  const float s = __builtin_amdgcn_sqrtf(tiny ? v * 0x1p64f : v);
  return tiny ? s * 0x1p-32f : s;
}

// The decay joins the update, not a factor 1 - lr wd, which has steps of 6e-8 (lr wd = 1e-7 would
// be 1.2e-7, 2e-8 nothing, for every weight and step alike).  Infinite weights stay what they are.
__device__ __forceinline__ void update(float (&p)[8], const float (&m)[8], const float (&v)[8],
                                       const AdamStep& st, float decay, float eps) {
  const float rate = st.lr * st.c1;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float den = __builtin_fmaf(root(v[e]), st.c2, eps);
    const float x = rate * m[e] * __builtin_amdgcn_rcpf(den);
    p[e] -= __builtin_fmaf(decay, __builtin_amdgcn_fmed3f(p[e], -0x1.fffffep127f, 0x1.fffffep127f), x);
  }
}

// A thread's 8 values with states in 8 bits: the moments in m and v, their codes and
// exponents written.  All lanes of the wavefront take part (left <= 0: with nothing).
constexpr int kBeyondM = 255 << 3, kBeyondV = 255 << 4;   // left of the border: not a finite float32
template <bool FULL>
__device__ __forceinline__ void step_codes(const AdamArgs& a, const AdamTensor& t, const AdamStep& st, int64_t i,
                                           int64_t left, const float (&g)[8], float (&m)[8], float (&v)[8]) {
  const uint2 mc = load_codes<FULL>(t.m, i, left), vc = load_codes<FULL>(t.v, i, left);
  const int64_t blk = i / kBlock;
  const bool here = FULL || left > 0;
  const int mb = here ? (t.m_exp[blk] - 15) * 8 : 0, vb = here ? (t.v_exp[blk] - 15) * 16 : 0;
  const uint32_t x0 = static_cast<uint32_t>(i) * 0xBB67AE85u + static_cast<uint32_t>(i >> 32) * 0x6A09E667u +
                      (st.seed ^ t.key);
  uint32_t mh[8], vh[8];
  int mt[8], vt[8], mmost = 16 << 3, vmost = 16 << 4;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const double gd = static_cast<double>(g[e]) * st.scale;
    const double md = mix(a.b1, decode_m(code_of(mc, e), mb), a.a1, gd);
    const double vd = mix(a.b2, decode_v(code_of(vc, e), vb), a.a2, gd * gd);
    m[e] = static_cast<float>(md);
    v[e] = static_cast<float>(vd);
    const uint32_t rnd = random_bits(x0 + e * 0xBB67AE85u);
    mh[e] = static_cast<uint32_t>(__double2hiint(md));
    vh[e] = static_cast<uint32_t>(__double2hiint(vd));
    mt[e] = static_cast<int>(((mh[e] & 0x7FFFFFFFu) + ((rnd & 0xFFFF) << 1)) >> 17) - ((1023 - 127) << 3);
    vt[e] = static_cast<int>(((vh[e] & 0x7FFFFFFFu) + (rnd >> 16)) >> 16) - ((1023 - 127) << 4);
    mmost = max(mmost, mt[e]);
    vmost = max(vmost, vt[e]);
  }
  // (values that are not finite as float32 do not count; they are rare enough to branch on)
  const bool odd = __any(mmost >= kBeyondM || vmost >= kBeyondV);
  if (odd) {
    mmost = 16 << 3;
    vmost = 16 << 4;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (vt[e] >= kBeyondV && mt[e] < kBeyondM) mt[e] = 0;
      mmost = max(mmost, mt[e] < kBeyondM ? mt[e] : 0);
      vmost = max(vmost, vt[e] < kBeyondV ? vt[e] : 0);
    }
  }
  const int mtop = row16_max(mmost) >> 3, vtop = row16_max(vmost) >> 4;
  uint32_t mq[8], vq[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int c = mt[e] - (mtop - 15) * 8;
    mq[e] = c > 0 ? c | (mh[e] >> 24 & 128) : 0;
    vq[e] = max(vt[e] - (vtop - 15) * 16, static_cast<int>(min(vh[e], 1u)));   // a v above 0 stays so
  }
  if (odd) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (mt[e] >= kBeyondM) mq[e] = 128;
      if (vt[e] >= kBeyondV) vq[e] = 255;
    }
  }
  store_codes<FULL>(t.m, i, left, mq);
  store_codes<FULL>(t.v, i, left, vq);
  if (here && threadIdx.x % (kBlock / 8) == 0) {
    t.m_exp[blk] = static_cast<uint8_t>(mtop);
    t.v_exp[blk] = static_cast<uint8_t>(vtop);
  }
}

template <bool FULL>
__device__ __forceinline__ void step_tile(const AdamArgs& a, const AdamTensor& t, const AdamStep& st, int64_t i,
                                          float decay) {
  const int64_t left = t.n - i;
  float g[8], p[8], m[8], v[8];
  load8<FULL>(t.g, t.g16, i, left, g);
  if (t.master) load8<FULL>(t.master, false, i, left, p);
  else load8<FULL>(t.p, t.p16, i, left, p);
  if (t.m_exp) {
    step_codes<FULL>(a, t, st, i, left, g, m, v);
  } else {
    load8<FULL>(t.m, false, i, left, m);
    load8<FULL>(t.v, false, i, left, v);
    const float b1 = static_cast<float>(a.b1), b2 = static_cast<float>(a.b2);
    const float a1 = static_cast<float>(a.a1), a2 = static_cast<float>(a.a2);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      g[e] *= st.scale;
      m[e] = b1 * m[e] + a1 * g[e];
      v[e] = b2 * v[e] + a2 * (g[e] * g[e]);
    }
    store8<FULL>(t.m, false, i, left, m);
    store8<FULL>(t.v, false, i, left, v);
  }
  update(p, m, v, st, decay, a.eps);
  if (t.master) store8<FULL>(t.master, false, i, left, p);
  store8<FULL>(t.p, t.p16, i, left, p);
}

__global__ __launch_bounds__(kAdamThreads) void adamw_kernel(const AdamArgs a) {
  AdamStep st = {a.lr, a.c1, a.c2, a.grad_scale ? *a.grad_scale : 1.f, a.seed};
  if (a.schedule) {
    st.lr = a.schedule->lr;
    st.c1 = a.schedule->c1;
    st.c2 = a.schedule->c2;
    st.seed = a.schedule->seed;
  }
  const int ti = find_tensor(a, blockIdx.x);
  const AdamTensor& t = a.t[ti];
  int64_t i0 = static_cast<int64_t>(static_cast<int>(blockIdx.x) - t.first) * a.tiles * kTile;
  const float decay = st.lr * t.decay;
  for (int k = 0; k < a.tiles && i0 < t.n; ++k, i0 += kTile) {
    if (i0 + kTile <= t.n) step_tile<true>(a, t, st, i0 + threadIdx.x * 8, decay);
    else step_tile<false>(a, t, st, i0 + threadIdx.x * 8, decay);
  }
}

// The values of 8-bit states: t.m, t.v to the 32-bit t.p and t.master.  Four values a
// thread and store, so that every store of a wavefront covers whole lines.
__global__ __launch_bounds__(kAdamThreads) void adamw_unpack_kernel(const AdamArgs a) {
  const int ti = find_tensor(a, blockIdx.x);
  const AdamTensor& t = a.t[ti];
  const int64_t i0 = static_cast<int64_t>(static_cast<int>(blockIdx.x) - t.first) * a.tiles * kTile;
  for (int k = 0; k < 2 * a.tiles; ++k) {
    const int64_t i = i0 + k * (kTile / 2) + threadIdx.x * 4, left = t.n - i;
    if (left <= 0) break;
    const int mb = (t.m_exp[i / kBlock] - 15) * 8, vb = (t.v_exp[i / kBlock] - 15) * 16;
    const uint8_t *mc = static_cast<const uint8_t*>(t.m) + i, *vc = static_cast<const uint8_t*>(t.v) + i;
    float* m = static_cast<float*>(t.p) + i;
    float* v = t.master + i;
    if (left >= 4) {
      const uint32_t x = *reinterpret_cast<const uint32_t*>(mc), y = *reinterpret_cast<const uint32_t*>(vc);
      floatx4 p, q;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        p[e] = decode_m(x >> (8 * e) & 255, mb);
        q[e] = decode_v(y >> (8 * e) & 255, vb);
      }
      *reinterpret_cast<floatx4*>(m) = p;
      *reinterpret_cast<floatx4*>(v) = q;
    } else {
      for (int e = 0; e < left; ++e) {
        m[e] = decode_m(mc[e], mb);
        v[e] = decode_v(vc[e], vb);
      }
    }
  }
}

bool tensor_ok(const moe_adamw_tensor& t) {
  if (t.n < 0 || !dtype_ok(t.p_dtype) || !dtype_ok(t.g_dtype)) return false;
  if (!(t.weight_decay >= 0) || !(t.weight_decay < INFINITY)) return false;
  if (!t.m_exp != !t.v_exp || (t.master && t.p_dtype == MOE_F32)) return false;
  if (t.n == 0) return true;
  return t.p && t.g && t.m && t.v && aligned16(t.p) && aligned16(t.g) && aligned16(t.master) &&
         aligned16(t.m) && aligned16(t.v);
}

// Launches kernel(args) over the tensors, kList a launch.  `each` fills in a tensor.
template <typename F, typename K>
moe_status for_lists(hipStream_t s, const char* name, int count, const moe_adamw_tensor* ts, AdamArgs a,
                     F&& each, K kernel) {
  // as many tiles a chunk as leave every CU sixteen workgroups, 4 at the most
  int64_t all = 0;
  for (int i = 0; i < count; ++i) all += (ts[i].n + kTile - 1) / kTile;
  a.tiles = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(4, all / (16 * num_cus()))));
  const int64_t chunk = static_cast<int64_t>(a.tiles) * kTile;
  int at = 0;
  while (at < count) {
    a.count = 0;
    int64_t chunks = 0;
    for (; at < count && a.count < kList; ++at) {
      if (ts[at].n == 0) continue;
      const int64_t more = (ts[at].n + chunk - 1) / chunk;
      if (chunks + more > 0x7FFFFFFF) break;   // the next launch's
      AdamTensor& t = a.t[a.count++];
      t = {};
      t.n = ts[at].n;
      t.m = ts[at].m;
      t.v = ts[at].v;
      t.m_exp = ts[at].m_exp;
      t.v_exp = ts[at].v_exp;
      t.first = static_cast<int>(chunks);
      each(t, at);
      chunks += more;
    }
    if (a.count == 0) break;
    a.chunks = static_cast<int>(chunks);
    MOE_TIMED(name, s);
    kernel<<<a.chunks, kAdamThreads, 0, s>>>(a);
    MOE_LAUNCH_CHECK();
  }
  return MOE_OK;
}

}  // namespace
}  // namespace moe

using namespace moe;

extern "C" size_t moe_adamw_blocks(int64_t n) {
  return n < 0 ? 0 : static_cast<size_t>((n + kBlock - 1) / kBlock);
}

extern "C" moe_status moe_adamw(void* stream, int count, const moe_adamw_tensor* tensors, double lr,
                                double beta1, double beta2, double eps, int64_t step, uint32_t seed,
                                const float* grad_scale, const moe_adamw_schedule* schedule) {
  auto fine = [](double v) { return v >= 0 && v < INFINITY; };
  if (count < 0 || (count > 0 && !tensors) || step < 1) return MOE_EINVAL;
  // (the hardware takes a subnormal divisor for zero: 0 / eps would be NaN)
  if (!fine(lr) || !fine(beta1) || !fine(beta2) || beta1 >= 1 || beta2 >= 1 || !fine(eps) ||
      !(static_cast<float>(eps) >= 0x1p-126f))
    return MOE_EINVAL;
  if ((reinterpret_cast<uintptr_t>(schedule) | reinterpret_cast<uintptr_t>(grad_scale)) & 3) return MOE_EINVAL;
  for (int i = 0; i < count; ++i)
    if (!tensor_ok(tensors[i]) || tensors[i].n > int64_t(1) << 40) return MOE_EINVAL;
  AdamArgs a{};
  a.lr = static_cast<float>(lr);
  a.c1 = static_cast<float>(1 / (1 - std::pow(beta1, static_cast<double>(step))));
  a.c2 = static_cast<float>(1 / std::sqrt(1 - std::pow(beta2, static_cast<double>(step))));
  a.eps = static_cast<float>(eps);
  a.b1 = beta1;
  a.b2 = beta2;
  a.a1 = 1 - beta1;
  a.a2 = 1 - beta2;
  a.seed = seed;
  a.grad_scale = grad_scale;
  a.schedule = schedule;
  return for_lists(static_cast<hipStream_t>(stream), "adamw", count, tensors, a,
                   [&](AdamTensor& t, int i) {
                     t.p = tensors[i].p;
                     t.g = tensors[i].g;
                     t.master = tensors[i].master;
                     t.decay = static_cast<float>(tensors[i].weight_decay);
                     t.key = static_cast<uint32_t>(i + 1) * 0x9E3779B9u;
                     t.p16 = tensors[i].p_dtype == MOE_BF16;
                     t.g16 = tensors[i].g_dtype == MOE_BF16;
                   },
                   adamw_kernel);
}

extern "C" moe_status moe_adamw_unpack(void* stream, int count, const moe_adamw_tensor* tensors,
                                       float* const* m, float* const* v) {
  if (count < 0 || (count > 0 && (!tensors || !m || !v))) return MOE_EINVAL;
  for (int i = 0; i < count; ++i) {
    const moe_adamw_tensor& t = tensors[i];
    if (t.n < 0 || t.n > int64_t(1) << 40) return MOE_EINVAL;
    if (t.n > 0 && (!t.m || !t.v || !t.m_exp || !t.v_exp || !m[i] || !v[i] || !aligned16(t.m) ||
                    !aligned16(t.v) || !aligned16(m[i]) || !aligned16(v[i])))
      return MOE_EINVAL;
  }
  return for_lists(static_cast<hipStream_t>(stream), "adamw_unpack", count, tensors, AdamArgs{},
                   [&](AdamTensor& t, int i) {
                     t.p = m[i];
                     t.master = v[i];
                   },
                   adamw_unpack_kernel);
}
