// pcs_rotary.cu -- rotary positions with several axes, and the append that
// writes rotated keys and values into the pages of a cache.
//
// k_rotate   y = R x per token and head: pair i turns by the angle
//            pos[axis of i] * freq[i].  R is orthogonal, so its gradient is
//            the turn by the opposite angle (inverse).  Every element is read
//            and written once and costs three flops: the bound is HBM.
//            A block takes a few tokens: their cosines and sines are computed
//            once into shared memory and serve all heads of all tensors, which
//            is what keeps the trigonometry (some 40 instructions a pair) off
//            the critical path; then each thread moves units of 16 bytes, or
//            of one pair where something is not aligned to 16 bytes.
//            With a cache (PAGED) the rows of keys and values go to the slots
//            of the tokens' positions.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "pcs_attend.h"
#include "pcs_internal.h"

namespace pcs {
namespace {

constexpr int kThreads = 256;
constexpr int kTokens = 8;     // tokens of a block at most
constexpr int kPairs = 128;    // pairs of a head at most
constexpr int kUnroll = 4;     // units in flight per thread

__device__ __forceinline__ void grid_dependency() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// Cosine and sine of position times frequency, the product in two floats: the
// position is split so that both parts are exact floats, each product's
// rounding error comes from a fused multiply-add, and the sum's from Knuth's
// two-sum.  (One rounding of a position of 10^5 would cost 0.004 rad.)  The
// rest turns the result: by two terms of its series while it is below 2^-8
// (what is left out is below 2^-26), by its own sine and cosine at positions
// beyond.
__device__ __forceinline__ float2 cos_sin(int32_t pos, float f) {
  const float hi = static_cast<float>(pos & ~0xfff), lo = static_cast<float>(pos & 0xfff);
  const float a = hi * f, ae = fmaf(hi, f, -a);
  const float b = lo * f, be = fmaf(lo, f, -b);
  const float s = a + b, t = s - a;
  const float rest = (((a - (s - t)) + (b - t)) + ae) + be;
  float sn, cs, rs = rest, rc = fmaf(-0.5f * rest, rest, 1.0f);
  sincosf(s, &sn, &cs);
  if (fabsf(rest) > 0.00390625f) sincosf(rest, &rs, &rc);
  return make_float2(fmaf(cs, rc, -sn * rs), fmaf(sn, rc, cs * rs));
}

template <typename T>
__device__ __forceinline__ float to_float(T x) { return static_cast<float>(x); }
template <typename T>
__device__ __forceinline__ T from_float(float x);
template <>
__device__ __forceinline__ float from_float<float>(float x) { return x; }
template <>
__device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// N elements that are moved together.
template <typename T, int N>
struct alignas(sizeof(T) * N) Run {
  T e[N];
};

// Where a token's row of the cache is: byte offsets, or -1.
struct Place {
  int64_t k, v;
};

__device__ __forceinline__ Place place_of(const RotArgs& a, int64_t t) {
  const BatchDev& b = a.batch;
  int s, at, m;
  if (b.q_off) {
    int lo = 0, hi = b.sessions;  // the last session whose first token is at most t
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (__ldg(b.q_off + mid) <= t) lo = mid;
      else hi = mid;
    }
    s = lo;
    const int32_t o = __ldg(b.q_off + s);
    m = __ldg(b.q_off + s + 1) - o;
    at = static_cast<int>(t - o);
    if (at < 0 || at >= m) return {-1, -1};
  } else {
    s = static_cast<int>(t / b.each);
    m = b.each;
    at = static_cast<int>(t - static_cast<int64_t>(s) * m);
  }
  const CacheDev& c = a.cache;
  const int64_t len = __ldg(b.lens + s), p = len - m + at;
  if (p < 0) {
    atomicOr(a.err, kDevErrIndex);
    return {-1, -1};
  }
  if (c.ring_rows && p >= c.sinks && p < len - c.ring_rows) return {-1, -1};
  const uint32_t slot = c.slot_of(static_cast<uint32_t>(p));
  if (slot >= static_cast<uint32_t>(c.slots)) {
    atomicOr(a.err, kDevErrIndex);
    return {-1, -1};
  }
  const uint32_t page = c.page_rows.div(slot);
  const int64_t row = static_cast<int64_t>(slot - page * c.page_rows.d) * c.row_bytes;
  const int64_t e = s * c.table_stride + page;
  const int32_t kp = __ldg(c.table + e);
  const int32_t vp = c.v_table ? __ldg(c.v_table + e) : kp;
  Place r = {-1, -1};
  if (kp >= 0 && kp < c.n_pages) r.k = kp * c.page_bytes + row;
  else if (kp != -1) atomicOr(a.err, kDevErrIndex);
  if (vp >= 0 && vp < c.n_pages) r.v = vp * c.page_bytes + row;
  else if (vp != -1) atomicOr(a.err, kDevErrIndex);
  return r;
}

// Units of a turned head: `turn` units of VE pairs' worth, then the elements
// behind them; of a copied head: elements.  VE elements a unit (1: one pair or
// one element).
template <typename T, int VE, bool IL, bool PAGED>
__global__ void __launch_bounds__(kThreads)
    k_rotate(const __grid_constant__ RotArgs a, int per_block, int turn, int units_turned,
             int units_plain, FastDiv by_units, FastDiv by_turned, FastDiv by_plain) {
  __shared__ float2 cs[kTokens * kPairs];
  __shared__ Place place[kTokens];
  grid_dependency();
  const int64_t t0 = static_cast<int64_t>(blockIdx.x) * per_block;
  const int nt = static_cast<int>(a.tokens - t0 < per_block ? a.tokens - t0 : per_block);
  for (int i = threadIdx.x; i < nt * a.pairs; i += kThreads) {
    const int t = i / a.pairs, p = i - t * a.pairs;
    int axis = 0;
    while (axis < a.axes - 1 && p >= a.axis_end[axis]) ++axis;
    float2 x = cos_sin(__ldg(a.pos + (t0 + t) * a.axes + axis), __ldg(a.freq + p));
    if (a.inverse) x.y = -x.y;
    cs[i] = x;
  }
  if (PAGED && threadIdx.x < nt) place[threadIdx.x] = place_of(a, t0 + threadIdx.x);
  __syncthreads();

  constexpr bool kPairRuns = !IL;  // the halves of a pair lie in two runs
  using V = Run<T, VE>;
  const int turned_heads = a.plain ? a.t[a.plain - 1].heads : 0;
  const uint32_t units_head = turned_heads * units_turned;
  const uint32_t total = nt * by_units.d;
  for (uint32_t u0 = threadIdx.x; u0 < total; u0 += kThreads * kUnroll) {
    V x[kUnroll], y[kUnroll];
    uint8_t* dst[kUnroll];
    int what[kUnroll];  // the first pair of a turned unit, -1: copied, -2: nothing
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) {
      const uint32_t u = u0 + k * kThreads;
      what[k] = -2;
      if (u >= total) continue;
      const uint32_t t = by_units.div(u);
      uint32_t r = u - t * by_units.d;
      int head, e, w = -1;  // head of the call, first element, first pair
      if (r < units_head) {
        head = by_turned.div(r);
        r -= head * units_turned;
        if (static_cast<int>(r) < turn) {
          if (VE == 1) w = r, e = IL ? 2 * r : r;
          else w = IL ? r * (VE / 2) : r * VE, e = r * VE;
        } else {
          e = 2 * a.pairs + (r - turn) * VE;
        }
      } else {
        r -= units_head;
        const uint32_t h = by_plain.div(r);
        head = turned_heads + h;
        e = (r - h * units_plain) * VE;
      }
      int n = 0;
      while (head >= a.t[n].heads) ++n;
      const RotSlot& z = a.t[n];
      const int h = head - (n ? a.t[n - 1].heads : 0);
      const uint8_t* src = z.src + (t0 + t) * z.src_token + h * z.src_head + e * sizeof(T);
      if (PAGED && z.role) {
        const int64_t row = z.role == 1 ? place[t].k : place[t].v;
        if (row < 0) continue;
        dst[k] = (z.role == 1 ? a.cache.k : a.cache.v) + row + h * a.cache.head_bytes + e * sizeof(T);
      } else {
        dst[k] = z.dst + (t0 + t) * z.dst_token + h * z.dst_head + e * sizeof(T);
      }
      x[k] = *reinterpret_cast<const V*>(src);
      if (w >= 0) {
        if (kPairRuns) y[k] = *reinterpret_cast<const V*>(src + a.pairs * sizeof(T));
        else if (VE == 1) y[k] = *reinterpret_cast<const V*>(src + sizeof(T));
        w += t * a.pairs;
      }
      what[k] = w;
    }
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) {
      if (what[k] == -2) continue;
      if (what[k] >= 0) {
        if (kPairRuns || VE == 1) {
#pragma unroll
          for (int i = 0; i < VE; ++i) {
            const float2 c = cs[what[k] + i];
            const float p = to_float(x[k].e[i]), q = to_float(y[k].e[i]);
            x[k].e[i] = from_float<T>(p * c.x - q * c.y);
            y[k].e[i] = from_float<T>(p * c.y + q * c.x);
          }
          *reinterpret_cast<V*>(dst[k] + (kPairRuns ? a.pairs : 1) * sizeof(T)) = y[k];
        } else {
#pragma unroll
          for (int i = 0; i < VE; i += 2) {
            const float2 c = cs[what[k] + i / 2];
            const float p = to_float(x[k].e[i]), q = to_float(x[k].e[i + 1 < VE ? i + 1 : i]);
            x[k].e[i] = from_float<T>(p * c.x - q * c.y);
            x[k].e[i + 1 < VE ? i + 1 : i] = from_float<T>(p * c.y + q * c.x);
          }
        }
      }
      *reinterpret_cast<V*>(dst[k]) = x[k];
    }
  }
}

template <typename T, int VE, bool IL, bool PAGED>
cudaError_t launch(const RotArgs& a, int sm_count, cudaStream_t stream) {
  const int turn = a.pairs == 0 ? 0 : VE == 1 ? a.pairs : IL ? 2 * a.pairs / VE : a.pairs / VE;
  const int units_turned = turn + (a.head_dim - 2 * a.pairs) / VE;
  const int units_plain = a.head_dim / VE;
  const int turned_heads = a.plain ? a.t[a.plain - 1].heads : 0;
  const int plain_heads = a.t[a.n - 1].heads - turned_heads;
  FastDiv by_units, by_turned, by_plain;
  by_units.set(turned_heads * units_turned + plain_heads * units_plain);
  by_turned.set(units_turned);
  by_plain.set(units_plain);
  // Few tokens: a block each, for latency; many: up to kTokens a block, which
  // shares the setup among them while every SM still has two blocks.
  const int64_t share = a.tokens / (2 * sm_count);
  const int per_block = static_cast<int>(share < 1 ? 1 : share > kTokens ? kTokens : share);
  const int64_t grid = (a.tokens + per_block - 1) / per_block;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(grid));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, k_rotate<T, VE, IL, PAGED>, a, per_block, turn, units_turned,
                            units_plain, by_units, by_turned, by_plain);
}

template <typename T>
cudaError_t by_form(const RotArgs& a, bool paged, bool vec, int sm_count, cudaStream_t stream) {
  constexpr int V = 16 / sizeof(T);
  if constexpr (sizeof(T) == 2) {
    if (paged)
      return vec ? (a.interleaved ? launch<T, V, true, true>(a, sm_count, stream)
                                  : launch<T, V, false, true>(a, sm_count, stream))
                 : (a.interleaved ? launch<T, 1, true, true>(a, sm_count, stream)
                                  : launch<T, 1, false, true>(a, sm_count, stream));
  }
  return vec ? (a.interleaved ? launch<T, V, true, false>(a, sm_count, stream)
                              : launch<T, V, false, false>(a, sm_count, stream))
             : (a.interleaved ? launch<T, 1, true, false>(a, sm_count, stream)
                              : launch<T, 1, false, false>(a, sm_count, stream));
}

}  // namespace

cudaError_t launch_rotate(const RotArgs& a, uint32_t dtype, bool paged, bool vec, int sm_count,
                          cudaStream_t stream) {
  if (a.tokens == 0) return cudaSuccess;
  switch (dtype) {
    case PCS_DT_F16: return by_form<__half>(a, paged, vec, sm_count, stream);
    case PCS_DT_BF16: return by_form<__nv_bfloat16>(a, paged, vec, sm_count, stream);
    default: return by_form<float>(a, paged, vec, sm_count, stream);
  }
}

}  // namespace pcs
