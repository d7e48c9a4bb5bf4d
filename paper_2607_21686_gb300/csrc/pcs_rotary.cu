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
//            the critical path; then each thread moves units of 16 bytes, of 8
//            or 4 where the pairs' halves are no whole vectors, or of one pair
//            where something is not aligned.  With a cache (PAGED) the rows of
//            keys and values go to the slots of the tokens' positions.
//            49,153 tokens of 32 + 8 heads of 128 in float16, neighbours: 163 us,
//            6.2 TB/s (92 % of the measured copy rate), halves 152 us; 23,000 new
//            tokens of 24 sessions, 16 heads of 64: 48 us, 5.9 TB/s.  What is left is
//            instructions (two thirds of the issue slots are taken) and a block's
//            look-ups before its first load.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "pcs_attend.h"
#include "pcs_internal.h"

namespace pcs {
namespace {

constexpr int kThreads = 256;
constexpr int kTokens = 4;     // tokens of a block at most
constexpr int kPairs = 128;    // pairs of a head at most

__device__ __forceinline__ void grid_dependency() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// x + y as a float and what its rounding left (Knuth's two-sum).
__device__ __forceinline__ float two_sum(float x, float y, float& left) {
  const float s = x + y, t = s - x;
  left = (x - (s - t)) + (y - t);
  return s;
}

// Cosine and sine of position times frequency, the product in two floats: the
// position is split so that both parts are exact floats, each product's
// rounding error comes from a fused multiply-add, and the sums' from two_sum.
// (One rounding of a position of 10^5 would cost 0.004 rad.)  The rest turns the
// result: by two terms of its series while it is below 2^-8 (what is left out is
// below 2^-26), by its own sine and cosine at positions beyond, where its
// rounding (2^-17 rad at 2^31) turns them by one term.
__device__ __forceinline__ float2 cos_sin(int32_t pos, float f) {
  const float hi = static_cast<float>(pos & ~0xfff), lo = static_cast<float>(pos & 0xfff);
  const float a = __fmul_rn(hi, f), ae = fmaf(hi, f, -a);
  const float b = __fmul_rn(lo, f), be = fmaf(lo, f, -b);
  float e, left_e, left;
  const float s = two_sum(a, b, e);
  const float rest = two_sum(two_sum(e, ae, left_e), be, left);
  float sn, cs, rs = rest, rc = fmaf(-0.5f * rest, rest, 1.0f);
  sincosf(s, &sn, &cs);
  if (fabsf(rest) > 0.00390625f) {
    float rs1, rc1;
    sincosf(rest, &rs1, &rc1);
    left += left_e;
    rs = fmaf(rc1, left, rs1);
    rc = fmaf(-rs1, left, rc1);
  }
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

// The last of the sessions whose first token is at most t, by one warp: 32
// probes at a time.
__device__ __forceinline__ int session_of(const BatchDev& b, int64_t t, int lane) {
  int lo = 0, n = b.sessions;  // it is among [lo, lo + n)
  while (n > 1) {
    const int step = (n + 31) / 32;
    const int i = lo + lane * step;
    const unsigned m = __ballot_sync(0xffffffffu, lane * step < n && __ldg(b.q_off + i) <= t);
    const int k = m ? 31 - __clz(m) : 0;
    lo += k * step;
    n = min(step, n - k * step);
  }
  return lo;
}

__device__ __forceinline__ Place place_of(const RotArgs& a, int64_t t, int s) {
  const BatchDev& b = a.batch;
  int at, m;
  if (b.q_off) {
    int32_t o = __ldg(b.q_off + s), end = __ldg(b.q_off + s + 1);
    while (t >= end && s + 1 < b.sessions) {
      ++s;
      o = end;
      end = __ldg(b.q_off + s + 1);
    }
    m = end - o;
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
  if (kp < 0 || kp >= c.n_pages || vp < 0 || vp >= c.n_pages) {  // neither of them is written
    if (kp < -1 || kp >= c.n_pages || vp < -1 || vp >= c.n_pages) atomicOr(a.err, kDevErrIndex);
    return {-1, -1};
  }
  return {kp * c.page_bytes + row, vp * c.page_bytes + row};
}

// How a block's threads share out a head: `units` side by side, `at_once` heads.
// (A head has at most 256 elements, so no more units than there are threads.)
struct Share {
  int32_t units, at_once;
  FastDiv by_units;
  void set(int units_) {
    units = units_;
    at_once = kThreads / units_;
    by_units.set(units_);
  }
};
struct Shares {
  Share turned, plain;             // heads that are turned, that are copied
  FastDiv by_heads[kRotTensors];   // by a tensor's heads
};

__device__ __forceinline__ int64_t times(uint32_t n, int64_t stride) {
  return static_cast<int64_t>(static_cast<uint64_t>(n) * static_cast<uint64_t>(stride));
}

// Units of VE elements, or with halves (a pair's elements lie in two runs) VE
// of each; VE 1: one pair or one element.  Turns the pairs from `cs` on, `live`
// of which there are (neighbours: a unit may end in elements that stay).
template <typename T, int VE, bool IL>
__device__ __forceinline__ void turn_unit(Run<T, VE>& x, Run<T, VE>& y, const float2* cs, int live) {
  if constexpr (VE == 1) {
    const float2 c = cs[0];
    const float p = to_float(x.e[0]), q = to_float(y.e[0]);
    x.e[0] = from_float<T>(p * c.x - q * c.y);
    y.e[0] = from_float<T>(p * c.y + q * c.x);
  } else {
    const float4* c4 = reinterpret_cast<const float4*>(cs);
    constexpr int kPairsHere = IL ? VE / 2 : VE;
#pragma unroll
    for (int i = 0; i < kPairsHere; i += 2) {
      const float4 c = c4[i / 2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const float co = k ? c.z : c.x, si = k ? c.w : c.y;
        T& u = IL ? x.e[2 * (i + k)] : x.e[i + k];
        T& v = IL ? x.e[2 * (i + k) + 1] : y.e[i + k];
        const float p = to_float(u), q = to_float(v);
        if (IL && i + k >= live) continue;
        u = from_float<T>(p * co - q * si);
        v = from_float<T>(p * si + q * co);
      }
    }
  }
}

// A token's cosines and sines begin at a multiple of 32 bytes.
__device__ __forceinline__ int pairs_row(const RotArgs& a) { return (a.pairs + 3) & ~3; }

// A block's tokens [t0, t0 + nt) and tensors [n0, n1); their cosines and sines,
// and the rows of the cache they go to, are in shared memory after this.
struct BlockWork {
  int64_t t0;
  int nt, n0, n1;
};
template <bool PAGED>
__device__ __forceinline__ BlockWork block_setup(const RotArgs& a, int per_block, float2* cs, Place* place) {
  grid_dependency();
  BlockWork b;
  b.t0 = static_cast<int64_t>(blockIdx.x) * per_block;
  b.nt = static_cast<int>(a.tokens - b.t0 < per_block ? a.tokens - b.t0 : per_block);
  b.n0 = gridDim.y > 1 ? blockIdx.y : 0;
  b.n1 = gridDim.y > 1 ? b.n0 + 1 : a.n;
  const int tid = threadIdx.x, lane = tid & 31;
  if (PAGED && tid >= kThreads - 32 && a.t[b.n1 - 1].role) {  // the last warp looks the tokens up
    const int s = a.batch.q_off ? session_of(a.batch, b.t0, lane) : 0;
    if (lane < b.nt) place[lane] = place_of(a, b.t0 + lane, s);
  }
  if (b.n0 < a.plain)
    for (int i = tid; i < b.nt * a.pairs; i += kThreads) {
      const int t = i / a.pairs, p = i - t * a.pairs;
      int axis = 0;
      while (axis < a.axes - 1 && p >= a.axis_end[axis]) ++axis;
      float2 x = cos_sin(__ldg(a.pos + (b.t0 + t) * a.axes + axis), __ldg(a.freq + p));
      if (a.inverse) x.y = -x.y;
      cs[t * pairs_row(a) + p] = x;
    }
  __syncthreads();
  return b;
}

template <typename T, int VE, bool IL, bool PAGED>
__global__ void __launch_bounds__(kThreads, 7)
    k_rotate(const __grid_constant__ RotArgs a, const __grid_constant__ Shares shares, int per_block, int turn) {
  using V = Run<T, VE>;
  constexpr bool kTwo = !IL || VE == 1;         // a turned unit has two runs
  __shared__ __align__(32) float2 cs[kTokens * kPairs + 4];
  __shared__ Place place[kTokens];
  const BlockWork b = block_setup<PAGED>(a, per_block, cs, place);
  const int64_t t0 = b.t0;
  const int nt = b.nt, n0 = b.n0, n1 = b.n1, tid = threadIdx.x;
  const int row = pairs_row(a);
  const int64_t second = (IL ? 1 : a.pairs) * static_cast<int64_t>(sizeof(T));  // from a pair's first element
  for (int n = n0; n < n1; ++n) {
    const RotSlot& z = a.t[n];
    const Share& sh = n < a.plain ? shares.turned : shares.plain;
    const int turned = n < a.plain ? turn : 0;
    const int heads = z.heads - (n ? a.t[n - 1].heads : 0), total = nt * heads;
    const int h0 = sh.by_units.div(tid), r = tid - h0 * sh.units;
    if (h0 >= sh.at_once) continue;
    const bool turns = r < turned;
    const int pair = VE == 1 ? r : IL ? r * (VE / 2) : r * VE;
    const int e = (turns ? (VE == 1 && IL ? 2 * r : r * VE) : (turned ? (VE > 1 && IL ? turned * VE : 2 * a.pairs) : 0) + (r - turned) * VE) *
                  static_cast<int>(sizeof(T));
    const uint8_t* const src0 = z.src + t0 * z.src_token;
    // A unit at a time, of as many threads as an SM's registers hold (49,153 tokens
    // of 32 + 8 heads of 128, neighbours: when that took 165 us, two units of fewer
    // threads took 184 us, four 186 us, eight 286 us).
    for (int p = h0; p < total; p += sh.at_once) {
      // (t is never below zero.  The branch keeps the compiler from moving all that
      // follows from t's place ahead of the loop, where it does not fit the 32
      // registers that seven blocks an SM leave: 217 us without it, 164 us with.)
      const int t = shares.by_heads[n].div(p), h = p - t * heads;
      if (t < 0) continue;
      const uint8_t* src = src0 + times(t, z.src_token) + times(h, z.src_head) + e;
      V x = *reinterpret_cast<const V*>(src), y;
      if (kTwo && turns) y = *reinterpret_cast<const V*>(src + second);
      uint8_t* dst;
      if (PAGED && z.role) {
        const int64_t at = z.role == 1 ? place[t].k : place[t].v;
        if (at < 0) continue;
        dst = (z.role == 1 ? a.cache.k : a.cache.v) + at + times(h, a.cache.head_bytes) + e;
      } else {
        dst = z.dst + (t0 + t) * z.dst_token + times(h, z.dst_head) + e;
      }
      if (turns) {
        turn_unit<T, VE, IL>(x, y, cs + t * row + pair, a.pairs - pair);
        if (kTwo) *reinterpret_cast<V*>(dst + second) = y;
      }
      *reinterpret_cast<V*>(dst) = x;
    }
  }
}

// Few tokens: a block for each and each tensor, for latency; many: up to
// kTokens a block, which shares the setup among them and all tensors while
// every SM still has two blocks.
cudaLaunchConfig_t config(const RotArgs& a, int sm_count, int* per_block, cudaLaunchAttribute* attr, cudaStream_t stream) {
  const int64_t share = a.tokens / (2 * sm_count);
  *per_block = static_cast<int>(share < 1 ? 1 : share > kTokens ? kTokens : share);
  attr->id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr->val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>((a.tokens + *per_block - 1) / *per_block), share < 2 ? a.n : 1);
  cfg.blockDim = dim3(kThreads);
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cfg;
}

template <typename T, int VE, bool IL, bool PAGED>
cudaError_t launch(const RotArgs& a, int sm_count, cudaStream_t stream) {
  const int turn = a.pairs == 0 ? 0 : VE == 1 ? a.pairs : IL ? (2 * a.pairs + VE - 1) / VE : a.pairs / VE;
  Shares shares;
  shares.turned.set(VE > 1 && IL ? a.head_dim / VE : turn + (a.head_dim - 2 * a.pairs) / VE);
  shares.plain.set(a.head_dim / VE);
  for (int n = 0; n < a.n; ++n) shares.by_heads[n].set(a.t[n].heads - (n ? a.t[n - 1].heads : 0));
  int per_block;
  cudaLaunchAttribute attr;
  const cudaLaunchConfig_t cfg = config(a, sm_count, &per_block, &attr, stream);
  return cudaLaunchKernelEx(&cfg, k_rotate<T, VE, IL, PAGED>, a, shares, per_block, turn);
}

// The widest units of whole vectors (neighbours: of vectors that may end in
// elements that stay; halves: a half is a number of whole units, for a thread has
// both elements of its pairs).  49,153 tokens of 32 + 8 heads of 128: 64 pairs, in
// units of 16 bytes, 152 us; 60 pairs, of 8 bytes, 172 us; 62, of 4 bytes, 240 us;
// pair by pair 389 us.
template <typename T, bool PAGED>
cudaError_t by_unit(const RotArgs& a, bool vec, int sm_count, cudaStream_t stream) {
  constexpr int V = 16 / sizeof(T);
  if (a.interleaved)
    return vec ? launch<T, V, true, PAGED>(a, sm_count, stream) : launch<T, 1, true, PAGED>(a, sm_count, stream);
  if (vec && a.pairs % V == 0) return launch<T, V, false, PAGED>(a, sm_count, stream);
  if constexpr (V == 8)
    if (vec && a.pairs % 4 == 0) return launch<T, 4, false, PAGED>(a, sm_count, stream);
  if (vec && a.pairs % 2 == 0) return launch<T, 2, false, PAGED>(a, sm_count, stream);
  return launch<T, 1, false, PAGED>(a, sm_count, stream);
}

template <typename T>
cudaError_t by_form(const RotArgs& a, bool paged, bool vec, int sm_count, cudaStream_t stream) {
  if constexpr (sizeof(T) == 2)
    if (paged) return by_unit<T, true>(a, vec, sm_count, stream);
  return by_unit<T, false>(a, vec, sm_count, stream);
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
