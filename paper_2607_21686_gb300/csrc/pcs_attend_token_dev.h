// pcs_attend_token_dev.h -- the kernel for few query rows a key head over a cache of
// 16-bit elements (pcs_attend_token.cu says what it does and what it measured), and
// the parts of it that the one over 8-bit caches shares.
#pragma once

#include "pcs_attend_dev.h"

namespace pcs {
namespace {

constexpr int kWarps = kTokenWarps;
constexpr int kThreads = 32 * kWarps;
constexpr int kTile = 16;
constexpr unsigned kFull = 0xffffffffu;
// A row's running maximum is raised only when a score exceeds it by 2^8: the
// weights stay below 256 (times 2^kLift), and raising it (a reduction over the warp and a
// pass over the sums) is rare.
constexpr float kSlack = 8.0f;

__device__ __forceinline__ void ldm4(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(at)
               : "memory");
}
__device__ __forceinline__ void ldm4t(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(at)
               : "memory");
}
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
template <typename T>
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void mma<__half>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma<__nv_bfloat16>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Stages of a warp's ring: the loads in flight on an SM have to cover its
// share of HBM (44 GB/s) times the latency, some 64 KB.
template <int DP>
constexpr int kStagesOf = DP == 64 ? 4 : 3;
template <int DP>
constexpr uint32_t kStageBytes = 2 * kTile * DP * 2;
template <int DP>
constexpr uint32_t kRingBytes = kWarps * kStagesOf<DP> * kStageBytes<DP>;

// Blocks that one SM holds: as many rings as its 227 KB of shared memory take
// (2 KB a block for the rest), and as its registers do -- 32 rows of 64 dims want
// some 250 a thread, two blocks' worth.  The compiler is held to it, so that what
// the host takes for one wave of parts is one.  (One session of 100,000 tokens,
// 32 rows of 64 dims: 36 us; 47 us when three blocks were counted on.)  32 rows of
// 128 dims take all 255 registers, and 68 bytes of a thread's values spill.
template <int DP, int NT>
constexpr int kResident = DP == 64 && NT == 4 ? 2 : static_cast<int>(227 * 1024 / (kRingBytes<DP> + 2048));

// Floats of a row of a warp's sums.
template <int DP>
constexpr int kPadOf = DP + 4;

// Joined sums of one row pair of dims; `w` parts with maxima m, totals l.
struct Joined {
  float x, y, top, total;
};

// Joins the sums, maxima and totals that the warps have left in shared memory, and
// the parts of a session: the last part, or a part's own rows where there is one.
template <typename T, int DP, int NT>
__device__ __forceinline__ void join_parts(const AttendArgs& a, const SessionView& view, uint8_t* smem, int s, int head,
                                           int sp) {
  constexpr int kRows = 8 * NT, kPad = kPadOf<DP>;
  __shared__ uint32_t last;
  const int tid = threadIdx.x, rows = view.m * a.group, head_dim = a.cache.head_dim;
  float* sums = reinterpret_cast<float*>(smem);           // [warp][row][kPad]
  float* tops = sums + kWarps * kRows * kPad;             // [warp][row]
  float* totals = tops + kWarps * kRows;
  constexpr float kLn2 = 0.693147180559945309f;
  auto write = [&](int row, int d, const Joined& j) {
    const uint32_t tok = a.by_group.div(row);
    const int64_t t = view.q0 + tok;
    const int h = head * a.group + (row - tok * a.group);
    const float inv = j.total == 0.0f ? 0.0f : 1.0f / j.total;
    if (d < head_dim)
      *reinterpret_cast<uint32_t*>(a.out.data + t * a.out.token_bytes + h * a.out.head_bytes + d * 2) =
          pack2<T>(j.x * inv, j.y * inv);
    if (d == 0 && a.lse)
      a.lse[t * (static_cast<int64_t>(a.cache.heads) * a.group) + h] =
          j.total == 0.0f ? -INFINITY : fmaf(j.top - kLift<T>, kLn2, logf(j.total));
  };
  const int64_t pair = static_cast<int64_t>(s) * a.cache.heads + head;
  const int64_t part_floats = static_cast<int64_t>(kRows) * (DP + 2);
  float* part = a.part + pair * a.splits * part_floats;
  for (int i = tid; i < rows * (DP / 2); i += kThreads) {
    const int row = i / (DP / 2), d = i % (DP / 2) * 2;
    float m = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) m = fmaxf(m, tops[w * kRows + row]);
    Joined j = {0.0f, 0.0f, m, 0.0f};
    const float at = m == -INFINITY ? 0.0f : m;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float f = exp2_fast(tops[w * kRows + row] - at);
      const float* r = sums + (w * kRows + row) * kPad + d;
      j.x = fmaf(r[0], f, j.x);
      j.y = fmaf(r[1], f, j.y);
      j.total = fmaf(totals[w * kRows + row], f, j.total);
    }
    if (a.splits == 1) {
      write(row, d, j);
    } else {
      float* p = part + sp * part_floats;
      *reinterpret_cast<float2*>(p + row * DP + d) = make_float2(j.x, j.y);
      if (d == 0) {
        p[kRows * DP + row] = j.top;
        p[kRows * DP + kRows + row] = j.total;
      }
    }
  }
  if (a.splits == 1 || a.ticket == nullptr) return;

  // The part that ends last joins all, in the parts' order.
  __threadfence();
  __syncthreads();
  if (tid == 0) last = atomicInc(a.ticket + pair, a.splits - 1) == static_cast<uint32_t>(a.splits - 1);
  __syncthreads();
  if (!last) return;
  __threadfence();
  constexpr int kMine = kRows * DP / 2 / kThreads;  // pairs of dims a thread joins at most
  float* factors = sums;                            // [part][row]: 2^(its maximum - the row's)
  for (int row = tid; row < rows; row += kThreads) {
    float m = -INFINITY;
    for (int w = 0; w < a.splits; ++w) m = fmaxf(m, __ldcg(part + w * part_floats + kRows * DP + row));
    const float at = m == -INFINITY ? 0.0f : m;
    float total = 0.0f;
    for (int w = 0; w < a.splits; ++w) {
      const float* p = part + w * part_floats + kRows * DP + row;
      const float f = exp2_fast(__ldcg(p) - at);
      factors[w * kRows + row] = f;
      total = fmaf(__ldcg(p + kRows), f, total);
    }
    tops[row] = m;
    totals[row] = total;
  }
  __syncthreads();
  float2 x[kMine];
#pragma unroll
  for (int k = 0; k < kMine; ++k) x[k] = make_float2(0.0f, 0.0f);
#pragma unroll 2
  for (int w = 0; w < a.splits; ++w) {
#pragma unroll
    for (int k = 0; k < kMine; ++k) {
      const int i = tid + k * kThreads, row = i / (DP / 2), d = i % (DP / 2) * 2;
      if (row >= rows) continue;
      const float2 y = __ldcg(reinterpret_cast<const float2*>(part + w * part_floats + row * DP + d));
      const float f = factors[w * kRows + row];
      x[k].x = fmaf(y.x, f, x[k].x);
      x[k].y = fmaf(y.y, f, x[k].y);
    }
  }
#pragma unroll
  for (int k = 0; k < kMine; ++k) {
    const int i = tid + k * kThreads, row = i / (DP / 2), d = i % (DP / 2) * 2;
    if (row < rows) write(row, d, Joined{x[k].x, x[k].y, tops[row], totals[row]});
  }
}

// TREE: the new tokens are nodes of a tree.
template <typename T, int DP, int NT, bool TREE>
__global__ void __launch_bounds__(kThreads, (kResident<DP, NT>))
    k_attend_token(const __grid_constant__ AttendArgs a) {
  constexpr int kStages = kStagesOf<DP>;
  constexpr uint32_t kStage = kStageBytes<DP>;
  constexpr int kChunks = DP / 8;            // 16-byte chunks of a row
  constexpr int kRowsAtOnce = 32 / kChunks;  // rows one copy instruction of a warp moves
  constexpr int kRows = 8 * NT;
  constexpr int kPad = kPadOf<DP>;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ uint32_t valid[kWarps][kStages];
  __shared__ TreeNode nodes[TREE ? PCS_TREE_MAX : 1];
  static_assert(kWarps * (kRows * (kPad + 2)) * 4 <= kRingBytes<DP>, "the join reuses the ring");

  attend_dependency();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int g = lane >> 2, q4 = lane & 3;
  const int head = blockIdx.x % a.cache.heads;
  const int sp = blockIdx.x / a.cache.heads % a.splits;
  const int s = blockIdx.x / a.cache.heads / a.splits;
  const SessionView view = session_view(a, s);
  if (view.m <= 0) return;  // the same in every part
  const int rows = view.m * a.group;
  if (!rows_there(a, view, tid == 0)) return;  // (max_new tokens' rows are at most kRows)
  const int head_dim = a.cache.head_dim;
  const uint32_t ring = smem_addr(smem) + warp * kStages * kStage;
  if (head_dim < DP) {  // chunks that no copy writes
    for (uint32_t i = lane * 16; i < kStages * kStage; i += 512)
      *reinterpret_cast<uint4*>(smem + warp * kStages * kStage + i) = make_uint4(0, 0, 0, 0);
    __syncwarp();
  }

  // This part's tiles; the warp takes every kWarps-th one.
  const int tiles = (view.seen + kTile - 1) / kTile;
  const int per = (tiles + a.splits - 1) / a.splits;
  const int t_end = min(tiles, (sp + 1) * per);
  int t_next = sp * per + warp;  // the next tile whose places are looked up

  const uint8_t* kbase = a.cache.k + head * a.cache.head_bytes;
  const uint8_t* vbase = a.cache.v + head * a.cache.head_bytes;
  // Lanes 0..15 (and again 16..31) look up a row each.
  auto look = [&](int t) {
    RowPlace r = {kNoRow, kNoRow};
    const int e = t * kTile + (lane & 15);
    if (t < t_end && e < view.seen) r = row_place(a, s, seen_position(view, e));
    return r;
  };
  const int chunk = lane % kChunks, row0 = lane / kChunks;
  auto copy = [&](const RowPlace& r, int stage) {
    const uint32_t there = __ballot_sync(kFull, r.k != kNoRow) & 0xffffu;
    if (lane == 0) valid[warp][stage] = there;
    const uint32_t base = ring + stage * kStage;
#pragma unroll
    for (int i = 0; i < kTile / kRowsAtOnce; ++i) {
      const int row = i * kRowsAtOnce + row0;
      const uint32_t ko = __shfl_sync(kFull, r.k, row), vo = __shfl_sync(kFull, r.v, row);
      const bool in = ko != kNoRow;
      if (chunk * 8 < head_dim) {
        const uint32_t at = base + row * (DP * 2) + ((chunk ^ (row & 7)) << 4);
        copy16(at, row_at(a, kbase, in ? ko : 0) + chunk * 16, in);
        copy16(at + kStage / 2, row_at(a, vbase, in ? vo : 0) + chunk * 16, in);
      }
    }
  };

  RowPlace place = look(t_next);
#pragma unroll
  for (int i = 0; i < kStages - 1; ++i) {
    if (t_next < t_end) copy(place, i);
    asm volatile("cp.async.commit_group;" ::: "memory");
    t_next += kWarps;
    place = look(t_next);
  }

  // Query rows as the second operand: dims 2 q4, +1 (+8, +9) of row g.
  uint32_t qf[NT][DP / 16][2];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int r = n * 8 + g;
    const uint32_t tok = a.by_group.div(r);
    const uint8_t* q = a.q.data + (view.q0 + tok) * a.q.token_bytes +
                       (head * a.group + (r - tok * a.group)) * a.q.head_bytes;
#pragma unroll
    for (int k = 0; k < DP / 16; ++k)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int d = k * 16 + i * 8 + q4 * 2;
        qf[n][k][i] = r < rows && d < head_dim ? *reinterpret_cast<const uint32_t*>(q + d * 2) : 0u;
      }
  }
  // New tokens of the rows this thread has scores of.
  const bool many = view.m > 1;
  int32_t new_token[NT][2];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int i = 0; i < 2; ++i)
      new_token[n][i] = TREE ? min(static_cast<int>(a.by_group.div(n * 8 + q4 * 2 + i)), view.m - 1)
                             : static_cast<int>(a.by_group.div(n * 8 + q4 * 2 + i));

  // Ranges of the first and the last new token.  (Nodes of a tree: what all of them
  // see of the context.)
  RowRange low = row_range(a, view, view.first);
  const RowRange high = row_range(a, view, view.first + view.m - 1);
  if constexpr (TREE) {
    low.hi = context_end(view);
    tree_nodes(a, view, tid, nodes);
    __syncthreads();
  }
  // Which of the tokens from place b on the rows of new token t see, as bits.
  auto sees = [&](int32_t t, int b) {
    if constexpr (TREE) return tree_row(a, view, nodes[t]).bits(b);
    return row_range(a, view, view.first + t).bits(b);
  };

  float o[DP / 16][NT][4];
  float top[NT][2], total[NT][2];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    top[n][0] = top[n][1] = -INFINITY;
    total[n][0] = total[n][1] = 0.0f;
#pragma unroll
    for (int i = 0; i < DP / 16; ++i) o[i][n][0] = o[i][n][1] = o[i][n][2] = o[i][n][3] = 0.0f;
  }

  int stage = 0;
  for (int t = sp * per + warp; t < t_end; t += kWarps) {
    asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
    __syncwarp();
    {
      const int into = stage == 0 ? kStages - 1 : stage - 1;
      if (t_next < t_end) copy(place, into);
      asm volatile("cp.async.commit_group;" ::: "memory");
      t_next += kWarps;
      place = look(t_next);
    }
    const uint32_t kat = ring + stage * kStage, vat = kat + kStage / 2;
    float c[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n) c[n][0] = c[n][1] = c[n][2] = c[n][3] = 0.0f;
#pragma unroll
    for (int k = 0; k < DP / 16; ++k) {
      uint32_t f[4];
      const int row = lane & 15;
      ldm4(f, kat + row * (DP * 2) + (((k * 2 + (lane >> 4)) ^ (row & 7)) << 4));
#pragma unroll
      for (int n = 0; n < NT; ++n) mma<T>(c[n], f, qf[n][k][0], qf[n][k][1]);
    }
    const uint32_t there = valid[warp][stage];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) c[n][i] *= a.scale_log2;
    const int e0 = t * kTile;
    const bool part = many && !(e0 + kTile - 1 <= low.hi && (e0 >= high.lo || e0 + kTile <= low.first));
    if (part || there != 0xffffu) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint32_t m = there & (part ? sees(new_token[n][i], e0) : kFull);
          if (!(m >> g & 1)) c[n][i] = -INFINITY;
          if (!(m >> (g + 8) & 1)) c[n][2 + i] = -INFINITY;
        }
    }
    bool raise = false;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 2; ++i) raise |= fmaxf(c[n][i], c[n][2 + i]) > top[n][i] + kSlack;
    if (__any_sync(kFull, raise)) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float m = fmaxf(c[n][i], c[n][2 + i]);
          m = fmaxf(m, __shfl_xor_sync(kFull, m, 4));
          m = fmaxf(m, __shfl_xor_sync(kFull, m, 8));
          m = fmaxf(m, __shfl_xor_sync(kFull, m, 16));
          m = fmaxf(m, top[n][i]);
          const float f = m == -INFINITY ? 1.0f : exp2_fast(top[n][i] - m);
          top[n][i] = m;
          total[n][i] *= f;
#pragma unroll
          for (int d = 0; d < DP / 16; ++d) {
            o[d][n][i] *= f;
            o[d][n][2 + i] *= f;
          }
        }
    }
    uint32_t w[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const float m0 = top[n][0] == -INFINITY ? 0.0f : top[n][0] - kLift<T>;
      const float m1 = top[n][1] == -INFINITY ? 0.0f : top[n][1] - kLift<T>;
      const float p0 = exp2_fast(c[n][0] - m0), p1 = exp2_fast(c[n][1] - m1);
      const float p2 = exp2_fast(c[n][2] - m0), p3 = exp2_fast(c[n][3] - m1);
      total[n][0] += p0 + p2;
      total[n][1] += p1 + p3;
      w[n][0] = transposed(pack2<T>(p0, p1));
      w[n][1] = transposed(pack2<T>(p2, p3));
    }
    auto values = [&](uint32_t (&f)[4], int d) {
      const int row = (lane & 7) + (lane >> 4) * 8;
      ldm4t(f, vat + row * (DP * 2) + (((d * 2 + ((lane >> 3) & 1)) ^ (row & 7)) << 4));
    };
    // (A tree has many rows that see a tile in part: they are told apart only where
    // some value is infinite or NaN.)
    bool apart = part;
    if (TREE && part) {
      bool any = false;
#pragma unroll
      for (int d = 0; d < DP / 16; ++d) {
        uint32_t f[4];
        values(f, d);
        any |= has_specials<T>(make_uint4(f[0], f[1], f[2], f[3]));
      }
      apart = __any_sync(kFull, any);
    }
    if (!apart) {
#pragma unroll
      for (int d = 0; d < DP / 16; ++d) {
        uint32_t f[4];
        values(f, d);
#pragma unroll
        for (int n = 0; n < NT; ++n) mma<T>(o[d][n], f, w[n][0], w[n][1]);
      }
    } else {
      // Tokens that some rows see and others do not: a weight of 0 would not
      // keep an infinity or a NaN out, so each new token's rows take what the
      // values come to with those it does not see taken out.
      for (int i = 0; i < view.m; ++i) {
        const uint32_t m = sees(i, e0) >> (2 * q4);
        uint32_t in[2];  // of tokens 2 q4, +1 and 8 more
#pragma unroll
        for (int h = 0; h < 2; ++h)
          in[h] = (m >> (8 * h) & 1 ? 0xffffu : 0u) | (m >> (8 * h + 1) & 1 ? 0xffff0000u : 0u);
        bool mine[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int h = 0; h < 2; ++h) mine[n][h] = new_token[n][h] == i;
#pragma unroll
        for (int d = 0; d < DP / 16; ++d) {
          uint32_t f[4];
          values(f, d);
          f[0] &= in[0], f[1] &= in[0], f[2] &= in[1], f[3] &= in[1];
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            // (A tree's products come on top of the sums, as above, where its rows are not
            // told apart: what is taken out changes no rounding of what stays.)
            float x[4];
#pragma unroll
            for (int h = 0; h < 4; ++h) x[h] = TREE ? o[d][n][h] : 0.0f;
            mma<T>(x, f, w[n][0], w[n][1]);
#pragma unroll
            for (int h = 0; h < 4; ++h)
              if (mine[n][h & 1]) o[d][n][h] = TREE ? x[h] : o[d][n][h] + x[h];
          }
        }
      }
    }
    __syncwarp();  // the stage may be filled again
    stage = stage + 1 == kStages ? 0 : stage + 1;
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      total[n][i] += __shfl_xor_sync(kFull, total[n][i], 4);
      total[n][i] += __shfl_xor_sync(kFull, total[n][i], 8);
      total[n][i] += __shfl_xor_sync(kFull, total[n][i], 16);
    }

  // Join the warps.
  __syncthreads();
  float* sums = reinterpret_cast<float*>(smem);           // [warp][row][kPad]
  float* tops = sums + kWarps * kRows * kPad;             // [warp][row]
  float* totals = tops + kWarps * kRows;
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int row = n * 8 + q4 * 2 + i;
      float* r = sums + (warp * kRows + row) * kPad;
#pragma unroll
      for (int d = 0; d < DP / 16; ++d) {
        r[d * 16 + g] = o[d][n][i];
        r[d * 16 + 8 + g] = o[d][n][2 + i];
      }
      if (g == 0) {
        tops[warp * kRows + row] = top[n][i];
        totals[warp * kRows + row] = total[n][i];
      }
    }
  __syncthreads();

  join_parts<T, DP, NT>(a, view, smem, s, head, sp);
}

}  // namespace
}  // namespace pcs
