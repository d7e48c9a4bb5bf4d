// pcs_attend_token.cu -- attention of one new token, or of a few, of every
// session over a paged cache of keys and values.
//
// k_attend_token  o = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m), s_j = scale
//                 q.k_j, over the tokens a new token sees, in one pass with
//                 running m and sums.  Every key and value row is used by the
//                 few query rows of its head alone (at most 32), so the bound
//                 is HBM.  A block takes one session, key head and part of the
//                 visible tokens; each of its warps walks tiles of 16 tokens
//                 through a ring of its own in shared memory, filled by
//                 16-byte asynchronous copies (pages of any size, no barrier
//                 between the warps), and the warps' and then the parts'
//                 results are joined by their maxima.
//                 Tokens are the rows of the matrix instruction (m16n8k16) and
//                 query rows its columns: keys and values come out of shared
//                 memory as the first operand, eight query rows cost one
//                 column tile, and the weights turn from result to operand
//                 with one transposing move per 8 x 8.  (That instruction is
//                 busy 6 % of the time while HBM is the bound: the fifth-
//                 generation tensor cores, which want 128 rows, have nothing to
//                 add here.)
//                 256 sessions over windows of 1,024 tokens, 16 heads of 64 in
//                 bfloat16: 170 us, 6.3 TB/s (95 % of the measured copy rate);
//                 four tokens over 200,001, 8 key heads of 128: 125 us, 6.6 TB/s.
//                 A second product with what the weights' rounding left of them
//                 took 175 us there, and 10 % more with 32 rows a key head: the
//                 weights stay in 16 bits.
//                 k_attend_token_join joins more parts than kTokenOwnJoin.
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

// Joined sums of one row pair of dims; `w` parts with maxima m, totals l.
struct Joined {
  float x, y, top, total;
};

template <typename T, int DP, int NT>
__global__ void __launch_bounds__(kThreads, (kResident<DP, NT>))
    k_attend_token(const __grid_constant__ AttendArgs a) {
  constexpr int kStages = kStagesOf<DP>;
  constexpr uint32_t kStage = kStageBytes<DP>;
  constexpr int kChunks = DP / 8;            // 16-byte chunks of a row
  constexpr int kRowsAtOnce = 32 / kChunks;  // rows one copy instruction of a warp moves
  constexpr int kRows = 8 * NT;
  constexpr int kPad = DP + 4;               // floats of a row of a warp's sums
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ uint32_t valid[kWarps][kStages];
  __shared__ uint32_t last;
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
  // Positions of the rows this thread has scores of.
  const bool many = view.m > 1;
  int32_t pos[NT][2];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int i = 0; i < 2; ++i)
      pos[n][i] = view.first + static_cast<int>(a.by_group.div(n * 8 + q4 * 2 + i));

  // Ranges of the first and the last new token.
  const RowRange low = row_range(a, view, view.first), high = row_range(a, view, view.first + view.m - 1);

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
          const uint32_t m = there & (part ? row_range(a, view, pos[n][i]).bits(e0) : kFull);
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
    if (!part) {
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
        const uint32_t m = row_range(a, view, view.first + i).bits(e0) >> (2 * q4);
        uint32_t in[2];  // of tokens 2 q4, +1 and 8 more
#pragma unroll
        for (int h = 0; h < 2; ++h)
          in[h] = (m >> (8 * h) & 1 ? 0xffffu : 0u) | (m >> (8 * h + 1) & 1 ? 0xffff0000u : 0u);
        bool mine[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int h = 0; h < 2; ++h) mine[n][h] = pos[n][h] == view.first + i;
#pragma unroll
        for (int d = 0; d < DP / 16; ++d) {
          uint32_t f[4];
          values(f, d);
          f[0] &= in[0], f[1] &= in[0], f[2] &= in[1], f[3] &= in[1];
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            float x[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            mma<T>(x, f, w[n][0], w[n][1]);
#pragma unroll
            for (int h = 0; h < 4; ++h)
              if (mine[n][h & 1]) o[d][n][h] += x[h];
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

// Joins many parts: a block per row, whose warps take every kWarps-th part.
template <typename T, int DP, int NT>
__global__ void __launch_bounds__(kThreads) k_attend_token_join(const __grid_constant__ AttendArgs a) {
  constexpr int kRows = 8 * NT;
  __shared__ float sums[kWarps][DP], tops[kWarps], totals[kWarps];
  attend_dependency();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t pair = blockIdx.x / kRows;
  const int row = static_cast<int>(blockIdx.x % kRows);
  const int s = static_cast<int>(pair / a.cache.heads), head = static_cast<int>(pair % a.cache.heads);
  const SessionView view = session_rows(a, s);
  if (row >= view.m * a.group || !rows_there(a, view, false)) return;
  const int64_t part_floats = static_cast<int64_t>(kRows) * (DP + 2);
  const float* part = a.part + pair * a.splits * part_floats;
  float m = -INFINITY;
  for (int w = threadIdx.x; w < a.splits; w += kThreads) m = fmaxf(m, __ldcg(part + w * part_floats + kRows * DP + row));
#pragma unroll
  for (int k = 16; k > 0; k /= 2) m = fmaxf(m, __shfl_xor_sync(kFull, m, k));
  if (lane == 0) tops[warp] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWarps; ++w) m = fmaxf(m, tops[w]);
  const float at = m == -INFINITY ? 0.0f : m;
  float x[DP / 32] = {}, total = 0.0f;
#pragma unroll 8
  for (int w = warp; w < a.splits; w += kWarps) {
    const float* p = part + w * part_floats;
    const float f = exp2_fast(__ldcg(p + kRows * DP + row) - at);
    total = fmaf(__ldcg(p + kRows * DP + kRows + row), f, total);
#pragma unroll
    for (int k = 0; k < DP / 64; ++k) {
      const float2 y = __ldcg(reinterpret_cast<const float2*>(p + row * DP + 64 * k + 2 * lane));
      x[2 * k] = fmaf(y.x, f, x[2 * k]);
      x[2 * k + 1] = fmaf(y.y, f, x[2 * k + 1]);
    }
  }
#pragma unroll
  for (int k = 0; k < DP / 64; ++k)
    *reinterpret_cast<float2*>(&sums[warp][64 * k + 2 * lane]) = make_float2(x[2 * k], x[2 * k + 1]);
  if (lane == 0) totals[warp] = total;
  __syncthreads();
  total = 0.0f;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) total += totals[w];
  const float inv = total == 0.0f ? 0.0f : 1.0f / total;
  const uint32_t tok = a.by_group.div(row);
  const int h = head * a.group + (row - static_cast<int>(tok) * a.group);
  for (int d = 2 * threadIdx.x; d < a.cache.head_dim; d += 2 * kThreads) {
    float2 y = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      y.x += sums[w][d];
      y.y += sums[w][d + 1];
    }
    *reinterpret_cast<uint32_t*>(a.out.data + (view.q0 + tok) * a.out.token_bytes + h * a.out.head_bytes + d * 2) =
        pack2<T>(y.x * inv, y.y * inv);
  }
  if (threadIdx.x == 0 && a.lse)
    a.lse[(view.q0 + tok) * (static_cast<int64_t>(a.cache.heads) * a.group) + h] =
        total == 0.0f ? -INFINITY : fmaf(m - kLift<T>, 0.693147180559945309f, logf(total));
}

template <typename T, int DP, int NT>
cudaError_t launch(const AttendArgs& a, bool join, cudaStream_t stream) {
  auto k = k_attend_token<T, DP, NT>;
  static SmemLimit limit;
  if (cudaError_t e = limit.set(k, kRingBytes<DP>)) return e;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(a.batch.sessions) * a.cache.heads * a.splits);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kRingBytes<DP>;
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (join) {
    cfg.gridDim = dim3(static_cast<unsigned>(static_cast<int64_t>(a.batch.sessions) * a.cache.heads * 8 * NT));
    cfg.dynamicSmemBytes = 0;
    return cudaLaunchKernelEx(&cfg, k_attend_token_join<T, DP, NT>, a);
  }
  return cudaLaunchKernelEx(&cfg, k, a);
}

template <typename T>
cudaError_t by_size(const AttendArgs& a, int rows, bool join, cudaStream_t stream) {
  if (a.cache.head_dim <= 64)
    return rows <= 8 ? launch<T, 64, 1>(a, join, stream) : rows <= 16 ? launch<T, 64, 2>(a, join, stream)
                                                               : launch<T, 64, 4>(a, join, stream);
  return rows <= 8 ? launch<T, 128, 1>(a, join, stream) : rows <= 16 ? launch<T, 128, 2>(a, join, stream)
                                                              : launch<T, 128, 4>(a, join, stream);
}

}  // namespace

int attend_token_blocks_per_sm(int head_dim, int rows) {
  if (head_dim <= 64) return rows <= 16 ? kResident<64, 2> : kResident<64, 4>;
  return kResident<128, 4>;
}

cudaError_t launch_attend_token(const AttendArgs& a, uint32_t dtype, int rows, bool join, cudaStream_t stream) {
  return dtype == PCS_DT_F16 ? by_size<__half>(a, rows, join, stream) : by_size<__nv_bfloat16>(a, rows, join, stream);
}

}  // namespace pcs
