// pcs_attend_token8.cu -- attention of one new token, or of a few (a tree's nodes
// among them), of every session over a paged cache in 8 bits.
//
// k_attend_token8  The one-pass softmax of pcs_attend_token.cu over half the bytes:
//                 codes and a scale byte a head and token stream through each warp's
//                 ring as they are, and become float16 operands on their way from
//                 shared memory to the matrix instruction (E4M3 by the conversion
//                 instruction, I8 through 1024 + c; both exactly).  The scales, powers
//                 of two, stay out of the operands: a key's multiplies its scores, a
//                 value's its weights.  So what a row's weights refer to is not the
//                 largest score but the largest score + log2(scale): a token with a
//                 large weight and small values loses nothing beside one with a small
//                 weight and large values, and the total, in 32 bits, refers to the
//                 same.  Query rows become float16 times a power of two of their own,
//                 that no bfloat16 is too large for it.
//                 Operands of 16 bits take 4 codes a thread where two elements lay:
//                 keys as their first operand read 16-byte chunks by ldmatrix (a
//                 thread gets four neighbouring dims, so the instruction's k runs over
//                 dims in the order 0 1 4 5 8 9 12 13 2 3 6 7 .., and the query rows are
//                 read in the same one); values come out transposed by pairs of dims,
//                 whose bytes are sorted into even and odd dims (rows g and g + 8).
//                 A warp's tile is 32 tokens.  They come by tensor copies of boxes of 8
//                 to 32 rows of a page (BOX), codes and scale bytes apart, or row by row
//                 from pages whose size no such box divides.  (What bounds copies by the
//                 warps' lanes is their number: a scale byte of a row is a request of its
//                 own beside 64 or 128 bytes of codes.)
#include "pcs_attend_token_dev.h"
#include "pcs_codes_dev.h"

namespace pcs {
namespace {

constexpr int kTile8 = kTokenTile8;
template <int DP>
constexpr int kStages8 = DP == 64 ? 3 : 2;
// Codes of keys and of values, then scale bytes of each row: 16 heads' (BOX) or 4 heads'.
template <bool BOX>
constexpr int kScaleBytes = BOX ? 16 : 4;
template <int DP, bool BOX>
constexpr uint32_t kStage8 = 2 * kTile8 * (DP + kScaleBytes<BOX>);
// (Boxes begin at multiples of 1,024 bytes: room to get there.)
template <int DP, bool BOX>
constexpr uint32_t kRing8 = kWarps * kStages8<DP> * kStage8<DP, BOX> + (BOX ? 1024 : 0);
// The rings, or what the warps' results take, which lie over them at the end.
template <int DP, int NT>
constexpr uint32_t kJoin8 = kWarps * 8 * NT * (kPadOf<DP> + 2) * 4;
template <int DP, int NT, bool BOX>
constexpr uint32_t kSmem8 = kRing8<DP, BOX> > kJoin8<DP, NT> ? kRing8<DP, BOX> : kJoin8<DP, NT>;
template <int DP, int NT, bool BOX>
constexpr int kResident8 = NT == 4 ? 2 : NT == 2 ? (DP == 64 ? 3 : 2) : static_cast<int>(227 * 1024 / (kSmem8<DP, NT, BOX> + 3072));

// 4 bytes from global to shared memory, zeros where there is no source.
__device__ __forceinline__ void copy4(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(there ? 4 : 0) : "memory");
}
// Where chunk c of row r of a tile lies: eight rows' chunks in eight banks of 16 bytes.
template <int DP>
__device__ __forceinline__ uint32_t chunk_at(int r, int c) {
  return DP == 128 ? r * 128 + ((c ^ (r & 7)) << 4) : r * 64 + ((c ^ ((r >> 1) & 3)) << 4);
}
// Where a row's weights refer to before its first token: nothing is below it.
constexpr float kNothing = -1e30f;
// A weight beyond this, or times its value's scale beyond 2^15, raises the reference.
constexpr float kMostWeight = 1.2676506e30f;  // 2^100

// A box of rows: `x`, `y`, .. where it begins in the tensor.
__device__ __forceinline__ void box_of_codes(uint32_t to, uint64_t map, int head, int row, int page, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(to),
      "l"(map), "r"(0), "r"(head), "r"(row), "r"(page), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void box_of_scales(uint32_t to, uint64_t map, int byte, int row, int page, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(to),
      "l"(map), "r"(byte), "r"(row), "r"(page), "r"(bar)
      : "memory");
}

template <int CODES, int DP, int NT, bool BOX>
__global__ void __launch_bounds__(kThreads, (kResident8<DP, NT, BOX>))
    k_attend_token8(const __grid_constant__ AttendArgs a, const __grid_constant__ CodeMaps maps) {
  constexpr int kStages = kStages8<DP>;
  constexpr uint32_t kStage = kStage8<DP, BOX>;
  constexpr int kChunks = DP / 16;           // 16-byte chunks of a row
  constexpr int kRowsAtOnce = 32 / kChunks;  // rows one copy instruction of a warp moves
  constexpr int kRows = 8 * NT;
  constexpr int kPad = kPadOf<DP>;
  constexpr bool kEarly = NT == 1;           // registers hold a tile's values beside its scores
  constexpr float kUp = 7.0f;                // weights are 2^7 times higher, as kLift says
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ uint32_t valid[kWarps][kStages];
  __shared__ __align__(8) uint64_t bars[BOX ? kWarps * kStages : 1];
  __shared__ TreeNode nodes[PCS_TREE_MAX];

  attend_dependency();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int g = lane >> 2, q4 = lane & 3;
  const int head = blockIdx.x % a.cache.heads;
  const int sp = blockIdx.x / a.cache.heads % a.splits;
  const int s = blockIdx.x / a.cache.heads / a.splits;
  if (BOX && tid < 4) asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(maps.map[tid])) : "memory");
  SessionView view = session_rows(a, s);
  narrow(a, view, 0, view.m, BOX ? a.box_rows : 1);
  if (view.m <= 0) return;  // the same in every part
  const int rows = view.m * a.group;
  if (!rows_there(a, view, tid == 0)) return;  // (max_new tokens' rows are at most kRows)
  const int head_dim = a.cache.head_dim;
  const bool tree = a.parent != nullptr;
  uint8_t* const ring_ptr = smem + (BOX ? -smem_addr(smem) & 1023u : 0u) + warp * kStages * kStage;
  const uint32_t ring = smem_addr(ring_ptr), bar0 = smem_addr(bars) + 8 * warp * kStages;
  if (BOX) {
    if (lane == 0) {
      for (int i = 0; i < kStages; ++i) bar_init(bar0 + 8 * i, 1);
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
  } else if (head_dim < DP) {  // chunks that no copy writes
    for (uint32_t i = lane * 16; i < kStages * kStage; i += 512)
      *reinterpret_cast<uint4*>(ring_ptr + i) = make_uint4(0, 0, 0, 0);
    __syncwarp();
  }
  if (tree) {
    tree_nodes(a, view, tid, nodes);
    __syncthreads();
  }

  // This part's tiles; the warp takes every kWarps-th one.
  const int tiles = (view.seen + kTile8 - 1) / kTile8;
  const int per = (tiles + a.splits - 1) / a.splits;
  const int t_end = min(tiles, (sp + 1) * per);
  int t_next = sp * per + warp;  // the next tile whose places are looked up

  // What a tile's copies need to know, looked up one tile ahead of them: a lane's row, or
  // (BOX) a lane's box of rows, of which there are 32 / box_rows a tile.
  using Ahead = std::conditional_t<BOX, Box, RowPlace>;
  const int box_shift = BOX ? 31 - __clz(a.box_rows) : 0, boxes = kTile8 >> box_shift;
  auto look = [&](int t) {
    if constexpr (BOX) {
      Box x = {-1, -1, 0};
      const int e = t * kTile8 + lane * a.box_rows;
      if (t < t_end && lane < boxes && e < view.seen) x = box_place(a, s, view, e);
      return x;
    } else {
      RowPlace r = {kNoRow, kNoRow};
      const int e = t * kTile8 + lane;
      if (t < t_end && e < view.seen) r = row_place(a, s, seen_position(view, e));
      return r;
    }
  };
  // The bytes of a row that hold the head's scale byte.
  constexpr int kScales = kScaleBytes<BOX>;
  const int scale_from = head & -kScales, scale_byte = head & (kScales - 1);
  auto copy = [&](Ahead& r, int t, int stage) {
    const uint32_t base = ring + stage * kStage;
    if constexpr (BOX) {
      settle(a, r);
      const int e = t * kTile8 + lane;
      const bool mine = __shfl_sync(kFull, r.k, lane >> box_shift) < a.cache.n_pages && !(e >= view.gap0 && e < view.gap1);
      const uint32_t there = __ballot_sync(kFull, mine);
      const uint32_t bar = bar0 + 8 * stage;
      if (lane == 0) {
        valid[warp][stage] = there;
        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(kStage) : "memory");
      }
      for (int k = 0; k < boxes; ++k) {
        const int kp = __shfl_sync(kFull, r.k, k), vp = __shfl_sync(kFull, r.v, k), row = __shfl_sync(kFull, r.row, k);
        const uint32_t at = k * a.box_rows;
        if (lane == 0) {
          box_of_codes(base + at * DP, reinterpret_cast<uint64_t>(maps.map[0]), head, row, kp, bar);
          box_of_codes(base + (kTile8 + at) * DP, reinterpret_cast<uint64_t>(maps.map[1]), head, row, vp, bar);
          box_of_scales(base + 2 * kTile8 * DP + at * kScales, reinterpret_cast<uint64_t>(maps.map[2]), scale_from, row, kp, bar);
          box_of_scales(base + 2 * kTile8 * DP + (kTile8 + at) * kScales, reinterpret_cast<uint64_t>(maps.map[3]), scale_from, row,
                        vp, bar);
        }
      }
    } else {
      const int chunk = lane % kChunks, row0 = lane / kChunks;
      const uint8_t* kbase = a.cache.k + head * a.cache.head_bytes;
      const uint8_t* vbase = a.cache.v + head * a.cache.head_bytes;
      const bool mine = r.k != kNoRow;
      const uint32_t there = __ballot_sync(kFull, mine);
      if (lane == 0) valid[warp][stage] = there;
#pragma unroll
      for (int i = 0; i < kTile8 / kRowsAtOnce; ++i) {
        const int row = i * kRowsAtOnce + row0;
        const uint32_t ko = __shfl_sync(kFull, r.k, row), vo = __shfl_sync(kFull, r.v, row);
        const bool in = ko != kNoRow;
        if (chunk * 16 < head_dim) {
          const uint32_t at = base + chunk_at<DP>(row, chunk);
          copy16(at, row_at(a, kbase, in ? ko : 0) + chunk * 16, in);
          copy16(at + kTile8 * DP, row_at(a, vbase, in ? vo : 0) + chunk * 16, in);
        }
      }
      // (A row is a multiple of 16 bytes, so the words that hold scales are in it.)
      const uint32_t words = base + 2 * kTile8 * DP + lane * 4;
      copy4(words, row_at(a, a.cache.k, mine ? r.k : 0) + a.cache.scale_at + scale_from, mine);
      copy4(words + kTile8 * 4, row_at(a, a.cache.v, mine ? r.v : 0) + a.cache.scale_at + scale_from, mine);
    }
  };

  Ahead place;
  {
    Ahead first[kStages];
#pragma unroll
    for (int i = 0; i < kStages; ++i) first[i] = look(t_next + i * kWarps);
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) {
      if (t_next < t_end) copy(first[i], t_next, i);
      if (!BOX) asm volatile("cp.async.commit_group;" ::: "memory");
      t_next += kWarps;
    }
    place = first[kStages - 1];
  }

  // Query rows as the second operand: of chunk k, dims 4 q4 .. +3 of row g, times
  // 2^-back, the power that puts the row's largest element at 2^14.
  uint32_t qf[NT][DP / 16][2];
  float back[NT][2];  // of the rows this thread has scores of, times the scale
  const bool half = a.dtype == PCS_DT_F16;
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int r = n * 8 + g;
    const uint32_t tok = a.by_group.div(r);
    const uint8_t* q = a.q.data + (view.q0 + tok) * a.q.token_bytes +
                       (head * a.group + (r - tok * a.group)) * a.q.head_bytes;
    float top = 0.0f;
#pragma unroll
    for (int k = 0; k < DP / 16; ++k) {
      const int d = k * 16 + q4 * 4;
      uint2 x = make_uint2(0, 0);
      if (r < rows && d < head_dim) x = *reinterpret_cast<const uint2*>(q + d * 2);
      qf[n][k][0] = x.x;
      qf[n][k][1] = x.y;
    }
    auto value = [&](uint32_t x) {
      return half ? __half22float2(*reinterpret_cast<const __half2*>(&x))
                  : make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u));
    };
#pragma unroll
    for (int k = 0; k < DP / 16; ++k)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float2 x = value(qf[n][k][i]);
        top = fmaxf(top, fmaxf(fabsf(x.x), fabsf(x.y)));
      }
    top = fmaxf(top, __shfl_xor_sync(kFull, top, 1));
    top = fmaxf(top, __shfl_xor_sync(kFull, top, 2));
    // (Rows with an infinity stay as they are, very small ones are not raised above 2^-86.)
    int e = static_cast<int>(__float_as_uint(top) >> 23) - 127;
    e = e > 127 ? 14 : max(e, -100);
    const float up = __uint_as_float(static_cast<uint32_t>(127 + 14 - e) << 23);
#pragma unroll
    for (int k = 0; k < DP / 16; ++k)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float2 x = value(qf[n][k][i]);
        qf[n][k][i] = pack2<__half>(x.x * up, x.y * up);
      }
    const float down = fmaxf(__uint_as_float(static_cast<uint32_t>(127 - 14 + e) << 23) * a.scale_log2, 1.2e-38f);
#pragma unroll
    for (int i = 0; i < 2; ++i) back[n][i] = __shfl_sync(kFull, down, (q4 * 2 + i) * 4);
  }
  // New tokens of the rows this thread has scores of.
  const bool many = view.m > 1;
  int32_t new_token[NT][2];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int i = 0; i < 2; ++i) new_token[n][i] = min(static_cast<int>(a.by_group.div(n * 8 + q4 * 2 + i)), view.m - 1);

  // Ranges of the first and the last new token.  (Nodes of a tree: what all of them
  // see of the context.)
  RowRange low = row_range(a, view, view.first);
  const RowRange high = row_range(a, view, view.first + view.m - 1);
  if (tree) low.hi = context_end(view);
  // Which of the tokens from place b on the rows of new token t see, as bits.
  auto sees = [&](int32_t t, int b) {
    return tree ? tree_row(a, view, nodes[t]).bits(b) : row_range(a, view, view.first + t).bits(b);
  };

  float o[DP / 16][NT][4];
  float refer[NT][2], total[NT][2];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    refer[n][0] = refer[n][1] = kNothing;
    total[n][0] = total[n][1] = 0.0f;
#pragma unroll
    for (int i = 0; i < DP / 16; ++i) o[i][n][0] = o[i][n][1] = o[i][n][2] = o[i][n][3] = 0.0f;
  }

  int stage = 0;
  uint32_t phase = 0;
  bool ok = true;
  for (int t = sp * per + warp; t < t_end; t += kWarps) {
    if (!BOX) {
      asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
      __syncwarp();
    }
    {
      const int into = stage == 0 ? kStages - 1 : stage - 1;
      if (t_next < t_end) copy(place, t_next, into);
      if (!BOX) asm volatile("cp.async.commit_group;" ::: "memory");
      t_next += kWarps;
      place = look(t_next);
    }
    if (BOX) {
      ok = __all_sync(kFull, bar_wait(bar0 + 8 * stage, phase)) != 0;
      if (!ok) break;
    }
    const uint32_t kat = ring + stage * kStage, vat = kat + kTile8 * DP;
    // This lane's row's scales.
    const uint8_t* scales = ring_ptr + stage * kStage + 2 * kTile8 * DP + lane * kScales + scale_byte;
    const float ks = scale_value(scales[0]), vs = scale_value(scales[kTile8 * kScales]);
    const uint32_t there = valid[warp][stage];
    const int e0 = t * kTile8;
    // (Boxes begin ahead of what is seen and end behind it.)
    const bool part = (BOX || many) && !(e0 + kTile8 - 1 <= low.hi && (e0 >= high.lo || e0 + kTile8 <= low.first));

    // Two chunks of 16 dims of the tokens 16 h .. +15: pairs of dims by pairs of tokens.
    auto values = [&](uint32_t (&f)[4], int h, int k) {
      ldm4t(f, vat + chunk_at<DP>(h * 16 + (lane & 15), 2 * k + (lane >> 4)));
    };
    // All that the tile gives is on its way out of shared memory before any of it is used.
    uint32_t kf[2][DP / 32][4], vf[2][DP / 32][4];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int k = 0; k < DP / 32; ++k) ldm4(kf[h][k], kat + chunk_at<DP>(h * 16 + (lane & 15), 2 * k + (lane >> 4)));
    if (kEarly) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int k = 0; k < DP / 32; ++k) values(vf[h][k], h, k);
    }
    // Scores of tokens 16 h + g, + 8, but for the rows' factors.
    float c[2][NT][4];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int n = 0; n < NT; ++n) c[h][n][0] = c[h][n][1] = c[h][n][2] = c[h][n][3] = 0.0f;
#pragma unroll
    for (int k = 0; k < DP / 32; ++k)
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t x[4];
          four_halves<CODES>(kf[h][k][2 * j], x[0], x[2]);
          four_halves<CODES>(kf[h][k][2 * j + 1], x[1], x[3]);
#pragma unroll
          for (int n = 0; n < NT; ++n) mma<__half>(c[h][n], x, qf[n][2 * k + j][0], qf[n][2 * k + j][1]);
        }
    float vscale[2][2];  // of token 16 h + 8 j + g
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float y = __shfl_sync(kFull, ks, h * 16 + j * 8 + g);
        vscale[h][j] = __shfl_sync(kFull, vs, h * 16 + j * 8 + g);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          c[h][n][2 * j] *= y;
          c[h][n][2 * j + 1] *= y;
        }
      }
    const bool masked = part || there != kFull;
    uint32_t seen[NT][2];  // bits of the tokens that a row sees
    if (masked) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          seen[n][i] = (there & (part ? sees(new_token[n][i], e0) : kFull)) >> g;
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < 2; ++j)
              if (!(seen[n][i] >> (h * 16 + j * 8) & 1)) c[h][n][2 * j + i] = -INFINITY;
        }
    }
    // Weights 2^(score - reference), p; times the values' scales, v.
    float p[2][NT][4], v[2][NT][4];
    auto weigh = [&] {
      float most = 0.0f, largest = 0.0f;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const int z = 2 * j + i;
              p[h][n][z] = exp2_fast(fmaf(c[h][n][z], back[n][i], -refer[n][i]));
              v[h][n][z] = p[h][n][z] * vscale[h][j];
              largest = fmaxf(largest, p[h][n][z]);
              most = fmaxf(most, v[h][n][z]);
            }
      return most > 32768.0f || largest > kMostWeight;
    };
    if (__any_sync(kFull, weigh())) {
      // The reference becomes the largest score + log2(scale), less 7 as kUp says, and
      // at least what keeps the largest weight below 2^93.
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float m = -INFINITY, w = -INFINITY;
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              const float x = c[h][n][2 * j + i] * back[n][i];
              const int e = static_cast<int>(__float_as_uint(vscale[h][j]) >> 23) - 127;  // (255: below any other)
              m = fmaxf(m, x);
              w = fmaxf(w, x + static_cast<float>(e > 127 ? -127 : e));
            }
#pragma unroll
          for (int k = 4; k <= 16; k *= 2) {
            m = fmaxf(m, __shfl_xor_sync(kFull, m, k));
            w = fmaxf(w, __shfl_xor_sync(kFull, w, k));
          }
          const float to = fmaxf(fmaxf(w - kUp, m - 93.0f), refer[n][i]);
          const float f = exp2_fast(refer[n][i] - to);
          refer[n][i] = to;
          total[n][i] *= f;
#pragma unroll
          for (int d = 0; d < DP / 16; ++d) {
            o[d][n][i] *= f;
            o[d][n][2 + i] *= f;
          }
        }
      weigh();
    }
    if (masked) {  // (a scale that stands for NaN would go through a weight of 0)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < 2; ++j)
              if (!(seen[n][i] >> (h * 16 + j * 8) & 1)) v[h][n][2 * j + i] = 0.0f;
    }
    uint32_t w[2][NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        total[n][0] += p[h][n][0] + p[h][n][2];
        total[n][1] += p[h][n][1] + p[h][n][3];
        w[h][n][0] = transposed(pack2<__half>(v[h][n][0], v[h][n][1]));
        w[h][n][1] = transposed(pack2<__half>(v[h][n][2], v[h][n][3]));
      }
    // The first operand of one of them: even dims are its rows g, odd ones its rows g + 8.
    auto operand = [&](uint32_t (&x)[4], uint32_t early, uint32_t late) {
      four_halves<CODES>(__byte_perm(early, 0, 0x3120), x[0], x[1]);
      four_halves<CODES>(__byte_perm(late, 0, 0x3120), x[2], x[3]);
    };
    // (Only the NaN of 8-bit floats would go through a weight of 0: tokens that some rows
    // see and others do not are told apart where there is one.)
    bool apart = false;
    if (CODES == kCodesE4M3 && part) {
      uint32_t nan = 0;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int k = 0; k < DP / 32; ++k) {
          uint32_t f[4];
          values(f, h, k);
#pragma unroll
          for (int i = 0; i < 4; ++i) nan |= (f[i] & 0x7f7f7f7fu) + 0x01010101u;
        }
      apart = __any_sync(kFull, (nan & 0x80808080u) != 0);
    }
    if (!apart) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int k = 0; k < DP / 32; ++k) {
          uint32_t x[4];
          if (!kEarly) values(vf[h][k], h, k);
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            operand(x, vf[h][k][2 * j], vf[h][k][2 * j + 1]);
#pragma unroll
            for (int n = 0; n < NT; ++n) mma<__half>(o[2 * k + j][n], x, w[h][n][0], w[h][n][1]);
          }
        }
    } else {
      for (int i = 0; i < view.m; ++i) {
        const uint32_t m = sees(i, e0) >> (2 * q4);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t in[2];  // of tokens 16 h + 2 q4, +1 and 8 more
#pragma unroll
          for (int z = 0; z < 2; ++z)
            in[z] = (m >> (16 * h + 8 * z) & 1 ? 0xffffu : 0u) | (m >> (16 * h + 8 * z + 1) & 1 ? 0xffff0000u : 0u);
#pragma unroll
          for (int k = 0; k < DP / 32; ++k) {
            uint32_t f[4], x[4];
            values(f, h, k);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              operand(x, f[2 * j] & in[0], f[2 * j + 1] & in[1]);
#pragma unroll
              for (int n = 0; n < NT; ++n) {
                float y[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                mma<__half>(y, x, w[h][n][0], w[h][n][1]);
#pragma unroll
                for (int z = 0; z < 4; ++z)
                  if (new_token[n][z & 1] == i) o[2 * k + j][n][z] += y[z];
              }
            }
          }
        }
      }
    }
    __syncwarp();  // the stage may be filled again
    stage = stage + 1 == kStages ? 0 : stage + 1;
    if (stage == 0) phase ^= 1;
  }
  if (!BOX) asm volatile("cp.async.wait_all;" ::: "memory");
  if (!ok) {  // a copy did not come: it and those behind it get as long again, then the block ends
    for (int t = t_next - kStages * kWarps; t < min(t_next, t_end); t += kWarps) {
      bar_wait(bar0 + 8 * stage, phase);
      stage = stage + 1 == kStages ? 0 : stage + 1;
      if (stage == 0) phase ^= 1;
    }
    if (lane == 0) atomicOr(a.err, kDevErrTimeout);
  }

#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      total[n][i] += __shfl_xor_sync(kFull, total[n][i], 4);
      total[n][i] += __shfl_xor_sync(kFull, total[n][i], 8);
      total[n][i] += __shfl_xor_sync(kFull, total[n][i], 16);
    }
  __syncthreads();
  const float lift = half ? kLift<__half> : kLift<__nv_bfloat16>;
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
      for (int d = 0; d < DP / 16; ++d)
        *reinterpret_cast<float2*>(r + d * 16 + 2 * g) = make_float2(o[d][n][i], o[d][n][2 + i]);
      if (g == 0) {
        // (The join takes kLift off again, where the result's type has one.)
        tops[warp * kRows + row] = refer[n][i] == kNothing ? -INFINITY : refer[n][i] + lift;
        totals[warp * kRows + row] = total[n][i];
      }
    }
  __syncthreads();
  if (half)
    join_parts<__half, DP, NT>(a, view, smem, s, head, sp);
  else
    join_parts<__nv_bfloat16, DP, NT>(a, view, smem, s, head, sp);
}

template <int CODES, int DP, int NT, bool BOX>
cudaError_t launch(const AttendArgs& a, const CodeMaps& maps, cudaStream_t stream) {
  auto k = k_attend_token8<CODES, DP, NT, BOX>;
  static SmemLimit limit;
  if (cudaError_t e = limit.set(k, kSmem8<DP, NT, BOX>)) return e;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(a.batch.sessions) * a.cache.heads * a.splits);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kSmem8<DP, NT, BOX>;
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, k, a, maps);
}

template <int CODES, bool BOX>
cudaError_t by_size(const AttendArgs& a, int rows, const CodeMaps& maps, cudaStream_t stream) {
  if (a.cache.head_dim <= 64)
    return rows <= 8    ? launch<CODES, 64, 1, BOX>(a, maps, stream)
           : rows <= 16 ? launch<CODES, 64, 2, BOX>(a, maps, stream)
                        : launch<CODES, 64, 4, BOX>(a, maps, stream);
  return rows <= 8    ? launch<CODES, 128, 1, BOX>(a, maps, stream)
         : rows <= 16 ? launch<CODES, 128, 2, BOX>(a, maps, stream)
                      : launch<CODES, 128, 4, BOX>(a, maps, stream);
}
template <int CODES>
cudaError_t by_form(const AttendArgs& a, int rows, const CodeMaps& maps, cudaStream_t stream) {
  return a.box_rows ? by_size<CODES, true>(a, rows, maps, stream) : by_size<CODES, false>(a, rows, maps, stream);
}

}  // namespace

int attend_token8_blocks_per_sm(int head_dim, int rows) {
  const int n = rows <= 8 ? 1 : rows <= 16 ? 2 : 4;
  if (head_dim <= 64) return n == 1 ? kResident8<64, 1, true> : n == 2 ? kResident8<64, 2, true> : kResident8<64, 4, true>;
  return n == 1 ? kResident8<128, 1, true> : n == 2 ? kResident8<128, 2, true> : kResident8<128, 4, true>;
}

cudaError_t launch_attend_token8(const AttendArgs& a, int rows, const CodeMaps& maps, cudaStream_t stream) {
  return a.cache.codes == kCodesE4M3 ? by_form<kCodesE4M3>(a, rows, maps, stream) : by_form<kCodesI8>(a, rows, maps, stream);
}

}  // namespace pcs
