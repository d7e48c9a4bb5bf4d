// pcs_attend_token8.cu -- attention of one new token, or of a few (a tree's nodes
// among them), of every session over a paged cache in 8 bits.
//
// k_attend_token8  The one-pass softmax of pcs_attend_token.cu over half the bytes:
//                 codes and a scale byte a head and token stream through each warp's
//                 ring as they are, and become float16 operands on their way from
//                 shared memory to the matrix instruction (E4M3 by the conversion
//                 instruction, I8 through 1024 + c; both exactly).  The scales, powers
//                 of two, stay out of the operands: a key's multiplies its scores, a
//                 value's is added to the logarithm of its weights.  So a row has two
//                 running maxima: that of its scores, which the total refers to, and
//                 that of score + log2(scale), which the weights of the sums refer to
//                 -- a token with a large weight and small values loses nothing
//                 beside one with a small weight and large values.  Query rows
//                 become float16 times a power of two of their own, that no bfloat16
//                 is too large for it.
//                 Operands of 16 bits take 4 codes a thread where two elements lay:
//                 keys as their first operand read 16-byte chunks by ldmatrix (a
//                 thread gets four neighbouring dims, so the instruction's k runs over
//                 dims in the order 0 1 4 5 8 9 12 13 2 3 6 7 .., and the query rows are
//                 read in the same one); values come out transposed by pairs of dims,
//                 whose bytes are sorted into even and odd dims (rows g and g + 8).
//                 A warp's tile is 32 tokens: a lane looks up one of them.
#include "pcs_attend_token_dev.h"
#include "pcs_codes_dev.h"

namespace pcs {
namespace {

constexpr int kTile8 = 32;
// Stages of a warp's ring: 64 to 100 KB in flight on an SM, as with 16 bits.
template <int DP>
constexpr int kStages8 = DP == 64 ? 4 : 3;
// Codes of keys and of values, then a word of scale bytes of each row.
template <int DP>
constexpr uint32_t kStage8 = 2 * kTile8 * DP + 2 * kTile8 * 4;
template <int DP>
constexpr uint32_t kRing8 = kWarps * kStages8<DP> * kStage8<DP>;
template <int DP, int NT>
constexpr int kResident8 = DP == 64 && NT == 4 ? 2 : static_cast<int>(227 * 1024 / (kRing8<DP> + 4096));

// 4 bytes from global to shared memory, zeros where there is no source.
__device__ __forceinline__ void copy4(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(there ? 4 : 0) : "memory");
}
// Where chunk c of row r of a tile lies: eight rows' chunks in eight banks of 16 bytes.
template <int DP>
__device__ __forceinline__ uint32_t chunk_at(int r, int c) {
  return DP == 128 ? r * 128 + ((c ^ (r & 7)) << 4) : r * 64 + ((c ^ ((r >> 1) & 3)) << 4);
}
// log2 of a scale; NaN for its NaN.
__device__ __forceinline__ float scale_log2_of(uint32_t b) {
  return b == 255 ? __uint_as_float(0x7fc00000u) : static_cast<float>(static_cast<int>(b) - 127);
}

template <int CODES, int DP, int NT>
__global__ void __launch_bounds__(kThreads, (kResident8<DP, NT>))
    k_attend_token8(const __grid_constant__ AttendArgs a) {
  constexpr int kStages = kStages8<DP>;
  constexpr uint32_t kStage = kStage8<DP>;
  constexpr int kChunks = DP / 16;           // 16-byte chunks of a row
  constexpr int kRowsAtOnce = 32 / kChunks;  // rows one copy instruction of a warp moves
  constexpr int kRows = 8 * NT;
  constexpr int kPad = kPadOf<DP>;
  constexpr float kUp = 7.0f;                // weights are 2^7 times higher, as kLift says
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ uint32_t valid[kWarps][kStages];
  __shared__ TreeNode nodes[PCS_TREE_MAX];
  static_assert(kWarps * (kRows * (kPad + 2)) * 4 <= kRing8<DP>, "the join reuses the ring");

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
  const bool tree = a.parent != nullptr;
  const uint32_t ring = smem_addr(smem) + warp * kStages * kStage;
  if (head_dim < DP) {  // chunks that no copy writes
    for (uint32_t i = lane * 16; i < kStages * kStage; i += 512)
      *reinterpret_cast<uint4*>(smem + warp * kStages * kStage + i) = make_uint4(0, 0, 0, 0);
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

  const uint8_t* kbase = a.cache.k + head * a.cache.head_bytes;
  const uint8_t* vbase = a.cache.v + head * a.cache.head_bytes;
  // The aligned word that holds the head's scale byte.  (A row is a multiple of 16 bytes.)
  const int scale_word = a.cache.scale_at + (head & ~3), scale_byte = head & 3;
  auto look = [&](int t) {
    RowPlace r = {kNoRow, kNoRow};
    const int e = t * kTile8 + lane;
    if (t < t_end && e < view.seen) r = row_place(a, s, seen_position(view, e));
    return r;
  };
  const int chunk = lane % kChunks, row0 = lane / kChunks;
  auto copy = [&](const RowPlace& r, int stage) {
    const bool mine = r.k != kNoRow;
    const uint32_t there = __ballot_sync(kFull, mine);
    if (lane == 0) valid[warp][stage] = there;
    const uint32_t base = ring + stage * kStage;
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
    const uint32_t words = base + 2 * kTile8 * DP + lane * 4;
    copy4(words, row_at(a, a.cache.k, mine ? r.k : 0) + scale_word, mine);
    copy4(words + kTile8 * 4, row_at(a, a.cache.v, mine ? r.v : 0) + scale_word, mine);
  };

  RowPlace place = look(t_next);
#pragma unroll
  for (int i = 0; i < kStages - 1; ++i) {
    if (t_next < t_end) copy(place, i);
    asm volatile("cp.async.commit_group;" ::: "memory");
    t_next += kWarps;
    place = look(t_next);
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
    const float down = __uint_as_float(static_cast<uint32_t>(127 - 14 + e) << 23) * a.scale_log2;
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
  float top[NT][2], mark[NT][2], total[NT][2];  // maxima of scores, of scores with the values' scales
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    top[n][0] = top[n][1] = mark[n][0] = mark[n][1] = -INFINITY;
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
    const uint32_t kat = ring + stage * kStage, vat = kat + kTile8 * DP;
    const uint8_t* scales = smem + (warp * kStages + stage) * kStage + 2 * kTile8 * DP + scale_byte;
    const uint32_t there = valid[warp][stage];
    const int e0 = t * kTile8;
    const bool part = many && !(e0 + kTile8 - 1 <= low.hi && (e0 >= high.lo || e0 + kTile8 <= low.first));

    // c: scores of tokens 16 h + g, + 8; cv: with the logarithm of the values' scales.
    float c[2][NT][4], cv[2][NT][4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int n = 0; n < NT; ++n) c[h][n][0] = c[h][n][1] = c[h][n][2] = c[h][n][3] = 0.0f;
#pragma unroll
      for (int k = 0; k < DP / 32; ++k) {
        uint32_t f[4];
        ldm4(f, kat + chunk_at<DP>(h * 16 + (lane & 15), 2 * k + (lane >> 4)));
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          uint32_t x[4];
          four_halves<CODES>(f[2 * j], x[0], x[2]);
          four_halves<CODES>(f[2 * j + 1], x[1], x[3]);
#pragma unroll
          for (int n = 0; n < NT; ++n) mma<__half>(c[h][n], x, qf[n][2 * k + j][0], qf[n][2 * k + j][1]);
        }
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {  // token 16 h + 8 i + g
        const int row = h * 16 + i * 8 + g;
        const float ks = scale_value(scales[row * 4]), vl = scale_log2_of(scales[(kTile8 + row) * 4]);
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            c[h][n][2 * i + j] *= ks * back[n][j];
            cv[h][n][2 * i + j] = c[h][n][2 * i + j] + vl;
          }
      }
    }
    if (part || there != kFull) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint32_t m = there & (part ? sees(new_token[n][i], e0) : kFull);
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < 2; ++j)
              if (!(m >> (h * 16 + j * 8 + g) & 1)) c[h][n][2 * j + i] = cv[h][n][2 * j + i] = -INFINITY;
        }
    }
    bool raise = false;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        raise |= fmaxf(fmaxf(c[0][n][i], c[0][n][2 + i]), fmaxf(c[1][n][i], c[1][n][2 + i])) > top[n][i] + kSlack;
        raise |= fmaxf(fmaxf(cv[0][n][i], cv[0][n][2 + i]), fmaxf(cv[1][n][i], cv[1][n][2 + i])) > mark[n][i] + kSlack;
      }
    if (__any_sync(kFull, raise)) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float m = fmaxf(fmaxf(c[0][n][i], c[0][n][2 + i]), fmaxf(c[1][n][i], c[1][n][2 + i]));
          float w = fmaxf(fmaxf(cv[0][n][i], cv[0][n][2 + i]), fmaxf(cv[1][n][i], cv[1][n][2 + i]));
#pragma unroll
          for (int k = 4; k <= 16; k *= 2) {
            m = fmaxf(m, __shfl_xor_sync(kFull, m, k));
            w = fmaxf(w, __shfl_xor_sync(kFull, w, k));
          }
          m = fmaxf(m, top[n][i]);
          w = fmaxf(w, mark[n][i]);
          total[n][i] *= m == -INFINITY ? 1.0f : exp2_fast(top[n][i] - m);
          const float f = w == -INFINITY ? 1.0f : exp2_fast(mark[n][i] - w);
          top[n][i] = m;
          mark[n][i] = w;
#pragma unroll
          for (int d = 0; d < DP / 16; ++d) {
            o[d][n][i] *= f;
            o[d][n][2 + i] *= f;
          }
        }
    }
    uint32_t w[2][NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const float m0 = top[n][0] == -INFINITY ? 0.0f : top[n][0], m1 = top[n][1] == -INFINITY ? 0.0f : top[n][1];
      const float w0 = mark[n][0] == -INFINITY ? 0.0f : mark[n][0] - kUp, w1 = mark[n][1] == -INFINITY ? 0.0f : mark[n][1] - kUp;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        total[n][0] += exp2_fast(c[h][n][0] - m0) + exp2_fast(c[h][n][2] - m0);
        total[n][1] += exp2_fast(c[h][n][1] - m1) + exp2_fast(c[h][n][3] - m1);
        w[h][n][0] = transposed(pack2<__half>(exp2_fast(cv[h][n][0] - w0), exp2_fast(cv[h][n][1] - w1)));
        w[h][n][1] = transposed(pack2<__half>(exp2_fast(cv[h][n][2] - w0), exp2_fast(cv[h][n][3] - w1)));
      }
    }
    // Two chunks of 16 dims of the tokens 16 h .. +15: pairs of dims by pairs of tokens.
    auto values = [&](uint32_t (&f)[4], int h, int k) {
      ldm4t(f, vat + chunk_at<DP>(h * 16 + (lane & 15), 2 * k + (lane >> 4)));
    };
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
          uint32_t f[4], x[4];
          values(f, h, k);
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            operand(x, f[2 * j], f[2 * j + 1]);
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
  }
  asm volatile("cp.async.wait_all;" ::: "memory");

  // Sums and totals that refer to the scores' maximum, as the join takes them (2^kLift of
  // the result's type higher).
  const float lift = half ? kLift<__half> : kLift<__nv_bfloat16>;
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      total[n][i] += __shfl_xor_sync(kFull, total[n][i], 4);
      total[n][i] += __shfl_xor_sync(kFull, total[n][i], 8);
      total[n][i] += __shfl_xor_sync(kFull, total[n][i], 16);
      total[n][i] *= exp2_fast(lift);
    }
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
      const float f = mark[n][i] == -INFINITY ? 1.0f : exp2_fast(mark[n][i] - kUp - top[n][i] + lift);
#pragma unroll
      for (int d = 0; d < DP / 16; ++d)
        *reinterpret_cast<float2*>(r + d * 16 + 2 * g) = make_float2(o[d][n][i] * f, o[d][n][2 + i] * f);
      if (g == 0) {
        tops[warp * kRows + row] = top[n][i];
        totals[warp * kRows + row] = total[n][i];
      }
    }
  __syncthreads();
  if (half)
    join_parts<__half, DP, NT>(a, view, smem, s, head, sp);
  else
    join_parts<__nv_bfloat16, DP, NT>(a, view, smem, s, head, sp);
}

template <int CODES, int DP, int NT>
cudaError_t launch(const AttendArgs& a, cudaStream_t stream) {
  auto k = k_attend_token8<CODES, DP, NT>;
  static SmemLimit limit;
  if (cudaError_t e = limit.set(k, kRing8<DP>)) return e;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(a.batch.sessions) * a.cache.heads * a.splits);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kRing8<DP>;
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, k, a);
}

template <int CODES>
cudaError_t by_size(const AttendArgs& a, int rows, cudaStream_t stream) {
  if (a.cache.head_dim <= 64)
    return rows <= 8 ? launch<CODES, 64, 1>(a, stream) : rows <= 16 ? launch<CODES, 64, 2>(a, stream) : launch<CODES, 64, 4>(a, stream);
  return rows <= 8 ? launch<CODES, 128, 1>(a, stream) : rows <= 16 ? launch<CODES, 128, 2>(a, stream) : launch<CODES, 128, 4>(a, stream);
}

}  // namespace

int attend_token8_blocks_per_sm(int head_dim, int rows) {
  if (head_dim <= 64) return rows <= 16 ? kResident8<64, 2> : kResident8<64, 4>;
  return kResident8<128, 4>;
}

cudaError_t launch_attend_token8(const AttendArgs& a, int rows, cudaStream_t stream) {
  return a.cache.codes == kCodesE4M3 ? by_size<kCodesE4M3>(a, rows, stream) : by_size<kCodesI8>(a, rows, stream);
}

}  // namespace pcs
