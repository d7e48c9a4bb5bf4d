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
//                 A block takes one, two or four key heads of a session and a part of
//                 its tokens, a warp a head (or a half, a quarter of the tiles of one), in
//                 tiles of 32 tokens.  Tensor copies bring boxes of 8 to 32 rows of a page,
//                 of all the block's heads at once, and the scale bytes of 16 heads beside
//                 them; the warps send them in turn.  (What bounds copies by the warps'
//                 lanes is their number: a scale byte is a request of its own beside 64 or
//                 128 bytes of codes.)
//                 256 sessions over windows of 1,024 tokens, 16 heads of 64, E4M3: 102 us,
//                 5.4 TB/s (79 % of the measured copy rate; 1.7 waves of equal blocks); 48
//                 sessions of 1 to 12,000 tokens, 32 over 8 heads of 128, I8: 104 us.  The
//                 copies alone, a warp a head, took 94 us of the first.
// k_attend_token8_rows  The same from pages whose size no such box divides: each warp
//                 copies rows of tiles of its own (the 48 sessions in pages of 25: 139 us).
#include "pcs_attend_token_dev.h"
#include "pcs_codes_dev.h"

namespace pcs {
namespace {

constexpr int kTile8 = kTokenTile8;

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
constexpr float kNothing = -3e38f;
// A weight beyond this, or times its value's scale beyond 2^15, raises the reference.
constexpr float kMostWeight = 1.2676506e30f;  // 2^100

// A warp's query rows over the tiles that it takes.
template <int CODES, int DP, int NT>
struct TokenRows {
  static constexpr int H = NT == 4 ? 1 : 2;     // halves of a tile, 16 tokens, that are in registers at once
  static constexpr bool kEarly = NT == 1;       // a tile's values beside its scores
  static constexpr float kUp = 7.0f;            // weights are 2^7 times higher, as kLift says
  uint32_t qf[NT][DP / 16][2];
  float back[NT][2];       // of the rows this thread has scores of, times the scale
  int32_t new_token[NT][2];
  float o[DP / 16][NT][4];
  float refer[NT][2], total[NT][2];
  int lane, g, q4, m_new;

  __device__ __forceinline__ void begin(const AttendArgs& a, const SessionView& view, int head, int lane_) {
    lane = lane_, g = lane >> 2, q4 = lane & 3, m_new = view.m;
    const int rows = view.m * a.group;
    // Query rows as the second operand: of chunk k, dims 4 q4 .. +3 of row g, times
    // 2^-back, the power that puts the row's largest element at 2^14.
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
        if (r < rows && d < a.cache.head_dim) x = *reinterpret_cast<const uint2*>(q + d * 2);
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
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        new_token[n][i] = min(static_cast<int>(a.by_group.div(n * 8 + q4 * 2 + i)), view.m - 1);
        refer[n][i] = kNothing;
        total[n][i] = 0.0f;
      }
#pragma unroll
      for (int i = 0; i < DP / 16; ++i) o[i][n][0] = o[i][n][1] = o[i][n][2] = o[i][n][3] = 0.0f;
    }
  }

  // Tokens [e0, e0 + 32): keys and values in shared memory, at(h, k) the offset of this
  // lane's chunk of chunks 2 k and 2 k + 1 of half h; the scales of token e0 + lane; which
  // tokens are in the cache; whether some row does not see all (sees: a new token's bits).
  template <typename At, typename Sees>
  __device__ __forceinline__ void tile(uint32_t kat, uint32_t vat, const At& at, float ks, float vs, int e0, uint32_t there, bool part,
                                       const Sees& sees) {
#pragma unroll 1
    for (int h0 = 0; h0 < 2; h0 += H) halves(kat, vat, at, ks, vs, e0, there, part, sees, h0);
  }

  template <typename At, typename Sees>
  __device__ __forceinline__ void halves(uint32_t kat, uint32_t vat, const At& at, float ks, float vs, int e0, uint32_t there, bool part,
                                         const Sees& sees, int h0) {
    // All that the tile gives is on its way out of shared memory before any of it is used.
    uint32_t kf[H][DP / 32][4], vf[H][DP / 32][4];
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int k = 0; k < DP / 32; ++k) ldm4(kf[h][k], kat + at(h0 + h, k));
    if (kEarly) {
#pragma unroll
      for (int h = 0; h < H; ++h)
#pragma unroll
        for (int k = 0; k < DP / 32; ++k) ldm4t(vf[h][k], vat + at(h0 + h, k));
    }
    // Scores of tokens 16 h + g, + 8, but for the rows' factors.
    float c[H][NT][4];
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int n = 0; n < NT; ++n) c[h][n][0] = c[h][n][1] = c[h][n][2] = c[h][n][3] = 0.0f;
#pragma unroll
    for (int k = 0; k < DP / 32; ++k)
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int h = 0; h < H; ++h) {
          uint32_t x[4];
          four_halves<CODES>(kf[h][k][2 * j], x[0], x[2]);
          four_halves<CODES>(kf[h][k][2 * j + 1], x[1], x[3]);
#pragma unroll
          for (int n = 0; n < NT; ++n) mma<__half>(c[h][n], x, qf[n][2 * k + j][0], qf[n][2 * k + j][1]);
        }
    float vscale[H][2];  // of token 16 h + 8 j + g
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float y = __shfl_sync(kFull, ks, (h0 + h) * 16 + j * 8 + g);
        vscale[h][j] = __shfl_sync(kFull, vs, (h0 + h) * 16 + j * 8 + g);
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
          seen[n][i] = (there & (part ? sees(new_token[n][i], e0) : kFull)) >> (16 * h0 + g);
#pragma unroll
          for (int h = 0; h < H; ++h)
#pragma unroll
            for (int j = 0; j < 2; ++j)
              if (!(seen[n][i] >> (h * 16 + j * 8) & 1)) c[h][n][2 * j + i] = -INFINITY;
        }
    }
    // Weights 2^(score - reference), p; times the values' scales, v.
    float p[H][NT][4], v[H][NT][4];
    auto weigh = [&] {
      float most = 0.0f, largest = 0.0f;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int h = 0; h < H; ++h)
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
          for (int h = 0; h < H; ++h)
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
          for (int h = 0; h < H; ++h)
#pragma unroll
            for (int j = 0; j < 2; ++j)
              if (!(seen[n][i] >> (h * 16 + j * 8) & 1)) v[h][n][2 * j + i] = 0.0f;
    }
    uint32_t w[H][NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int h = 0; h < H; ++h) {
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
    // (Only the NaN of 8-bit floats would go through a weight of 0: where there is one among
    // tokens that some rows do not see, or rows that a box brought along that are nobody's,
    // as those behind the end of a ring, each new token takes the codes of what it sees.)
    bool apart = false;
    if (CODES == kCodesE4M3 && masked) {
      uint32_t nan = 0;
#pragma unroll
      for (int h = 0; h < H; ++h)
#pragma unroll
        for (int k = 0; k < DP / 32; ++k) {
          uint32_t f[4];
          ldm4t(f, vat + at(h0 + h, k));
#pragma unroll
          for (int i = 0; i < 4; ++i) nan |= (f[i] & 0x7f7f7f7fu) + 0x01010101u;
        }
      apart = __any_sync(kFull, (nan & 0x80808080u) != 0);
    }
    if (!apart) {
#pragma unroll
      for (int h = 0; h < H; ++h)
#pragma unroll
        for (int k = 0; k < DP / 32; ++k) {
          uint32_t x[4];
          if (!kEarly) ldm4t(vf[h][k], vat + at(h0 + h, k));
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            operand(x, vf[h][k][2 * j], vf[h][k][2 * j + 1]);
#pragma unroll
            for (int n = 0; n < NT; ++n) mma<__half>(o[2 * k + j][n], x, w[h][n][0], w[h][n][1]);
          }
        }
    } else {
      for (int i = 0; i < m_new; ++i) {
        const uint32_t m = (there & (part ? sees(i, e0) : kFull)) >> (16 * h0 + 2 * q4);
#pragma unroll
        for (int h = 0; h < H; ++h) {
          uint32_t in[2];  // of tokens 16 h + 2 q4, +1 and 8 more
#pragma unroll
          for (int z = 0; z < 2; ++z)
            in[z] = (m >> (16 * h + 8 * z) & 1 ? 0xffffu : 0u) | (m >> (16 * h + 8 * z + 1) & 1 ? 0xffff0000u : 0u);
#pragma unroll
          for (int k = 0; k < DP / 32; ++k) {
            uint32_t f[4], x[4];
            ldm4t(f, vat + at(h0 + h, k));
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              operand(x, f[2 * j] & in[0], f[2 * j + 1] & in[1]);
#pragma unroll
              for (int n = 0; n < NT; ++n) {
                // (On top of the sums, in the order of the products above: what is taken
                // out changes no rounding of what stays.)
                float y[4];
#pragma unroll
                for (int z = 0; z < 4; ++z) y[z] = o[2 * k + j][n][z];
                mma<__half>(y, x, w[h][n][0], w[h][n][1]);
#pragma unroll
                for (int z = 0; z < 4; ++z)
                  if (new_token[n][z & 1] == i) o[2 * k + j][n][z] = y[z];
              }
            }
          }
        }
      }
    }
  }

  // The rows' totals over the warp.
  __device__ __forceinline__ void end() {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        total[n][i] += __shfl_xor_sync(kFull, total[n][i], 4);
        total[n][i] += __shfl_xor_sync(kFull, total[n][i], 8);
        total[n][i] += __shfl_xor_sync(kFull, total[n][i], 16);
      }
  }
};

// ---- Boxes of rows ---------------------------------------------------------------------

// A block's turn is its warps' tiles: those of its heads, or several of one's.  Codes of
// keys and of values of a turn, each box with its heads one behind the other; then scale
// bytes of 16 heads, of keys and of values.
// Three turns, two of them on their way: 139 KB an SM with heads of 64 and four blocks, 135 KB
// with heads of 128 and two.  (48 sessions of 1 to 12,000 tokens, 8 heads of 128: 106 us, 108
// us with two turns of three blocks; heads of 64, 256 sessions: 104 us, three blocks of four
// turns 128 us, five of two 118 us.)
constexpr int kStages8 = 3;
template <int DP, int HEADS>
constexpr uint32_t kStage8 = 2 * kWarps * kTile8 * DP + 2 * (kWarps / HEADS) * kTile8 * 16;
// (Boxes begin at multiples of 1,024 bytes: room to get there.)
template <int DP, int HEADS>
constexpr uint32_t kSmem8 = kStages8 * kStage8<DP, HEADS> + 1024;
// Blocks that one SM holds, by its registers and by its shared memory.
template <int DP, int NT>
constexpr int kByRegisters8 = NT == 4 ? 2 : NT == 2 ? (DP == 64 ? 3 : 2) : DP == 64 ? 4 : 2;
template <int DP, int NT, int HEADS>
constexpr int kResident8 = kByRegisters8<DP, NT> * (kSmem8<DP, HEADS> + 3 * 1024) <= 227 * 1024
                               ? kByRegisters8<DP, NT>
                               : static_cast<int>(227 * 1024 / (kSmem8<DP, HEADS> + 3 * 1024));

__device__ __forceinline__ void box_of_codes(uint32_t to, uint64_t map, int row, int head, int page, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(to),
      "l"(map), "r"(0), "r"(row), "r"(head), "r"(page), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void box_of_scales(uint32_t to, uint64_t map, int byte, int row, int page, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(to),
      "l"(map), "r"(byte), "r"(row), "r"(page), "r"(bar)
      : "memory");
}

template <int CODES, int DP, int NT, int HEADS>
__global__ void __launch_bounds__(kThreads, (kResident8<DP, NT, HEADS>))
    k_attend_token8(const __grid_constant__ AttendArgs a, const __grid_constant__ CodeMaps maps) {
  constexpr int kStages = kStages8;
  constexpr uint32_t kStage = kStage8<DP, HEADS>;
  constexpr int kTiles = kWarps / HEADS;        // tiles of a turn
  constexpr uint32_t kCodeBytes = kWarps * kTile8 * DP, kScaleBytes = kTiles * kTile8 * 16;
  constexpr int kRows = 8 * NT;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ uint32_t valid[kStages][kTiles];
  __shared__ __align__(8) uint64_t bars[2 * kStages];  // filled, free
  __shared__ TreeNode nodes[PCS_TREE_MAX];

  attend_dependency();
  const int tid = threadIdx.x, warp = __shfl_sync(kFull, tid >> 5, 0), lane = tid & 31;
  const int groups = a.cache.heads / HEADS;
  const int head0 = blockIdx.x % groups * HEADS;
  const int sp = blockIdx.x / groups % a.splits;
  int s = blockIdx.x / groups / a.splits;
  if (a.ranked) {
    s = ranked_session(a.batch, s, tid, kThreads, reinterpret_cast<uint32_t*>(smem));
    // The ring lies over its numbers: what this thread wrote and read comes before the tensor
    // copies behind the barrier below.
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  const int head = head0 + warp % HEADS, turn = warp / HEADS;  // this warp's head, and its tile of a turn
  if (tid < 4) asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(maps.map[tid])) : "memory");
  SessionView view = session_rows(a, s);
  narrow(a, view, 0, view.m, a.box_rows);
  if (view.m <= 0) return;  // the same in every part
  const int rows = view.m * a.group;
  if (!rows_there(a, view, tid == 0)) return;  // (max_new tokens' rows are at most kRows)
  const bool tree = a.parent != nullptr;
  const uint32_t ring = (smem_addr(smem) + 1023) & ~1023u, bar0 = smem_addr(bars);
  uint8_t* const ring_ptr = smem + (ring - smem_addr(smem));
  auto full = [&](int stage) { return bar0 + 8 * stage; };
  auto empty = [&](int stage) { return bar0 + 8 * (kStages + stage); };
  if (tid == 0) {
    for (int i = 0; i < kStages; ++i) {
      bar_init(full(i), 1);
      bar_init(empty(i), kWarps);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (tree) tree_nodes(a, view, tid, nodes);
  __syncthreads();

  // This part's turns.
  const int all = (view.seen + kTile8 * kTiles - 1) / (kTile8 * kTiles);
  const int per = (all + a.splits - 1) / a.splits;
  const int begin = min(all, sp * per), turns = min(all, begin + per) - begin;

  // A lane's box of the rows of turn i, of which there are `boxes`.
  const int shift = 31 - __clz(a.box_rows), boxes = kTiles * kTile8 >> shift;
  auto look = [&](int i) {
    Box x = {-1, -1, 0};
    const int e = ((begin + i) * kTiles * kTile8) + (lane << shift);
    if (i < turns && lane < boxes && e < view.seen) x = box_place(a, s, view, e);
    return x;
  };
  auto send = [&](Box x, int i, int stage) {
    settle(a, x);
    const uint32_t at = ring + stage * kStage, bar = full(stage);
#pragma unroll
    for (int k = 0; k < kTiles; ++k) {
      const int r = k * kTile8 + lane, e = (begin + i) * kTiles * kTile8 + r;
      const bool in = __shfl_sync(kFull, x.k, r >> shift) < a.cache.n_pages && !(e >= view.gap0 && e < view.gap1);
      const uint32_t there = __ballot_sync(kFull, in);
      if (lane == 0) valid[stage][k] = there;
    }
    if (lane == 0) asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(kStage) : "memory");
    for (int k = 0; k < boxes; ++k) {
      const int kp = __shfl_sync(kFull, x.k, k), vp = __shfl_sync(kFull, x.v, k), row = __shfl_sync(kFull, x.row, k);
      const uint32_t codes = at + (k << shift) * HEADS * DP, scales = at + 2 * kCodeBytes + (k << shift) * 16;
      if (lane == 0) {
        box_of_codes(codes, reinterpret_cast<uint64_t>(maps.map[0]), row, head0, kp, bar);
        box_of_codes(codes + kCodeBytes, reinterpret_cast<uint64_t>(maps.map[1]), row, head0, vp, bar);
        box_of_scales(scales, reinterpret_cast<uint64_t>(maps.map[2]), head0 & ~15, row, kp, bar);
        box_of_scales(scales + kScaleBytes, reinterpret_cast<uint64_t>(maps.map[3]), head0 & ~15, row, vp, bar);
      }
    }
  };
  // The first turns are sent by a warp each; then warp i % kWarps sends turn i + kStages - 1
  // when it comes to turn i, whose stage was used up in the turn before.
  static_assert(kStages - 1 <= kWarps, "a warp a stage");
  if (warp < kStages - 1 && warp < turns) send(look(warp), warp, warp);
  Box ahead = look(warp + kStages - 1);

  TokenRows<CODES, DP, NT> work;
  work.begin(a, view, head, lane);
  // Ranges of the first and the last new token.  (Nodes of a tree: what all of them
  // see of the context.)
  RowRange low = row_range(a, view, view.first);
  const RowRange high = row_range(a, view, view.first + view.m - 1);
  if (tree) low.hi = context_end(view);
  // Which of the tokens from place b on the rows of new token t see, as bits.
  auto sees = [&](int32_t t, int b) {
    return tree ? tree_row(a, view, nodes[t]).bits(b) : row_range(a, view, view.first + t).bits(b);
  };
  // Where this lane's rows of its warp's tile lie in a turn's codes: row 16 h + (lane & 15)
  // of it in box r >> shift, at the warp's head.
  uint32_t row_at_h[2], chunk[DP / 32];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int r = h * 16 + (lane & 15), b = (turn * kTile8 + r) >> shift;
    row_at_h[h] = ((((b * HEADS + warp % HEADS) << shift) + (r & (a.box_rows - 1)))) * DP;
  }
#pragma unroll
  for (int k = 0; k < DP / 32; ++k)  // (the swizzle goes by a row's number modulo 8, as boxes have at least 8)
    chunk[k] = chunk_at<DP>(lane & 7, 2 * k + (lane >> 4)) - (lane & 7) * DP;
  auto at = [&](int h, int k) { return row_at_h[h] + chunk[k]; };

  bool ok = true;
  int stage = 0;
  uint32_t phase = 0;
  for (int i = 0; i < turns; ++i) {
    if (i + kStages - 1 < turns && i % kWarps == warp) {
      const int into = stage == 0 ? kStages - 1 : stage - 1;  // the stage of turn i - 1
      if (i > 0) ok = __all_sync(kFull, bar_wait(empty(into), phase ^ (stage == 0 ? 1 : 0))) != 0;
      if (!ok) break;
      send(ahead, i + kStages - 1, into);
      ahead = look(i + kWarps + kStages - 1);
    }
    ok = __all_sync(kFull, bar_wait(full(stage), phase)) != 0;
    if (!ok) break;
    const int e0 = ((begin + i) * kTiles + turn) * kTile8;
    if (e0 < view.seen) {
      const uint32_t codes = ring + stage * kStage;
      const uint8_t* scales = ring_ptr + stage * kStage + 2 * kCodeBytes + (turn * kTile8 + lane) * 16 + (head & 15);
      // (Boxes begin ahead of what is seen and end behind it.)
      const bool part = !(e0 + kTile8 - 1 <= low.hi && (e0 >= high.lo || e0 + kTile8 <= low.first));
      work.tile(codes, codes + kCodeBytes, at, scale_value(scales[0]), scale_value(scales[kScaleBytes]), e0, valid[stage][turn], part,
                sees);
    }
    __syncwarp();
    if (lane == 0) bar_arrive(empty(stage));
    stage = stage + 1 == kStages ? 0 : stage + 1;
    if (stage == 0) phase ^= 1;
  }
  if (!ok) {
    // A copy did not come.  Those that this warp knows of get as long again, then the
    // block ends: every warp that gives up does so, so none is on its way then.
    for (int k = 0; k < kStages; ++k) bar_wait(full(k), phase ^ (k < stage ? 1 : 0));
    if (lane == 0) atomicOr(a.err, kDevErrTimeout);
  }
  work.end();

  // A warp's result is its part's: one of splits * kTiles of its head.
  const int parts = a.splits * kTiles, part = sp * kTiles + turn;
  const int64_t pair = static_cast<int64_t>(s) * a.cache.heads + head;
  const int64_t part_floats = static_cast<int64_t>(kRows) * (DP + 2);
  const bool half = a.dtype == PCS_DT_F16;
  const int g = lane >> 2, q4 = lane & 3;
  // Row `row`'s dims d, d + 1 and, from one thread, its log sum of exponentials.
  auto write = [&](int row, int d, float x, float y, float inv) {
    const uint32_t tok = a.by_group.div(row);
    if (d < a.cache.head_dim)
      *reinterpret_cast<uint32_t*>(a.out.data + (view.q0 + tok) * a.out.token_bytes +
                                   (head * a.group + (row - static_cast<int>(tok) * a.group)) * a.out.head_bytes + d * 2) =
          half ? pack2<__half>(x * inv, y * inv) : pack2<__nv_bfloat16>(x * inv, y * inv);
  };
  auto write_lse = [&](int row, float top, float total) {
    const uint32_t tok = a.by_group.div(row);
    if (a.lse)
      a.lse[(view.q0 + tok) * (static_cast<int64_t>(a.cache.heads) * a.group) + head * a.group + (row - static_cast<int>(tok) * a.group)] =
          total == 0.0f ? -INFINITY : fmaf(top, 0.693147180559945309f, logf(total));
  };
  if (parts == 1) {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int row = n * 8 + q4 * 2 + i;
        if (row >= rows) continue;
        const float total = work.total[n][i], inv = total == 0.0f ? 0.0f : 1.0f / total;
#pragma unroll
        for (int d = 0; d < DP / 16; ++d) write(row, d * 16 + 2 * g, work.o[d][n][i], work.o[d][n][2 + i], inv);
        if (g == 0) write_lse(row, work.refer[n][i], total);
      }
    return;
  }
  float* mine = a.part + (pair * parts + part) * part_floats;
  // (A join in a launch of its own takes kLift off the maxima, where the result's type has one.)
  const float lift = a.ticket ? 0.0f : half ? kLift<__half> : kLift<__nv_bfloat16>;
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int row = n * 8 + q4 * 2 + i;
      if (row >= rows) continue;
#pragma unroll
      for (int d = 0; d < DP / 16; ++d)
        *reinterpret_cast<float2*>(mine + row * DP + d * 16 + 2 * g) = make_float2(work.o[d][n][i], work.o[d][n][2 + i]);
      if (g == 0) {
        mine[kRows * DP + row] = work.refer[n][i] == kNothing ? -INFINITY : work.refer[n][i] + lift;
        mine[kRows * DP + kRows + row] = work.total[n][i];
      }
    }
  if (a.ticket == nullptr) return;

  // The part that ends last joins all, in the parts' order: a part a lane for a row's
  // factors, then two dims a lane.
  __threadfence();
  __syncwarp();
  uint32_t before = 0;
  if (lane == 0) before = atomicInc(a.ticket + pair, parts - 1);
  if (__shfl_sync(kFull, before, 0) != static_cast<uint32_t>(parts - 1)) return;
  __threadfence();
  const float* first = a.part + pair * parts * part_floats;
  for (int row = 0; row < rows; ++row) {
    float top = -INFINITY, total = 0.0f;
    if (lane < parts) {
      top = __ldcg(first + lane * part_floats + kRows * DP + row);
      total = __ldcg(first + lane * part_floats + kRows * DP + kRows + row);
    }
    float m = top;
#pragma unroll
    for (int k = 16; k > 0; k /= 2) m = fmaxf(m, __shfl_xor_sync(kFull, m, k));
    const float factor = exp2_fast(top - (m == -INFINITY ? 0.0f : m));
    total *= factor;
#pragma unroll
    for (int k = 16; k > 0; k /= 2) total += __shfl_xor_sync(kFull, total, k);
    float2 x[DP / 64];
#pragma unroll
    for (int d = 0; d < DP / 64; ++d) x[d] = make_float2(0.0f, 0.0f);
#pragma unroll 4
    for (int w = 0; w < parts; ++w) {
      const float f = __shfl_sync(kFull, factor, w);
#pragma unroll
      for (int d = 0; d < DP / 64; ++d) {
        const float2 y = __ldcg(reinterpret_cast<const float2*>(first + w * part_floats + row * DP + 64 * d + 2 * lane));
        x[d].x = fmaf(y.x, f, x[d].x);
        x[d].y = fmaf(y.y, f, x[d].y);
      }
    }
    const float inv = total == 0.0f ? 0.0f : 1.0f / total;
#pragma unroll
    for (int d = 0; d < DP / 64; ++d) write(row, 64 * d + 2 * lane, x[d].x, x[d].y, inv);
    if (lane == 0) write_lse(row, m, total);
  }
}

// ---- Rows one by one ---------------------------------------------------------------------

template <int DP>
constexpr int kRowStages = DP == 64 ? 3 : 2;
// Codes of keys and of values, then a word of scale bytes of each row.
template <int DP>
constexpr uint32_t kRowStage = 2 * kTile8 * (DP + 4);
// The rings, or what the warps' results take, which lie over them at the end.
template <int DP>
constexpr uint32_t kRowRing = kWarps * kRowStages<DP> * kRowStage<DP>;
template <int DP, int NT>
constexpr uint32_t kRowJoin = kWarps * 8 * NT * (kPadOf<DP> + 2) * 4;
template <int DP, int NT>
constexpr uint32_t kRowSmem = kRowRing<DP> > kRowJoin<DP, NT> ? kRowRing<DP> : kRowJoin<DP, NT>;

template <int CODES, int DP, int NT>
__global__ void __launch_bounds__(kThreads, (kByRegisters8<DP, NT>))
    k_attend_token8_rows(const __grid_constant__ AttendArgs a) {
  constexpr int kStages = kRowStages<DP>;
  constexpr uint32_t kStage = kRowStage<DP>;
  constexpr int kChunks = DP / 16;           // 16-byte chunks of a row
  constexpr int kRowsAtOnce = 32 / kChunks;  // rows one copy instruction of a warp moves
  constexpr int kRows = 8 * NT;
  constexpr int kPad = kPadOf<DP>;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ uint32_t valid[kWarps][kStages];
  __shared__ TreeNode nodes[PCS_TREE_MAX];

  attend_dependency();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int g = lane >> 2, q4 = lane & 3;
  const int head = blockIdx.x % a.cache.heads;
  const int sp = blockIdx.x / a.cache.heads % a.splits;
  const int s = blockIdx.x / a.cache.heads / a.splits;
  const SessionView view = session_view(a, s);
  if (view.m <= 0) return;  // the same in every part
  if (!rows_there(a, view, tid == 0)) return;  // (max_new tokens' rows are at most kRows)
  const int head_dim = a.cache.head_dim;
  const bool tree = a.parent != nullptr;
  uint8_t* const ring_ptr = smem + warp * kStages * kStage;
  const uint32_t ring = smem_addr(ring_ptr);
  if (head_dim < DP) {  // chunks that no copy writes
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

  RowPlace place;
  {
    RowPlace ahead[kStages];
#pragma unroll
    for (int i = 0; i < kStages; ++i) ahead[i] = look(t_next + i * kWarps);
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) {
      if (t_next < t_end) copy(ahead[i], i);
      asm volatile("cp.async.commit_group;" ::: "memory");
      t_next += kWarps;
    }
    place = ahead[kStages - 1];
  }
  TokenRows<CODES, DP, NT> work;
  work.begin(a, view, head, lane);
  const bool many = view.m > 1;
  // Ranges of the first and the last new token.  (Nodes of a tree: what all of them
  // see of the context.)
  RowRange low = row_range(a, view, view.first);
  const RowRange high = row_range(a, view, view.first + view.m - 1);
  if (tree) low.hi = context_end(view);
  // Which of the tokens from place b on the rows of new token t see, as bits.
  auto sees = [&](int32_t t, int b) {
    return tree ? tree_row(a, view, nodes[t]).bits(b) : row_range(a, view, view.first + t).bits(b);
  };
  auto at = [&](int h, int k) { return chunk_at<DP>(h * 16 + (lane & 15), 2 * k + (lane >> 4)); };
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
    const uint32_t kat = ring + stage * kStage;
    const uint8_t* scales = ring_ptr + stage * kStage + 2 * kTile8 * DP + lane * 4 + scale_byte;
    const int e0 = t * kTile8;
    const bool part = many && !(e0 + kTile8 - 1 <= low.hi && (e0 >= high.lo || e0 + kTile8 <= low.first));
    work.tile(kat, kat + kTile8 * DP, at, scale_value(scales[0]), scale_value(scales[kTile8 * 4]), e0, valid[warp][stage], part, sees);
    __syncwarp();  // the stage may be filled again
    stage = stage + 1 == kStages ? 0 : stage + 1;
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  work.end();

  __syncthreads();
  const bool half = a.dtype == PCS_DT_F16;
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
        *reinterpret_cast<float2*>(r + d * 16 + 2 * g) = make_float2(work.o[d][n][i], work.o[d][n][2 + i]);
      if (g == 0) {
        // (The join takes kLift off again, where the result's type has one.)
        tops[warp * kRows + row] = work.refer[n][i] == kNothing ? -INFINITY : work.refer[n][i] + lift;
        totals[warp * kRows + row] = work.total[n][i];
      }
    }
  __syncthreads();
  if (half)
    join_parts<__half, DP, NT>(a, view, smem, s, head, sp);
  else
    join_parts<__nv_bfloat16, DP, NT>(a, view, smem, s, head, sp);
}

cudaLaunchConfig_t config(int64_t blocks, uint32_t smem, cudaLaunchAttribute* attr, cudaStream_t stream) {
  attr->id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr->val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(blocks));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cfg;
}

template <int CODES, int DP, int NT, int HEADS>
cudaError_t launch_boxes(const AttendArgs& a, const CodeMaps& maps, cudaStream_t stream) {
  auto k = k_attend_token8<CODES, DP, NT, HEADS>;
  static SmemLimit limit;
  if (cudaError_t e = limit.set(k, kSmem8<DP, HEADS>)) return e;
  cudaLaunchAttribute attr;
  const cudaLaunchConfig_t cfg =
      config(static_cast<int64_t>(a.batch.sessions) * (a.cache.heads / HEADS) * a.splits, kSmem8<DP, HEADS>, &attr, stream);
  return cudaLaunchKernelEx(&cfg, k, a, maps);
}

template <int CODES, int DP, int NT>
cudaError_t launch(const AttendArgs& a, const CodeMaps& maps, cudaStream_t stream) {
  if (a.box_rows)
    return a.box_heads == 4   ? launch_boxes<CODES, DP, NT, 4>(a, maps, stream)
           : a.box_heads == 2 ? launch_boxes<CODES, DP, NT, 2>(a, maps, stream)
                              : launch_boxes<CODES, DP, NT, 1>(a, maps, stream);
  auto k = k_attend_token8_rows<CODES, DP, NT>;
  static SmemLimit limit;
  if (cudaError_t e = limit.set(k, kRowSmem<DP, NT>)) return e;
  cudaLaunchAttribute attr;
  const cudaLaunchConfig_t cfg =
      config(static_cast<int64_t>(a.batch.sessions) * a.cache.heads * a.splits, kRowSmem<DP, NT>, &attr, stream);
  return cudaLaunchKernelEx(&cfg, k, a);
}

template <int CODES>
cudaError_t by_size(const AttendArgs& a, int rows, const CodeMaps& maps, cudaStream_t stream) {
  if (a.cache.head_dim <= 64)
    return rows <= 8    ? launch<CODES, 64, 1>(a, maps, stream)
           : rows <= 16 ? launch<CODES, 64, 2>(a, maps, stream)
                        : launch<CODES, 64, 4>(a, maps, stream);
  return rows <= 8    ? launch<CODES, 128, 1>(a, maps, stream)
         : rows <= 16 ? launch<CODES, 128, 2>(a, maps, stream)
                      : launch<CODES, 128, 4>(a, maps, stream);
}

}  // namespace

int attend_token8_blocks_per_sm(int head_dim, int rows) {
  const int n = rows <= 8 ? 1 : rows <= 16 ? 2 : 4;
  if (head_dim <= 64) return n == 1 ? kResident8<64, 1, 4> : n == 2 ? kResident8<64, 2, 4> : kResident8<64, 4, 4>;
  return n == 1 ? kResident8<128, 1, 4> : n == 2 ? kResident8<128, 2, 4> : kResident8<128, 4, 4>;
}

cudaError_t launch_attend_token8(const AttendArgs& a, int rows, const CodeMaps& maps, cudaStream_t stream) {
  return a.cache.codes == kCodesE4M3 ? by_size<kCodesE4M3>(a, rows, maps, stream) : by_size<kCodesI8>(a, rows, maps, stream);
}

}  // namespace pcs
