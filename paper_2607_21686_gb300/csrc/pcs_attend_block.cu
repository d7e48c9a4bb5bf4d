// pcs_attend_block.cu -- attention of blocks of new tokens (frames, prompts)
// over a paged cache of keys and values.
//
// k_attend_block  The same one-pass softmax as the token kernel's, with enough
//                 query rows per key head that the matrix products bound it
//                 (4 head_dim flops per visible pair of row and token): they
//                 run on the fifth-generation tensor cores.  A block takes one
//                 session, key head and 256 rows (query heads of a key head
//                 side by side, then tokens) as two tiles of 128, and walks
//                 the tokens they see in tiles of 128.  Per tile and row tile
//                 S = Q K^T goes to tensor memory, four warps turn it into
//                 weights (a thread per row), write them back as the first
//                 operand of O += P V, which stays in tensor memory too; while
//                 one row tile is with its warps the other one has the matrix
//                 unit.  Keys and values come into rings in shared memory in
//                 the 128-byte swizzled layout the matrix unit reads: one warp
//                 sends tensor copies of boxes of 8 to 128 rows of a page
//                 (BOX), or three copy row by row, 16 bytes at a time, from
//                 pages whose size no such box divides.
//                 A tile that some rows see in part may hold infinities or NaN
//                 in values those rows must not see, and 0 * inf is NaN: there
//                 the copying warps replace them by zeros, and the rows that
//                 do see them take them up at the end.
//                 A prompt of 8,000 tokens, 32 query heads over 8 of 128 in
//                 bfloat16: 367 us, 1.43 PFLOP/s (75 % of the measured matrix
//                 rate), with inputs that come from memory; 349 us in a loop over
//                 three sets of them; by rows 867 us.  The matrix unit is busy
//                 52 % of a 4,096-token prompt's 111 us.  When that took 129 us,
//                 leaving out the warps' work on the scores saved 31 us, the products
//                 15 us and the exponentials 5 us: what bounds it is the chain
//                 of both with the hand-overs between them, and at windows and
//                 short sessions the 6 us a block takes to its first scores and
//                 from its last ones.  Some values of a thread spill (68 to 100
//                 bytes stored, 112 to 232 loaded, by form).
// k_attend_join   joins the parts of rows whose tokens were split over blocks.
#include "pcs_attend_dev.h"
#include "pcs_attend_rounds.h"

namespace pcs {
namespace {

constexpr int kTile = 128;              // rows of a row tile, tokens of a tile
// Warps 0-3 and 4-7: a row tile each, a thread a row; 8: matrix products; 9-11:
// copies.
constexpr int kSoftWarps = 8;
constexpr int kMmaWarp = 8;
constexpr int kCopyWarp = 9;
constexpr int kCopyWarps = 3;
constexpr int kThreads = 32 * (kCopyWarp + kCopyWarps);
// Registers of a thread: the launch's 168 shared out anew, 256 x 224 + 128 x 56
// = 384 x 168.
constexpr int kSoftRegs = 224, kOtherRegs = 56;
constexpr int kLag = 2;                 // copies in flight behind the newest
constexpr int kValid = 8;               // tiles whose masks are kept
constexpr unsigned kFull = 0xffffffffu;
constexpr float kSlack = 8.0f;          // as in the token kernel
constexpr long long kWaitCycles = 4000000000ll;

// Tiles of keys and of values in shared memory, each a ring of its own: a warp
// that waits for values alone then sees every phase of their barriers.  (In one
// ring of five, keys and values took turns in a buffer; a warp that waited for
// its values while the keys before them were still on their way took the phase
// before those for its own.)
template <int DP>
constexpr int kKeyTiles = DP == 64 ? 4 : 2;
template <int DP, bool BOX>
constexpr int kValueTiles = DP == 64 ? 4 : BOX ? 3 : 2;
template <int DP, bool BOX>
constexpr int kBuffers = kKeyTiles<DP> + kValueTiles<DP, BOX>;
template <int DP>
constexpr uint32_t kTileBytes = kTile * DP * 2;
template <int DP, bool BOX>
constexpr uint32_t kSmemBytes = (2 + kBuffers<DP, BOX>) * kTileBytes<DP> + 1024;

__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}
// Bounded wait for the phase of the given parity; false: it gave up.
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity) {
  if (bar_try(bar, parity)) return true;
  const long long t0 = clock64();
  while (!bar_try(bar, parity))
    if (clock64() - t0 > kWaitCycles) return false;
  return true;
}

// A barrier expects `bytes`; a box of rows of a pool for them.
__device__ __forceinline__ void fill_begins(uint32_t bar, uint32_t bytes, uint32_t one) {
  asm volatile(
      "{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %2, 0;\n\t"
      "@q mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n\t}" ::"r"(bar),
      "r"(bytes), "r"(one)
      : "memory");
}
__device__ __forceinline__ void copy_box(uint32_t to, uint64_t map, int d, int head, int row, int page, uint32_t bar,
                                         uint32_t one) {
  asm volatile(
      "{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %7, 0;\n\t"
      "@q cp.async.bulk.tensor.4d.shared::cta.global.tile.mbarrier::complete_tx::bytes "
      "[%0], [%1, {%2, %3, %4, %5}], [%6];\n\t}" ::"r"(to),
      "l"(map), "r"(d), "r"(head), "r"(row), "r"(page), "r"(bar), "r"(one)
      : "memory");
}

// ---- Tensor memory and its matrix instruction ----------------------------------

// Shared-memory operand in 128-byte rows of a 128-byte swizzle: the low word of
// its descriptor (`lead` bytes lie between 64-element columns of a transposed
// one) and the high one (eight rows are 1,024 bytes).
__device__ __forceinline__ uint32_t operand(uint32_t at, uint32_t lead) { return (at >> 4) | (lead >> 4) << 16; }
constexpr uint32_t kOperandHigh = (1024 >> 4) | 1u << 14 | 2u << 29;
// One thread of a warp.
__device__ __forceinline__ uint32_t elected() {
  uint32_t is;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(is));
  return is;
}
// 128 x N products of 16-bit elements into 32-bit floats; b_across: the second
// operand lies with its columns, not its rows, in 128-byte rows.
template <typename T>
__device__ __forceinline__ constexpr uint32_t instruction(uint32_t n, bool b_across) {
  const uint32_t type = sizeof(T) == 2 && std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
  return (1u << 4) | (type << 7) | (type << 10) | ((b_across ? 1u : 0u) << 16) | ((n >> 3) << 17) |
         ((128u >> 4) << 24);
}
// The matrix instruction and its commit are run by the whole warp and take
// effect in the one thread that `one` is set in: its operands then stay in
// uniform registers, where it wants them.  Issued by one thread of a branch of
// its own, every instruction took some 120 cycles instead of the 64 it keeps
// the unit busy for.
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t i, bool add, uint32_t one) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t.reg .b64 a, b;\n\tmov.b64 a, {%1, %6};\n\tmov.b64 b, {%2, %6};\n\t"
      "setp.ne.u32 p, %4, 0;\n\tsetp.ne.u32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n\t}" ::"r"(d),
      "r"(a), "r"(b), "r"(i), "r"(add ? 1u : 0u), "r"(one), "n"(kOperandHigh)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t i, bool add, uint32_t one) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t.reg .b64 b;\n\tmov.b64 b, {%2, %6};\n\t"
      "setp.ne.u32 p, %4, 0;\n\tsetp.ne.u32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n\t}" ::"r"(d),
      "r"(a), "r"(b), "r"(i), "r"(add ? 1u : 0u), "r"(one), "n"(kOperandHigh)
      : "memory");
}
// The barrier's arrival when everything issued so far has finished.
__device__ __forceinline__ void mma_commit(uint32_t bar, uint32_t one) {
  asm volatile(
      "{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %1, 0;\n\t"
      "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar),
      "r"(one)
      : "memory");
}
__device__ __forceinline__ void fence_before() {
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
}
__device__ __forceinline__ void fence_after() {
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
}
// 32 columns of this warp's 32 lanes, a lane per thread.
__device__ __forceinline__ void tm_load(uint32_t (&r)[32], uint32_t at) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,"
      "%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]),
        "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]),
        "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]),
        "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(at)
      : "memory");
}
__device__ __forceinline__ void tm_store(uint32_t at, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,"
      "%26,%27,%28,%29,%30,%31,%32};" ::"r"(at),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
      "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]),
      "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]),
      "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
// Barriers of the threads of a row tile, and of the copying warps.
__device__ __forceinline__ void row_tile_sync(int t) { asm volatile("barrier.cta.sync %0, 128;" ::"r"(1 + t) : "memory"); }
__device__ __forceinline__ void copy_sync() {
  asm volatile("barrier.cta.sync 3, %0;" ::"n"(32 * kCopyWarps) : "memory");
}
__device__ __forceinline__ void tm_store16(uint32_t at, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(at),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
      "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void tm_loaded() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tm_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Two floats side by side, and operations on both.
__device__ __forceinline__ uint64_t pair(float x, float y) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
  return r;
}
__device__ __forceinline__ void unpair(uint64_t p, float& x, float& y) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(p));
}
__device__ __forceinline__ uint64_t fma2(uint64_t x, uint64_t y, uint64_t z) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(x), "l"(y), "l"(z));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t x, uint64_t y) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(x), "l"(y));
  return r;
}
__device__ __forceinline__ float max3(float x, float y, float z) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(x), "f"(y), "f"(z));
  return r;
}

// Columns of tensor memory: scores, sums and weights of the row tiles.  Heads of
// 64 leave room for weights beside the scores, so that the next tile's scores
// are made while this one's weights are (kAhead); with heads of 128 the weights
// lie over the scores they came from.
constexpr uint32_t kScores = 0, kSums = 256;
template <int DP>
constexpr bool kAhead = DP == 64;
template <int DP>
constexpr uint32_t kWeights = DP == 64 ? 384 : 0;
template <int DP>
constexpr uint32_t kWeightsStep = DP == 64 ? 64 : kTile;

// What a block's rows see, the same for all its warps.
struct Work {
  SessionView all;    // the session
  SessionView view;   // what these rows see
  int32_t rows;       // of the session and key head
  int32_t row0;       // the block's first
  int32_t tile0, tiles;
  int32_t pmin, pmax; // positions of the block's rows
};

__device__ __forceinline__ Work block_work(const AttendArgs& a, int s, int blk, int sp) {
  Work w;
  w.all = session_rows(a, s);
  w.rows = max(w.all.m, 0) * a.group;
  w.row0 = blk * 2 * kTile;
  w.tiles = 0;
  if (w.row0 >= w.rows || !rows_there(a, w.all, false)) return w;
  const int t0 = a.by_group.div(w.row0);
  const int t1 = a.by_group.div(min(w.row0 + 2 * kTile, w.rows) - 1);
  w.view = w.all;
  narrow(a, w.view, t0, t1 + 1, a.box_rows > 0 ? a.box_rows : 1);
  w.pmin = w.all.first + t0;
  w.pmax = w.all.first + t1;
  const int n = (w.view.seen + kTile - 1) / kTile;
  const int per = (n + a.splits - 1) / a.splits;
  w.tile0 = min(n, sp * per);
  w.tiles = min(n, w.tile0 + per) - w.tile0;
  return w;
}

// Of row tile t.
__device__ __forceinline__ RowsRange tile_range(const AttendArgs& a, const Work& w, int t) {
  const int r0 = w.row0 + t * kTile, r1 = min(r0 + kTile, w.rows) - 1;
  return rows_range(a, w.view, w.all.first + static_cast<int>(a.by_group.div(r0)),
                    w.all.first + static_cast<int>(a.by_group.div(r1)));
}

// 16-bit elements (two in a word) whose exponent is all ones.
template <typename T>
__device__ __forceinline__ uint32_t specials(uint32_t x) {
  const uint32_t e = std::is_same<T, __half>::value ? 0x7c00u : 0x7f80u;
  return ((x & e) == e ? 0xffffu : 0u) | ((x >> 16 & e) == e ? 0xffff0000u : 0u);
}

// A box of rows: pages of its keys and values as the table has them, the first
// row in them.  The page ids are on their way from memory until settle().
struct Box {
  int32_t k, v, row;
};
// The box at place e of a view.
__device__ __forceinline__ Box box_place(const AttendArgs& a, int s, const SessionView& w, int32_t e) {
  const CacheDev& c = a.cache;
  const uint32_t slot = box_slot(a, w, e);
  if (slot >= static_cast<uint32_t>(c.slots)) {
    atomicOr(a.err, kDevErrIndex);
    return {-1, -1, 0};
  }
  const uint32_t page = c.page_rows.div(slot);
  const int64_t at = s * c.table_stride + page;
  Box x;
  x.k = __ldg(c.table + at);
  x.v = __ldg((c.v_table ? c.v_table : c.table) + at);
  x.row = slot - page * c.page_rows.d;
  return x;
}
// Page n_pages, whose rows come out as zeros, for what is not in the cache.
__device__ __forceinline__ void settle(const AttendArgs& a, Box& x) {
  const int32_t n = a.cache.n_pages;
  if (x.k < 0 || x.k >= n || x.v < 0 || x.v >= n) {
    if (x.k < -1 || x.k >= n || x.v < -1 || x.v >= n) atomicOr(a.err, kDevErrIndex);
    x.k = x.v = n;
  }
}

// Whether some of eight elements are infinite or NaN: the lowest bit of an
// exponent added to one of all ones carries into the sign's place.
template <typename T>
__device__ __forceinline__ bool has_specials(const uint4& v) {
  constexpr uint32_t e = std::is_same<T, __half>::value ? 0x7c007c00u : 0x7f807f80u;
  constexpr uint32_t one = std::is_same<T, __half>::value ? 0x04000400u : 0x00800080u;
  return ((((v.x & e) + one) | ((v.y & e) + one) | ((v.z & e) + one) | ((v.w & e) + one)) & 0x80008000u) != 0;
}
// Zeros for them; whether there were any.
template <typename T>
__device__ __forceinline__ bool take_out(uint4* at, uint4 v) {
  if (!has_specials<T>(v)) return false;
  const uint4 m = make_uint4(specials<T>(v.x), specials<T>(v.y), specials<T>(v.z), specials<T>(v.w));
  v.x &= ~m.x, v.y &= ~m.y, v.z &= ~m.z, v.w &= ~m.w;
  *at = v;
  return true;
}

// MAKERS: warps that send tensor copies of boxes of rows (the other copying warps
// look values over); 0: rows are copied one by one.  Boxes of eight rows are
// sixteen or thirty-two a tile, more than one warp can send in a tile's time: two
// warps take keys and values (8,000-token prompt in pages of 8: 411 us by one,
// 358 us by two; in pages of 16: 349 and 353 us).
template <typename T, int DP, int MAKERS>
__global__ void __launch_bounds__(kThreads, 1)
    k_attend_block(const __grid_constant__ AttendArgs a, const __grid_constant__ TensorMaps maps, int blocks) {
  constexpr bool BOX = MAKERS > 0;
  constexpr int kRing = kBuffers<DP, BOX>, kKeys = kKeyTiles<DP>, kValues = kValueTiles<DP, BOX>;
  using Fills = Rings<kKeys, kValues>;
  using Bars = Barriers<kKeys, kValues, BOX>;
  auto buf_of = [](int i) { return Fills::buffer(i); };
  auto use_of = [](int i) { return Fills::use(i); };
  constexpr uint32_t kBytes = kTileBytes<DP>;
  constexpr uint32_t kPanel = kTile * 128;  // 64 columns of a tile
  constexpr int kChunks = DP / 8;
  extern __shared__ __align__(16) uint8_t raw[];
  __shared__ __align__(8) uint64_t bars[Bars::kCount];
  __shared__ uint32_t tmem_at;
  __shared__ __align__(16) uint32_t valid[kValid][4];  // a bit per token that is in the cache
  __shared__ uint32_t special;
  __shared__ uint32_t places[2][2][BOX ? 1 : kTile];      // tile, keys or values, row: offsets (not BOX)

  attend_dependency();
  const int tid = threadIdx.x, warp = __shfl_sync(kFull, tid >> 5, 0), lane = tid & 31;
  if (BOX && warp == kCopyWarp && lane < 2)
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(lane ? maps.v : maps.k)) : "memory");
  int b = blockIdx.x;
  const int head = b % a.cache.heads;
  b /= a.cache.heads;
  const int sp = b % a.splits;
  b /= a.splits;
  const int s = b % a.batch.sessions;
  const int blk = blocks - 1 - b / a.batch.sessions;  // the longest first
  const Work w = block_work(a, s, blk, sp);
  if (w.row0 >= w.rows || !rows_there(a, w.all, tid == 0)) return;
  const int nq = w.rows - w.row0 > kTile ? 2 : 1;  // row tiles

  const uint32_t smem = (smem_addr(raw) + 1023) & ~1023u;
  const uint32_t qat = smem, ring = smem + 2 * kBytes;
  uint8_t* const ring_ptr = raw + (ring - smem_addr(raw));
  const uint32_t bar0 = smem_addr(bars);
  const uint32_t q_full = bar0 + 8 * Bars::q_full(), drained = bar0 + 8 * Bars::drained();
  auto kv_full = [&](int i) { return bar0 + 8 * Bars::kv_full(i); };
  auto kv_empty = [&](int i) { return bar0 + 8 * Bars::kv_empty(i); };
  auto s_full = [&](int t) { return bar0 + 8 * Bars::s_full(t); };
  auto p_full = [&](int t) { return bar0 + 8 * Bars::p_full(t); };
  auto o_full = [&](int t) { return bar0 + 8 * Bars::o_full(t); };
  auto s_read = [&](int t) { return bar0 + 8 * Bars::s_read(t); };  // kAhead: scores are in registers
  auto v_fine = [&](int j) { return bar0 + 8 * Bars::v_fine(j); };  // BOX: the values of tile j are looked over
  if (tid == 0) {
    Bars::each(kTile, 32 * kSoftWarps / 2 * nq, BOX ? 1 : 32 * kCopyWarps, 32 * (kCopyWarps - MAKERS),
               [&](int i, int count) { bar_init(bar0 + 8 * i, count); });
    special = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(&tmem_at))
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = tmem_at;
  bool ok = true;

  // This lane's 16-byte chunk of a row of a tile: kAtOnce rows an instruction.
  constexpr int kAtOnce = 32 / kChunks;
  const int chunk = lane % kChunks, sub = lane / kChunks;
  const bool mine = chunk * 8 < a.cache.head_dim;
  auto spot = [](int row, int c) { return (c >> 3) * kPanel + row * 128 + (((c & 7) ^ (row & 7)) << 4); };

  if (warp >= kSoftWarps) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
    if (warp >= kCopyWarp && w.tiles > 0) {
    // ---- Copying warps.  Fill i: keys of tile i / 2, or its values ----
    const int c = warp - kCopyWarp;
    const RowsRange range = rows_range(a, w.view, w.pmin, w.pmax);
    if constexpr (BOX) {
      if (c < MAKERS) {
        // Fills the rings, a lane per box of rows.
        const uint32_t one = elected();
        const uint64_t kmap = reinterpret_cast<uint64_t>(maps.k), vmap = reinterpret_cast<uint64_t>(maps.v);
        const int rows = a.box_rows, boxes = kTile / rows;
        auto look = [&](int t) {
          Box x = {-1, -1, 0};
          const int e = t * kTile + lane * rows;
          if (lane < boxes && e < w.view.seen) x = box_place(a, s, w.view, e);
          return x;
        };
        Box box, next = look(w.tile0);
        int sent = 2 * w.tiles;
        for (int i = c; i < 2 * w.tiles; i += MAKERS) {
          const int buf = buf_of(i), use = use_of(i);
          if (use > 0) ok = bar_wait(kv_empty(buf), (use - 1) & 1);
          ok = __all_sync(kFull, ok);
          if (!ok) {
            sent = i;
            break;
          }
          if (MAKERS == 2 || (i & 1) == 0) {
            box = next;
            if (i / 2 + 1 < w.tiles) next = look(w.tile0 + i / 2 + 1);
            settle(a, box);
            // A bit per token of the tile: its box is in the cache.
            const uint32_t there = __ballot_sync(kFull, lane < boxes && box.k < a.cache.n_pages);
            if (lane < 4 && (i & 1) == 0) {
              uint32_t m = 0;
              for (int k = 0; k < 32; k += 8)
                if (there >> ((lane * 32 + k) / rows) & 1) m |= 0xffu << k;
              const int32_t e = (w.tile0 + i / 2) * kTile + lane * 32;
              m &= ~(RowRange::upto(w.view.gap1 - e) & ~RowRange::upto(w.view.gap0 - e));
              valid[(i / 2) % kValid][lane] = m;
            }
            __syncwarp();
          }
          fill_begins(kv_full(buf), kBytes, one);
          for (int k = 0; k < boxes; ++k) {
            const int row = __shfl_sync(kFull, box.row, k), page = __shfl_sync(kFull, i & 1 ? box.v : box.k, k);
#pragma unroll
            for (int d = 0; d < DP / 64; ++d)
              copy_box(ring + buf * kBytes + d * kPanel + k * rows * 128, i & 1 ? vmap : kmap, d * 64, head, row, page,
                       kv_full(buf), one);
          }
        }
        // No copy is on its way into a block that has ended, whoever gave up.
        const bool landed =
            Fills::drain(c, MAKERS, sent, [&](int f) { return bar_wait(kv_full(buf_of(f)), use_of(f) & 1); });
        ok = ok && landed;
      } else {
        // The others look values over.
        for (int i = 1; i < 2 * w.tiles && ok; i += 2) {
          const int buf = buf_of(i);
          ok = bar_wait(kv_full(buf), use_of(i) & 1);
          ok = __all_sync(kFull, ok);
          if (!ok) break;
          if (!range.whole_and_filled(w.tile0 + i / 2)) {
            uint4* tile = reinterpret_cast<uint4*>(ring_ptr + buf * kBytes);
            bool any = false;
            constexpr int kFlight = 8;  // vectors in flight
            constexpr int step = 32 * (kCopyWarps - MAKERS);
            for (int k = (c - MAKERS) * 32 + lane; k < static_cast<int>(kBytes / 16); k += kFlight * step) {
              uint4 v[kFlight];
#pragma unroll
              for (int u = 0; u < kFlight; ++u) v[u] = tile[k + u * step];
#pragma unroll
              for (int u = 0; u < kFlight; ++u) any |= take_out<T>(tile + k + u * step, v[u]);
            }
            if (any) special = 1;
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          }
          bar_arrive(v_fine(i / 2));
        }
      }
    } else {
      constexpr int kGroups = kTile / kAtOnce;  // warp c moves every kCopyWarps-th
      if (!mine)                                // chunks that no copy writes
        for (int i = 0; i < kRing; ++i)
          for (int g = c; g < kGroups; g += kCopyWarps)
            *reinterpret_cast<uint4*>(ring_ptr + i * kBytes + spot(g * kAtOnce + sub, chunk)) = make_uint4(0, 0, 0, 0);
      auto landed = [&](int i) {
        if ((i & 1) && !range.whole_and_filled(w.tile0 + i / 2) && mine) {
          uint8_t* tile = ring_ptr + buf_of(i) * kBytes;
          bool any = false;
          for (int g = c; g < kGroups; g += kCopyWarps)
            any |= take_out<T>(reinterpret_cast<uint4*>(tile + spot(g * kAtOnce + sub, chunk)),
                               *reinterpret_cast<const uint4*>(tile + spot(g * kAtOnce + sub, chunk)));
          if (any) special = 1;
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        bar_arrive(kv_full(buf_of(i)));
      };
      // Rows' places of tile t, of the call's tile w.tile0 + t.
      auto look = [&](int t) {
        for (int r = c * 32 + lane; r < kTile; r += 32 * kCopyWarps) {
          RowPlace x = {kNoRow, kNoRow};
          const int e = (w.tile0 + t) * kTile + r;
          if (e < w.view.seen) x = row_place(a, s, seen_position(w.view, e));
          places[t & 1][0][r] = x.k;
          places[t & 1][1][r] = x.v;
          const uint32_t there = __ballot_sync(kFull, x.k != kNoRow);
          if (lane == 0) valid[t % kValid][r >> 5] = there;
        }
      };
      look(0);
      const uint8_t* kbase = a.cache.k + head * a.cache.head_bytes + chunk * 16;
      const uint8_t* vbase = a.cache.v + head * a.cache.head_bytes + chunk * 16;
      ok = in_rounds(
          2 * w.tiles,
          [&](int i) {
            const int use = use_of(i);
            return __all_sync(kFull, use == 0 || bar_wait(kv_empty(buf_of(i)), (use - 1) & 1)) != 0;
          },
          // The tile's places are written, the ones before the last are used up.
          [&] { copy_sync(); },
          [&](int i) {
            const uint8_t* base = i & 1 ? vbase : kbase;
            const uint32_t* place = places[(i / 2) & 1][i & 1];
            const uint32_t tile = ring + buf_of(i) * kBytes;
#pragma unroll 4
            for (int g = c; g < kGroups; g += kCopyWarps) {
              const uint32_t o = place[g * kAtOnce + sub];
              const bool in = o != kNoRow;
              if (mine) copy16(tile + spot(g * kAtOnce + sub, chunk), row_at(a, base, in ? o : 0), in);
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
            if ((i & 1) == 0 && i / 2 + 1 < w.tiles) look(i / 2 + 1);
            asm volatile("cp.async.wait_group %0;" ::"n"(kLag) : "memory");
            if (i >= kLag) landed(i - kLag);
          });
      asm volatile("cp.async.wait_all;" ::: "memory");
      if (ok)
        for (int i = max(0, 2 * w.tiles - kLag); i < 2 * w.tiles; ++i) landed(i);
    }
    }
    // ---- The warp that feeds the matrix unit ----
    if (warp == kMmaWarp && w.tiles > 0) {
      // Everything an instruction's operands and this loop go by is the same in
      // all lanes, and made so that it is seen to be (a reduction over the
      // warp): operands then lie in uniform registers.  Moved there one by one
      // they held the instructions 80 cycles apart.
      const uint32_t one = elected(), mem = __reduce_max_sync(kFull, tmem);
      const int tiles = static_cast<int>(__reduce_max_sync(kFull, static_cast<uint32_t>(w.tiles)));
      const int row_tiles = static_cast<int>(__reduce_max_sync(kFull, static_cast<uint32_t>(nq)));
      constexpr uint32_t kQK = instruction<T>(kTile, false), kPV = instruction<T>(DP, true);
      const uint32_t q0 = operand(qat, 16), k0 = operand(ring, 16), v0 = operand(ring, kPanel);
      auto scores = [&](int t, int i) {  // S = Q K^T of row tile t, keys of fill i
        const uint32_t q = q0 + t * (kBytes >> 4), k = k0 + buf_of(i) * (kBytes >> 4);
#pragma unroll
        for (int d = 0; d < DP / 16; ++d) {
          const uint32_t at = ((d >> 2) * kPanel + (d & 3) * 32) >> 4;
          mma_ss(mem + kScores + t * kTile, q + at, k + at, kQK, d > 0, one);
        }
      };
      auto sums = [&](int t, int i, bool add) {  // O += P V, values of fill i
        const uint32_t v = v0 + buf_of(i) * (kBytes >> 4);
#pragma unroll
        for (int k = 0; k < kTile / 16; ++k)
          mma_ts(mem + kSums + t * DP, mem + kWeights<DP> + t * kWeightsStep<DP> + k * 8, v + k * (2048 >> 4), kPV,
                 add || k > 0, one);
      };
      const RowsRange range0 = tile_range(a, w, 0), range1 = tile_range(a, w, nq - 1);
      auto some = [&](int t, int j) { return __any_sync(kFull, (t ? range1 : range0).some(w.tile0 + j)); };
      int done[2] = {0, 0};  // tiles taken
      ok = __all_sync(kFull, bar_wait(q_full, 0));
      int given[2] = {0, 0};  // scores made
      // S of row tile t and tile j, whose keys are there.
      auto next_scores = [&](int t, int j) {
        if (some(t, j)) {
          if (kAhead<DP> && given[t] > 0) ok = __all_sync(kFull, bar_wait(s_read(t), (given[t] - 1) & 1));
          if (!ok) return;
          fence_after();
          scores(t, 2 * j);
          mma_commit(s_full(t), one);
          given[t] += 1;
        }
      };
      // O += P V of row tile t and tile j, whose values are there.
      auto next_sums = [&](int t, int j) {
        if (some(t, j)) {
          ok = __all_sync(kFull, bar_wait(p_full(t), done[t] & 1));
          if (!ok) return;
          fence_after();
          sums(t, 2 * j + 1, done[t] > 0);
          done[t] += 1;
          mma_commit(o_full(t), one);
        }
      };
      auto keys = [&](int j) {
        ok = __all_sync(kFull, ok && bar_wait(kv_full(buf_of(2 * j)), use_of(2 * j) & 1));
        fence_after();
      };
      if (ok) keys(0);
      for (int t = 0; t < row_tiles && ok; ++t) next_scores(t, 0);
      if (ok) mma_commit(kv_empty(0), one);
      for (int j = 0; j < tiles && ok; ++j) {
        const int vi = 2 * j + 1, ki = 2 * j + 2;
        const bool more = j + 1 < tiles;
        // Everything that is not on the way from weights to scores is waited
        // for before them: a wait takes some 200 cycles even if it is over.
        if (more) keys(j + 1);
        if (kAhead<DP> && more) {
          for (int t = 0; t < row_tiles && ok; ++t) next_scores(t, j + 1);
          mma_commit(kv_empty(buf_of(ki)), one);
        }
        ok = ok && bar_wait(kv_full(buf_of(vi)), use_of(vi) & 1);
        if (BOX) ok = ok && bar_wait(v_fine(j), (j / kValues) & 1);
        ok = __all_sync(kFull, ok);
        if (!ok) break;
        next_sums(0, j);
        if (row_tiles == 1) mma_commit(kv_empty(buf_of(vi)), one);
        if (!kAhead<DP> && more && ok) {
          next_scores(0, j + 1);
          if (row_tiles == 1) mma_commit(kv_empty(buf_of(ki)), one);
        }
        if (row_tiles == 2 && ok) {
          next_sums(1, j);
          mma_commit(kv_empty(buf_of(vi)), one);
          if (!kAhead<DP> && more && ok) {
            next_scores(1, j + 1);
            mma_commit(kv_empty(buf_of(ki)), one);
          }
        }
      }
      // Nor are products or their arrivals at barriers, when tensor memory is
      // given back.
      mma_commit(drained, one);
      const bool finished = bar_wait(drained, 0);
      ok = ok && finished;
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftRegs));
    // ---- A thread per row: weights, running maximum and total ----
    const int t = warp >> 2;
    if (t < nq) {
      const int row = (warp & 3) * 32 + lane, r = w.row0 + t * kTile + row;
      const bool there = r < w.rows;
      const uint32_t tok = a.by_group.div(there ? r : w.rows - 1);
      // Query rows, zeros behind the last: kAtOnce rows an instruction.
#pragma unroll
      for (int g = 0; g < kTile / kAtOnce / 4; ++g) {
        const int i = (g * 4 + (warp & 3)) * kAtOnce + sub, ri = w.row0 + t * kTile + i;
        const bool in = ri < w.rows;
        const uint32_t ti = a.by_group.div(in ? ri : 0);
        const int h = head * a.group + (in ? ri - static_cast<int>(ti) * a.group : 0);
        const bool live = mine && in;
        copy16(qat + t * kBytes + spot(i, chunk),
               a.q.data + (live ? (w.all.q0 + ti) * a.q.token_bytes + h * a.q.head_bytes + chunk * 16 : 0), live);
      }
      asm volatile("cp.async.wait_all;" ::: "memory");
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      bar_arrive(q_full);
      const uint32_t lanes = static_cast<uint32_t>(warp & 3) << 21;  // its warp's lanes of tensor memory
      const uint32_t sc = tmem + kScores + t * kTile + lanes, su = tmem + kSums + t * DP + lanes,
                     we = tmem + kWeights<DP> + t * kWeightsStep<DP> + lanes;
      const RowRange sees = row_range(a, w.view, w.all.first + static_cast<int32_t>(tok));
      const RowsRange range = tile_range(a, w, t);
      float top = -INFINITY, total = 0.0f;
      int done = 0;
      for (int j = 0; j < w.tiles; ++j) {
        const int tile = w.tile0 + j;
        if (!range.some(tile)) continue;
        ok = ok && bar_wait(s_full(t), done & 1);
        __syncwarp();
        fence_after();
        uint32_t x[4][32];
        tm_load(x[0], sc);
        tm_load(x[1], sc + 32);
        tm_loaded();
        tm_load(x[2], sc + 64);
        tm_load(x[3], sc + 96);
        float mx[4];
        auto highest = [&](int c) {
          mx[c] = __uint_as_float(x[c][0]);
#pragma unroll
          for (int k = 1; k < 31; k += 2) mx[c] = max3(mx[c], __uint_as_float(x[c][k]), __uint_as_float(x[c][k + 1]));
          mx[c] = fmaxf(mx[c], __uint_as_float(x[c][31]));
        };
        const uint4 in = *reinterpret_cast<const uint4*>(valid[j % kValid]);
        if (range.whole(tile) && (in.x & in.y & in.z & in.w) == kFull) {
          highest(0);
          highest(1);
          tm_loaded();
        } else {
          tm_loaded();
          const uint32_t m4[4] = {in.x, in.y, in.z, in.w};
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            // (Most 32 by 32 pieces of a tile on the diagonal are seen whole.)
            const uint32_t m = m4[c] & sees.bits(tile * kTile + c * 32);
            if (__all_sync(kFull, m == kFull)) continue;
#pragma unroll
            for (int k = 0; k < 32; ++k)
              if (!(m >> k & 1)) x[c][k] = 0xff800000u;  // -inf
          }
          highest(0);
          highest(1);
        }
        if (kAhead<DP>) {
          fence_before();
          bar_arrive(s_read(t));
        }
        highest(2);
        highest(3);
        const float high = fmaxf(max3(mx[0], mx[1], mx[2]), mx[3]) * a.scale_log2;
        if (kAhead<DP> && done > 0) {  // the weights before these are used up, the sums may be changed
          ok = ok && bar_wait(o_full(t), (done - 1) & 1);
          __syncwarp();
          fence_after();
        }
        const bool raise = high > top + kSlack;
        if (__any_sync(kFull, raise)) {
          const float to = raise ? high : top;
          const float f = raise ? exp2_fast(top - to) : 1.0f;
          top = to;
          total *= f;
          if (done > 0) {
#pragma unroll 1
            for (int c = 0; c < DP / 32; ++c) {
              uint32_t y[32];
              tm_load(y, su + c * 32);
              tm_loaded();
#pragma unroll
              for (int k = 0; k < 32; ++k) y[k] = __float_as_uint(__uint_as_float(y[k]) * f);
              tm_store(su + c * 32, y);
            }
          }
        }
        const float at = top == -INFINITY ? 0.0f : top - kLift<T>;
        const uint64_t scale2 = pair(a.scale_log2, a.scale_log2), at2 = pair(-at, -at);
        uint64_t sum[2] = {0, 0};
#pragma unroll
        for (int h = 0; h < 4; ++h) {
          uint32_t y[16];
#pragma unroll
          for (int k = 0; k < 16; ++k) {
            const uint32_t* z = &x[h][2 * k];
            float u, v;
            unpair(fma2(pair(__uint_as_float(z[0]), __uint_as_float(z[1])), scale2, at2), u, v);
            u = exp2_fast(u);
            v = exp2_fast(v);
            sum[k & 1] = add2(sum[k & 1], pair(u, v));
            y[k] = pack2<T>(u, v);
          }
          // (Heads of 128: over the first half of the scores, all of which are
          // in registers by now.)
          tm_store16(we + h * 16, y);
        }
        float u, v;
        unpair(add2(sum[0], sum[1]), u, v);
        total += u + v;
        tm_stored();
        fence_before();
        bar_arrive(p_full(t));
        done += 1;
      }
      // Whatever the copying warps took out of the values is known when they have
      // handed over the last ones.
      if (ok && w.tiles > 0) {
        const int last = w.tiles - 1, i = 2 * last + 1;
        ok = BOX ? bar_wait(v_fine(last), (last / kValues) & 1) : bar_wait(kv_full(buf_of(i)), use_of(i) & 1);
      }
      // (The sums before the last ones were done when the last scores were.)
      if (ok && done > 0) ok = bar_wait(o_full(t), (done - 1) & 1);
      __syncwarp();
      fence_after();
      constexpr float kLn2 = 0.693147180559945309f;
      const float inv = total == 0.0f ? 0.0f : 1.0f / total;
      const bool mend = *reinterpret_cast<volatile uint32_t*>(&special) != 0;
      float* part = a.part + (static_cast<int64_t>(blockIdx.x) * 2 + t) * (DP + 2) * kTile + row;
#pragma unroll 1
      for (int c = 0; c < DP / 32; ++c) {
        const int d0 = c * 32;
        uint32_t x[32];
        if (done > 0) {
          tm_load(x, su + c * 32);
          tm_loaded();
        } else {
#pragma unroll
          for (int k = 0; k < 32; ++k) x[k] = 0;
        }
        if (mend && there) {
          // Infinities and NaN among the values that this row sees in tiles
          // where zeros took their place.
          const RowsRange block = rows_range(a, w.view, w.pmin, w.pmax);
          for (int j = w.tile0; j < w.tile0 + w.tiles; ++j) {
            if (block.whole_and_filled(j)) continue;
            for (int e = j * kTile; e < min((j + 1) * kTile, w.view.seen); ++e) {
              if (!(sees.bits(e) & 1) || (e >= w.view.gap0 && e < w.view.gap1)) continue;
              const RowPlace pl = row_place(a, s, seen_position(w.view, e));
              if (pl.k == kNoRow) continue;
              const uint8_t* v = row_at(a, a.cache.v + head * a.cache.head_bytes, pl.v) + d0 * 2;
#pragma unroll
              for (int k = 0; k < 32; k += 2) {
                if (d0 + k >= a.cache.head_dim) continue;
                const uint32_t y = *reinterpret_cast<const uint32_t*>(v + 2 * k), m = specials<T>(y);
                T e0, e1;
                const uint16_t lo = static_cast<uint16_t>(y), hi = static_cast<uint16_t>(y >> 16);
                memcpy(&e0, &lo, 2);
                memcpy(&e1, &hi, 2);
                if (m & 0xffffu) x[k] = __float_as_uint(__uint_as_float(x[k]) + static_cast<float>(e0));
                if (m >> 16) x[k + 1] = __float_as_uint(__uint_as_float(x[k + 1]) + static_cast<float>(e1));
              }
            }
          }
        }
        if (a.splits > 1) {  // a column at a time: a warp's rows lie side by side
#pragma unroll
          for (int k = 0; k < 32; ++k) part[(d0 + k) * kTile] = __uint_as_float(x[k]);
        } else {  // over the query rows, which are used up
#pragma unroll
          for (int k = 0; k < 32; k += 8) {
            uint4 y;
            y.x = pack2<T>(__uint_as_float(x[k]) * inv, __uint_as_float(x[k + 1]) * inv);
            y.y = pack2<T>(__uint_as_float(x[k + 2]) * inv, __uint_as_float(x[k + 3]) * inv);
            y.z = pack2<T>(__uint_as_float(x[k + 4]) * inv, __uint_as_float(x[k + 5]) * inv);
            y.w = pack2<T>(__uint_as_float(x[k + 6]) * inv, __uint_as_float(x[k + 7]) * inv);
            *reinterpret_cast<uint4*>(ring_ptr - (2 - t) * kBytes + spot(row, (d0 + k) >> 3)) = y;
          }
        }
      }
      if (a.splits > 1) {
        part[DP * kTile] = top;
        part[(DP + 1) * kTile] = total;
      } else {
        row_tile_sync(t);
#pragma unroll 4
        for (int g = warp & 3; g < kTile / kAtOnce; g += 4) {  // whole rows to memory
          const int i = g * kAtOnce + sub, ri = w.row0 + t * kTile + i;
          if (ri >= w.rows || !mine || !ok) continue;
          const uint32_t ti = a.by_group.div(ri);
          const int h = head * a.group + (ri - static_cast<int>(ti) * a.group);
          *reinterpret_cast<uint4*>(a.out.data + (w.all.q0 + ti) * a.out.token_bytes + h * a.out.head_bytes + chunk * 16) =
              *reinterpret_cast<const uint4*>(ring_ptr - (2 - t) * kBytes + spot(i, chunk));
        }
        if (ok && there && a.lse) {
          const int h = head * a.group + (r - static_cast<int>(tok) * a.group);
          a.lse[(w.all.q0 + tok) * (static_cast<int64_t>(a.cache.heads) * a.group) + h] =
              total == 0.0f ? -INFINITY : fmaf(top - kLift<T>, kLn2, logf(total));
        }
      }
    }
  }
  if (!ok && lane == 0) atomicOr(a.err, kDevErrTimeout);
  fence_before();
  __syncthreads();
  if (warp == kMmaWarp) {
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
  }
}

// Joins the parts of a row tile: a thread per row, 32 of its dims a block.
template <typename T, int DP>
__global__ void __launch_bounds__(kTile) k_attend_join(const __grid_constant__ AttendArgs a, int blocks) {
  attend_dependency();
  int b = blockIdx.x;
  const int d0 = b % (DP / 32) * 32;
  b /= DP / 32;
  const int t = b % 2;
  b /= 2;
  const int head = b % a.cache.heads;
  b /= a.cache.heads;
  const int s = b % a.batch.sessions, blk = blocks - 1 - b / a.batch.sessions;
  const SessionView v = session_rows(a, s);
  const int row = threadIdx.x, r = blk * 2 * kTile + t * kTile + row;
  if (!rows_there(a, v, false) || r >= v.m * a.group) return;
  // The parts of the blocks that the block kernel's numbering puts side by side.
  const int64_t first = static_cast<int64_t>(b) * a.splits * a.cache.heads + head;
  const int64_t step = static_cast<int64_t>(a.cache.heads) * 2 * (DP + 2) * kTile;
  const float* part = a.part + (first * 2 + t) * (DP + 2) * kTile + row;
  float top = -INFINITY;
  for (int w = 0; w < a.splits; ++w) top = fmaxf(top, __ldcg(part + w * step + DP * kTile));
  const float at = top == -INFINITY ? 0.0f : top;
  float o[32] = {}, total = 0.0f;
  for (int w = 0; w < a.splits; ++w) {
    const float f = exp2_fast(__ldcg(part + w * step + DP * kTile) - at);
    total = fmaf(__ldcg(part + w * step + (DP + 1) * kTile), f, total);
#pragma unroll
    for (int k = 0; k < 32; ++k) o[k] = fmaf(__ldcg(part + w * step + (d0 + k) * kTile), f, o[k]);
  }
  const float inv = total == 0.0f ? 0.0f : 1.0f / total;
  const uint32_t tok = a.by_group.div(r);
  const int h = head * a.group + (r - static_cast<int>(tok) * a.group);
  uint8_t* out = a.out.data + (v.q0 + tok) * a.out.token_bytes + h * a.out.head_bytes + d0 * 2;
#pragma unroll
  for (int k = 0; k < 32; k += 8) {
    if (d0 + k >= a.cache.head_dim) continue;
    uint4 y;
    y.x = pack2<T>(o[k] * inv, o[k + 1] * inv);
    y.y = pack2<T>(o[k + 2] * inv, o[k + 3] * inv);
    y.z = pack2<T>(o[k + 4] * inv, o[k + 5] * inv);
    y.w = pack2<T>(o[k + 6] * inv, o[k + 7] * inv);
    *reinterpret_cast<uint4*>(out + 2 * k) = y;
  }
  if (d0 == 0 && a.lse)
    a.lse[(v.q0 + tok) * (static_cast<int64_t>(a.cache.heads) * a.group) + h] =
        total == 0.0f ? -INFINITY : fmaf(top - kLift<T>, 0.693147180559945309f, logf(total));
}

cudaLaunchConfig_t config(int64_t grid, int threads, uint32_t smem, cudaLaunchAttribute* attr, cudaStream_t stream) {
  attr->id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr->val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(grid));
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cfg;
}

template <typename T, int DP, int MAKERS>
cudaError_t launch_form(const AttendArgs& a, int blocks, const TensorMaps& maps, cudaStream_t stream) {
  auto k = k_attend_block<T, DP, MAKERS>;
  constexpr uint32_t smem = kSmemBytes<DP, (MAKERS > 0)>;
  static SmemLimit limit;
  if (cudaError_t e = limit.set(k, smem)) return e;
  cudaLaunchAttribute attr;
  const cudaLaunchConfig_t cfg =
      config(static_cast<int64_t>(blocks) * a.batch.sessions * a.splits * a.cache.heads, kThreads, smem, &attr, stream);
  return cudaLaunchKernelEx(&cfg, k, a, maps, blocks);
}
template <typename T, int DP>
cudaError_t launch(const AttendArgs& a, int blocks, const TensorMaps& maps, cudaStream_t stream) {
  return a.box_rows == 0   ? launch_form<T, DP, 0>(a, blocks, maps, stream)
         : a.box_rows == 8 ? launch_form<T, DP, 2>(a, blocks, maps, stream)
                           : launch_form<T, DP, 1>(a, blocks, maps, stream);
}

template <typename T, int DP>
cudaError_t launch_join(const AttendArgs& a, int blocks, cudaStream_t stream) {
  cudaLaunchAttribute attr;
  const cudaLaunchConfig_t cfg =
      config(static_cast<int64_t>(blocks) * a.batch.sessions * a.cache.heads * 2 * (DP / 32), kTile, 0, &attr, stream);
  return cudaLaunchKernelEx(&cfg, k_attend_join<T, DP>, a, blocks);
}

}  // namespace

cudaError_t launch_attend_block(const AttendArgs& a, uint32_t dtype, int blocks, const TensorMaps& maps,
                                cudaStream_t stream) {
  if (dtype == PCS_DT_F16)
    return a.cache.head_dim <= 64 ? launch<__half, 64>(a, blocks, maps, stream) : launch<__half, 128>(a, blocks, maps, stream);
  return a.cache.head_dim <= 64 ? launch<__nv_bfloat16, 64>(a, blocks, maps, stream)
                                : launch<__nv_bfloat16, 128>(a, blocks, maps, stream);
}

cudaError_t launch_attend_join(const AttendArgs& a, uint32_t dtype, int blocks, cudaStream_t stream) {
  if (dtype == PCS_DT_F16)
    return a.cache.head_dim <= 64 ? launch_join<__half, 64>(a, blocks, stream) : launch_join<__half, 128>(a, blocks, stream);
  return a.cache.head_dim <= 64 ? launch_join<__nv_bfloat16, 64>(a, blocks, stream) : launch_join<__nv_bfloat16, 128>(a, blocks, stream);
}

}  // namespace pcs
