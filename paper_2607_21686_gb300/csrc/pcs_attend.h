// pcs_attend.h -- descriptors of the operators over a paged cache of keys and
// values (rotary positions, append, attention), shared by their host side
// (pcs_attend.cpp) and their kernels, and what that host side needs of a
// context (OpCall, in pcs_runtime.cpp).
#pragma once

#include <cstdint>

#include <cuda_runtime.h>

#include "pcs.h"

namespace pcs {

// ---- One call on a context ---------------------------------------------------

// Kernels of the operators, in the order of their names in the timing table.
enum OpKernel { kOpRotate, kOpAppend, kOpAttendToken, kOpAttendBlock, kOpAttendJoin };

// Words of a call that are zero on entry and have to be on exit.
constexpr int kOpWords = 1024;

// Message of the calling thread's last error, and the status itself.
pcs_status op_fail(pcs_status s, const char* fmt, ...) __attribute__((format(printf, 2, 3)));

// A call: names an NVTX range, holds the context and its device from begin()
// on, and the stream's workspace from scratch() to end().
class OpCall {
 public:
  OpCall(pcs_ctx* c, const char* name, void* stream);
  ~OpCall();
  OpCall(const OpCall&) = delete;
  OpCall& operator=(const OpCall&) = delete;
  pcs_status begin();
  // `bytes` of device memory (256-byte aligned) that are the call's until its
  // end on the stream, and kOpWords words.
  pcs_status scratch(uint64_t bytes, uint8_t** out, uint32_t** words);
  // Around each launch: counts and times it.
  void before(OpKernel k);
  pcs_status after(cudaError_t e);
  pcs_status end();
  cudaStream_t stream() const { return stream_; }
  uint32_t* errors() const;
  int sm_count() const;

 private:
  pcs_ctx* c_;
  cudaStream_t stream_;
  bool locked_ = false, scratch_ = false;
  void* scope_ = nullptr;
};

// ---- Division by a number known on the host ------------------------------------

// n / d for 0 <= n < 2^31 by a multiplication: with L = ceil(log2 d) and
// m = ceil(2^(31+L) / d), m d exceeds 2^(31+L) by less than 2^L, so the error
// of n m / 2^(31+L) stays below 1 / d (Granlund and Montgomery 1994).
struct FastDiv {
  uint32_t mul = 0, shift = 0, d = 1;
  void set(uint32_t by) {
    d = by;
    uint32_t l = 0;
    while ((1ull << l) < by) ++l;
    shift = 31 + l;
    mul = static_cast<uint32_t>(((1ull << shift) + by - 1) / by);
  }
  __host__ __device__ __forceinline__ uint32_t div(uint32_t n) const {
    return static_cast<uint32_t>((static_cast<uint64_t>(n) * mul) >> shift);
  }
};

// ---- The cache and the sessions of a call -----------------------------------------

struct CacheDev {
  uint8_t* k;
  uint8_t* v;
  const int32_t* table;
  const int32_t* v_table;  // null: the K pages' table
  int64_t table_stride;
  int64_t page_bytes, row_bytes, head_bytes;  // strides
  uint32_t unit, page_units, row_units;       // page and row strides in units of `unit` bytes,
                                              // in which every row's offset has 32 bits
  FastDiv page_rows, ring;
  int32_t n_pages, slots;   // slots a table has room for
  int32_t heads, head_dim;
  int32_t sinks;
  int32_t ring_rows;        // 0: none

  __host__ __device__ __forceinline__ uint32_t slot_of(uint32_t p) const {
    if (ring_rows == 0 || p < static_cast<uint32_t>(sinks)) return p;
    const uint32_t x = p - sinks;
    return sinks + x - ring.div(x) * ring.d;
  }
};

struct BatchDev {
  const int32_t* lens;
  const int32_t* q_off;  // null: `each` new tokens a session
  int64_t tokens;
  int32_t sessions, each, max_new;
};

// A tensor of heads: strides in bytes.
struct HeadsDev {
  uint8_t* data;
  int64_t token_bytes, head_bytes;
};

// ---- Rotary positions, append ------------------------------------------------------

constexpr int kRotTensors = 8;  // tensors of one call

struct RotSlot {
  const uint8_t* src;
  uint8_t* dst;          // null: the cache's keys (role 1) or values (role 2)
  int64_t src_token, src_head, dst_token, dst_head;  // strides in bytes
  int32_t heads;         // heads of this and of the tensors before it
  int32_t role;
};

struct RotArgs {
  RotSlot t[kRotTensors];
  int32_t n;               // tensors; those from `plain` on are copied, not turned
  int32_t plain;
  const int32_t* pos;
  const float* freq;
  int32_t axes;
  int32_t axis_end[4];     // pairs of the axes up to and with this one
  int32_t pairs;
  int32_t head_dim;
  int32_t interleaved, inverse;
  int64_t tokens;
  uint32_t* err;
  CacheDev cache;          // append only
  BatchDev batch;
};
// paged: some tensor goes to the cache.  vec: every address and a head are
// multiples of 16 bytes.
cudaError_t launch_rotate(const RotArgs& a, uint32_t dtype, bool paged, bool vec, int sm_count,
                          cudaStream_t stream);

// ---- Attention -------------------------------------------------------------------------

struct AttendArgs {
  CacheDev cache;
  BatchDev batch;
  HeadsDev q, out;
  float* lse;              // [tokens][q heads] or null
  float scale_log2;        // scale * log2(e)
  int32_t window;          // 0: everything before a token
  int32_t group;           // query heads per key head
  FastDiv by_group;
  int32_t splits;          // parts of a session's visible tokens
  float* part;             // partial results (splits > 1)
  uint32_t* ticket;        // token kernel: zero on entry and on exit; null: parts are joined later
  int32_t box_rows;        // block kernel: rows of a tensor copy, 0: rows are copied one by one
  uint32_t* err;
};

// One row is one query head of one new token; the token kernel takes all rows
// of a session and key head together.
constexpr int kTokenRowsMax = 32;
constexpr int kTokenWarps = 4;
// Floats of one partial result: its rows' sums, then their maxima and totals.
inline uint64_t token_part_floats(int rows, int head_dim) {
  const uint64_t padded = rows <= 8 ? 8 : rows <= 16 ? 16 : 32;
  return padded * ((head_dim <= 64 ? 64 : 128) + 2);
}
// Parts are joined by the block that ends last while there are at most
// kTokenOwnJoin of them (a.ticket), else by a second launch (`join`).
constexpr int kTokenOwnJoin = 16;
cudaError_t launch_attend_token(const AttendArgs& a, uint32_t dtype, int rows, bool join, cudaStream_t stream);
// Blocks of the token kernel that one SM holds, for `rows` rows a key head.
int attend_token_blocks_per_sm(int head_dim, int rows);

// The block kernel: a session and key head's rows in blocks of kBlockRows,
// `blocks` of them at most.  With splits > 1 a block's part is its rows' sums,
// maxima and totals; launch_attend_join joins them.
constexpr int kBlockRows = 256;
constexpr int kBlockTile = 128;  // tokens of a tile
inline uint64_t block_part_floats(int head_dim) { return kBlockRows * ((head_dim <= 64 ? 64 : 128) + 2); }
// maps: the keys' and the values' tensor maps (box_rows > 0), 128 bytes each.
struct alignas(64) TensorMaps {
  uint8_t k[128], v[128];
};
cudaError_t launch_attend_block(const AttendArgs& a, uint32_t dtype, int blocks, const TensorMaps& maps,
                                cudaStream_t stream);
cudaError_t launch_attend_join(const AttendArgs& a, uint32_t dtype, int blocks, cudaStream_t stream);

}  // namespace pcs
