// pcs_attend.cpp -- host side of the operators over a paged cache of keys and
// values: checks of arguments, the choice of a kernel and of its split.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>
#include <numeric>

#include <cuda.h>

#include "pcs.h"
#include "pcs_attend.h"

using namespace pcs;

namespace {

// CUDA's tensor map encoder; null if there is none.
using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                              const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                              CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeFn encoder() {
  static const EncodeFn fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess) {
      cudaGetLastError();
      p = nullptr;
    }
    return reinterpret_cast<EncodeFn>(p);
  }();
  return fn;
}

// A pool as elements, heads, rows and pages, copied by boxes of 64 elements of
// `rows` rows of a page, 128-byte swizzled.
bool encode_pool(const pcs_kv_cache& c, void* pool, int rows, uint8_t* map) {
  const EncodeFn fn = encoder();
  if (!fn) return false;
  const cuuint64_t dims[4] = {static_cast<cuuint64_t>(c.head_dim), static_cast<cuuint64_t>(c.heads),
                              static_cast<cuuint64_t>(c.page_rows), static_cast<cuuint64_t>(c.n_pages)};
  const cuuint64_t strides[3] = {2 * static_cast<cuuint64_t>(c.head_stride), 2 * static_cast<cuuint64_t>(c.row_stride),
                                 2 * static_cast<cuuint64_t>(c.page_stride)};
  const cuuint32_t box[4] = {64, 1, static_cast<cuuint32_t>(rows), 1}, step[4] = {1, 1, 1, 1};
  CUtensorMap m;
  static_assert(sizeof m == 128, "tensor map");
  if (fn(&m, c.dtype == PCS_DT_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, pool, dims,
         strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
         CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
    return false;
  std::memcpy(map, &m, sizeof m);
  return true;
}

// A cache in 8 bits: codes copied by boxes of `rows` rows of a page, of `heads` heads one
// behind the other, as they are or swizzled by 64 or 128 bytes as they are long; scale bytes
// of 16 heads of as many rows.
bool encode_codes(const pcs_kv_cache& c, const CacheDev& d, int rows, int heads, bool swizzled, CodeMaps* maps) {
  const EncodeFn fn = encoder();
  if (!fn) return false;
  for (int i = 0; i < 4; ++i) {
    uint8_t* pool = i & 1 ? d.v : d.k;
    CUtensorMap m;
    CUresult r;
    if (i < 2) {
      const cuuint64_t dims[4] = {static_cast<cuuint64_t>(c.head_dim), static_cast<cuuint64_t>(c.page_rows),
                                  static_cast<cuuint64_t>(c.heads), static_cast<cuuint64_t>(c.n_pages)};
      const cuuint64_t strides[3] = {static_cast<cuuint64_t>(c.row_stride), static_cast<cuuint64_t>(c.head_stride),
                                     static_cast<cuuint64_t>(c.page_stride)};
      const cuuint32_t wide = c.head_dim <= 64 ? 64 : 128;
      const cuuint32_t box[4] = {wide, static_cast<cuuint32_t>(rows), static_cast<cuuint32_t>(heads), 1}, step[4] = {1, 1, 1, 1};
      r = fn(&m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, pool, dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
             !swizzled    ? CU_TENSOR_MAP_SWIZZLE_NONE
             : wide == 64 ? CU_TENSOR_MAP_SWIZZLE_64B
                          : CU_TENSOR_MAP_SWIZZLE_128B,
             CU_TENSOR_MAP_L2_PROMOTION_NONE,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    } else {
      const cuuint64_t dims[3] = {static_cast<cuuint64_t>(c.heads), static_cast<cuuint64_t>(c.page_rows),
                                  static_cast<cuuint64_t>(c.n_pages)};
      const cuuint64_t strides[2] = {static_cast<cuuint64_t>(c.row_stride), static_cast<cuuint64_t>(c.page_stride)};
      const cuuint32_t box[3] = {16, static_cast<cuuint32_t>(rows), 1}, step[3] = {1, 1, 1};
      r = fn(&m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, pool + d.scale_at, dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
             CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    }
    if (r != CUDA_SUCCESS) return false;
    std::memcpy(maps->map[i], &m, sizeof m);
  }
  return true;
}

// Rows of the boxes that tensor copies can move: a power of two that divides a
// page, so that a tile's boxes never leave theirs.  0: rows are copied one by one
// (a prompt of 8,000 tokens, 32 query heads over 8, in pages of 16: 349 us with
// boxes; in pages of 17, by rows, 867 us).
int box_rows(const pcs_kv_cache& c, int most) {
  for (int r = most; r >= 8; r /= 2)
    if (c.page_rows % r == 0) return r;
  return 0;
}

bool aligned(const void* p, uint64_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

int elem_bytes(uint32_t dtype) {
  return dtype == PCS_DT_F16 || dtype == PCS_DT_BF16 ? 2 : dtype == PCS_DT_F32 ? 4 : 0;
}

// Anything thrown on the way (memory) becomes a status.
template <typename F>
pcs_status guarded(F&& f) {
  try {
    return f();
  } catch (const std::bad_alloc&) {
    return op_fail(PCS_E_NOMEM, "out of host memory");
  } catch (...) {
    return op_fail(PCS_E_CUDA, "unexpected failure on the host");
  }
}

pcs_status check_heads(const pcs_heads* h, const char* what, uint32_t dtype, int32_t head_dim) {
  if (!h) return op_fail(PCS_E_INVAL, "%s is null", what);
  if (h->reserved) return op_fail(PCS_E_INVAL, "%s: reserved must be 0", what);
  if (h->heads < 1 || h->heads > 65535) return op_fail(PCS_E_INVAL, "%s: %d heads", what, h->heads);
  if (h->dtype != dtype) return op_fail(PCS_E_INVAL, "%s: element type %u, expected %u", what, h->dtype, dtype);
  if (h->head_dim != head_dim)
    return op_fail(PCS_E_INVAL, "%s: heads of %d elements, expected %d", what, h->head_dim, head_dim);
  if (h->token_stride < 0 || h->head_stride < 0) return op_fail(PCS_E_INVAL, "%s: negative stride", what);
  if (!h->data) return op_fail(PCS_E_INVAL, "%s: data is null", what);
  if (!aligned(h->data, elem_bytes(dtype)))
    return op_fail(PCS_E_ALIGN, "%s: data is not aligned to its elements", what);
  return PCS_OK;
}

bool vector_rows(const pcs_heads& h) {
  const int e = elem_bytes(h.dtype);
  return aligned(h.data, 16) && h.token_stride * e % 16 == 0 && h.head_stride * e % 16 == 0;
}

pcs_status check_cache(const pcs_kv_cache* c, CacheDev* d) {
  if (!c) return op_fail(PCS_E_INVAL, "cache is null");
  if (!c->k || !c->v || !c->table) return op_fail(PCS_E_INVAL, "cache: null pools or table");
  const bool codes = c->dtype == PCS_DT_E4M3 || c->dtype == PCS_DT_I8;
  if (c->dtype != PCS_DT_F16 && c->dtype != PCS_DT_BF16 && !codes)
    return op_fail(PCS_E_INVAL, "cache: element type %u (F16, BF16, E4M3 or I8)", c->dtype);
  if (c->heads < 1 || c->heads > 65535) return op_fail(PCS_E_INVAL, "cache: %d heads", c->heads);
  const int32_t part = codes ? 16 : 8;  // elements of 16 bytes
  if (c->head_dim < part || c->head_dim > 128 || c->head_dim % part != 0)
    return op_fail(PCS_E_INVAL, "cache: heads of %d elements (a multiple of %d up to 128)", c->head_dim, part);
  if (c->n_pages < 1 || c->page_rows < 1 || c->table_pages < 1)
    return op_fail(PCS_E_INVAL, "cache: n_pages, page_rows and table_pages must be positive");
  const int64_t slots = static_cast<int64_t>(c->page_rows) * c->table_pages;
  if (slots > 0x7FFFFFFFll) return op_fail(PCS_E_INVAL, "cache: more than 2^31 - 1 slots a session");
  if (c->table_stride < c->table_pages)
    return op_fail(PCS_E_INVAL, "cache: table_stride is below table_pages");
  if (c->sinks < 0 || c->ring < 0) return op_fail(PCS_E_INVAL, "cache: negative sinks or ring");
  if (c->ring > 0 && static_cast<int64_t>(c->sinks) + c->ring > slots)
    return op_fail(PCS_E_INVAL, "cache: sinks + ring exceed the %lld slots of a table",
                   static_cast<long long>(slots));
  if (c->page_stride < 0 || c->row_stride < 0 || c->head_stride < 0)
    return op_fail(PCS_E_INVAL, "cache: negative stride");
  if (!aligned(c->k, 16) || !aligned(c->v, 16) || c->page_stride % part || c->row_stride % part || c->head_stride % part)
    return op_fail(PCS_E_ALIGN, "cache: pools and strides must be multiples of 16 bytes");
  if (codes) {
    if (c->head_stride < c->head_dim || c->head_stride > 0x7FFF)
      return op_fail(PCS_E_INVAL, "cache: head_stride %lld of %d codes", static_cast<long long>(c->head_stride), c->head_dim);
    d->scale_at = static_cast<int32_t>(c->heads * c->head_stride);
    if (c->row_stride < static_cast<int64_t>(d->scale_at) + c->heads)
      return op_fail(PCS_E_INVAL, "cache: rows of %lld bytes do not hold %d heads and their scales",
                     static_cast<long long>(c->row_stride), c->heads);
  }
  const int64_t size = codes ? 1 : 2;
  d->codes = c->dtype == PCS_DT_E4M3 ? kCodesE4M3 : c->dtype == PCS_DT_I8 ? kCodesI8 : kElements16;
  d->k = static_cast<uint8_t*>(c->k);
  d->v = static_cast<uint8_t*>(c->v);
  d->table = c->table;
  d->v_table = c->v_table;
  d->table_stride = c->table_stride;
  d->page_bytes = size * c->page_stride;
  d->row_bytes = size * c->row_stride;
  d->head_bytes = size * c->head_stride;
  const uint64_t unit = std::gcd(static_cast<uint64_t>(d->page_bytes), static_cast<uint64_t>(d->row_bytes));
  d->unit = static_cast<uint32_t>(std::min<uint64_t>(std::max<uint64_t>(unit, 16), 0x7FFFFFF0u));
  if (d->page_bytes % d->unit || d->row_bytes % d->unit) d->unit = 16;
  const uint64_t pu = d->page_bytes / d->unit, ru = d->row_bytes / d->unit;
  if (pu > 0xFFFFFFFEull || ru > 0xFFFFFFFEull ||
      pu * (c->n_pages - 1) > 0xFFFFFFFEull - std::min<uint64_t>(ru * (c->page_rows - 1), 0xFFFFFFFEull))
    return op_fail(PCS_E_INVAL, "cache: rows lie more than 2^32 common divisors (%u bytes) of their strides apart",
                   d->unit);
  d->page_units = static_cast<uint32_t>(pu);
  d->row_units = static_cast<uint32_t>(ru);
  d->page_rows.set(c->page_rows);
  if (c->ring) d->ring.set(c->ring);
  d->n_pages = c->n_pages;
  d->slots = static_cast<int32_t>(slots);
  d->heads = c->heads;
  d->head_dim = c->head_dim;
  d->sinks = c->sinks;
  d->ring_rows = c->ring;
  return PCS_OK;
}

pcs_status check_batch(const pcs_kv_batch* b, BatchDev* d) {
  if (!b) return op_fail(PCS_E_INVAL, "batch is null");
  if (b->reserved) return op_fail(PCS_E_INVAL, "batch: reserved must be 0");
  if (b->sessions < 0 || b->tokens < 0 || b->tokens > 0x7FFFFFFFll || b->max_new < 0 || b->max_len < 0)
    return op_fail(PCS_E_INVAL, "batch: negative or too large counts");
  if (b->sessions == 0 && b->tokens > 0) return op_fail(PCS_E_INVAL, "batch: tokens without sessions");
  if (b->sessions > 0 && !b->lens) return op_fail(PCS_E_INVAL, "batch: lens is null");
  if (b->q_off) {
    if (b->tokens > 0 && b->max_new < 1) return op_fail(PCS_E_INVAL, "batch: max_new is needed with q_off");
  } else if (b->sessions > 0 && b->tokens % b->sessions != 0) {
    return op_fail(PCS_E_INVAL, "batch: %lld tokens do not share out over %d sessions",
                   static_cast<long long>(b->tokens), b->sessions);
  }
  d->lens = b->lens;
  d->q_off = b->q_off;
  d->tokens = b->tokens;
  d->sessions = b->sessions;
  d->each = b->q_off || b->sessions == 0 ? 0 : static_cast<int32_t>(b->tokens / b->sessions);
  d->max_new = b->q_off ? static_cast<int32_t>(std::min<int64_t>(b->max_new, b->tokens)) : d->each;
  return PCS_OK;
}

pcs_status check_rotary(const pcs_rotary* r, int32_t head_dim, RotArgs* a) {
  if (r->axes < 1 || r->axes > 4) return op_fail(PCS_E_INVAL, "rotary: %d axes (1 to 4)", r->axes);
  if (r->flags & ~(PCS_ROT_INTERLEAVED | PCS_ROT_INVERSE))
    return op_fail(PCS_E_INVAL, "rotary: unknown flags 0x%x", r->flags);
  int64_t pairs = 0;
  for (int i = 0; i < 4; ++i) {
    if (r->pairs[i] < 0 || (i >= r->axes && r->pairs[i] != 0))
      return op_fail(PCS_E_INVAL, "rotary: %d pairs on axis %d of %d", r->pairs[i], i, r->axes);
    pairs += r->pairs[i];
    a->axis_end[i] = static_cast<int32_t>(std::min<int64_t>(pairs, 0x7FFFFFFF));
  }
  if (2 * pairs > head_dim)
    return op_fail(PCS_E_INVAL, "rotary: %lld pairs in heads of %d elements", static_cast<long long>(pairs), head_dim);
  if (pairs > 0 && (!r->pos || !r->freq)) return op_fail(PCS_E_INVAL, "rotary: pos or freq is null");
  a->pos = r->pos;
  a->freq = r->freq;
  a->axes = r->axes;
  a->pairs = static_cast<int32_t>(pairs);
  a->interleaved = (r->flags & PCS_ROT_INTERLEAVED) != 0;
  a->inverse = (r->flags & PCS_ROT_INVERSE) != 0;
  return PCS_OK;
}

void add_tensor(RotArgs* a, const pcs_heads& x, const pcs_heads* y, int role) {
  const int e = elem_bytes(x.dtype);
  RotSlot& t = a->t[a->n];
  t.src = static_cast<const uint8_t*>(x.data);
  t.src_token = x.token_stride * e;
  t.src_head = x.head_stride * e;
  t.dst = y ? static_cast<uint8_t*>(y->data) : nullptr;
  t.dst_token = y ? y->token_stride * e : 0;
  t.dst_head = y ? y->head_stride * e : 0;
  t.heads = x.heads + (a->n ? a->t[a->n - 1].heads : 0);
  t.role = role;
  a->n += 1;
}

// Whether heads are whole vectors.
bool vector_parts(const RotArgs& a, uint32_t dtype) { return a.head_dim % (16 / elem_bytes(dtype)) == 0; }

// Working memory of a call.  A stream's own is handed from call to call by events,
// which a graph that is run again and again cannot follow: a call that is being
// captured gets memory of its own, that no other graph or call uses, for the
// context's lifetime.  Its words are put to zero in the graph.
pcs_status working_memory(OpCall& call, uint64_t bytes, uint8_t** out, uint32_t** words) {
  cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
  cudaError_t e = cudaStreamIsCapturing(call.stream(), &capture);
  if (e != cudaSuccess) {
    cudaGetLastError();
    return op_fail(PCS_E_CUDA, "the stream's capture: %s", cudaGetErrorString(e));
  }
  if (capture == cudaStreamCaptureStatusNone) return call.scratch(bytes, out, words);
  constexpr uint64_t head = 4 * static_cast<uint64_t>(kOpWords);
  void* p = nullptr;
  cudaStreamCaptureMode mode = cudaStreamCaptureModeRelaxed;
  cudaThreadExchangeStreamCaptureMode(&mode);
  e = cudaMalloc(&p, head + bytes);
  cudaThreadExchangeStreamCaptureMode(&mode);
  if (e != cudaSuccess) {
    cudaGetLastError();
    return op_fail(PCS_E_NOMEM, "cannot allocate %llu bytes for a captured call", static_cast<unsigned long long>(head + bytes));
  }
  call.keep(p);
  e = cudaMemsetAsync(p, 0, head, call.stream());
  if (e != cudaSuccess) return op_fail(PCS_E_CUDA, "%s", cudaGetErrorString(e));
  *words = static_cast<uint32_t*>(p);
  *out = static_cast<uint8_t*>(p) + head;
  return PCS_OK;
}

uint64_t round_up_256(uint64_t x) { return (x + 255) / 256 * 256; }
// Working memory for codes that are turned into elements ahead of attention over them.
constexpr uint64_t kWidenMost = 1ull << 30;

// A tree's nodes, and tokens of which some are kept, all have to be in the cache.
pcs_status check_ring(const CacheDev& c, const BatchDev& b) {
  if (c.ring_rows && b.max_new > c.ring_rows)
    return op_fail(PCS_E_INVAL, "%d new tokens in a ring of %d slots", b.max_new, c.ring_rows);
  return PCS_OK;
}

pcs_status attend(const char* name, pcs_ctx* ctx, const pcs_kv_cache* cache, const pcs_kv_batch* batch,
                  const pcs_attend_params* params, bool tree, const int32_t* parent, const pcs_heads* q,
                  const pcs_heads* out, float* lse, void* stream) {
  return guarded([&]() -> pcs_status {
    OpCall call(ctx, name, stream);
    if (!ctx) return op_fail(PCS_E_INVAL, "ctx is null");
    AttendArgs a = {};
    pcs_status st = check_cache(cache, &a.cache);
    if (!st) st = check_batch(batch, &a.batch);
    if (st) return st;
    if (!params) return op_fail(PCS_E_INVAL, "params is null");
    if (params->flags || params->reserved)
      return op_fail(PCS_E_INVAL, "params: flags (0x%x) and reserved must be 0", params->flags);
    if (params->window < 0) return op_fail(PCS_E_INVAL, "negative window");
    if (!(params->scale >= 0.0f) || std::isinf(params->scale))
      return op_fail(PCS_E_INVAL, "scale must be finite and positive (0: 1 / sqrt(head_dim))");
    if (a.batch.tokens == 0) return PCS_OK;
    const bool codes = a.cache.codes != kElements16;
    if (codes && q && q->dtype != PCS_DT_F16 && q->dtype != PCS_DT_BF16)
      return op_fail(PCS_E_INVAL, "q: element type %u (F16 or BF16)", q->dtype);
    const uint32_t dtype = codes && q ? q->dtype : cache->dtype;
    st = check_heads(q, "q", dtype, cache->head_dim);
    if (!st) st = check_heads(out, "out", dtype, cache->head_dim);
    if (st) return st;
    if (q->heads % cache->heads != 0)
      return op_fail(PCS_E_INVAL, "%d query heads over %d heads of the cache", q->heads, cache->heads);
    if (out->heads != q->heads) return op_fail(PCS_E_INVAL, "q and out differ in heads");
    if (!vector_rows(*q) || !vector_rows(*out))
      return op_fail(PCS_E_ALIGN, "q, out and their strides must be multiples of 16 bytes");
    a.q = {static_cast<uint8_t*>(q->data), 2 * q->token_stride, 2 * q->head_stride};
    a.out = {static_cast<uint8_t*>(out->data), 2 * out->token_stride, 2 * out->head_stride};
    a.lse = lse;
    const double scale = params->scale > 0.0f ? params->scale : 1.0 / std::sqrt(double(cache->head_dim));
    a.scale_log2 = static_cast<float>(scale * 1.4426950408889634);
    a.window = params->window;
    a.group = q->heads / cache->heads;
    a.by_group.set(a.group);

    a.dtype = dtype;
    if (tree) {
      if (!parent) return op_fail(PCS_E_INVAL, "parent is null");
      if (a.batch.max_new > PCS_TREE_MAX)
        return op_fail(PCS_E_INVAL, "a tree of %d tokens (at most %d)", a.batch.max_new, PCS_TREE_MAX);
      if ((st = check_ring(a.cache, a.batch))) return st;
      a.parent = parent;
    }

    const int64_t rows = static_cast<int64_t>(a.batch.max_new) * a.group;
    // Few rows of a key head, bound by HBM, go to the token kernel: up to 16, and
    // up to 32 where sessions and heads alone would leave SMs without a block of
    // the other one.  (64 sessions of 500 to 4,000 tokens, 4 key heads of 128:
    // 8 rows 60 us, and 79 us by blocks; 16 rows 69 and 79; 32 rows 113 and 80.
    // One session of 100,000 tokens, 32 rows: 60 and 112 us.)
    const int64_t pairs = static_cast<int64_t>(a.batch.sessions) * cache->heads;
    if ((st = call.begin())) return st;
    a.err = call.errors();
    const bool few = rows <= 16 || (rows <= kTokenRowsMax && pairs < call.sm_count());
    // Tokens that the rows of a block see at most, as far as the host knows: a
    // hint for the split, which is right for any length.
    int64_t seen = cache->ring ? static_cast<int64_t>(cache->sinks) + cache->ring : a.cache.slots;
    if (batch->max_len) seen = std::min<int64_t>(seen, batch->max_len);
    const int64_t all_seen = a.window ? std::min<int64_t>(seen, static_cast<int64_t>(cache->sinks) + a.window + a.batch.max_new) : seen;
    const int64_t tokens = few || tree ? a.batch.max_new : std::min<int64_t>(a.batch.max_new, kBlockRows / a.group + 2);
    if (a.window) seen = std::min<int64_t>(seen, static_cast<int64_t>(cache->sinks) + a.window + tokens);
    if (few) {
      const int n_rows = static_cast<int>(rows);
      CodeMaps maps;
      if (codes) {
        a.box_rows = box_rows(*cache, kTokenTile8);
        a.box_heads = cache->heads % 4 == 0 ? 4 : cache->heads % 2 == 0 ? 2 : 1;
        if (a.box_rows && !encode_codes(*cache, a.cache, a.box_rows, a.box_heads, true, &maps)) a.box_rows = 0;
      }
      const bool boxes = codes && a.box_rows > 0;
      const int64_t resident =
          static_cast<int64_t>(call.sm_count()) *
          (codes ? attend_token8_blocks_per_sm(cache->head_dim, n_rows) : attend_token_blocks_per_sm(cache->head_dim, n_rows));
      const int64_t tiles = (seen + 15) / 16;
      // Parts for a wave of blocks, of two tiles a warp at least; and of several
      // sessions, whose lengths may differ, up to four waves of parts of eight
      // tiles a warp.  (48 sessions of 1 to 12,000 tokens: 217 us in one wave,
      // 196 us in four; one of 200,001 tokens, when measured: 163 and 196 us.)
      int64_t splits = std::min(resident / pairs, tiles / (2 * kTokenWarps));
      if (splits > kTokenOwnJoin) splits = std::max<int64_t>(kTokenOwnJoin, std::min(splits, tiles / (4 * kTokenWarps)));
      if (a.batch.sessions > 1)
        splits = std::max(splits, std::min(4 * resident / pairs, tiles / (8 * kTokenWarps)));
      // Blocks over codes that take several heads: a warp's result is a part of its head's.
      // Of several sessions whose lengths may differ by much (no window or ring makes them
      // alike), the longest come first and there are parts for two waves and a quarter.  (48
      // sessions of 1 to 12,000 tokens, 8 heads of 128: 131 us in one wave as they come, 106 us
      // so; 128 over windows of 2,048, 16 heads of 64: 97 us whole, 114 us in three parts.)
      int64_t each = 1;
      if (boxes) {
        each = kTokenWarps / a.box_heads;
        const int64_t blocks = pairs / a.box_heads, turns = (tiles + 2 * each - 1) / (2 * each);
        splits = std::min(resident / blocks, turns / 2);
        if (splits * each > kTokenOwnJoin) splits = std::max<int64_t>(kTokenOwnJoin / each, std::min(splits, turns / 4));
        const int64_t longest = batch->max_len ? batch->max_len : cache->ring ? INT32_MAX : a.cache.slots;
        a.ranked = a.batch.sessions > 1 && a.batch.sessions <= kRankMost && tiles >= 128 && seen >= longest;
        if (a.ranked) splits = std::max(splits, std::min((9 * resident / 4 + blocks / 2) / blocks, turns / 16));
      }
      splits = std::max<int64_t>(splits, 1);
      const int64_t parts = splits * each;
      // (Warps over codes join alone what is little: each of their parts waits for its writes.
      // 64 sessions in two parts of a row: 33 us, 39 us by a second launch; the 48 of above in
      // eleven of four rows 115 and 106 us.)
      const bool own = parts <= kTokenOwnJoin && pairs <= kOpWords && (!boxes || parts * rows <= 16);
      a.splits = static_cast<int32_t>(splits);
      if (pairs * parts > 0x7FFFFFFFll) return op_fail(PCS_E_INVAL, "too many sessions and heads in one call");
      if (parts > 1) {
        uint8_t* ws = nullptr;
        uint32_t* words = nullptr;
        st = working_memory(call, 4 * token_part_floats(n_rows, cache->head_dim) * pairs * parts, &ws, &words);
        if (st) return st;
        a.part = reinterpret_cast<float*>(ws);
        a.ticket = own ? words : nullptr;
      }
      call.before(kOpAttendToken);
      st = call.after(codes ? launch_attend_token8(a, n_rows, maps, call.stream())
                            : launch_attend_token(a, dtype, n_rows, false, call.stream()));
      if (!st && parts > 1 && !own) {
        a.splits = static_cast<int32_t>(parts);
        call.before(kOpAttendJoin);
        st = call.after(launch_attend_token(a, dtype, n_rows, true, call.stream()));
      }
      return st ? st : call.end();
    }
    const int64_t blocks = (rows + kBlockRows - 1) / kBlockRows;
    if (blocks > 0x7FFFFFFFll / pairs) return op_fail(PCS_E_INVAL, "too many sessions and heads in one call");
    const int64_t tiles = (seen + kBlockTile - 1) / kBlockTile;
    int64_t splits = std::max<int64_t>(1, std::min(call.sm_count() / (pairs * blocks), tiles / 4));
    a.splits = static_cast<int32_t>(splits);
    // (Parts are numbered by their blocks: a launch that joins them takes sessions as they come.)
    a.ranked = splits == 1 && a.batch.sessions > 1 && a.batch.sessions <= kRankMost;
    const uint64_t parts = splits > 1 ? round_up_256(4 * block_part_floats(cache->head_dim) * splits * pairs * blocks) : 0;
    // Codes that several blocks of rows go over are turned into elements once, ahead of
    // them, where that takes no more than kWidenMost and there is memory for it.  (Trees of 60
    // nodes over 16 sessions of 500 to 9,000 tokens, 8 heads of 128, two, three and four blocks
    // of rows: 188 to 192, 265 and 301 us, over the codes 178 to 186, 312 and 364 us; 8,000
    // tokens, the last 128, 192 and 512: 53, 52 and 76 us, over the codes 52, 57 and 107 us; two
    // blocks of a frame of heads of 64: 32 and 28 us.)
    pcs_kv_cache wide;
    const uint64_t pages = static_cast<uint64_t>(a.batch.sessions) * cache->table_pages;
    const uint64_t pool = codes ? pages * cache->page_rows * (2ull * cache->heads * cache->head_dim) : 0;
    bool widen = codes && blocks > 1 && 2 * pool <= kWidenMost;
    const uint64_t table = widen ? round_up_256(4 * pages) : 0;
    uint8_t* ws = nullptr;
    if (parts || widen) {
      uint32_t* words = nullptr;
      st = working_memory(call, parts + (widen ? table + 2 * pool : 0), &ws, &words);
      if (st == PCS_E_NOMEM && widen) {  // the kernel over codes needs none of it
        widen = false;
        st = parts ? working_memory(call, parts, &ws, &words) : PCS_OK;
      }
      if (st) return st;
      a.part = parts ? reinterpret_cast<float*>(ws) : nullptr;
    }
    if (widen) {
      const WidenTo to = {ws + parts + table, ws + parts + table + pool, reinterpret_cast<int32_t*>(ws + parts),
                          2ll * cache->heads * cache->head_dim};
      a.box_rows = box_rows(*cache, kBlockTile);
      call.before(kOpWiden);
      if ((st = call.after(launch_widen(a, to, all_seen, call.stream())))) return st;
      wide = *cache;
      wide.k = to.k, wide.v = to.v, wide.table = to.table, wide.v_table = nullptr;
      wide.table_stride = cache->table_pages;
      wide.head_stride = cache->head_dim;
      wide.row_stride = static_cast<int64_t>(cache->heads) * cache->head_dim;
      wide.page_stride = wide.row_stride * cache->page_rows;
      wide.n_pages = static_cast<int32_t>(pages);
      wide.dtype = dtype;
      cache = &wide;
      if ((st = check_cache(cache, &a.cache))) return st;
    }
    a.box_rows = box_rows(*cache, kBlockTile);
    if (codes && !widen) {
      CodeMaps maps;
      if (a.box_rows && !encode_codes(*cache, a.cache, a.box_rows, 1, false, &maps)) a.box_rows = 0;
      call.before(kOpAttendBlock);
      const auto launch = a.cache.codes == kCodesE4M3 ? launch_attend_block_e4m3 : launch_attend_block_i8;
      st = call.after(launch(a, dtype, static_cast<int>(blocks), maps, call.stream()));
    } else {
      TensorMaps maps = {};
      if (a.box_rows &&
          !(encode_pool(*cache, cache->k, a.box_rows, maps.k) && encode_pool(*cache, cache->v, a.box_rows, maps.v)))
        a.box_rows = 0;
      call.before(kOpAttendBlock);
      st = call.after(launch_attend_block(a, dtype, static_cast<int>(blocks), maps, call.stream()));
    }
    if (st) return st;
    if (splits > 1) {
      call.before(kOpAttendJoin);
      if ((st = call.after(launch_attend_join(a, dtype, static_cast<int>(blocks), call.stream())))) return st;
    }
    return call.end();
  });
}

}  // namespace

extern "C" {

pcs_status pcs_rotate(pcs_ctx* ctx, const pcs_rotary* rotary, const pcs_heads* x, const pcs_heads* y,
                      int32_t n, int64_t tokens, void* stream) {
  return guarded([&]() -> pcs_status {
    OpCall call(ctx, "pcs_rotate", stream);
    if (!ctx) return op_fail(PCS_E_INVAL, "ctx is null");
    if (!rotary) return op_fail(PCS_E_INVAL, "rotary is null");
    if (n < 0 || n > kRotTensors) return op_fail(PCS_E_INVAL, "%d tensors (at most %d)", n, kRotTensors);
    if (tokens < 0 || tokens > 0x7FFFFFFFll) return op_fail(PCS_E_INVAL, "bad number of tokens");
    if (n == 0 || tokens == 0) return PCS_OK;
    if (!x || !y) return op_fail(PCS_E_INVAL, "x or y is null");
    const uint32_t dtype = x[0].dtype;
    const int32_t dim = x[0].head_dim;
    if (!elem_bytes(dtype)) return op_fail(PCS_E_INVAL, "element type %u (F16, BF16 or F32)", dtype);
    if (dim < 1 || dim > 256) return op_fail(PCS_E_INVAL, "heads of %d elements (1 to 256)", dim);
    RotArgs a = {};
    a.head_dim = dim;
    a.tokens = tokens;
    pcs_status st = check_rotary(rotary, dim, &a);
    bool vec = vector_parts(a, dtype);
    for (int i = 0; i < n && !st; ++i) {
      st = check_heads(x + i, "x", dtype, dim);
      if (!st) st = check_heads(y + i, "y", dtype, dim);
      if (!st && x[i].heads != y[i].heads) st = op_fail(PCS_E_INVAL, "x and y differ in heads");
      if (st) break;
      vec = vec && vector_rows(x[i]) && vector_rows(y[i]);
      add_tensor(&a, x[i], y + i, 0);
    }
    if (st) return st;
    a.plain = n;
    if ((st = call.begin())) return st;
    a.err = call.errors();
    call.before(kOpRotate);
    return call.after(launch_rotate(a, dtype, false, vec, call.sm_count(), call.stream()));
  });
}

pcs_status pcs_kv_append(pcs_ctx* ctx, const pcs_kv_cache* cache, const pcs_kv_batch* batch,
                         const pcs_rotary* rotary, const pcs_heads* k, const pcs_heads* v,
                         const pcs_heads* q, const pcs_heads* q_out, void* stream) {
  return guarded([&]() -> pcs_status {
    OpCall call(ctx, "pcs_kv_append", stream);
    if (!ctx) return op_fail(PCS_E_INVAL, "ctx is null");
    RotArgs a = {};
    pcs_status st = check_cache(cache, &a.cache);
    if (!st) st = check_batch(batch, &a.batch);
    if (st) return st;
    if (a.batch.tokens == 0) return PCS_OK;
    // (A cache in 8 bits takes either 16-bit type.)
    const bool codes = a.cache.codes != kElements16;
    if (codes && k && k->dtype != PCS_DT_F16 && k->dtype != PCS_DT_BF16)
      return op_fail(PCS_E_INVAL, "k: element type %u (F16 or BF16)", k->dtype);
    const uint32_t dtype = codes && k ? k->dtype : cache->dtype;
    a.head_dim = cache->head_dim;
    a.tokens = a.batch.tokens;
    a.axes = 1;
    if (rotary) st = check_rotary(rotary, a.head_dim, &a);
    if (!st) st = check_heads(k, "k", dtype, a.head_dim);
    if (!st) st = check_heads(v, "v", dtype, a.head_dim);
    if (st) return st;
    if (k->heads != cache->heads || v->heads != cache->heads)
      return op_fail(PCS_E_INVAL, "k and v must have the cache's %d heads", cache->heads);
    if (!q != !q_out) return op_fail(PCS_E_INVAL, "q and q_out go together");
    bool vec = vector_parts(a, dtype) && vector_rows(*k) && vector_rows(*v);
    if (q) {
      st = check_heads(q, "q", dtype, a.head_dim);
      if (!st) st = check_heads(q_out, "q_out", dtype, a.head_dim);
      if (st) return st;
      if (q->heads != q_out->heads) return op_fail(PCS_E_INVAL, "q and q_out differ in heads");
      vec = vec && vector_rows(*q) && vector_rows(*q_out);
      add_tensor(&a, *q, q_out, 0);
    }
    add_tensor(&a, *k, nullptr, 1);
    a.plain = a.n;
    add_tensor(&a, *v, nullptr, 2);
    if ((st = call.begin())) return st;
    a.err = call.errors();
    if (codes) {
      call.before(kOpStore);
      return call.after(launch_store(a, dtype, vec, call.sm_count(), call.stream()));
    }
    call.before(kOpAppend);
    return call.after(launch_rotate(a, dtype, true, vec, call.sm_count(), call.stream()));
  });
}

pcs_status pcs_attend(pcs_ctx* ctx, const pcs_kv_cache* cache, const pcs_kv_batch* batch,
                      const pcs_attend_params* params, const pcs_heads* q, const pcs_heads* out,
                      float* lse, void* stream) {
  return attend("pcs_attend", ctx, cache, batch, params, false, nullptr, q, out, lse, stream);
}

pcs_status pcs_attend_tree(pcs_ctx* ctx, const pcs_kv_cache* cache, const pcs_kv_batch* batch,
                           const pcs_attend_params* params, const int32_t* parent, const pcs_heads* q,
                           const pcs_heads* out, float* lse, void* stream) {
  return attend("pcs_attend_tree", ctx, cache, batch, params, true, parent, q, out, lse, stream);
}

pcs_status pcs_kv_keep(pcs_ctx* ctx, const pcs_kv_cache* cache, const pcs_kv_batch* batch, const int32_t* index,
                       int64_t index_stride, int32_t most, const int32_t* count, int32_t* lens_out, void* stream) {
  return guarded([&]() -> pcs_status {
    OpCall call(ctx, "pcs_kv_keep", stream);
    if (!ctx) return op_fail(PCS_E_INVAL, "ctx is null");
    KeepArgs a = {};
    pcs_status st = check_cache(cache, &a.cache);
    if (!st) st = check_batch(batch, &a.batch);
    if (st) return st;
    if (a.batch.sessions == 0) return PCS_OK;
    if (!index || !count) return op_fail(PCS_E_INVAL, "index or count is null");
    if (most < 0 || index_stride < most)
      return op_fail(PCS_E_INVAL, "index: rows of %d elements, %lld apart", most, static_cast<long long>(index_stride));
    if ((st = check_ring(a.cache, a.batch))) return st;
    a.index = index;
    a.index_stride = index_stride;
    a.count = count;
    a.lens_out = lens_out;
    a.most = most;
    if ((st = call.begin())) return st;
    a.err = call.errors();
    call.before(kOpKeep);
    return call.after(launch_keep(a, call.stream()));
  });
}

pcs_status pcs_kv_read(pcs_ctx* ctx, const pcs_kv_cache* cache, const pcs_kv_batch* batch, const pcs_heads* k,
                       const pcs_heads* v, void* stream) {
  return guarded([&]() -> pcs_status {
    OpCall call(ctx, "pcs_kv_read", stream);
    if (!ctx) return op_fail(PCS_E_INVAL, "ctx is null");
    ReadArgs a = {};
    pcs_status st = check_cache(cache, &a.cache);
    if (!st) st = check_batch(batch, &a.batch);
    if (st) return st;
    if (a.batch.tokens == 0 || (!k && !v)) return PCS_OK;
    a.dtype = k ? k->dtype : v->dtype;
    const bool fits = a.cache.codes == kElements16 ? a.dtype == cache->dtype : elem_bytes(a.dtype) != 0;
    if (!fits) return op_fail(PCS_E_INVAL, "k, v: element type %u of a cache of type %u", a.dtype, cache->dtype);
    const pcs_heads* out[2] = {k, v};
    for (int i = 0; i < 2 && !st; ++i) {
      const char* what = i ? "v" : "k";
      if (!out[i]) continue;
      st = check_heads(out[i], what, a.dtype, cache->head_dim);
      if (st) break;
      if (out[i]->heads != cache->heads) return op_fail(PCS_E_INVAL, "%s must have the cache's %d heads", what, cache->heads);
      if (!vector_rows(*out[i])) return op_fail(PCS_E_ALIGN, "%s and its strides must be multiples of 16 bytes", what);
      const int e = elem_bytes(a.dtype);
      a.out[i] = {static_cast<uint8_t*>(out[i]->data), e * out[i]->token_stride, e * out[i]->head_stride};
    }
    if (st) return st;
    if ((st = call.begin())) return st;
    a.err = call.errors();
    call.before(kOpRead);
    return call.after(launch_read(a, call.sm_count(), call.stream()));
  });
}

}  // extern "C"
