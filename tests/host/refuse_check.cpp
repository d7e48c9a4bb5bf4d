// Checks of what the operators over a paged cache refuse, without a GPU: their host
// side (csrc/pcs_attend.cpp) is compiled into this program over a stand-in for a call on
// a context and for the kernels' launchers, which count what would have been launched.
// Prints "ok" or the first failure.
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <string>
#include <vector>

#include "pcs_attend.cpp"

static std::vector<std::string> g_launched;
static std::string g_message;

namespace pcs {

pcs_status op_fail(pcs_status s, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  std::vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  g_message = buf;
  return s;
}
OpCall::OpCall(pcs_ctx* c, const char*, void*) : c_(c) {}
OpCall::~OpCall() {}
pcs_status OpCall::begin() { return PCS_OK; }
pcs_status OpCall::scratch(uint64_t bytes, uint8_t** out, uint32_t** words) {
  static std::vector<uint32_t> w(kOpWords);
  *out = reinterpret_cast<uint8_t*>(uintptr_t{1} << 40);  // (never looked at)
  *words = w.data();
  g_launched.push_back("scratch of " + std::to_string(bytes));
  return PCS_OK;
}
void OpCall::keep(void*) {}
void OpCall::before(OpKernel) {}
pcs_status OpCall::after(cudaError_t e) { return e == cudaSuccess ? PCS_OK : PCS_E_CUDA; }
pcs_status OpCall::end() { return PCS_OK; }
uint32_t* OpCall::errors() const { return nullptr; }
int OpCall::sm_count() const { return 152; }

static cudaError_t launched(const char* what) {
  g_launched.push_back(what);
  return cudaSuccess;
}
cudaError_t launch_rotate(const RotArgs&, uint32_t, bool, bool, int, cudaStream_t) { return launched("rotate"); }
cudaError_t launch_store(const RotArgs&, uint32_t, bool, int, cudaStream_t) { return launched("store"); }
cudaError_t launch_read(const ReadArgs&, int, cudaStream_t) { return launched("read"); }
cudaError_t launch_keep(const KeepArgs&, cudaStream_t) { return launched("keep"); }
cudaError_t launch_widen(const AttendArgs&, const WidenTo&, int64_t, cudaStream_t) { return launched("widen"); }
cudaError_t launch_attend_token(const AttendArgs& a, uint32_t, int, bool join, cudaStream_t) {
  return launched(join ? "token join" : a.parent ? "token tree" : "token");
}
cudaError_t launch_attend_token8(const AttendArgs& a, int, const CodeMaps&, cudaStream_t) { return launched(a.parent ? "token8 tree" : "token8"); }
int attend_token_blocks_per_sm(int, int) { return 2; }
int attend_token8_blocks_per_sm(int, int) { return 3; }
cudaError_t launch_attend_block(const AttendArgs& a, uint32_t, int, const TensorMaps&, cudaStream_t) { return launched(a.parent ? "block tree" : "block"); }
cudaError_t launch_attend_block_e4m3(const AttendArgs& a, uint32_t, int, const CodeMaps&, cudaStream_t) { return launched(a.parent ? "block8 tree" : "block8"); }
cudaError_t launch_attend_block_i8(const AttendArgs& a, uint32_t, int, const CodeMaps&, cudaStream_t) { return launched(a.parent ? "block8 tree" : "block8"); }
cudaError_t launch_attend_join(const AttendArgs&, uint32_t, int, cudaStream_t) { return launched("join"); }

}  // namespace pcs

extern "C" {
cudaError_t cudaGetDriverEntryPointByVersion(const char*, void** f, unsigned, unsigned long long, cudaDriverEntryPointQueryResult*) {
  *f = nullptr;
  return cudaErrorNotSupported;
}
cudaError_t cudaGetLastError() { return cudaSuccess; }
const char* cudaGetErrorString(cudaError_t) { return "stand-in"; }
cudaError_t cudaStreamIsCapturing(cudaStream_t, cudaStreamCaptureStatus* s) {
  *s = cudaStreamCaptureStatusNone;
  return cudaSuccess;
}
cudaError_t cudaThreadExchangeStreamCaptureMode(cudaStreamCaptureMode*) { return cudaSuccess; }
cudaError_t cudaMalloc(void**, size_t) { return cudaErrorMemoryAllocation; }
cudaError_t cudaMemsetAsync(void*, int, size_t, cudaStream_t) { return cudaSuccess; }
}

static int g_line = 0;
static bool g_bad = false;
static void want(int line, pcs_status got, pcs_status expected, size_t launches) {
  if (!g_bad && (got != expected || g_launched.size() != launches)) {
    g_bad = true;
    g_line = line;
    std::printf("line %d: status %d, expected %d, %zu launched (%s)\n", line, got, expected, g_launched.size(), g_message.c_str());
  }
  g_launched.clear();
}
#define REFUSED(status, call) want(__LINE__, call, status, 0)
#define DONE(n, call) want(__LINE__, call, PCS_OK, n)

int main() {
  pcs_ctx* const ctx = reinterpret_cast<pcs_ctx*>(uintptr_t{64});
  auto dev = [](uint64_t off = 0) { return reinterpret_cast<void*>((uintptr_t{1} << 41) + off); };
  const int32_t* ints = static_cast<const int32_t*>(dev());
  // 2 heads of 64 codes, rows of 160 bytes, pages of 16.
  const pcs_kv_cache cache = {dev(), dev(1 << 20), ints, nullptr, 8, 16 * 160, 160, 64, 20, 8, 16, 2, 64, 0, 0, PCS_DT_E4M3};
  const pcs_kv_batch batch = {ints, nullptr, 6, 2, 0, 0, 0};
  const pcs_attend_params par = {0.0f, 0, 0, 0};
  const pcs_heads k = {dev(), 128, 64, 2, 64, PCS_DT_BF16, 0}, q = {dev(), 256, 64, 4, 64, PCS_DT_BF16, 0};
  int32_t* lens = static_cast<int32_t*>(dev());

  DONE(1, pcs_kv_append(ctx, &cache, &batch, nullptr, &k, &k, &q, &q, nullptr));
  DONE(1, pcs_kv_read(ctx, &cache, &batch, &k, &k, nullptr));
  DONE(1, pcs_kv_keep(ctx, &cache, &batch, ints, 3, 3, ints, lens, nullptr));
  DONE(1, pcs_attend(ctx, &cache, &batch, &par, &q, &q, nullptr, nullptr));
  DONE(1, pcs_attend_tree(ctx, &cache, &batch, &par, ints, &q, &q, nullptr, nullptr));

  // Caches in 8 bits.
  struct {
    pcs_status status;
    void (*change)(pcs_kv_cache*);
  } caches[] = {
      {PCS_E_INVAL, [](pcs_kv_cache* c) { c->head_dim = 8; }},      {PCS_E_INVAL, [](pcs_kv_cache* c) { c->head_dim = 72; }},
      {PCS_E_INVAL, [](pcs_kv_cache* c) { c->head_dim = 144; }},    {PCS_E_ALIGN, [](pcs_kv_cache* c) { c->row_stride = 168; }},
      {PCS_E_INVAL, [](pcs_kv_cache* c) { c->row_stride = 128; }},  {PCS_E_INVAL, [](pcs_kv_cache* c) { c->head_stride = 48; }},
      {PCS_E_ALIGN, [](pcs_kv_cache* c) { c->head_stride = 72; }},  {PCS_E_ALIGN, [](pcs_kv_cache* c) { c->page_stride += 8; }},
      {PCS_E_INVAL, [](pcs_kv_cache* c) { c->head_stride = 80; }},  {PCS_E_INVAL, [](pcs_kv_cache* c) { c->dtype = PCS_DT_U8; }},
      {PCS_E_INVAL, [](pcs_kv_cache* c) { c->dtype = 10; }},        {PCS_E_INVAL, [](pcs_kv_cache* c) { c->head_stride = 1 << 15; }},
      {PCS_E_ALIGN, [](pcs_kv_cache* c) { c->k = static_cast<uint8_t*>(c->k) + 8; }},
      {PCS_E_INVAL, [](pcs_kv_cache* c) { c->v = nullptr; }},
      {PCS_E_INVAL, [](pcs_kv_cache* c) { c->page_stride = 1ll << 40, c->n_pages = 1 << 20; }},
  };
  for (const auto& x : caches) {
    pcs_kv_cache c = cache;
    x.change(&c);
    REFUSED(x.status, pcs_kv_append(ctx, &c, &batch, nullptr, &k, &k, nullptr, nullptr, nullptr));
    REFUSED(x.status, pcs_kv_read(ctx, &c, &batch, &k, &k, nullptr));
    REFUSED(x.status, pcs_kv_keep(ctx, &c, &batch, ints, 3, 3, ints, lens, nullptr));
    REFUSED(x.status, pcs_attend(ctx, &c, &batch, &par, &q, &q, nullptr, nullptr));
    REFUSED(x.status, pcs_attend_tree(ctx, &c, &batch, &par, ints, &q, &q, nullptr, nullptr));
  }
  {
    pcs_kv_cache c = cache;  // heads apart, scales behind them
    c.head_stride = 80, c.row_stride = 176, c.page_stride = 16 * 176;
    DONE(1, pcs_attend(ctx, &c, &batch, &par, &q, &q, nullptr, nullptr));
  }

  // Types of queries, keys and values over 8 bits: either of 16, the same in a call.
  pcs_heads k32 = k, k16 = k, q16 = q, q32 = q;
  k32.dtype = q32.dtype = PCS_DT_F32;
  k16.dtype = q16.dtype = PCS_DT_F16;
  DONE(1, pcs_kv_append(ctx, &cache, &batch, nullptr, &k16, &k16, &q16, &q16, nullptr));
  DONE(1, pcs_attend(ctx, &cache, &batch, &par, &q16, &q16, nullptr, nullptr));
  REFUSED(PCS_E_INVAL, pcs_kv_append(ctx, &cache, &batch, nullptr, &k16, &k, nullptr, nullptr, nullptr));
  REFUSED(PCS_E_INVAL, pcs_kv_append(ctx, &cache, &batch, nullptr, &k, &k, &q16, &q16, nullptr));
  REFUSED(PCS_E_INVAL, pcs_kv_append(ctx, &cache, &batch, nullptr, &k32, &k32, nullptr, nullptr, nullptr));
  REFUSED(PCS_E_INVAL, pcs_kv_append(ctx, &cache, &batch, nullptr, nullptr, &k, nullptr, nullptr, nullptr));
  REFUSED(PCS_E_INVAL, pcs_attend(ctx, &cache, &batch, &par, &q, &q16, nullptr, nullptr));
  REFUSED(PCS_E_INVAL, pcs_attend(ctx, &cache, &batch, &par, &q32, &q32, nullptr, nullptr));
  REFUSED(PCS_E_INVAL, pcs_attend(ctx, &cache, &batch, &par, nullptr, &q, nullptr, nullptr));

  // Reads.
  DONE(1, pcs_kv_read(ctx, &cache, &batch, &k32, &k32, nullptr));
  DONE(1, pcs_kv_read(ctx, &cache, &batch, nullptr, &k16, nullptr));
  DONE(0, pcs_kv_read(ctx, &cache, &batch, nullptr, nullptr, nullptr));
  REFUSED(PCS_E_INVAL, pcs_kv_read(ctx, &cache, &batch, &k, &k16, nullptr));
  REFUSED(PCS_E_INVAL, pcs_kv_read(ctx, &cache, &batch, &q, nullptr, nullptr));
  REFUSED(PCS_E_INVAL, pcs_kv_read(nullptr, &cache, &batch, &k, &k, nullptr));
  REFUSED(PCS_E_INVAL, pcs_kv_read(ctx, nullptr, &batch, &k, &k, nullptr));
  REFUSED(PCS_E_INVAL, pcs_kv_read(ctx, &cache, nullptr, &k, &k, nullptr));
  pcs_heads bad = k;
  bad.token_stride = 132;
  REFUSED(PCS_E_ALIGN, pcs_kv_read(ctx, &cache, &batch, &bad, nullptr, nullptr));
  bad = k;
  bad.data = dev(2);
  REFUSED(PCS_E_ALIGN, pcs_kv_read(ctx, &cache, &batch, &k, &bad, nullptr));
  bad = k;
  bad.reserved = 1;
  REFUSED(PCS_E_INVAL, pcs_kv_read(ctx, &cache, &batch, &k, &bad, nullptr));
  pcs_heads kw = k;
  kw.dtype = PCS_DT_U8;
  REFUSED(PCS_E_INVAL, pcs_kv_read(ctx, &cache, &batch, &kw, nullptr, nullptr));
  const pcs_kv_cache wide = {dev(), dev(1 << 20), ints, nullptr, 8, 16 * 128, 128, 64, 20, 8, 16, 2, 64, 0, 0, PCS_DT_BF16};
  DONE(1, pcs_kv_read(ctx, &wide, &batch, &k, &k, nullptr));
  REFUSED(PCS_E_INVAL, pcs_kv_read(ctx, &wide, &batch, &k16, &k16, nullptr));
  REFUSED(PCS_E_INVAL, pcs_kv_read(ctx, &wide, &batch, &k32, &k32, nullptr));

  // Trees.
  REFUSED(PCS_E_INVAL, pcs_attend_tree(ctx, &cache, &batch, &par, nullptr, &q, &q, nullptr, nullptr));
  pcs_kv_batch many = {ints, nullptr, 130, 2, 0, 0, 0};
  REFUSED(PCS_E_INVAL, pcs_attend_tree(ctx, &cache, &many, &par, ints, &q, &q, nullptr, nullptr));
  many = {ints, ints, 130, 2, 65, 0, 0};
  REFUSED(PCS_E_INVAL, pcs_attend_tree(ctx, &wide, &many, &par, ints, &q, &q, nullptr, nullptr));
  many = {ints, ints, 70, 2, 64, 0, 0};
  DONE(1, pcs_attend_tree(ctx, &wide, &many, &par, ints, &q, &q, nullptr, nullptr));
  pcs_attend_params odd = par;
  odd.flags = 1;
  REFUSED(PCS_E_INVAL, pcs_attend_tree(ctx, &cache, &batch, &odd, ints, &q, &q, nullptr, nullptr));
  odd = par;
  odd.window = -1;
  REFUSED(PCS_E_INVAL, pcs_attend_tree(ctx, &cache, &batch, &odd, ints, &q, &q, nullptr, nullptr));
  REFUSED(PCS_E_INVAL, pcs_attend_tree(nullptr, &cache, &batch, &par, ints, &q, &q, nullptr, nullptr));
  pcs_kv_cache ring = cache;
  ring.ring = 2;
  REFUSED(PCS_E_INVAL, pcs_attend_tree(ctx, &ring, &batch, &par, ints, &q, &q, nullptr, nullptr));
  ring.ring = 3;
  DONE(1, pcs_attend_tree(ctx, &ring, &batch, &par, ints, &q, &q, nullptr, nullptr));
  pcs_kv_batch none = {ints, nullptr, 0, 2, 0, 0, 0};
  DONE(0, pcs_attend_tree(ctx, &ring, &none, &par, nullptr, nullptr, nullptr, nullptr, nullptr));

  // Keep.
  ring.ring = 2;
  REFUSED(PCS_E_INVAL, pcs_kv_keep(ctx, &ring, &batch, ints, 3, 3, ints, lens, nullptr));
  REFUSED(PCS_E_INVAL, pcs_kv_keep(ctx, &cache, &batch, nullptr, 3, 3, ints, lens, nullptr));
  REFUSED(PCS_E_INVAL, pcs_kv_keep(ctx, &cache, &batch, ints, 3, 3, nullptr, lens, nullptr));
  REFUSED(PCS_E_INVAL, pcs_kv_keep(ctx, &cache, &batch, ints, 2, 3, ints, lens, nullptr));
  REFUSED(PCS_E_INVAL, pcs_kv_keep(ctx, &cache, &batch, ints, 3, -1, ints, lens, nullptr));
  REFUSED(PCS_E_INVAL, pcs_kv_keep(nullptr, &cache, &batch, ints, 3, 3, ints, lens, nullptr));
  DONE(1, pcs_kv_keep(ctx, &cache, &batch, ints, 3, 3, ints, nullptr, nullptr));
  const pcs_kv_batch nobody = {nullptr, nullptr, 0, 0, 0, 0, 0};
  DONE(0, pcs_kv_keep(ctx, &cache, &nobody, nullptr, 0, 0, nullptr, nullptr, nullptr));

  // Which kernels: few rows, one block of them, several (codes widened ahead), and several
  // over tables too large for that.
  auto runs = [&](const pcs_kv_cache& c, int64_t tokens, std::vector<std::string> names, int line) {
    const pcs_kv_batch b = {ints, nullptr, tokens, 2, 0, 0, 0};
    const pcs_status st = pcs_attend(ctx, &c, &b, &par, &q, &q, nullptr, nullptr);
    std::vector<std::string> got;
    for (const std::string& s : g_launched)
      if (s.compare(0, 7, "scratch")) got.push_back(s);
    if (!g_bad && (st || got != names)) {
      g_bad = true;
      std::printf("line %d: status %d, %zu launches, first %s\n", line, st, got.size(), got.empty() ? "none" : got[0].c_str());
    }
    g_launched.clear();
  };
  runs(cache, 2, {"token8"}, __LINE__);
  runs(cache, 100, {"block8"}, __LINE__);
  runs(cache, 400, {"widen", "block"}, __LINE__);
  pcs_kv_cache vast = cache;
  vast.table_pages = vast.table_stride = 1 << 20;
  runs(vast, 400, {"block8", "join"}, __LINE__);
  if (g_bad) return 1;
  std::puts("ok");
}
