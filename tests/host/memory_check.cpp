// Checks of what attention does where working memory cannot be had, without a GPU: its host
// side (csrc/pcs_attend.cpp) is compiled into this program over a stand-in for a call on a
// context, whose memory ends at a limit, and for the kernels' launchers, which write down
// what would have been launched.  Prints "ok" or the first failure.
#include <cstdarg>
#include <cstdio>
#include <string>
#include <vector>

#include "pcs_attend.cpp"

static std::vector<std::string> g_launched;
static uint64_t g_limit = ~0ull, g_given = 0;
static bool g_capturing = false;
static pcs_status g_scratch_status = PCS_E_NOMEM;  // of a call beyond the limit
static const void* g_part = nullptr;
alignas(256) static uint8_t g_memory[1 << 20];

namespace pcs {

pcs_status op_fail(pcs_status s, const char*, ...) { return s; }
OpCall::OpCall(pcs_ctx* c, const char*, void*) : c_(c) {}
OpCall::~OpCall() {}
pcs_status OpCall::begin() { return PCS_OK; }
pcs_status OpCall::scratch(uint64_t bytes, uint8_t** out, uint32_t** words) {
  static uint32_t w[kOpWords];
  if (bytes > g_limit) return g_scratch_status;
  *out = g_memory;
  *words = w;
  g_given = bytes;
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
static cudaError_t block(const char* what, const AttendArgs& a) {
  g_part = a.part;
  if ((a.splits > 1) != (a.part != nullptr)) return launched("parts without memory");
  return launched(what);
}
cudaError_t launch_rotate(const RotArgs&, uint32_t, bool, bool, int, cudaStream_t) { return launched("rotate"); }
cudaError_t launch_store(const RotArgs&, uint32_t, bool, int, cudaStream_t) { return launched("store"); }
cudaError_t launch_read(const ReadArgs&, int, cudaStream_t) { return launched("read"); }
cudaError_t launch_keep(const KeepArgs&, cudaStream_t) { return launched("keep"); }
cudaError_t launch_widen(const AttendArgs&, const WidenTo&, int64_t, cudaStream_t) { return launched("widen"); }
cudaError_t launch_attend_token(const AttendArgs&, uint32_t, int, bool, cudaStream_t) { return launched("token"); }
cudaError_t launch_attend_token8(const AttendArgs&, int, const CodeMaps&, cudaStream_t) { return launched("token8"); }
int attend_token_blocks_per_sm(int, int) { return 2; }
int attend_token8_blocks_per_sm(int, int) { return 3; }
cudaError_t launch_attend_block(const AttendArgs&, uint32_t, int, const TensorMaps&, cudaStream_t) { return launched("block"); }
cudaError_t launch_attend_block_e4m3(const AttendArgs& a, uint32_t, int, const CodeMaps&, cudaStream_t) {
  return a.cache.codes == kCodesE4M3 ? block("block8", a) : launched("wrong codes");
}
cudaError_t launch_attend_block_i8(const AttendArgs& a, uint32_t, int, const CodeMaps&, cudaStream_t) {
  return a.cache.codes == kCodesI8 ? block("block8", a) : launched("wrong codes");
}
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
  *s = g_capturing ? cudaStreamCaptureStatusActive : cudaStreamCaptureStatusNone;
  return cudaSuccess;
}
cudaError_t cudaThreadExchangeStreamCaptureMode(cudaStreamCaptureMode*) { return cudaSuccess; }
cudaError_t cudaMalloc(void** p, size_t bytes) {
  if (bytes > g_limit) return cudaErrorMemoryAllocation;
  *p = g_memory;
  g_given = bytes;
  return cudaSuccess;
}
cudaError_t cudaMemsetAsync(void*, int, size_t, cudaStream_t) { return cudaSuccess; }
}

int main() {
  bool bad = false;
  pcs_ctx* const ctx = reinterpret_cast<pcs_ctx*>(uintptr_t{64});
  auto dev = [](uint64_t off = 0) { return reinterpret_cast<void*>((uintptr_t{1} << 41) + off); };
  const int32_t* ints = static_cast<const int32_t*>(dev());
  // 2 heads of 64 codes, rows of 160 bytes, pages of 16, 320 slots a session.
  pcs_kv_cache cache = {dev(), dev(1 << 20), ints, nullptr, 20, 16 * 160, 160, 64, 20, 20, 16, 2, 64, 0, 0, PCS_DT_E4M3};
  const pcs_attend_params par = {0.0f, 0, 0, 0};
  const pcs_heads q = {dev(), 256, 64, 4, 64, PCS_DT_BF16, 0};
  auto runs = [&](int line, const pcs_kv_cache& c, int64_t tokens, bool tree, pcs_status status, std::vector<std::string> names) {
    const pcs_kv_batch b = {ints, nullptr, tokens, 1, 0, 0, 0};
    g_part = nullptr;
    const pcs_status st = tree ? pcs_attend_tree(ctx, &c, &b, &par, ints, &q, &q, nullptr, nullptr)
                               : pcs_attend(ctx, &c, &b, &par, &q, &q, nullptr, nullptr);
    if (!bad && (st != status || g_launched != names)) {
      bad = true;
      std::printf("line %d: status %d, %zu launches, first %s\n", line, st, g_launched.size(), g_launched.empty() ? "none" : g_launched[0].c_str());
    }
    g_launched.clear();
  };
  for (int i = 0; i < 4; ++i) {
    g_capturing = i & 1;
    cache.dtype = i & 2 ? PCS_DT_I8 : PCS_DT_E4M3;
    // Memory for widened codes: there, not there.  (Two key heads, 300 tokens of two rows: three
    // blocks.)
    g_limit = ~0ull;
    runs(__LINE__, cache, 300, false, PCS_OK, {"widen", "block"});
    const uint64_t whole = g_given;
    g_limit = whole - 1;
    runs(__LINE__, cache, 300, false, PCS_OK, {"block8"});
    g_limit = 0;
    runs(__LINE__, cache, 300, false, PCS_OK, {"block8"});
    // Parts as well, of 2,048 slots: those have to be had.
    pcs_kv_cache longer = cache;
    longer.table_pages = longer.table_stride = 128;
    g_limit = ~0ull;
    runs(__LINE__, longer, 300, false, PCS_OK, {"widen", "block", "join"});
    g_limit = g_given - 1;
    runs(__LINE__, longer, 300, false, PCS_OK, {"block8", "join"});
    const uint64_t parts = g_given;
    g_limit = parts - 1;
    runs(__LINE__, longer, 300, false, PCS_E_NOMEM, {});
    g_limit = parts;
    runs(__LINE__, longer, 300, false, PCS_OK, {"block8", "join"});
    // Other errors are no lack of memory.
    g_scratch_status = PCS_E_CUDA;
    g_limit = 0;
    if (!g_capturing) runs(__LINE__, longer, 300, false, PCS_E_CUDA, {});
    g_scratch_status = PCS_E_NOMEM;
    // One block of rows is never widened.
    runs(__LINE__, cache, 60, true, PCS_OK, {"block8"});
  }
  if (bad) return 1;
  std::puts("ok");
}
