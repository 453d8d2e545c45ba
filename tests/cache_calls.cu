// Host check of what bdkv_attention queues in the library's own workspace: the entry points (cache_api.cu) linked with
// a record in the place of the CUDA runtime calls they make and of the kernels' launches. Each argument is a stream
// handle and a bound on the lengths, "handle:max_kv_len"; a line of output for each call:
//   <status> <what was queued, in order: free malloc wait(stream) parts(stream) join(stream) record(stream)>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <string>

#include "cache/cache_api.cu"

namespace {

std::string g_log;
void* g_workspace;

void note(const char* what) { g_log += std::string(" ") + what; }
void note(const char* what, cudaStream_t st) {
  g_log += std::string(" ") + what + "(" + std::to_string(reinterpret_cast<uintptr_t>(st)) + ")";
}

}  // namespace

namespace bdkv {
cudaError_t launch_tables(const bdkv_tables_args&, int, cudaStream_t) { return cudaSuccess; }
cudaError_t launch_write(const bdkv_cache&, const bdkv_rows&, const bdkv_rows&, const int64_t*, int64_t, int,
                         cudaStream_t) {
  return cudaSuccess;
}
cudaError_t launch_attn_rows(const AttnArgs& a, cudaStream_t st) {
  if (a.n_split > 1 && a.part_o != g_workspace) note("elsewhere");
  note("parts", st);
  return cudaSuccess;
}
cudaError_t launch_attn_tiles(const AttnArgs& a, cudaStream_t st) { return launch_attn_rows(a, st); }
cudaError_t launch_attn_join(const AttnArgs&, cudaStream_t st) { return note("join", st), cudaSuccess; }
cudaError_t tiles_status(cudaStream_t, uint32_t* bits) { return *bits = 0, cudaSuccess; }
}  // namespace bdkv

extern "C" {
cudaError_t __wrap_cudaGetDevice(int* d) { return *d = 0, cudaSuccess; }
cudaError_t __wrap_cudaSetDevice(int) { return cudaSuccess; }
cudaError_t __wrap_cudaGetLastError() { return cudaSuccess; }
cudaError_t __wrap_cudaDeviceGetAttribute(int* v, cudaDeviceAttr a, int) {
  *v = a == cudaDevAttrComputeCapabilityMajor ? 10 : a == cudaDevAttrComputeCapabilityMinor ? 3 : 152;
  return cudaSuccess;
}
cudaError_t __wrap_cudaStreamIsCapturing(cudaStream_t, cudaStreamCaptureStatus* s) {
  return *s = cudaStreamCaptureStatusNone, cudaSuccess;
}
cudaError_t __wrap_cudaEventCreateWithFlags(cudaEvent_t* e, unsigned) {
  return *e = reinterpret_cast<cudaEvent_t>(uintptr_t(8)), cudaSuccess;
}
cudaError_t __wrap_cudaEventDestroy(cudaEvent_t) { return cudaSuccess; }
cudaError_t __wrap_cudaEventRecord(cudaEvent_t, cudaStream_t st) { return note("record", st), cudaSuccess; }
cudaError_t __wrap_cudaStreamWaitEvent(cudaStream_t st, cudaEvent_t, unsigned) { return note("wait", st), cudaSuccess; }
cudaError_t __wrap_cudaMalloc(void** p, size_t n) {
  note("malloc");
  g_workspace = *p = std::malloc(n);
  return cudaSuccess;
}
cudaError_t __wrap_cudaFree(void* p) {
  note("free");
  std::free(p);
  return cudaSuccess;
}
}

int main(int argc, char** argv) {
  bdkv_cache c = {};
  uint8_t* some = reinterpret_cast<uint8_t*>(uintptr_t(1) << 20);  // never dereferenced
  c.k = c.v = c.k_scale = c.v_scale = some;
  c.n_pages = 4096, c.page_size = 16, c.n_heads = 2, c.head_dim = 64;
  for (int64_t* s : {c.k_stride, c.v_stride}) s[0] = 16 * 2 * 64, s[1] = 2 * 64, s[2] = 64;
  c.k_scale_stride = c.v_scale_stride = 2;
  for (int i = 1; i < argc; ++i) {
    bdkv_attention_args a = {};
    a.q.data = a.out.data = some;
    a.q.dtype = a.out.dtype = BDKV_BF16;
    a.q.stride_token = a.out.stride_token = 8 * 64, a.q.stride_head = a.out.stride_head = 64;
    a.block_table = a.kv_lens = a.query_start = reinterpret_cast<int32_t*>(some);
    a.table_stride = a.max_blocks = 4096;
    a.n_seq = 2, a.n_q_heads = 8, a.max_q_len = 1, a.mask_block = 1, a.scale = 0.125f;
    a.stream = reinterpret_cast<void*>(static_cast<uintptr_t>(std::atoi(argv[i])));
    a.max_kv_len = std::atoi(std::strchr(argv[i], ':') + 1);
    g_log.clear();
    const int rc = bdkv_attention(&c, &a);
    std::printf("%d%s\n", rc, g_log.c_str());
  }
  return 0;
}
