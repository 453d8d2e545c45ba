// What the entry points of the cache libraries share: argument checks and the library-owned workspaces. Everything here is
// private to the translation unit that includes it, so each library has workspaces of its own.
#pragma once

#include <algorithm>
#include <atomic>
#include <climits>
#include <mutex>
#include <utility>

#include "cache.h"

namespace {

// Compute capability and SM count of the current device, cached (0 = unknown, -1 = another device than sm_103).
std::atomic<int> g_sms[64];

int check_device(int* sms) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return BD_ERR_CUDA;
  if (dev < 0 || dev >= 64) return BD_ERR_DEVICE;
  int s = g_sms[dev].load(std::memory_order_relaxed);
  if (s == 0) {
    int maj = 0, mnr = 0, n = 0;
    if (cudaDeviceGetAttribute(&maj, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&mnr, cudaDevAttrComputeCapabilityMinor, dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
      return BD_ERR_CUDA;
    s = maj == 10 && mnr == 3 ? n : -1;
    g_sms[dev].store(s, std::memory_order_relaxed);
  }
  *sms = s;
  return s > 0 ? BD_OK : BD_ERR_DEVICE;
}

int cuda_status(cudaError_t e) {
  if (e == cudaSuccess) return BD_OK;
  return e == cudaErrorNoKernelImageForDevice || e == cudaErrorInvalidDeviceFunction ? BD_ERR_DEVICE : BD_ERR_CUDA;
}

bool aligned(const void* p, uintptr_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

bool page_size_ok(int p) { return p == 16 || p == 32 || p == 64 || p == 128 || p == 256; }

constexpr int64_t MAX_STRIDE = int64_t(1) << 40;
constexpr int MAX_KV = 1 << 30;  // the kernels count a part's end, and tokens a few tiles behind it, in 32 bits

int check_strides(const int64_t* s, int n, int64_t multiple) {
  for (int i = 0; i < n; ++i) {
    if (s[i] < 0 || s[i] > MAX_STRIDE) return BD_ERR_SHAPE;
    if (s[i] % multiple != 0) return BD_ERR_ALIGN;
  }
  return BD_OK;
}

int check_cache(const bdkv_cache& c) {
  if (!page_size_ok(c.page_size) || c.n_heads < 1 || c.n_heads > 1024 || c.head_dim < 16 || c.head_dim > 128 ||
      c.head_dim % 16 != 0)
    return BD_ERR_SHAPE;
  if (c.n_pages < 0 || c.n_pages > INT_MAX || c.k_scale_stride < 0 || c.v_scale_stride < 0 ||
      c.k_scale_stride > MAX_STRIDE || c.v_scale_stride > MAX_STRIDE)
    return BD_ERR_SHAPE;
  if (int rc = check_strides(c.k_stride, 3, 16)) return rc;
  if (int rc = check_strides(c.v_stride, 3, 16)) return rc;
  if (c.n_pages > 0 && (!c.k || !c.v || !c.k_scale || !c.v_scale)) return BD_ERR_NULL;
  return aligned(c.k, 16) && aligned(c.v, 16) ? BD_OK : BD_ERR_ALIGN;
}

int check_rows(const bdkv_rows& r) {
  if (r.dtype != BDKV_BF16 && r.dtype != BDKV_F16) return BD_ERR_DTYPE;
  const int64_t s[2] = {r.stride_token, r.stride_head};
  if (int rc = check_strides(s, 2, 8)) return rc;
  return aligned(r.data, 16) ? BD_OK : BD_ERR_ALIGN;
}

// A cache that is written: its codes, and its scales, must not lie on one another. (Keys and values may be the same
// memory, if a user stores the same in both.)
int check_cache_apart(const bdkv_cache& c) {
  for (const int64_t* s : {c.k_stride, c.v_stride}) {
    std::pair<int64_t, int64_t> d[3] = {{s[0], c.n_pages}, {s[1], c.page_size}, {s[2], c.n_heads}};  // stride, extent
    std::sort(d, d + 3);
    __int128 span = c.head_dim;  // of what the smaller strides reach
    for (const auto& [stride, extent] : d) {
      if (extent <= 1) continue;
      if (stride < span) return BD_ERR_ARG;
      span += static_cast<__int128>(stride) * (extent - 1);
    }
  }
  return c.n_pages > 1 && std::min(c.k_scale_stride, c.v_scale_stride) < c.n_heads ? BD_ERR_ARG : BD_OK;
}

// Rows that are written must not lie on one another, as far as strides show it: the number of tokens is not known here,
// so where a head's tokens lie closer than its heads, the heads' distance is not checked.
int check_rows_apart(const bdkv_rows& r, int64_t heads, int64_t dim, bool many_tokens) {
  if ((heads > 1 && r.stride_head < dim) || (many_tokens && r.stride_token < dim)) return BD_ERR_ARG;
  if (heads > 1 && many_tokens && r.stride_token >= r.stride_head && r.stride_token < (heads - 1) * r.stride_head + dim)
    return BD_ERR_ARG;
  return BD_OK;
}

// The library's own workspace of a device. All calls share it: each waits for the last one's end, also on what looks like
// the same stream (a handle may be a destroyed stream's, or the per-thread default stream's of another thread).
struct Workspace {
  void* data = nullptr;
  size_t bytes = 0;
  cudaEvent_t used = nullptr;
};
std::mutex g_mu;
Workspace g_ws[64];

int own_workspace(size_t bytes, cudaStream_t st, Workspace** out) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return BD_ERR_CUDA;
  cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
  if (cudaStreamIsCapturing(st, &capture) != cudaSuccess) return BD_ERR_CUDA;
  if (capture != cudaStreamCaptureStatusNone) return BD_ERR_WORKSPACE;
  Workspace& w = g_ws[dev];
  if (w.used == nullptr && cudaEventCreateWithFlags(&w.used, cudaEventDisableTiming) != cudaSuccess) return BD_ERR_CUDA;
  if (w.bytes < bytes) {
    if (w.data) cudaFree(w.data);  // synchronises the device: no call can still use it
    w.data = nullptr;
    w.bytes = 0;
    if (cudaMalloc(&w.data, bytes) != cudaSuccess) {
      cudaGetLastError();
      return BD_ERR_CUDA;
    }
    w.bytes = bytes;
  } else if (cudaStreamWaitEvent(st, w.used) != cudaSuccess) {
    return BD_ERR_CUDA;
  }
  *out = &w;
  return BD_OK;
}

int free_workspaces() {
  std::lock_guard<std::mutex> lock(g_mu);
  int cur = 0;
  if (cudaGetDevice(&cur) != cudaSuccess) return BD_ERR_CUDA;
  for (int dev = 0; dev < 64; ++dev) {
    Workspace& w = g_ws[dev];
    if (w.used == nullptr || cudaSetDevice(dev) != cudaSuccess) continue;
    if (w.data) cudaFree(w.data);
    cudaEventDestroy(w.used);
    w = Workspace();
  }
  cudaSetDevice(cur);
  return BD_OK;
}

}  // namespace
