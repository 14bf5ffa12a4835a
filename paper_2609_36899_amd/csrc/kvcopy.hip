// KV snapshot and restore: page gather to, and scatter from, pinned host memory; and copies of
// pages within a caller's pools.
//
// A trajectory that departs is snapshotted from device memory to host memory
// over PCIe, freeing its pages while the host copy keeps it available (paper:
// Design, "KV Preparation for Late-Bound Placement", phase 1).  The host copy
// is page-major, [page][layer][K|V][Hkv][16 * Dh], so any prefix range of
// pages is one contiguous byte range.  Each work group moves one
// (page, layer, K|V) block of Hkv * 16 * Dh elements with 16-byte accesses.
#include "hip_common.h"
#include "kernels.h"

#include <algorithm>

namespace pdec {

namespace {

__global__ __launch_bounds__(256) void kv_page_copy_kernel(
    const int32_t* __restrict__ pages, int n_layers, int64_t n_pool_pages, int64_t block_bytes,
    char* __restrict__ pool, char* __restrict__ host, int to_host) {
  const int i = blockIdx.x;                 // page index within the sequence
  const int lk = blockIdx.y;                // layer * 2 + kind
  const int64_t dev_off = ((int64_t)lk * n_pool_pages + pages[i]) * block_bytes;
  const int64_t host_off = ((int64_t)i * n_layers * 2 + lk) * block_bytes;
  const int64_t n16 = block_bytes / 16;
  u32x4* d = (u32x4*)(pool + dev_off);
  u32x4* h = (u32x4*)(host + host_off);
  for (int64_t j = threadIdx.x; j < n16; j += 256) {
    if (to_host)
      h[j] = d[j];
    else
      d[j] = h[j];
  }
}

// Pages of a caller's pools to other places of the same pools: a work group per pair and part
// of a page, two units a thread: bound by memory, and many short groups keep more of it under way
// than few long ones.  What is written is not read again here, and passes by the caches.  8190
// pages of 18 KB over and over: 8 units a thread 158 us, 4 49, 2 50, 1 56, written past the caches
// 2 units 41 and 1 41; others each time, from HBM: 67, 4.5 TB/s read and written (a large copy
// 4.9).  Attention over the copies right behind them takes as long in all either way: 8000 pages
// of 10 KB 78 us past the caches and 79, of 18 KB 93 and 92, 1000 pages of eight layers 257 and
// 257, 222 and 224.  T is the widest unit that every part of the pool's pages is a whole number of.
constexpr int kCopyEach = 2, kCopyUnits = kCopyEach * 256;  // of a thread, of a part
template <typename T>
__device__ __forceinline__ void copy_part(const char* from, char* to, int64_t n) {
  T x[kCopyEach];
#pragma unroll
  for (int i = 0; i < kCopyEach; ++i)
    if (i * 256 + threadIdx.x < n) x[i] = ((const T*)from)[i * 256 + threadIdx.x];
#pragma unroll
  for (int i = 0; i < kCopyEach; ++i)
    if (i * 256 + threadIdx.x < n) __builtin_nontemporal_store(x[i], (T*)to + i * 256 + threadIdx.x);
}
// Pools whose pages are whole 16-byte units are copied by these, others by 4 bytes or by one.
__host__ __device__ inline int copy_unit(const void* pool, int64_t bytes) {
  const uint64_t bits = (uint64_t)pool | (uint64_t)bytes;
  return bits % 16 == 0 ? 16 : bits % 4 == 0 ? 4 : 1;
}
__host__ __device__ inline int64_t copy_parts(const void* pool, int64_t bytes) {
  const int64_t part = (int64_t)copy_unit(pool, bytes) * kCopyUnits;
  return (bytes + part - 1) / part;
}

__global__ __launch_bounds__(256) void page_copy_kernel(PageCopyArgs a) {
  const int64_t src = a.src[blockIdx.x], dst = a.dst[blockIdx.x];
  if (src < 0 || src >= a.n_pages || dst < 0 || dst >= a.n_pages || src == dst) return;
  int p = 0;
  int64_t part = blockIdx.y;
  while (true) {
    int64_t n = 0;
    for (; p < a.n_pools; ++p) {
      n = copy_parts(a.pool[p], a.bytes[p]);
      if (part < n) break;
      part -= n;
    }
    if (p == a.n_pools) return;
    const int64_t bytes = a.bytes[p];
    const int unit = copy_unit(a.pool[p], bytes);
    const int64_t at = part * unit * kCopyUnits, left = bytes / unit - part * kCopyUnits;
    const char* from = (const char*)a.pool[p] + src * bytes + at;
    char* to = (char*)a.pool[p] + dst * bytes + at;
    if (unit == 16) copy_part<u32x4>(from, to, left);
    else if (unit == 4) copy_part<uint32_t>(from, to, left);
    else copy_part<uint8_t>(from, to, left);
    part += gridDim.y;
  }
}

int64_t page_copy_parts(const PageCopyArgs& a) {
  int64_t n = 0;
  for (int p = 0; p < a.n_pools; ++p) n += copy_parts(a.pool[p], a.bytes[p]);
  return n;
}

}  // namespace

hipError_t launch_page_copy(const PageCopyArgs& a, hipStream_t stream) {
  if (a.n_pairs == 0 || a.n_pools == 0) return hipSuccess;
  const dim3 grid(a.n_pairs, (uint32_t)std::min<int64_t>(page_copy_parts(a), 65535));
  page_copy_kernel<<<grid, 256, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_kv_page_copy(int n_pages, const int32_t* pages_dev, int n_layers,
                               int64_t n_pool_pages, int64_t block_bytes, void* pool,
                               void* host_dev_ptr, int to_host, hipStream_t stream) {
  if (n_pages == 0) return hipSuccess;
  const dim3 grid(n_pages, 2 * n_layers);
  kv_page_copy_kernel<<<grid, 256, 0, stream>>>(pages_dev, n_layers, n_pool_pages, block_bytes,
                                               (char*)pool, (char*)host_dev_ptr, to_host);
  return hipGetLastError();
}

}  // namespace pdec
