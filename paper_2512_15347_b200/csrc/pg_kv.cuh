// Shared pieces of the token-rollout calls: the cache descriptor as the kernels see it, its
// argument checks, element conversions.
#pragma once

#include "pg_common.cuh"

#include <cuda_fp16.h>

#include <atomic>

namespace pg {

constexpr int kStatusTimeout = 2;   // status bit 1: a bounded wait ran out
constexpr int kStatusIndex = 4;     // status bit 2: an index from device memory was out of range
constexpr int kStatusPages = 8;     // status bit 3: no free page, or a row's table is full

// Every call's workspace begins with this many bytes of counters that are zero between calls; what lies behind them is written
// before it is read.  So one buffer may serve all calls of a stream.
constexpr size_t kCounterBytes = 4096;

// One layer of the cache, by value in the kernel parameters.  Strides in elements.
struct KvView {
  void *k, *v;
  int64_t page_stride, layer_stride;
  int32_t* table;
  const int32_t* len;
  int32_t* grown;
  int32_t* status;
  int n_layers, n_pages, n_kv_heads, page_size, head_dim, n_rows, max_pages;
};

// Rows and pages of a cache, rows of a fork: a loop over as many in steps of a CTA still ends inside 32 bits.
constexpr int32_t kMostItems = 0x7FF00000;

// Checks that need no device access.  The product of all sizes must stay addressable in 63 bits.
inline int kv_check(const pg_kv* c) {
  if (!c) return PG_EINVAL;
  if (c->dtype != PG_F32 && c->dtype != PG_BF16 && c->dtype != PG_F16) return PG_EINVAL;
  if (c->n_layers < 1 || c->n_pages < 1 || c->n_kv_heads < 1 || c->page_size < 1) return PG_EINVAL;
  if (c->head_dim < 8 || c->head_dim > 256 || (c->head_dim & 7)) return PG_EINVAL;
  if (c->n_rows < 0 || c->max_pages < 1) return PG_EINVAL;
  if (c->n_rows > kMostItems || c->n_pages > kMostItems) return PG_EINVAL;
  if (((int64_t)c->max_pages + 1) * c->page_size > 0x80000000LL - 4096) return PG_EINVAL;   // a length rounded up to a page fits
  const int64_t head = (int64_t)c->page_size * c->head_dim;
  if (head > ((int64_t)1 << 40) / c->n_kv_heads) return PG_EINVAL;
  if (c->page_stride < head * c->n_kv_heads || (c->page_stride & 7)) return PG_EINVAL;
  if (c->page_stride > ((int64_t)1 << 60) / c->n_pages) return PG_EINVAL;
  if (c->layer_stride < 0 || (c->layer_stride & 7)) return PG_EINVAL;
  if (c->n_layers > 1 && (c->layer_stride < head * c->n_kv_heads ||
                          c->layer_stride > ((int64_t)1 << 60) / c->n_layers)) return PG_EINVAL;
  if (!c->k || !c->v || (((uintptr_t)c->k | (uintptr_t)c->v) & 15)) return PG_EINVAL;
  if (c->n_rows > 0 && (!c->table || !c->len)) return PG_EINVAL;
  return PG_OK;
}

inline KvView kv_view(const pg_kv* c, int32_t* status) {
  KvView v;
  v.k = c->k;
  v.v = c->v;
  v.page_stride = c->page_stride;
  v.layer_stride = c->n_layers > 1 ? c->layer_stride : 0;
  v.table = c->table;
  v.len = c->len;
  v.grown = c->grown;
  v.status = status;
  v.n_layers = c->n_layers;
  v.n_pages = c->n_pages;
  v.n_kv_heads = c->n_kv_heads;
  v.page_size = c->page_size;
  v.head_dim = c->head_dim;
  v.n_rows = c->n_rows;
  v.max_pages = c->max_pages;
  return v;
}

// Lets a kernel use `bytes` of dynamic shared memory; asked of the runtime once per kernel and device.
template <typename Kernel>
inline int allow_shared(Kernel* kernel, int bytes, std::atomic<uint64_t>& done) {
  int dev = 0;
  PG_CUDA(cudaGetDevice(&dev));
  if (dev < 64 && (done.load(std::memory_order_acquire) >> dev & 1)) return PG_OK;
  PG_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes));
  if (dev < 64) done.fetch_or(1ull << dev, std::memory_order_release);
  return PG_OK;
}

inline size_t dtype_bytes(int dtype) { return dtype == PG_F32 ? 4 : 2; }

// n / d for 0 <= n < 2^31 by a multiplication (d >= 1): m = ceil(2^(32+s) / d), s = ceil(log2 d) - 1.
struct FastDiv {
  uint32_t d, m, s;
};
inline FastDiv fast_div(uint32_t d) {
  FastDiv f{d, 0, 0};
  if (d > 1) {
    uint32_t s = 0;
    while ((1ull << (s + 1)) < d) ++s;
    f.s = s;
    f.m = (uint32_t)((((unsigned __int128)1 << (32 + s)) + d - 1) / d);
  }
  return f;
}

#ifdef __CUDACC__
__device__ __forceinline__ uint32_t div_by(uint32_t n, const FastDiv& f) {
  return f.d == 1 ? n : __umulhi(n, f.m) >> f.s;
}
__device__ __forceinline__ void flag(int32_t* status, int bit) {
  if (status) atomicOr(status, bit);
}

// A row's length, kept inside what its table can hold.
__device__ __forceinline__ int checked_len(const KvView& kv, int n) {
  const int most = kv.max_pages * kv.page_size;
  if ((unsigned int)n > (unsigned int)most) {
    flag(kv.status, kStatusIndex);
    return n < 0 ? 0 : most;
  }
  return n;
}
__device__ __forceinline__ int row_len(const KvView& kv, int row) { return checked_len(kv, kv.len[row]); }

// Whether pg_kv_extend has last found room for n new tokens of a row, as far as the cache keeps that.
__device__ __forceinline__ bool has_room(const KvView& kv, int row, int n) { return !kv.grown || n <= kv.grown[row]; }

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }
#endif

}  // namespace pg
