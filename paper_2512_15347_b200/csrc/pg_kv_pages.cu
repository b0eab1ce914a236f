// Pages of the key-value cache: forking, dropping and reordering rows (pg_kv_fork), packing the pool
// (pg_kv_pack), room for new tokens (pg_kv_extend) and writing them (pg_kv_append).
//
// A page's count is the number of rows that refer to it.  Counts move by integer atomics, whose result
// does not depend on their order, and free pages are always taken lowest first through a scan of the
// counts, so that tables, counts and pools come out the same on every run.
#include "pg_kv.cuh"
#include "pg_trace.cuh"

#include <algorithm>

namespace pg {

// ---------------------------------------------------------------- scans in one CTA
constexpr int kScanThreads = 1024;          // of the kernels that are one CTA

// Exclusive prefix sum over the CTA; *total gets the sum.  All threads call.
template <typename Int>
__device__ __forceinline__ Int block_scan(Int v, Int* total) {
  __shared__ Int warp_sums[kScanThreads / 32 + 1];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  Int x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const Int y = __shfl_up_sync(0xFFFFFFFFu, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();                       // the previous call's readers are done
  if (lane == 31) warp_sums[warp] = x;
  __syncthreads();
  if (warp == 0) {
    Int s = lane < (int)(blockDim.x >> 5) ? warp_sums[lane] : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const Int y = __shfl_up_sync(0xFFFFFFFFu, s, o);
      if (lane >= o) s += y;
    }
    warp_sums[lane] = s;
  }
  __syncthreads();
  *total = warp_sums[(blockDim.x >> 5) - 1];
  return x - v + (warp ? warp_sums[warp - 1] : 0);
}

// Hands the free pages (refs == 0), lowest first, to take(k, page) for k < wanted; returns how many
// there were (at most wanted).  One CTA.
template <typename Take>
__device__ __forceinline__ int take_free(const int32_t* refs, int n_pages, int wanted, Take take) {
  // A warp looks at 1024 counts a round, 32 coalesced loads of 32; the ballot over load i is what lane i keeps.
  const int lane = threadIdx.x & 31;
  int found = 0;
  for (int base = 0; base < n_pages && found < wanted; base += blockDim.x * 32) {
    const int w0 = base + (threadIdx.x - lane) * 32, p = w0 + lane * 32;
    uint32_t free = 0;
    if (w0 < n_pages) {
#pragma unroll 16
      for (int i = 0; i < 32; ++i) {
        const int at = w0 + i * 32 + lane;
        const uint32_t b = __ballot_sync(0xFFFFFFFFu, at < n_pages && __ldcg(&refs[at]) == 0);
        if (lane == i) free = b;
      }
    }
    int total;
    int k = found + block_scan(__popc(free), &total);
    for (; free; free &= free - 1, ++k)
      if (k < wanted) take(k, p + __ffs(free) - 1);
    found += total;
  }
  __syncthreads();
  return min(found, wanted);
}

// Counts to their output, by one CTA (few pages: a launch less than a copy of its own).
constexpr int kCopyCounts = 1 << 17;         // pages up to which the one-CTA kernels do it
__device__ __forceinline__ void copy_counts(const int32_t* from, int32_t* to, int n) {
  if ((((uintptr_t)from | (uintptr_t)to) & 15) == 0) {
#pragma unroll 4
    for (int i = threadIdx.x; i < n / 4; i += blockDim.x) ((int4*)to)[i] = ((const int4*)from)[i];
    for (int i = n / 4 * 4 + threadIdx.x; i < n; i += blockDim.x) to[i] = from[i];
  } else {
#pragma unroll 4
    for (int i = threadIdx.x; i < n; i += blockDim.x) to[i] = from[i];
  }
  __syncthreads();
}

// ---------------------------------------------------------------- copies of whole pages
// Pairs (from, to) in device memory, their number too.  A page of one layer and one of k / v is
// contiguous but for its stride: kv heads * page_size * head_dim elements.  An item is one 32 KB piece of
// `run` consecutive pairs: forks of one row follow each other and have the same source, which is then read once a run.
// Bound: HBM.  The first table_ctas CTAs remap the table instead (pack).
struct CopyParams {
  KvView kv;
  const int2* pairs;
  const int32_t* n_pairs;
  int64_t page_words, stride_words, layer_words;   // 16-byte words
  int pieces, run;                                  // CTA-sized pieces of a page
  const int32_t* to;
  int32_t* table_out;
  unsigned table_ctas;
};
constexpr int kCopyThreads = 256;
constexpr int kCopyPer = 8;
constexpr int kCopyWords = kCopyThreads * kCopyPer; // 32 KB a piece

__device__ __forceinline__ void remap_table(const CopyParams& p) {
  const KvView& kv = p.kv;
  const int64_t entries = (int64_t)kv.n_rows * kv.max_pages;
  for (int64_t i = (int64_t)blockIdx.x * kCopyThreads + threadIdx.x; i < entries; i += (int64_t)p.table_ctas * kCopyThreads) {
    const int row = (int)(i / kv.max_pages), j = (int)(i - (int64_t)row * kv.max_pages);
    const int n = row_len(kv, row), pages = (n + kv.page_size - 1) / kv.page_size;
    int to = -1;
    if (j < pages) {
      const int page = kv.table[i];
      if ((unsigned int)page < (unsigned int)kv.n_pages) to = p.to[page];
      if (to < 0) flag(kv.status, kStatusIndex);
    }
    p.table_out[i] = to;
  }
}

__global__ void __launch_bounds__(kCopyThreads) copy_pages_kernel(const __grid_constant__ CopyParams p) {
  if (blockIdx.x < p.table_ctas) return remap_table(p);
  const int n_pairs = *p.n_pairs, per_run = p.pieces * p.kv.n_layers * 2;
  const int64_t items = (int64_t)((n_pairs + p.run - 1) / p.run) * per_run;
  for (int64_t item = blockIdx.x - p.table_ctas; item < items; item += gridDim.x - p.table_ctas) {
    const int first = (int)(item / per_run) * p.run;
    int rest = (int)(item % per_run);
    const int piece = rest % p.pieces;
    rest /= p.pieces;
    uint4* pool = (uint4*)((rest & 1) ? p.kv.v : p.kv.k) + (rest >> 1) * p.layer_words + (int64_t)piece * kCopyWords;
    const int n = (int)min((int64_t)kCopyWords, p.page_words - (int64_t)piece * kCopyWords);
    uint4 w[kCopyPer];
    int held = -1;
    for (int k = first; k < min(first + p.run, n_pairs); ++k) {
      const int2 move = p.pairs[k];
      if (move.x != held) {
        const uint4* from = pool + move.x * p.stride_words;
#pragma unroll
        for (int i = 0; i < kCopyPer; ++i) {
          const int at = threadIdx.x + i * kCopyThreads;
          if (at < n) w[i] = __ldcs(from + at);
        }
        held = move.x;
      }
      uint4* to = pool + move.y * p.stride_words;
#pragma unroll
      for (int i = 0; i < kCopyPer; ++i) {
        const int at = threadIdx.x + i * kCopyThreads;
        if (at < n) __stcs(to + at, w[i]);
      }
    }
  }
}

// CTA-sized pieces of a page of one layer; 0 if a copy in all layers would have more of them than 32 bits count.
static int copy_pieces(const pg_kv* kv) {
  const int64_t words = (int64_t)kv->n_kv_heads * kv->page_size * kv->head_dim * (int64_t)dtype_bytes(kv->dtype) / 16;
  const int64_t pieces = (words + kCopyWords - 1) / kCopyWords;
  return pieces > 0x7FFFFFFFLL / 2 / kv->n_layers ? 0 : (int)pieces;
}

static int launch_copy(const pg_kv* kv, const KvView& view, const int2* pairs, const int32_t* n_pairs, int64_t most, int run,
                       const int32_t* to, int32_t* table_out, cudaStream_t st) {
  const int64_t b = (int64_t)dtype_bytes(kv->dtype);
  CopyParams p;
  p.kv = view;
  p.pairs = pairs;
  p.n_pairs = n_pairs;
  p.page_words = (int64_t)kv->n_kv_heads * kv->page_size * kv->head_dim * b / 16;
  p.stride_words = kv->page_stride * b / 16;
  p.layer_words = view.layer_stride * b / 16;
  const int64_t pieces = copy_pieces(kv);
  p.pieces = (int)pieces;
  p.run = run;
  p.to = to;
  p.table_out = table_out;
  const int64_t entries = table_out ? (int64_t)kv->n_rows * kv->max_pages : 0;
  p.table_ctas = (unsigned)std::min<int64_t>((entries + kCopyThreads * 4 - 1) / (kCopyThreads * 4), 148);
  const int64_t items = (most + run - 1) / run * pieces * kv->n_layers * 2;
  copy_pages_kernel<<<p.table_ctas + (unsigned)std::min<int64_t>(std::max<int64_t>(items, 1), 148 * 64), kCopyThreads, 0, st>>>(p);
  PG_LAUNCH_CHECK();
  return PG_OK;
}

// ---------------------------------------------------------------- fork

struct ForkWork {            // in the caller's workspace
  unsigned int* ticket;      // counters
  int32_t* n_need;           // rows in need
  int32_t* n_pairs;          // copies to make
  int32_t* need;             // [n_out] 1 where new row i needs a page for its partly filled last page
  int2* pairs;               // [n_out]
};
static size_t fork_work(char* base, int64_t n_out, ForkWork* w) {
  auto up = [](size_t b) { return (b + 15) & ~(size_t)15; };
  const size_t need = up(n_out * 4), pairs = up(n_out * 8);
  if (w) {
    w->ticket = (unsigned int*)base;
    w->n_need = (int32_t*)(base + 4);
    base += kCounterBytes;
    w->n_pairs = (int32_t*)base;
    w->need = (int32_t*)(base + 16);
    w->pairs = (int2*)(base + 16 + need);
  }
  return kCounterBytes + 16 + need + pairs;
}

constexpr int kForkThreads = 256, kForkRows = 32;   // most old rows of a CTA
constexpr int kForkBatch = 12;                      // entries of src_rows a thread looks at a time

struct ForkParams {
  KvView kv;
  const int32_t* src;
  int32_t *table_out, *len_out, *refs;
  ForkWork w;
  int n_out, rows;           // rows: old rows of a CTA
};

// Pages for the rows that need one, and the list of copies.  One CTA, after all others.
__device__ __forceinline__ void fork_assign(const ForkParams& p) {
  const KvView& kv = p.kv;
  int wanted = 0;
  for (int base = 0; base < p.n_out; base += blockDim.x * 4) {     // pairs[k].x = the k-th row in need, for now
    const int i0 = base + threadIdx.x * 4;
    int need[4], mine = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      need[e] = i0 + e < p.n_out ? __ldcg(&p.w.need[i0 + e]) : 0;
      mine += need[e];
    }
    int total;
    int k = wanted + block_scan(mine, &total);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (need[e]) p.w.pairs[k++].x = i0 + e;
    wanted += total;
  }
  __syncthreads();
  const int found = take_free(p.refs, kv.n_pages, wanted, [&](int k, int page) { p.w.pairs[k].y = page; });
  constexpr int kAhead = 4;                           // rows of a thread whose look-ups are under way together
  for (int k0 = threadIdx.x; k0 < found; k0 += blockDim.x * kAhead) {
    int2 x[kAhead];
    int64_t last[kAhead];
    int from[kAhead];
#pragma unroll
    for (int e = 0; e < kAhead; ++e) {
      const int k = k0 + e * blockDim.x;
      x[e] = k < found ? p.w.pairs[k] : make_int2(-1, -1);
    }
#pragma unroll
    for (int e = 0; e < kAhead; ++e)
      last[e] = x[e].x >= 0 ? (int64_t)x[e].x * kv.max_pages + __ldcg(&p.len_out[x[e].x]) / kv.page_size : 0;
#pragma unroll
    for (int e = 0; e < kAhead; ++e) from[e] = x[e].x >= 0 ? __ldcg(&p.table_out[last[e]]) : 0;
#pragma unroll
    for (int e = 0; e < kAhead; ++e) {
      if (x[e].x < 0) continue;
      p.table_out[last[e]] = x[e].y;
      p.refs[x[e].y] = 1;
      p.w.pairs[k0 + e * blockDim.x].x = (unsigned int)from[e] < (unsigned int)kv.n_pages ? from[e] : x[e].y;
    }
  }
  for (int k = found + threadIdx.x; k < wanted; k += blockDim.x) {   // no page: the full pages remain
    const int i = p.w.pairs[k].x;
    const int full = __ldcg(&p.len_out[i]) / kv.page_size;
    p.table_out[(int64_t)i * kv.max_pages + full] = -1;
    p.len_out[i] = full * kv.page_size;
    flag(kv.status, kStatusPages);
  }
  if (threadIdx.x == 0) *p.w.n_pairs = found;
}

// A CTA takes `rows` old rows: it goes through src_rows once, 3072 entries at a time, and writes the table rows
// of their forks (CTA 0: also of entries that name no row); then the rows' pages change by (forks - 1), a
// partly filled last page by (min(forks, 1) - 1).  The last CTA to finish hands out the pages.
__global__ void __launch_bounds__(kForkThreads) fork_kernel(const __grid_constant__ ForkParams p) {
  __shared__ int forks[kForkRows], length[kForkRows], n_found, is_last;
  __shared__ int2 found[kForkThreads * kForkBatch];   // (new row, old row within the CTA or -1)
  const KvView& kv = p.kv;
  const int s0 = blockIdx.x * p.rows, n_rows = max(0, min(p.rows, kv.n_rows - s0));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if ((int)threadIdx.x < n_rows) {
    forks[threadIdx.x] = 0;
    length[threadIdx.x] = row_len(kv, s0 + threadIdx.x);
  }
  for (int base = 0; base < p.n_out; base += kForkThreads * kForkBatch) {
    int src[kForkBatch];
#pragma unroll
    for (int e = 0; e < kForkBatch; ++e) {
      const int i = base + e * kForkThreads + threadIdx.x;
      src[e] = i < p.n_out ? p.src[i] : 0;
    }
    __syncthreads();
    if (threadIdx.x == 0) n_found = 0;
    __syncthreads();
#pragma unroll
    for (int e = 0; e < kForkBatch; ++e) {
      const int i = base + e * kForkThreads + threadIdx.x;
      if (i >= p.n_out) continue;
      const int s = src[e];
      const bool none = (unsigned int)s >= (unsigned int)kv.n_rows;
      if ((unsigned int)(s - s0) < (unsigned int)n_rows) found[atomicAdd(&n_found, 1)] = make_int2(i, s - s0);
      else if (none && blockIdx.x == 0) found[atomicAdd(&n_found, 1)] = make_int2(i, s == -1 ? -1 : -2);
    }
    __syncthreads();
    // the first fork of a row in need of a page keeps the row's own: the smallest new row of the earliest batch
    for (int f = warp; f < n_found; f += kForkThreads / 32) {
      const int2 x = found[f];
      const int n = x.y >= 0 ? length[x.y] : 0, pages = (n + kv.page_size - 1) / kv.page_size;
      const int32_t* from = kv.table + (int64_t)(s0 + max(x.y, 0)) * kv.max_pages;
      int32_t* to = p.table_out + (int64_t)x.x * kv.max_pages;
      for (int j = lane; j < kv.max_pages; j += 32) {
        const int page = j < pages ? from[j] : -1;
        if (j < pages && (unsigned int)page >= (unsigned int)kv.n_pages) flag(kv.status, kStatusIndex);
        to[j] = page;
      }
      bool need = false;
      if (x.y >= 0 && n % kv.page_size != 0) {
        need = forks[x.y] > 0;                        // of earlier batches
        for (int g = lane; g < n_found && !need; g += 32) need = found[g].y == x.y && found[g].x < x.x;
        need = __any_sync(0xFFFFFFFFu, need);
      }
      if (lane == 0) {
        if (x.y == -2) flag(kv.status, kStatusIndex);
        p.len_out[x.x] = n;
        p.w.need[x.x] = need;
        if (need) atomicAdd(p.w.n_need, 1);
      }
    }
    __syncthreads();
    for (int f = threadIdx.x; f < n_found; f += kForkThreads)
      if (found[f].y >= 0) atomicAdd(&forks[found[f].y], 1);
  }
  __syncthreads();
  for (int r = warp; r < n_rows; r += kForkThreads / 32) {
    const int n = length[r], pages = (n + kv.page_size - 1) / kv.page_size, full = n / kv.page_size;
    const int all = forks[r] - 1, part = min(forks[r], 1) - 1;
    if (all == 0) continue;
    for (int j = lane; j < pages; j += 32) {
      const int page = kv.table[(int64_t)(s0 + r) * kv.max_pages + j];
      if ((unsigned int)page >= (unsigned int)kv.n_pages) flag(kv.status, kStatusIndex);
      else if (const int d = j < full ? all : part) atomicAdd(&p.refs[page], d);
    }
  }
  if (p.n_out == 0) return;
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) {
    is_last = atomicAdd(p.w.ticket, 1u) == gridDim.x - 1;
    if (is_last) *p.w.ticket = 0;
  }
  __syncthreads();
  if (!is_last) return;
  __threadfence();
  if (__ldcg(p.w.n_need) == 0) {
    if (threadIdx.x == 0) *p.w.n_pairs = 0;
    return;
  }
  fork_assign(p);
  if (threadIdx.x == 0) *p.w.n_need = 0;
}

// ---------------------------------------------------------------- pack

struct PackWork {          // in the caller's workspace, behind the counters
  int32_t* n_pairs;
  int32_t* to;         // [n_pages] new number of a page in use, -1 of a free one
  int2* pairs;         // [n_pages / 2 + 1] moves
};
static size_t pack_work(char* base, int64_t n_pages, PackWork* w) {
  auto up = [](size_t b) { return (b + 15) & ~(size_t)15; };
  const size_t to = up(n_pages * 4), pairs = up((n_pages / 2 + 1) * 8);
  if (w) {
    base += kCounterBytes;
    w->n_pairs = (int32_t*)base;
    w->to = (int32_t*)(base + 16);
    w->pairs = (int2*)(base + 16 + to);
  }
  return kCounterBytes + 16 + to + pairs;
}

struct PackParams {
  KvView kv;
  const int32_t* refs;
  int32_t *refs_out, *table_out, *page_map;
  PackWork w;
  int copy_refs;
};

// The k-th page in use at n_live or above moves into the k-th free page below n_live.  One CTA; a thread
// has eight pages at a time.
__global__ void __launch_bounds__(kScanThreads) pack_plan_kernel(const __grid_constant__ PackParams p) {
  constexpr int kPer = 8;
  const int n = p.kv.n_pages;
  int mine = 0, n_live, moves = 0;
  if (p.copy_refs) copy_counts(p.refs, p.refs_out, n);
#pragma unroll 4
  for (int i = threadIdx.x; i < n; i += kScanThreads) mine += p.refs[i] > 0;
  block_scan(mine, &n_live);
  int holes = 0;
  for (int base = 0; base < n; base += kScanThreads * kPer) {
    const int i0 = base + threadIdx.x * kPer;
    uint32_t hole = 0, mover = 0;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      const int i = i0 + e;
      if (i >= n) continue;
      const bool live = p.refs[i] > 0;
      hole |= (uint32_t)(i < n_live && !live) << e;
      mover |= (uint32_t)(i >= n_live && live) << e;
      p.w.to[i] = live ? i : -1;
    }
    int total;                                        // both counts in one scan: at most 8192 a batch
    const int before = block_scan(__popc(hole) | __popc(mover) << 16, &total);
    int kh = holes + (before & 0xFFFF), km = moves + (before >> 16);
    for (; hole; hole &= hole - 1) p.w.pairs[kh++].y = i0 + __ffs(hole) - 1;
    for (; mover; mover &= mover - 1) p.w.pairs[km++].x = i0 + __ffs(mover) - 1;
    holes += total & 0xFFFF;
    moves += total >> 16;
  }
  __syncthreads();
  for (int k = threadIdx.x; k < moves; k += kScanThreads) {
    const int2 m = p.w.pairs[k];
    p.w.to[m.x] = m.y;
    const int c = p.refs[m.x];
    p.refs_out[m.y] = c;
    p.refs_out[m.x] = 0;
  }
  if (threadIdx.x == 0) *p.w.n_pairs = moves;
  if (p.page_map) {
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kScanThreads) p.page_map[i] = p.w.to[i];
  }
}

// ---------------------------------------------------------------- extend

struct ExtendParams {
  KvView kv;
  const int32_t* n_new;
  int32_t *len_out, *refs;
  int n_uniform;
};

// One CTA: 12 us for one token in each of 768 rows, 26 us for 2100 pages of 64 rows.  Rows in chunks of 1024: pages wanted, their prefix, then the free pages in order.  1024 rows may want more
// than 2^31 pages together, so the prefix has 64 bits; past what the pool has it only says "none".
__global__ void __launch_bounds__(kScanThreads) extend_kernel(const __grid_constant__ ExtendParams p) {
  __shared__ int first[kScanThreads];           // pages handed to the chunk's rows before this one
  __shared__ int have[kScanThreads];
  const KvView& kv = p.kv;
  const int most = kv.max_pages * kv.page_size;
  bool dry = false;
  for (int base = 0; base < kv.n_rows; base += kScanThreads) {
    const int r = base + threadIdx.x;
    int n = 0, add = 0, old_pages = 0, want = 0;
    if (r < kv.n_rows) {
      n = row_len(kv, r);
      add = p.n_new ? p.n_new[r] : p.n_uniform;
      if (add < 0) { flag(kv.status, kStatusIndex); add = 0; }
      if (add > most - n) { flag(kv.status, kStatusPages); add = 0; }
      old_pages = (n + kv.page_size - 1) / kv.page_size;
      want = (n + add + kv.page_size - 1) / kv.page_size - old_pages;
    }
    long long total;
    const long long before = block_scan((long long)want, &total);
    first[threadIdx.x] = (int)min(before, 0x7FFFFFFFll);
    have[threadIdx.x] = old_pages;
    __syncthreads();
    int found = 0;
    if (total && !dry)
      found = take_free(p.refs, kv.n_pages, (int)min(total, (long long)kv.n_pages), [&](int k, int page) {
        int lo = 0, hi = kScanThreads - 1;                 // last row with first[row] <= k
        while (lo < hi) {
          const int mid = (lo + hi + 1) >> 1;
          if (first[mid] <= k) lo = mid; else hi = mid - 1;
        }
        kv.table[(int64_t)(base + lo) * kv.max_pages + have[lo] + k - first[lo]] = page;
        p.refs[page] = 1;
      });
    __syncthreads();
    const bool fits = before + want <= found || want == 0;
    const bool late = dry || (found < total && before + want > found);
    if (r < kv.n_rows) {
      const bool grown = fits && !late;
      if (!grown)                                      // the one row that got some of its pages gives them back
        for (int j = 0; j < min((long long)want, found - before); ++j) p.refs[kv.table[(int64_t)r * kv.max_pages + old_pages + j]] = 0;
      if (!grown && add) flag(kv.status, kStatusPages);
      p.len_out[r] = grown ? n + add : n;
      if (kv.grown) kv.grown[r] = grown ? add : 0;
    }
    dry = dry || found < total;
    __syncthreads();
  }
}

// ---------------------------------------------------------------- append

struct AppendParams {
  KvView kv;
  const uint4 *k_new, *v_new;
  const int32_t* start;
  int64_t new_words;        // 16-byte words between tokens
  int n_tokens, row_words;  // words of a token and head
  int elem_shift;           // log2 of the elements in a word
  FastDiv per_token, per_head;
};

constexpr int kAppendTokens = 8;

// A CTA writes eight tokens: the page of each is looked up once, then its words are moved.  Bound: HBM (80 us for 64 ragged
// prompts in fp32, 270 MB read and as many written).
__global__ void __launch_bounds__(256) append_kernel(const __grid_constant__ AppendParams p) {
  __shared__ int64_t slot[kAppendTokens];       // element offset of the token's head 0, -1: none
  const KvView& kv = p.kv;
  const int t0 = blockIdx.x * kAppendTokens;
  if (threadIdx.x < kAppendTokens) {
    const int t = t0 + threadIdx.x;
    int64_t at = -1;
    if (t < p.n_tokens) {
      int row = t, pos = -1;
      int last = 1;                             // place of the token from the row's end
      if (p.start) {
        int lo = 0, hi = kv.n_rows;             // first row whose end is past t
        while (lo < hi) {
          const int mid = (lo + hi) >> 1;
          if (p.start[mid + 1] <= t) lo = mid + 1; else hi = mid;
        }
        row = lo;
        if (row < kv.n_rows && t >= p.start[row]) {
          last = p.start[row + 1] - t;
          pos = row_len(kv, row) - last;
        }
      } else if (row < kv.n_rows) {
        pos = row_len(kv, row) - 1;
      }
      const bool left_out = row < kv.n_rows && !has_room(kv, row, last);
      if (pos >= 0 && !left_out) {
        const int page = kv.table[(int64_t)row * kv.max_pages + pos / kv.page_size];
        if ((unsigned int)page < (unsigned int)kv.n_pages)
          at = page * kv.page_stride + (int64_t)(pos % kv.page_size) * kv.head_dim;
      }
      if (at < 0 && !left_out) flag(kv.status, kStatusIndex);
    }
    slot[threadIdx.x] = at;
  }
  __syncthreads();
  // four words of K and of V a thread under way at a time
  constexpr int kAhead = 4;
  const int total = kAppendTokens * (int)p.per_token.d;
  for (int i0 = threadIdx.x; i0 < total; i0 += 256 * kAhead) {
    uint4 k[kAhead], v[kAhead];
    int64_t to[kAhead];
#pragma unroll
    for (int e = 0; e < kAhead; ++e) {
      const int i = i0 + e * 256;
      to[e] = -1;
      if (i >= total) continue;
      const int tok = (int)div_by(i, p.per_token), w = i - tok * (int)p.per_token.d;
      const int h = (int)div_by(w, p.per_head), c = w - h * p.row_words;
      const int64_t at = slot[tok];
      if (at < 0) continue;
      to[e] = ((at + (int64_t)h * kv.page_size * kv.head_dim) >> p.elem_shift) + c;
      const int64_t from = (t0 + tok) * p.new_words + w;
      k[e] = __ldcs(p.k_new + from);
      v[e] = __ldcs(p.v_new + from);
    }
#pragma unroll
    for (int e = 0; e < kAhead; ++e)
      if (to[e] >= 0) {
        ((uint4*)kv.k)[to[e]] = k[e];
        ((uint4*)kv.v)[to[e]] = v[e];
      }
  }
}

static bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return x < y + nb && y < x + na;
}

}  // namespace pg

extern "C" {

size_t pg_kv_fork_workspace_bytes(const pg_kv* kv, int32_t n_out) {
  if (pg::kv_check(kv) != PG_OK || n_out < 0 || n_out > pg::kMostItems || pg::copy_pieces(kv) == 0) return 0;
  return pg::fork_work(nullptr, n_out, nullptr);
}

int pg_kv_fork(const pg_kv* kv, int32_t n_out, const int32_t* src_rows, int32_t* table_out, int32_t* len_out,
               const int32_t* refs, int32_t* refs_out, void* workspace, size_t workspace_bytes, int32_t* status,
               void* stream) {
  pg::TraceRange trace_range("pg_kv_fork");
  const int rc = pg::kv_check(kv);
  if (rc != PG_OK) return rc;
  if (n_out < 0 || n_out > pg::kMostItems || pg::copy_pieces(kv) == 0 || !refs || !refs_out) return PG_EINVAL;
  if (n_out > 0 && (!src_rows || !table_out || !len_out)) return PG_EINVAL;
  if (!workspace || ((uintptr_t)workspace & 15) || workspace_bytes < pg_kv_fork_workspace_bytes(kv, n_out)) return PG_EINVAL;
  if ((int64_t)kv->n_rows + n_out > 0x7FFFFFFFLL) return PG_EINVAL;
  const size_t in_t = (size_t)kv->n_rows * kv->max_pages * 4, out_t = (size_t)n_out * kv->max_pages * 4;
  if (n_out > 0 && kv->n_rows > 0 &&
      (pg::overlap(table_out, out_t, kv->table, in_t) || pg::overlap(len_out, (size_t)n_out * 4, kv->len, (size_t)kv->n_rows * 4)))
    return PG_EINVAL;
  cudaStream_t st = (cudaStream_t)stream;
  if (refs != refs_out) PG_CUDA(cudaMemcpyAsync(refs_out, refs, (size_t)kv->n_pages * 4, cudaMemcpyDeviceToDevice, st));
  if (kv->n_rows + n_out == 0) return PG_OK;
  pg::ForkParams p;
  p.kv = pg::kv_view(kv, status);
  p.src = src_rows; p.table_out = table_out; p.len_out = len_out; p.refs = refs_out; p.n_out = n_out;
  pg::fork_work((char*)workspace, n_out, &p.w);
  // few old rows: one a CTA; many: as many as leave two CTAs per SM
  p.rows = (int)std::min<int64_t>(std::max<int64_t>(kv->n_rows / (148 * 2), 1), pg::kForkRows);
  const unsigned ctas = (unsigned)std::max<int64_t>(((int64_t)kv->n_rows + p.rows - 1) / p.rows, 1);
  pg::fork_kernel<<<ctas, pg::kForkThreads, 0, st>>>(p);
  PG_LAUNCH_CHECK();
  if (n_out == 0) return PG_OK;
  return pg::launch_copy(kv, p.kv, p.w.pairs, p.w.n_pairs, n_out, 8, nullptr, nullptr, st);
}

size_t pg_kv_pack_workspace_bytes(const pg_kv* kv) {
  if (pg::kv_check(kv) != PG_OK || pg::copy_pieces(kv) == 0) return 0;
  return pg::pack_work(nullptr, kv->n_pages, nullptr);
}

int pg_kv_pack(const pg_kv* kv, const int32_t* refs, int32_t* refs_out, int32_t* table_out, int32_t* page_map,
               void* workspace, size_t workspace_bytes, int32_t* status, void* stream) {
  pg::TraceRange trace_range("pg_kv_pack");
  const int rc = pg::kv_check(kv);
  if (rc != PG_OK) return rc;
  if (pg::copy_pieces(kv) == 0 || !refs || !refs_out || (kv->n_rows > 0 && !table_out)) return PG_EINVAL;
  if (!workspace || ((uintptr_t)workspace & 15) || workspace_bytes < pg_kv_pack_workspace_bytes(kv)) return PG_EINVAL;
  const size_t t = (size_t)kv->n_rows * kv->max_pages * 4;
  if (kv->n_rows > 0 && table_out != kv->table && pg::overlap(table_out, t, kv->table, t)) return PG_EINVAL;
  cudaStream_t st = (cudaStream_t)stream;
  pg::PackParams p;
  p.copy_refs = refs != refs_out && kv->n_pages <= pg::kCopyCounts;
  if (refs != refs_out && !p.copy_refs)
    PG_CUDA(cudaMemcpyAsync(refs_out, refs, (size_t)kv->n_pages * 4, cudaMemcpyDeviceToDevice, st));
  p.kv = pg::kv_view(kv, status);
  p.refs = refs; p.refs_out = refs_out; p.table_out = table_out; p.page_map = page_map;
  pg::pack_work((char*)workspace, kv->n_pages, &p.w);
  pg::pack_plan_kernel<<<1, pg::kScanThreads, 0, st>>>(p);
  PG_LAUNCH_CHECK();
  return pg::launch_copy(kv, p.kv, p.w.pairs, p.w.n_pairs, kv->n_pages / 2, 1, p.w.to, kv->n_rows > 0 ? table_out : nullptr, st);
}

int pg_kv_extend(const pg_kv* kv, const int32_t* n_new, int32_t n_uniform, int32_t* len_out, const int32_t* refs,
                 int32_t* refs_out, int32_t* status, void* stream) {
  pg::TraceRange trace_range("pg_kv_extend");
  const int rc = pg::kv_check(kv);
  if (rc != PG_OK) return rc;
  if ((!n_new && n_uniform < 0) || !refs || !refs_out || (kv->n_rows > 0 && !len_out)) return PG_EINVAL;
  cudaStream_t st = (cudaStream_t)stream;
  if (refs != refs_out) PG_CUDA(cudaMemcpyAsync(refs_out, refs, (size_t)kv->n_pages * 4, cudaMemcpyDeviceToDevice, st));
  if (kv->n_rows == 0) return PG_OK;
  pg::ExtendParams p;
  p.kv = pg::kv_view(kv, status);
  p.n_new = n_new; p.n_uniform = n_uniform; p.len_out = len_out; p.refs = refs_out;
  pg::extend_kernel<<<1, pg::kScanThreads, 0, st>>>(p);
  PG_LAUNCH_CHECK();
  return PG_OK;
}

int pg_kv_append(const pg_kv* kv, int32_t layer, int32_t n_tokens, const void* k_new, const void* v_new,
                 int64_t new_stride, const int32_t* start, int32_t* status, void* stream) {
  pg::TraceRange trace_range("pg_kv_append");
  const int rc = pg::kv_check(kv);
  if (rc != PG_OK) return rc;
  if (layer < 0 || layer >= kv->n_layers || n_tokens < 0) return PG_EINVAL;
  if (!start && n_tokens != kv->n_rows) return PG_EINVAL;
  if (n_tokens == 0) return PG_OK;
  const size_t b = pg::dtype_bytes(kv->dtype);
  const int64_t dense = (int64_t)kv->n_kv_heads * kv->head_dim;
  if (new_stride == 0) new_stride = dense;
  if (!k_new || !v_new || (((uintptr_t)k_new | (uintptr_t)v_new) & 15) || new_stride < dense || (new_stride * b & 15))
    return PG_EINVAL;
  pg::AppendParams p;
  p.kv = pg::kv_view(kv, status);
  p.kv.k = (char*)kv->k + (size_t)layer * p.kv.layer_stride * b;
  p.kv.v = (char*)kv->v + (size_t)layer * p.kv.layer_stride * b;
  p.k_new = (const uint4*)k_new; p.v_new = (const uint4*)v_new;
  p.start = start;
  p.new_words = new_stride * (int64_t)b / 16;
  p.n_tokens = n_tokens;
  p.row_words = (int)(kv->head_dim * b / 16);
  p.elem_shift = b == 4 ? 2 : 3;
  if ((int64_t)kv->n_kv_heads * p.row_words > (1 << 24)) return PG_EINVAL;
  p.per_token = pg::fast_div((uint32_t)(kv->n_kv_heads * p.row_words));
  p.per_head = pg::fast_div((uint32_t)p.row_words);
  pg::append_kernel<<<(unsigned)((n_tokens + (int64_t)pg::kAppendTokens - 1) / pg::kAppendTokens), 256, 0, (cudaStream_t)stream>>>(p);
  PG_LAUNCH_CHECK();
  return PG_OK;
}

int pg_kv_status(const int32_t* status, void* stream) {
  if (!status) return PG_EINVAL;
  int32_t word = 0;
  PG_CUDA(cudaMemcpyAsync(&word, status, sizeof(word), cudaMemcpyDeviceToHost, (cudaStream_t)stream));
  PG_CUDA(cudaStreamSynchronize((cudaStream_t)stream));
  if (word & pg::kStatusIndex) return PG_EINDEX;
  if (word & pg::kStatusTimeout) return PG_ETIMEOUT;
  if (word & pg::kStatusPages) return PG_ENOPAGES;
  return PG_OK;
}

}  // extern "C"
