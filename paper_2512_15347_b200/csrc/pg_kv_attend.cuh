// Pieces shared by the attention kernels: parameters, the shared part of a group, asynchronous copies.
#pragma once

#include "pg_kv.cuh"

namespace pg {

constexpr int kSms = 148;
constexpr int kMaxWarps = 8;
constexpr int kMaxHeads = 16;                 // query heads of a (row, kv head) piece
constexpr size_t kTicketBytes = 4096;         // >= 4 * kSms

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

struct AttendParams {
  KvView kv;
  const void* q;
  const void *k_new, *v_new;
  void* out;
  float* lse;
  const int32_t* shared;
  int64_t q_stride, new_stride, out_stride;   // elements
  int n_q_heads, per_kv, group;
  int n_split, piece_heads;                   // pieces per kv head, query heads of a piece
  float scale_log2;                           // scale * log2(e)
  FastDiv page;
  // shared pages of groups (shared != null), pg_kv_shared.cu
  int q_blocks, block_rows, block_queries;    // query blocks of a (group, kv head); rows and places of queries of a block
  long long* line;                            // [groups + 1]: the groups' first tiles on the line of shared tiles, and the quota
  float* shared_out;                          // [CTAs + units]: (m, l) [block_queries][2], then o [block_queries][head_dim]
  unsigned int* tickets;                      // [CTAs], zero between calls
  float* parts;                               // [2 * CTAs][REGS * 32 + 2 * kMaxHeads]
  float* dumps;                               // [CTAs][kWarps][REGS * 32]
};

#ifdef __CUDACC__
__device__ __forceinline__ uint32_t div_by(uint32_t n, const FastDiv& f) {
  return f.d == 1 ? n : __umulhi(n, f.m) >> f.s;
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t shared_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void copy_async(uint32_t dst, const void* src, bool some) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(some ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// ---------------------------------------------------------------- pages shared by a group
constexpr int kTile = 64;            // tokens of a tile of the shared part
constexpr int kMinShared = 64;       // fewer shared tokens are read row by row

// Tokens of group g that are computed once for its rows: whole tiles, and at least the last token of
// the first row (through whose table they are read) stays outside.
__device__ __forceinline__ int group_tokens(const AttendParams& p, int g) {
  if (!p.shared) return 0;
  const int n = min(p.shared[g], checked_len(p.kv, p.kv.len[g * p.group]) - 1);
  return n < kMinShared ? 0 : n / kTile * kTile;
}

// Where the shared part of a (row, piece) lies: its unit's line of tiles was cut at multiples of `quota`
// tiles, CTA c left the part of unit u in block c + u (the pairs (c, u) that occur form a monotone path).
struct SharedParts {
  int cta0, cta1, unit, column;      // cta1 < cta0: none
};
__device__ __forceinline__ SharedParts shared_parts(const AttendParams& p, int row, int head0) {
  const int g = row / p.group, tiles = group_tokens(p, g) / kTile;
  const int h = head0 / p.per_kv, n = row - g * p.group, block = n / p.block_rows;
  const int local = h * p.q_blocks + block;
  SharedParts s;
  s.cta0 = 0;
  s.cta1 = -1;
  if (tiles == 0) return s;
  const long long first = p.line[g] + (long long)local * tiles, quota = p.line[p.kv.n_rows / p.group];
  s.cta0 = (int)(first / quota);
  s.cta1 = (int)((first + tiles - 1) / quota);
  s.unit = g * p.kv.n_kv_heads * p.q_blocks + local;
  s.column = (n - block * p.block_rows) * p.per_kv + head0 - h * p.per_kv;
  return s;
}
__device__ __forceinline__ float* shared_part(const AttendParams& p, const SharedParts& s, int cta) {
  return p.shared_out + (size_t)(cta + s.unit) * p.block_queries * (p.kv.head_dim + 2);
}
#endif

// pg_kv_shared.cu: the shared part of groups against the queries of all their rows
bool shared_blocks(int group, int per_kv, int head_dim, int* blocks, int* rows, int* queries);
int launch_shared(const AttendParams& p, int dtype, cudaStream_t stream);

}  // namespace pg
