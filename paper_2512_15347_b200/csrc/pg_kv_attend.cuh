// Pieces shared by the attention kernels: parameters, the shared part of a group, asynchronous copies.
#pragma once

#include "pg_kv.cuh"

namespace pg {

constexpr int kSms = 148;
constexpr int kMaxWarps = 8;
constexpr int kMaxHeads = 16;                 // query heads of a (row, kv head) piece
static_assert(kSms * sizeof(unsigned int) <= kCounterBytes, "a ticket for every CTA");

// The bounded waits of the attention; bit k of AttendParams::lost_waits makes those of kind k run out at once.
enum class TokenWait : int { kTiles, kStages, kQueries, kScores, kWeights, kProducts, kChunks, kKinds };

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
  int q_words, out_words;                     // rows of q / out on 4-byte boundaries
  float scale_log2;                           // scale * log2(e)
  uint32_t lost_waits;                        // pg_selftest_token_waits
  FastDiv page, group_div;
  // shared pages of groups (shared != null), pg_kv_shared.cu
  int q_blocks, block_rows, block_queries;    // query blocks of a (group, kv head); rows and places of queries of a block
  int2* spans;                                // [units]: first and last CTA with a part of the unit
  float* shared_out;                          // [CTAs + units]: (m, l) [block_queries][2], then o [block_queries][head_dim]
  unsigned int* tickets;                      // [CTAs], zero between calls
  float* parts;                               // [2 * CTAs][REGS * 32 + 2 * kMaxHeads]
  float* dumps;                               // [CTAs][kWarps][REGS * 32]
};

#ifdef __CUDACC__
__device__ __forceinline__ int wait_limit(const AttendParams& p, TokenWait kind, int limit) {
  return p.lost_waits >> (int)kind & 1u ? 0 : limit;
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

// The unit of (group, kv head) that holds the queries of the group's row n, and their first column in it.
// The line of all units' tiles was cut into parts; CTA c left its part of unit u in block c + u (the pairs (c, u)
// that occur form a monotone path), and spans[u] holds the first and the last c.
__device__ __forceinline__ int shared_unit(const AttendParams& p, int group, int n, int h, int* column) {
  const int block = p.q_blocks == 1 ? 0 : n / p.block_rows;
  *column = (n - block * p.block_rows) * p.per_kv;
  return (group * p.kv.n_kv_heads + h) * p.q_blocks + block;
}
__device__ __forceinline__ float* shared_block(const AttendParams& p, int cta, int unit) {
  return p.shared_out + (size_t)(cta + unit) * p.block_queries * (p.kv.head_dim + 2);
}
#endif

// pg_kv_shared.cu: the shared part of groups against the queries of all their rows
bool shared_blocks(int group, int per_kv, int head_dim, int* blocks, int* rows, int* queries);
int launch_shared(const AttendParams& p, int dtype, cudaStream_t stream);

}  // namespace pg
