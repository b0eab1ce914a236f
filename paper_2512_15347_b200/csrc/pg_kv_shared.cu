// The shared part of pg_kv_attend: the tokens whose pages all rows of a group have in common (a prompt
// after its expansion) against the queries of all those rows at once.
//
// A unit is (group, kv head, block of queries): S = Q K^T, O += P V with up to 128 queries as the rows of
// the product, so a group of N rows reads the shared keys and values once instead of N times, and the
// work becomes a dense product of group * per_kv flop per byte.  The fifth-generation tensor cores do it:
//   loader warps    gather 64-token tiles of K and V from the pages with 16-byte asynchronous copies,
//                   laid out in the 128-byte swizzle that the tensor cores read (K along its head
//                   dimension, V along it too, i.e. transposed as an operand), up to three tiles ahead
//   one MMA thread  issues S_t = Q_t K^T and O_t += P_t V into tensor memory
//   softmax warps   a warpgroup for each of the (up to two) 128-query tiles t: a thread owns a query row,
//                   reads its S, keeps its maximum and sum, writes P (rounded to the cache's type) to
//                   shared memory
// so that one tile's softmax runs under the other tile's products.  The maximum that P is taken against
// is only raised when it has grown by more than kSlack (in powers of two): P stays below 2^kSlack, sums
// stay exact, and O is rescaled a few times per unit instead of every tile.  fp16 has 2^15 of room above 1 and weights of full
// precision down to 2^-14 only: there the slack is smaller, and all weights are 2^kLift times as large (the rows' own part
// does the same; joins scale alike).
// The tiles of all units form one line cut into equal parts over the CTAs; every (CTA, unit) leaves its
// queries' (m, l, O), and the rows' own pieces start from them.
// Measured: 768 rows in groups of 48 (192 queries a kv head) over 2048 shared tokens, bf16, 8 kv heads x 128: about 66 us
// for 25.8 GFLOP and 134 MB; the legacy mma path took 140 us.  Bound now: latency, not a pipe - 3700 cycles for a 64-token tile
// on average, at 27 % of the tensor pipe, 27 % issue and 2.3 TB/s, with most stalls on loads; which of the roles holds the
// others up has not been measured.
// Every wait is bounded: when one runs out, status bit 1 is set and its warp leaves, then those that wait for it (the
// results are not valid; pg_kv_status returns PG_ETIMEOUT).  What the rows' own kernel follows is in place before the first wait.
#include "pg_kv_attend.cuh"

#include <type_traits>

namespace pg {

constexpr int kRows = 128;           // queries of a product
template <typename T> struct Room {            // of a weight of type T, in powers of two
  static constexpr float kSlack = 8.f, kLift = 0.f;
};
template <> struct Room<__half> {
  // Together at most 15.  768 rows in groups of 48 in fp16: 165.0 us with 8 + 7, 165.3 with 2 + 13, 166.3 with 0 + 15.
  static constexpr float kSlack = 2.f, kLift = 13.f;
};
constexpr float kFarScore = 4194304.f;         // 2^22: half a unit in the last place is 2^-2
constexpr int kWaitLimit = 1 << 14;

// Two tiles of 128 queries share the tensor memory with their scores up to head dim 128, one above.
static int slots_of(int head_dim) { return head_dim > 128 ? 1 : 2; }

bool shared_blocks(int group, int per_kv, int head_dim, int* blocks, int* rows, int* queries) {
  const int most = kRows * slots_of(head_dim);
  if (per_kv > most) return false;             // a row alone does not fit: its group is read row by row
  *blocks = (group + most / per_kv - 1) / (most / per_kv);
  *rows = (group + *blocks - 1) / *blocks;
  *queries = most;
  return true;
}

#ifdef __CUDACC__
// ---------------------------------------------------------------- tensor core, tensor memory, barriers
// Operand tiles: blocks of 64 elements (128 bytes) of the contiguous dimension, rows 128 bytes apart,
// 16-byte piece c of row r at c ^ (r & 7).
__device__ __forceinline__ uint32_t swizzled(int row, int piece) { return row * 128 + ((piece ^ (row & 7)) << 4); }
// Shared-memory matrix descriptor, 128-byte swizzle: address, leading and stride offsets in 16-byte units.
__device__ __forceinline__ uint64_t matrix_desc(uint32_t addr, uint32_t leading, uint32_t stride) {
  return (uint64_t)((addr >> 4) & 0x3FFF) | (uint64_t)(leading >> 4) << 16 | (uint64_t)(stride >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
// fp32 accumulation, 16-bit inputs of one type; b_mn: B is contiguous along N.
template <typename T>
__device__ __forceinline__ constexpr uint32_t instr_desc(int n, bool b_mn) {
  const uint32_t type = std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
  return 1u << 4 | type << 7 | type << 10 | (b_mn ? 1u << 16 : 0u) | (uint32_t)(n >> 3) << 17 | (uint32_t)(kRows >> 4) << 24;
}
__device__ __forceinline__ bool elected() {
  uint32_t one;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one));
  return one != 0;
}
__device__ __forceinline__ void mma_async(uint32_t d, uint64_t a, uint64_t b, uint32_t desc, bool accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d), "l"(a), "l"(b), "r"(desc), "r"((uint32_t)accumulate) : "memory");
}
__device__ __forceinline__ void commit_to(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tmem_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void to_async_proxy() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tmem_load32(float (&r)[32], uint32_t addr) {
  uint32_t* u = reinterpret_cast<uint32_t*>(r);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];\n\t"
      "tcgen05.wait::ld.sync.aligned;"                 // in one piece: nothing may use the registers before
      : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]), "=r"(u[9]),
        "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15]), "=r"(u[16]), "=r"(u[17]), "=r"(u[18]), "=r"(u[19]),
        "=r"(u[20]), "=r"(u[21]), "=r"(u[22]), "=r"(u[23]), "=r"(u[24]), "=r"(u[25]), "=r"(u[26]), "=r"(u[27]), "=r"(u[28]), "=r"(u[29]),
        "=r"(u[30]), "=r"(u[31])
      : "r"(addr)
      : "memory");
}
__device__ __forceinline__ void tmem_store32(const float (&r)[32], uint32_t addr) {
  const uint32_t* u = reinterpret_cast<const uint32_t*>(r);
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};"
      ::"r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7]), "r"(u[8]), "r"(u[9]),
        "r"(u[10]), "r"(u[11]), "r"(u[12]), "r"(u[13]), "r"(u[14]), "r"(u[15]), "r"(u[16]), "r"(u[17]), "r"(u[18]), "r"(u[19]),
        "r"(u[20]), "r"(u[21]), "r"(u[22]), "r"(u[23]), "r"(u[24]), "r"(u[25]), "r"(u[26]), "r"(u[27]), "r"(u[28]), "r"(u[29]),
        "r"(u[30]), "r"(u[31]), "r"(addr)
      : "memory");
}
__device__ __forceinline__ void tmem_wait_store() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ uint32_t pack_pair(float a, float b, __nv_bfloat16) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t pack_pair(float a, float b, __half) {
  const __half2 v = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// Two fp32 operations in one instruction.
__device__ __forceinline__ uint64_t pair_of_floats(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void floats_of_pair(uint64_t p, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(p)); }
__device__ __forceinline__ uint64_t fma_pair(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add_pair(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// A tile of the line: tile `tile` of unit `local` of group `group`, whose units have `tiles` tiles.
struct TilePlace {
  int group, tiles, local, tile;
  __device__ __forceinline__ void next_unit(const AttendParams& p, int units) {
    tile = 0;
    if (++local < units) return;
    local = 0;
    do {
      if (++group >= p.kv.n_rows / p.group) return;
      tiles = group_tokens(p, group) / kTile;
    } while (tiles == 0);
  }
};

template <int DP, int kSlots>
struct SharedLayout {
  static constexpr int kBlocks = DP / 64;                         // 64-element blocks of the head dimension
  static constexpr int kStages = 3 - (DP > 128);
  static constexpr int kKBytes = kBlocks * kTile * 128, kStageBytes = 2 * kKBytes;
  static constexpr int kQBytes = kBlocks * kRows * 128, kPBytes = kRows * 128;
  static constexpr int kBytes = kStages * kStageBytes + kSlots * (kQBytes + kPBytes) + 1024;
  static constexpr int kThreads = kSlots * kRows + kStages * 32 + 32;
  static constexpr int kColumns = 512;                             // tensor memory: two S and an O for every slot
  static_assert(kSlots * (2 * kTile + DP) <= kColumns, "tensor memory");
};

template <typename T, int DP, int kSlots>
__global__ void __launch_bounds__(SharedLayout<DP, kSlots>::kThreads, 1) shared_kernel(const __grid_constant__ AttendParams p) {
  using L = SharedLayout<DP, kSlots>;
  constexpr int kThreads = L::kThreads, kWarps = kThreads / 32, kStages = L::kStages;
  extern __shared__ char smem_raw[];
  __shared__ long long warp_sum_[kWarps];
  __shared__ int first_group;
  __shared__ long long first_tile;                    // within the group
  __shared__ uint32_t tmem_base;
  __shared__ __align__(8) uint64_t bars[2 * kStages + 5 * kSlots + 1];
  const KvView& kv = p.kv;
  // (broadcasts tell the compiler what is the same for the warp: the products' operands are uniform registers)
  const int warp = __shfl_sync(0xFFFFFFFFu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const int groups = kv.n_rows / p.group, units = kv.n_kv_heads * p.q_blocks;    // of a group
  char* smem = smem_raw + (-(int)shared_addr(smem_raw) & 1023);

  // planning, as for the rows' own chunks
  const int per = (groups + kThreads - 1) / kThreads;
  const int g0 = min((int)threadIdx.x * per, groups), g1 = min(g0 + per, groups);
  long long mine = 0;
  for (int g = g0; g < g1; ++g) mine += (long long)(group_tokens(p, g) / kTile) * units;
  long long upto = mine;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const long long y = __shfl_up_sync(0xFFFFFFFFu, upto, d);
    if (lane >= d) upto += y;
  }
  if (lane == 31) warp_sum_[warp] = upto;
  __syncthreads();
  long long total = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w < warp) upto += warp_sum_[w];
    total += warp_sum_[w];
  }
  // parts of at least four tiles: a part leaves more bytes behind than a tile has
  const long long quota = max((total + gridDim.x - 1) / gridDim.x, 4ll);
  const long long begin = blockIdx.x * quota;
  const int count = __shfl_sync(0xFFFFFFFFu, (int)max(0ll, min(quota, total - begin)), 0);
  if (count == 0) return;
  if (begin >= upto - mine && begin < upto) {
    long long rest = begin - (upto - mine);
    for (int g = g0; g < g1; ++g) {
      const long long n = (long long)(group_tokens(p, g) / kTile) * units;
      if (rest < n) {
        first_group = g;
        first_tile = rest;
        break;
      }
      rest -= n;
    }
  }

  // barriers: tiles full / empty; queries in place, S ready, P in place, O done for every slot
  const uint32_t bar0 = shared_addr(bars);
  auto full = [&](int s) { return bar0 + 8 * s; };
  auto empty = [&](int s) { return bar0 + 8 * (kStages + s); };
  auto q_full = [&](int t) { return bar0 + 8 * (2 * kStages + t); };
  auto p_full = [&](int t) { return bar0 + 8 * (2 * kStages + kSlots + t); };
  auto o_done = [&](int t) { return bar0 + 8 * (2 * kStages + 2 * kSlots + t); };
  auto s_full = [&](int t, int tile) { return bar0 + 8 * (2 * kStages + 3 * kSlots + 2 * t + (tile & 1)); };   // S is double buffered
  const uint32_t drained = bar0 + 8 * (2 * kStages + 5 * kSlots);
  if (threadIdx.x == 0) {
    auto init = [](uint32_t b, int n) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(b), "r"(n) : "memory"); };
    for (int s = 0; s < kStages; ++s) {
      init(full(s), 32);
      init(empty(s), 1);
    }
    for (int t = 0; t < kSlots; ++t) {
      init(q_full(t), kRows);
      init(s_full(t, 0), 1);
      init(s_full(t, 1), 1);
      init(p_full(t), kRows);
      init(o_done(t), 1);
    }
    init(drained, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kWarps - 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(shared_addr(&tmem_base)), "n"(L::kColumns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  tmem_before();
  __syncthreads();
  tmem_after();
  const uint32_t tmem = tmem_base;
  // A bounded wait of a whole warp.  The warp votes, so that it goes on or leaves as one: what follows the waits (tensor
  // memory, votes, shuffles) needs all its lanes.  A warp leaves at its first wait that runs out; those that depend on
  // it then run out too, one each.  (A flag that spared them the wait cost 1.9 us of the 164 of the 768 rows above.)
  auto wait = [&](uint32_t bar, int parity, TokenWait kind) -> bool {
    const bool there = mbarrier_wait_bounded(bar, (unsigned)parity & 1u, wait_limit(p, kind, kWaitLimit));
    if (!there) flag(kv.status, kStatusTimeout);
    return __all_sync(0xFFFFFFFFu, there) != 0;
  };

  TilePlace here;
  here.group = first_group;
  here.tiles = group_tokens(p, first_group) / kTile;
  here.local = (int)(first_tile / here.tiles);
  here.tile = (int)(first_tile - (long long)here.local * here.tiles);
  const uint32_t ring = shared_addr(smem), q_at = ring + kStages * L::kStageBytes, p_at = q_at + kSlots * L::kQBytes;
  // queries of a block: whole rows, in order; slot t takes 128 of them
  auto block_queries = [&](int local) {
    const int block = local % p.q_blocks;
    return (min(p.group, (block + 1) * p.block_rows) - block * p.block_rows) * p.per_kv;
  };

  if (warp < kSlots * 4) {
    // ------------------------------------------------------------ softmax: a thread per query
    const int t = warp >> 2, row = threadIdx.x & (kRows - 1);
    const uint32_t lanes = (uint32_t)(warp & 3) << 21;               // tensor-memory lanes 32 (warp % 4) ..
    const uint32_t s_addr = tmem + lanes + t * 2 * kTile, o_addr = tmem + lanes + kSlots * 2 * kTile + t * DP;
    const float scale = fabsf(p.scale_log2);                         // a negative one goes into the queries' signs
    const uint32_t sign = p.scale_log2 < 0.f ? 0x80008000u : 0u;
    const bool aligned = (((uintptr_t)p.q | (p.q_stride * sizeof(T))) & 15) == 0;
    int tiles_done = 0;                                              // of this slot
    bool ok = true;
    for (int done = 0; ok && done < count;) {
      const int n = min(here.tiles - here.tile, count - done);
      const int h = here.local / p.q_blocks, block = here.local - h * p.q_blocks;
      const int queries = block_queries(here.local);
      if (t * kRows < queries) {
        const int c = t * kRows + row, q = block * p.block_rows * p.per_kv + min(c, queries - 1), i = q / p.per_kv;
        const int r = here.group * p.group + i;
        // a row that ends inside the shared tokens reads them by itself
        const bool mine = c < queries && checked_len(kv, kv.len[r]) > here.tiles * kTile;
        const T* src = (const T*)p.q + r * p.q_stride + (int64_t)(h * p.per_kv + q - i * p.per_kv) * kv.head_dim;
        char* dst = smem + kStages * L::kStageBytes + t * L::kQBytes;
#pragma unroll 4
        for (int c8 = 0; c8 < DP / 8; ++c8) {
          uint4 w = make_uint4(0, 0, 0, 0);
          if (mine && c8 * 8 < kv.head_dim) {
            if (aligned) {
              w = *(const uint4*)(src + c8 * 8);
            } else {
              uint32_t u[4];
#pragma unroll
              for (int k = 0; k < 4; ++k)
                u[k] = *(const uint16_t*)(src + c8 * 8 + 2 * k) | (uint32_t)*(const uint16_t*)(src + c8 * 8 + 2 * k + 1) << 16;
              w = make_uint4(u[0], u[1], u[2], u[3]);
            }
          }
          *(uint4*)(dst + (c8 >> 3) * kRows * 128 + swizzled(row, c8 & 7)) = make_uint4(w.x ^ sign, w.y ^ sign, w.z ^ sign, w.w ^ sign);
        }
        to_async_proxy();
        tmem_before();
        arrive(q_full(t));
        float m = -INFINITY, l = 0.f;
        for (int k = 0; k < n; ++k) {
          if (!wait(s_full(t, tiles_done), tiles_done >> 1, TokenWait::kScores)) { ok = false; break; }
          tmem_after();
          float s[kTile];
          const uint32_t s_here = s_addr + (tiles_done & 1) * kTile;
          tmem_load32(*reinterpret_cast<float(*)[32]>(s), s_here);
          tmem_load32(*reinterpret_cast<float(*)[32]>(s + 32), s_here + 32);
          float tops[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int j = 0; j < kTile; j += 2) tops[(j >> 1) & 3] = fmaxf(fmaxf(tops[(j >> 1) & 3], s[j]), s[j + 1]);
          const float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])) * scale;
          // the previous product has read P and updated O
          if (k > 0 && !wait(o_done(t), tiles_done - 1, TokenWait::kProducts)) { ok = false; break; }
          // Far from zero a rounded product and the fused one below differ by more than a weight can hold: there the
          // scores are scaled first, as the maximum has been.
          float by = scale;
          if (__any_sync(0xFFFFFFFFu, fabsf(top) >= kFarScore)) {
#pragma unroll
            for (int j = 0; j < kTile; ++j) s[j] *= scale;
            by = 1.f;
          }
          constexpr float kSlack = Room<T>::kSlack, kLift = Room<T>::kLift;
          const bool raise = top > __fadd_rd(m, kSlack + kLift) || m == -INFINITY;
          const float up = __fadd_ru(top, -kLift);
          float f = 1.f;
          if (raise && up > m) {
            f = exp2_fast(m - up);
            m = up;
          }
          if (k > 0 && __any_sync(0xFFFFFFFFu, f != 1.f)) {
            tmem_after();
#pragma unroll 1
            for (int d = 0; d < DP; d += 32) {
              float o[32];
              tmem_load32(o, o_addr + d);
    #pragma unroll
              for (int j = 0; j < 32; ++j) o[j] *= f;
              tmem_store32(o, o_addr + d);
            }
            tmem_wait_store();
          }
          l *= f;
          const float off = m == -INFINITY ? 0.f : m;
          char* pd = smem + kStages * L::kStageBytes + kSlots * L::kQBytes + t * L::kPBytes;
          uint64_t sums[2] = {0, 0};
          const uint64_t scale2 = pair_of_floats(by, by), off2 = pair_of_floats(-off, -off);
#pragma unroll
          for (int c8 = 0; c8 < kTile / 8; ++c8) {
            uint32_t packed[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              float x, y;
              floats_of_pair(fma_pair(pair_of_floats(s[c8 * 8 + 2 * j], s[c8 * 8 + 2 * j + 1]), scale2, off2), x, y);
              x = exp2_fast(x);
              y = exp2_fast(y);
              sums[j & 1] = add_pair(sums[j & 1], pair_of_floats(x, y));
              packed[j] = pack_pair(x, y, T());
            }
            *(uint4*)(pd + swizzled(row, c8)) = make_uint4(packed[0], packed[1], packed[2], packed[3]);
          }
          float l0, l1;
          floats_of_pair(add_pair(sums[0], sums[1]), l0, l1);
          l += l0 + l1;
          to_async_proxy();
          tmem_before();
          arrive(p_full(t));
          ++tiles_done;
        }
        if (!ok || !wait(o_done(t), tiles_done - 1, TokenWait::kProducts)) { ok = false; break; }
        tmem_after();
        float* out = shared_block(p, blockIdx.x, here.group * units + here.local);
        if (mine) __stcg((float2*)out + c, make_float2(m, l));
        float* o_out = out + 2 * p.block_queries + (size_t)c * kv.head_dim;
#pragma unroll 1
        for (int d = 0; d < DP; d += 32) {
          float o[32];
          tmem_load32(o, o_addr + d);
          if (mine) {
#pragma unroll
            for (int j = 0; j < 32; j += 4)
              if (d + j < kv.head_dim) __stcg((float4*)(o_out + d + j), make_float4(o[j], o[j + 1], o[j + 2], o[j + 3]));
          }
        }
      }
      done += n;
      if (done < count) here.next_unit(p, units);
    }
  } else if (warp < kWarps - 1) {
    // ------------------------------------------------------------ loaders: a warp for each stage
    constexpr int kPieces = DP / 8, kToks = 32 / kPieces > 0 ? 32 / kPieces : 1;     // 16-byte pieces of a token, tokens at a time
    static_assert(kPieces <= 32, "a token at a time at most");
    const int stage = warp - kSlots * 4, piece = lane % kPieces;
    const bool inside = piece < kv.head_dim / 8;
    const uint32_t kb = ring + stage * L::kStageBytes + (piece >> 3) * kTile * 128, vb = kb + L::kKBytes;
    // The spans of the part's units, before any wait: the rows' own kernel follows them whatever happens here.  By the loader that is
    // needed last (the warp that issues the products: 1.1 us more for the 768 rows above).
    if (stage == kStages - 1 && lane == 0) {
      TilePlace unit = here;
      long long line = begin - here.tile;                            // the unit's first tile on the line
      for (int done = 0; done < count;) {                            // CTAs that share a unit write the same
        p.spans[unit.group * units + unit.local] = make_int2((int)(line / quota), (int)((line + unit.tiles - 1) / quota));
        line += unit.tiles;
        done += min(unit.tiles - unit.tile, count - done);
        if (done < count) unit.next_unit(p, units);
      }
    }
    __syncwarp();
    int at = 0;                                                      // tile of the part that `here` is at
    for (int k = stage; k < count; k += kStages) {
      for (; at < k; ++at)
        if (++here.tile == here.tiles) here.next_unit(p, units);
      // a lane looks up two tokens' pages
      int64_t from[kTile / 32];
#pragma unroll
      for (int i = 0; i < kTile / 32; ++i) {
        const int tok = here.tile * kTile + i * 32 + lane, page = (int)div_by(tok, p.page);
        const int entry = kv.table[(int64_t)here.group * p.group * kv.max_pages + page];
        const bool good = (unsigned int)entry < (unsigned int)kv.n_pages;
        if (!good) flag(kv.status, kStatusIndex);
        from[i] = good ? entry * kv.page_stride + ((int64_t)(here.local / p.q_blocks) * kv.page_size + tok - page * kv.page_size) * kv.head_dim : -1;
      }
      if (k >= kStages && !wait(empty(stage), k / kStages - 1, TokenWait::kStages)) break;
#pragma unroll
      for (int i = 0; i < kTile; i += kToks) {
        const int tok = i + lane / kPieces;
        const int64_t src = __shfl_sync(0xFFFFFFFFu, from[i / 32], tok & 31);
        const bool some = src >= 0 && inside;
        const int64_t e = some ? src + piece * 8 : 0;
        copy_async(kb + swizzled(tok, piece & 7), (const T*)kv.k + e, some);
        copy_async(vb + swizzled(tok, piece & 7), (const T*)kv.v + e, some);
      }
      copy_commit();
      copy_wait<0>();
      to_async_proxy();
      arrive(full(stage));
    }
    copy_wait<0>();
  } else {
    // ------------------------------------------------------------ one warp issues the products, by one of its threads
    const uint32_t tmem_u = __shfl_sync(0xFFFFFFFFu, tmem, 0);
    const uint32_t qk = instr_desc<T>(kTile, false), pv = instr_desc<T>(DP, true);
    int tiles_done[kSlots] = {}, units_done[kSlots] = {};
    bool ok = true;
    const bool issuer = elected();
    auto scores = [&](int t, int stage, int tile) {                  // tile: counted over the slot, picks the S buffer
      const uint32_t a = q_at + t * L::kQBytes, b = ring + stage * L::kStageBytes, d = tmem_u + (2 * t + (tile & 1)) * kTile;
      if (issuer) {
#pragma unroll
        for (int s = 0; s < DP / 16; ++s)
          mma_async(d, matrix_desc(a + (s >> 2) * kRows * 128 + (s & 3) * 32, 16, 1024),
                    matrix_desc(b + (s >> 2) * kTile * 128 + (s & 3) * 32, 16, 1024), qk, s > 0);
        commit_to(s_full(t, tile));
      }
      __syncwarp();
    };
    int k = 0;                                                       // tile of the part
    for (int done = 0; ok && done < count;) {
      const int n = __shfl_sync(0xFFFFFFFFu, min(here.tiles - here.tile, count - done), 0);
      const int slots = __shfl_sync(0xFFFFFFFFu, (block_queries(here.local) + kRows - 1) / kRows, 0);
      ok = wait(full(k % kStages), k / kStages, TokenWait::kTiles);
#pragma unroll
      for (int t = 0; t < kSlots; ++t)
        if (ok && t < slots) {
          ok = wait(q_full(t), units_done[t]++, TokenWait::kQueries);
          tmem_after();
          if (ok) scores(t, k % kStages, tiles_done[t]);
        }
      for (int i = 0; ok && i < n; ++i, ++k) {
        const int stage = k % kStages, next = (k + 1) % kStages;
        const uint32_t v = ring + stage * L::kStageBytes + L::kKBytes;
        if (i + 1 < n) {                                             // the next scores run under this tile's softmax
          ok = wait(full(next), (k + 1) / kStages, TokenWait::kTiles);
          tmem_after();
#pragma unroll
          for (int t = 0; t < kSlots; ++t)
            if (ok && t < slots) scores(t, next, tiles_done[t] + 1);
        }
#pragma unroll
        for (int t = 0; t < kSlots; ++t) {
          if (!ok || t >= slots) continue;
          ok = wait(p_full(t), tiles_done[t]++, TokenWait::kWeights);
          if (!ok) continue;
          tmem_after();
          const uint32_t a = p_at + t * L::kPBytes, d = tmem_u + kSlots * 2 * kTile + t * DP;
          if (issuer) {
#pragma unroll
            for (int s = 0; s < kTile / 16; ++s)
              mma_async(d, matrix_desc(a + s * 32, 16, 1024), matrix_desc(v + s * 2048, kTile * 128, 1024), pv, i > 0 || s > 0);
            commit_to(o_done(t));
            if (t == slots - 1) commit_to(empty(stage));
          }
          __syncwarp();
        }
      }
      done += n;
      if (done < count) here.next_unit(p, units);
    }
    if (issuer) commit_to(drained);                                  // no product is in flight when the CTA leaves, whoever gave up
    __syncwarp();
    if (!mbarrier_wait_bounded(drained, 0, kWaitLimit)) flag(kv.status, kStatusTimeout);
  }
  __syncwarp();
  tmem_before();
  __syncthreads();
  tmem_after();
  if (warp == kWarps - 1)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(L::kColumns));
}
#endif

template <typename T, int DP, int kSlots>
static int launch_shared_as(const AttendParams& p, cudaStream_t st) {
  using L = SharedLayout<DP, kSlots>;
  static_assert(L::kBytes <= 224 * 1024, "shared memory");
  auto kernel = shared_kernel<T, DP, kSlots>;
  static std::atomic<uint64_t> done{0};
  if (const int rc = allow_shared(kernel, L::kBytes, done)) return rc;
  kernel<<<kSms, L::kThreads, L::kBytes, st>>>(p);
  PG_LAUNCH_CHECK();
  return PG_OK;
}
template <typename T>
static int launch_shared_type(const AttendParams& p, cudaStream_t st) {
  if (p.kv.head_dim <= 64) return launch_shared_as<T, 64, 2>(p, st);
  if (p.kv.head_dim <= 128) return launch_shared_as<T, 128, 2>(p, st);
  return launch_shared_as<T, 256, 1>(p, st);
}
int launch_shared(const AttendParams& p, int dtype, cudaStream_t st) {
  return dtype == PG_BF16 ? launch_shared_type<__nv_bfloat16>(p, st) : launch_shared_type<__half>(p, st);
}

}  // namespace pg
