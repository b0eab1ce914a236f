// Attention of one new token per row over the paged cache (pg_kv_attend).
//
// For each query head:  out = sum_t p_t v_t,  p = softmax(scale q.k_t),  lse = ln sum_t exp(scale q.k_t),
// in one pass over the tokens with a running maximum m, sum l and accumulator o per warp:
//     m' = max(m, max_t x_t),  l' = l 2^(m-m') + sum 2^(x_t-m'),  o' = o 2^(m-m') + sum 2^(x_t-m') v_t
// with x = scale log2(e) q.k; two such triples over disjoint tokens join by the same rule, which is how
// warps, and the CTAs that share a row, are put together.
//
// Bound: HBM.  A token's K and V of one kv head are 4 D bytes (16-bit) for 4 D flops per query head that
// shares them, i.e. per_kv flop per byte; every byte is read once, by one warp, for all query heads of
// its kv head.
//
// Work split.  The unit is a chunk: the K and V of kChunk consecutive tokens of one (row, kv head).  All
// chunks of the call, ordered (row, kv head, chunk), form one line - each piece (row, kv head) a few units
// longer than it has chunks, for what it costs besides them - that the warps of the resident CTAs cut into
// equal parts, so ragged lengths, one long row and many short ones all balance; the cuts follow from the
// lengths in device memory (every CTA sums them itself), nothing is planned on the host.  A warp streams
// its run of the line through a ring of kStages buffers of its own and finishes the pieces that it sees
// whole without waiting for anybody.  The two it may share are joined once at the end, first in the CTA, and
// where a cut between CTAs has split a piece, by the CTA that arrives last (wait-free ticket; parts are
// added in CTA order, so the bits do not depend on who that is).
// Measured on a B200 (bf16 / fp16, 32 query and 8 kv heads x 128): one row of 131071 tokens 105 us (5.1 TB/s), 96 rows
// of 1..8192 tokens 82 us (4.4 TB/s).  Bound now: the former by HBM and the join of the 18 parts of a piece, the
// latter by latency: two warps a scheduler, each a chain of scores, maximum, exponentials and second product, issue 0.21
// instructions a cycle (stalled by results of fixed latency, looked-up lengths and pages, and copies, about alike).  fp32:
// 313 us and 258 us, 1.9 and 2.3 times what its bytes take.
#include "pg_kv_attend.cuh"
#include "pg_trace.cuh"

#include <cuda.h>

#include <type_traits>

namespace pg {

#ifdef __CUDACC__
__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ void expect_bytes(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_tensor(uint32_t dst, const CUtensorMap* map, int row, int page, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %2, %4}], [%5];" ::"r"(dst),
      "l"(map), "r"(0), "r"(row), "r"(page), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void copy_bulk(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes),
               "r"(bar)
               : "memory");
}
template <typename T>
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (sizeof(T) == 2 && std::is_same<T, __nv_bfloat16>::value)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack2(float a, float b, __nv_bfloat16) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t pack2(float a, float b, __half) {
  const __half2 v = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// ---------------------------------------------------------------- bodies: one warp, one chunk at a time
// A body holds a warp's triple for up to NT * 8 query heads over head dimensions padded to DP (copies
// fill what is past head_dim with zeros).  o[REGS] is its part of the accumulator; head_of / dim_of say
// which element lane `lane` holds in register i.

// 16-bit: tensor cores, with keys as the rows of the product (S^T = K Q^T, O^T = V^T P^T), so that a kv
// head with few query heads fills the n = 8 side instead of padding m = 16.  P^T comes from S^T's
// accumulators by an 8x8 register transposition; P is rounded to the cache's type for the product (the
// sum l is taken before the rounding): one more error of the size of the result's own rounding, and independent from token to
// token (bf16, 96 ragged rows: 1.6e-3 of the result against 1.5e-3 for the plain form in fp32).  fp16 has weights of full
// precision down to 2^-14 only, and none below 2^-25, which many small ones beside a large one would be missed by: its m is
// kept kLift powers of two below the largest score, so that P, l and o are 2^kLift times as large.
template <typename T, int DP, int NT, int kKeys>
struct MmaBody {
  static constexpr int kChunk = kKeys;
  static constexpr int kTiles = kChunk / 16;
  static constexpr int kRegs = DP / 16 * NT * 4;
  static constexpr int kRowBytes = DP * 2;
  static constexpr size_t kQBytes = 0;              // shared memory per warp for the queries
  static constexpr float kLift = std::is_same<T, __half>::value ? 15.f : 0.f;
  float o[kRegs];
  float m[NT][2], l[NT][2];
  uint32_t q[DP / 16][NT][2];

  static __device__ __forceinline__ int head_of(int i, int lane) { return (i >> 2) % NT * 8 + (lane & 3) * 2 + (i & 1); }
  static __device__ __forceinline__ int dim_of(int i, int lane) { return (i >> 2) / NT * 16 + (lane >> 2) + ((i >> 1) & 1) * 8; }
  // of four registers 4 u .. 4 u + 3, the heads are those of the first and of the kSecond-th; which one each has
  static constexpr int kSecond = 1;
  static __device__ __forceinline__ int pair_of(int j) { return j & 1; }
  // 16-byte piece c of token t: blocks of 64 elements, tokens 128 bytes apart, pieces swizzled so that eight
  // tokens' equal pieces hit all banks (the tensor copies' 128-byte swizzle)
  static __device__ __forceinline__ uint32_t piece_at(int t, int c) {
    return (c >> 3) * kChunk * 128 + t * 128 + (((c & 7) ^ (t & 7)) << 4);
  }

  // query(g): the vector of column g of the warp, or null; words: on 4-byte boundaries
  template <typename Query>
  __device__ __forceinline__ void load_queries(int dim, bool words, int lane, Query query) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const T* qh = query(nt * 8 + (lane >> 2));
#pragma unroll
      for (int s = 0; s < DP / 16; ++s)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int d = s * 16 + j * 8 + (lane & 3) * 2;
          uint32_t w = 0;
          if (qh && d < dim) {
            if (words) w = *(const uint32_t*)(qh + d);
            else w = *(const uint16_t*)(qh + d) | (uint32_t)*(const uint16_t*)(qh + d + 1) << 16;
          }
          q[s][nt][j] = w;
        }
    }
  }

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      m[nt][0] = m[nt][1] = -INFINITY;
      l[nt][0] = l[nt][1] = 0.f;
    }
#pragma unroll
    for (int i = 0; i < kRegs; ++i) o[i] = 0.f;
  }

  __device__ __forceinline__ void begin(const AttendParams& p, int row, int head0, int heads, int lane, char*) {
    const T* base = (const T*)p.q + row * p.q_stride + (int64_t)head0 * p.kv.head_dim;
    load_queries(p.kv.head_dim, p.q_words, lane, [&](int g) { return g < heads ? base + (int64_t)g * p.kv.head_dim : (const T*)nullptr; });
    clear();
  }

  // The triple of the group's shared tokens goes in front of a row's own (sums are per lane: one of the
  // eight lanes of a head starts with the whole l).
  __device__ __forceinline__ void join_shared(const AttendParams& p, int unit, int column, int heads, int lane) {
    const int2 span = __ldcg(&p.spans[unit]);
    if ((unsigned int)span.x >= (unsigned int)kSms || (unsigned int)span.y >= (unsigned int)kSms) {   // of no CTA: nothing to join
      flag(p.kv.status, kStatusTimeout);
      return;
    }
#pragma unroll 1
    for (int c = span.x; c <= span.y; ++c) {
      const float* part = shared_block(p, c, unit);
      float f[NT][2], g[NT][2];
      const float* col[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int head = min(nt * 8 + (lane & 3) * 2 + j, heads - 1);
          col[nt][j] = part + 2 * p.block_queries + (size_t)(column + head) * p.kv.head_dim;
          const float2 s = __ldcg((const float2*)part + column + head);
          const float m2 = fmaxf(m[nt][j], s.x), off = m2 == -INFINITY ? 0.f : m2;
          f[nt][j] = exp2_fast(m[nt][j] - off);
          g[nt][j] = exp2_fast(s.x - off);
          l[nt][j] = l[nt][j] * f[nt][j] + (lane < 4 ? s.y * g[nt][j] : 0.f);
          m[nt][j] = m2;
        }
#pragma unroll
      for (int i = 0; i < kRegs; ++i) {
        const int nt = (i >> 2) % NT, j = i & 1, d = dim_of(i, lane);
        const float y = d < p.kv.head_dim ? __ldcg(col[nt][j] + d) : 0.f;
        o[i] = o[i] * f[nt][j] + y * g[nt][j];
      }
    }
  }

  // keys [t0, t0 + kChunk) in kbuf / vbuf (shared addresses), of which [lo, hi) count
  __device__ __forceinline__ void step(const AttendParams& p, uint32_t kbuf, uint32_t vbuf, const char*, int t0, int lo, int hi,
                                       int lane) {
    step_masked(p, kbuf, vbuf, t0, lane, t0 >= lo && t0 + kChunk <= hi, [&](int t, int, int) { return t >= lo && t < hi; });
  }

  // whole: keep(key, nt, j) is true throughout
  template <typename Keep>
  __device__ __forceinline__ void step_masked(const AttendParams& p, uint32_t kbuf, uint32_t vbuf, int t0, int lane, bool whole,
                                              Keep keep) {
    float s[kTiles][NT][4];
#pragma unroll
    for (int mt = 0; mt < kTiles; ++mt)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[mt][nt][j] = 0.f;
#pragma unroll
    for (int ks = 0; ks < DP / 16; ++ks)
#pragma unroll
      for (int mt = 0; mt < kTiles; ++mt) {
        uint32_t a[4];
        ldmatrix4(a, kbuf + piece_at(mt * 16 + (lane & 15), ks * 2 + (lane >> 4)));
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) mma16816<T>(s[mt][nt], a, q[ks][nt][0], q[ks][nt][1]);
      }
    float top[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      top[nt][0] = top[nt][1] = -INFINITY;
#pragma unroll
      for (int mt = 0; mt < kTiles; ++mt)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float x = s[mt][nt][j] * p.scale_log2;
          if (!whole) {
            const int t = t0 + mt * 16 + (lane >> 2) + (j >> 1) * 8;
            if (!keep(t, nt, j & 1)) x = -INFINITY;
          }
          s[mt][nt][j] = x;
          top[nt][j & 1] = fmaxf(top[nt][j & 1], x);
        }
    }
#pragma unroll
    for (int d = 4; d < 32; d <<= 1)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int j = 0; j < 2; ++j) top[nt][j] = fmaxf(top[nt][j], __shfl_xor_sync(0xFFFFFFFFu, top[nt][j], d));
    bool rose = false;
    float f[NT][2], off[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float m2 = fmaxf(m[nt][j], __fadd_ru(top[nt][j], -kLift));     // upwards: no weight is above 2^kLift
        off[nt][j] = m2 == -INFINITY ? 0.f : m2;       // nothing counted yet: every weight below is 0
        f[nt][j] = exp2_fast(m[nt][j] - off[nt][j]);
        rose |= m2 != m[nt][j];
        m[nt][j] = m2;
      }
    if (__any_sync(0xFFFFFFFFu, rose)) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        l[nt][0] *= f[nt][0];
        l[nt][1] *= f[nt][1];
      }
#pragma unroll
      for (int i = 0; i < kRegs; ++i) o[i] *= f[(i >> 2) % NT][i & 1];
    }
    uint32_t b[kTiles][NT][2];
#pragma unroll
    for (int mt = 0; mt < kTiles; ++mt)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          w[j] = exp2_fast(s[mt][nt][j] - off[nt][j & 1]);
          l[nt][j & 1] += w[j];
        }
        b[mt][nt][0] = transpose8x8(pack2(w[0], w[1], T()));
        b[mt][nt][1] = transpose8x8(pack2(w[2], w[3], T()));
      }
#pragma unroll
    for (int dt = 0; dt < DP / 16; ++dt)
#pragma unroll
      for (int mt = 0; mt < kTiles; ++mt) {
        uint32_t a[4];
        ldmatrix4_trans(a, vbuf + piece_at(mt * 16 + (lane & 7) + (lane >> 4) * 8, dt * 2 + ((lane >> 3) & 1)));
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float(&c)[4] = *reinterpret_cast<float(*)[4]>(&o[(dt * NT + nt) * 4]);
          mma16816<T>(c, a, b[mt][nt][0], b[mt][nt][1]);
        }
      }
  }

  // o / l of a piece seen whole, sums[head] = (m, l).  An 8x8 transposition of the rounded values leaves
  // a lane with two neighbouring elements of one head.
  __device__ __forceinline__ void store(const AttendParams& p, const float2* sums, int row, int head0, int heads, int lane) {
    T* out = (T*)p.out + row * p.out_stride + (int64_t)head0 * p.kv.head_dim;
    float r[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float l = sums[nt * 8 + (lane & 3) * 2 + j].y;
        r[nt][j] = l == 0.f ? 0.f : 1.f / l;
      }
#pragma unroll
    for (int i = 0; i < kRegs; i += 2) {
      const int nt = (i >> 2) % NT;
      const uint32_t w = transpose8x8(pack2(o[i] * r[nt][0], o[i + 1] * r[nt][1], T()));
      const int head = nt * 8 + (lane >> 2), d = (i >> 2) / NT * 16 + ((i >> 1) & 1) * 8 + (lane & 3) * 2;
      if (head < heads && d < p.kv.head_dim) {
        T* at = out + (int64_t)head * p.kv.head_dim + d;
        if (p.out_words) {
          *(uint32_t*)at = w;
        } else {
          ((uint16_t*)at)[0] = (uint16_t)w;
          ((uint16_t*)at)[1] = (uint16_t)(w >> 16);
        }
      }
    }
  }

  // stats[head] = (m, l), by the lanes that hold them
  __device__ __forceinline__ void stats(float2* out, int lane) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float s = l[nt][j];
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
        if (lane < 4) out[nt * 8 + lane * 2 + j] = make_float2(m[nt][j], s);
      }
  }
};

// fp32: fused multiply-adds (the tensor cores would round the inputs).  Eight lanes share a key for the
// scores, every lane owns DP / 32 dimensions for the products with V; queries and weights pass through
// shared memory.
template <int DP, int NT>
struct F32Body {
  static constexpr int kChunk = DP <= 128 ? 16 : NT == 1 ? 8 : 4;
  static constexpr int kHeads = NT * 8;
  static constexpr int kPer = DP / 32;              // elements of o and v per lane and head
  static constexpr int kRegs = kHeads * kPer;
  static constexpr int kRowBytes = DP * 4;
  static constexpr int kKeys = kChunk / 4;          // keys of a lane
  static constexpr int kVec = DP / 32;              // 16-byte pieces of a key per lane
  static constexpr size_t kQBytes = kHeads * DP * 4 + kChunk * kHeads * 4;
  static constexpr float kLift = 0.f;
  float o[kRegs];
  float m[kHeads], l[kHeads];

  static __device__ __forceinline__ int head_of(int i, int) { return i / kPer; }
  static __device__ __forceinline__ int dim_of(int i, int lane) {
    const int j = i % kPer;
    return kPer == 2 ? lane * 2 + j : (j >> 2) * 128 + lane * 4 + (j & 3);
  }
  static constexpr int kSecond = 2;
  static __device__ __forceinline__ int pair_of(int j) { return kPer == 2 ? j >> 1 : 0; }
  static __device__ __forceinline__ uint32_t piece_at(int t, int c) { return t * kRowBytes + (c << 4); }

  __device__ __forceinline__ void begin(const AttendParams& p, int row, int head0, int heads, int lane, char* scratch) {
    float* q = (float*)scratch;
    const float* base = (const float*)p.q + row * p.q_stride + (int64_t)head0 * p.kv.head_dim;
    __syncwarp();
    for (int i = lane; i < kHeads * DP; i += 32) {
      const int g = i / DP, d = i - g * DP;
      q[i] = g < heads && d < p.kv.head_dim ? base[(int64_t)g * p.kv.head_dim + d] : 0.f;
    }
    __syncwarp();
#pragma unroll
    for (int i = 0; i < kRegs; ++i) o[i] = 0.f;
#pragma unroll
    for (int g = 0; g < kHeads; ++g) { m[g] = -INFINITY; l[g] = 0.f; }
  }

  __device__ __forceinline__ void join_shared(const AttendParams&, int, int, int, int) {}

  __device__ __forceinline__ void step(const AttendParams& p, uint32_t kbuf, uint32_t vbuf, char* scratch, int t0, int lo, int hi,
                                       int lane) {
    const char* kb = (const char*)__cvta_shared_to_generic(kbuf);
    const char* vb = (const char*)__cvta_shared_to_generic(vbuf);
    const float4* q = (const float4*)scratch;
    float* w = (float*)(scratch + kHeads * DP * 4);
    const int part = lane & 7, sub = lane >> 3;
    float4 k[kKeys][kVec];
#pragma unroll
    for (int a = 0; a < kKeys; ++a)
#pragma unroll
      for (int c = 0; c < kVec; ++c) k[a][c] = *(const float4*)(kb + piece_at(a * 4 + sub, c * 8 + part));
#pragma unroll
    for (int g = 0; g < kHeads; ++g) {
      if (g >= p.piece_heads) continue;
      float s[kKeys];
#pragma unroll
      for (int a = 0; a < kKeys; ++a) s[a] = 0.f;
#pragma unroll
      for (int c = 0; c < kVec; ++c) {
        const float4 x = q[g * (DP / 4) + c * 8 + part];
#pragma unroll
        for (int a = 0; a < kKeys; ++a)
          s[a] = fmaf(x.x, k[a][c].x, fmaf(x.y, k[a][c].y, fmaf(x.z, k[a][c].z, fmaf(x.w, k[a][c].w, s[a]))));
      }
      float top = -INFINITY;
#pragma unroll
      for (int a = 0; a < kKeys; ++a) {
#pragma unroll
        for (int d = 1; d < 8; d <<= 1) s[a] += __shfl_xor_sync(0xFFFFFFFFu, s[a], d);
        const int t = t0 + a * 4 + sub;
        s[a] = t < lo || t >= hi ? -INFINITY : s[a] * p.scale_log2;
        top = fmaxf(top, s[a]);
      }
      top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 8));
      top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 16));
      const float m2 = fmaxf(m[g], top), off = m2 == -INFINITY ? 0.f : m2;
      if (m2 != m[g]) {                              // the same for all lanes
        const float f = exp2_fast(m[g] - off);
        l[g] *= f;
#pragma unroll
        for (int i = 0; i < kPer; ++i) o[g * kPer + i] *= f;
        m[g] = m2;
      }
#pragma unroll
      for (int a = 0; a < kKeys; ++a) {
        const float e = exp2_fast(s[a] - off);
        l[g] += e;                                   // eight lanes count the same key
        if (part == 0) w[(a * 4 + sub) * kHeads + g] = e;
      }
    }
    __syncwarp();
#pragma unroll 4
    for (int t = 0; t < kChunk; ++t) {
      float v[kPer];
      if constexpr (kPer == 2) {
        const float2 x = *(const float2*)(vb + t * kRowBytes + lane * 8);
        v[0] = x.x; v[1] = x.y;
      } else {
#pragma unroll
        for (int c = 0; c < kPer / 4; ++c) {
          const float4 x = *(const float4*)(vb + t * kRowBytes + c * 512 + lane * 16);
          v[c * 4] = x.x; v[c * 4 + 1] = x.y; v[c * 4 + 2] = x.z; v[c * 4 + 3] = x.w;
        }
      }
#pragma unroll
      for (int g4 = 0; g4 < kHeads; g4 += 4) {
        if (g4 >= p.piece_heads) continue;
        const float4 e = *(const float4*)(w + t * kHeads + g4);
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          o[(g4 + 0) * kPer + i] = fmaf(e.x, v[i], o[(g4 + 0) * kPer + i]);
          if (g4 + 1 < p.piece_heads) o[(g4 + 1) * kPer + i] = fmaf(e.y, v[i], o[(g4 + 1) * kPer + i]);
          if (g4 + 2 < p.piece_heads) o[(g4 + 2) * kPer + i] = fmaf(e.z, v[i], o[(g4 + 2) * kPer + i]);
          if (g4 + 3 < p.piece_heads) o[(g4 + 3) * kPer + i] = fmaf(e.w, v[i], o[(g4 + 3) * kPer + i]);
        }
      }
    }
    __syncwarp();
  }

  __device__ __forceinline__ void store(const AttendParams& p, const float2* sums, int row, int head0, int heads, int lane) {
    float* out = (float*)p.out + row * p.out_stride + (int64_t)head0 * p.kv.head_dim;
#pragma unroll
    for (int g = 0; g < kHeads; ++g) {
      if (g >= heads) continue;
      const float l = sums[g].y, r = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int d = dim_of(i, lane);
        if (d < p.kv.head_dim) out[(int64_t)g * p.kv.head_dim + d] = o[g * kPer + i] * r;
      }
    }
  }

  __device__ __forceinline__ void stats(float2* out, int lane) {
#pragma unroll
    for (int g = 0; g < kHeads; ++g) {
      float s = l[g];
      s += __shfl_xor_sync(0xFFFFFFFFu, s, 8);
      s += __shfl_xor_sync(0xFFFFFFFFu, s, 16);
      if (lane == 0) out[g] = make_float2(m[g], s);
    }
  }
};

// ---------------------------------------------------------------- the line of chunks

// A piece costs its warp more than its chunks: queries are fetched, statistics joined, results
// written.  On the line every piece is therefore kPieceCost units longer than it has chunks (768 rows in groups
// of 48: 180, 169 and 163 us with 3, 5 and 8 units; 96 ragged rows: 87, 82 and 82 us).
constexpr int kPieceCost = 8;

// Tokens [lo, hi) of a row that the line covers, in chunks [c0, c1).
struct RowSpan {
  int lo, hi, c0, c1;
  __device__ __forceinline__ int chunks() const { return c1 - c0; }
  __device__ __forceinline__ int units() const { return c1 > c0 ? c1 - c0 + kPieceCost : 0; }
};
template <int kChunk>
__device__ __forceinline__ RowSpan row_span(const AttendParams& p, int shared_tokens, int len) {
  RowSpan s;
  s.hi = checked_len(p.kv, len);
  s.lo = shared_tokens < s.hi ? shared_tokens : 0;    // a row that ends inside the shared tokens reads them by itself
  s.c0 = s.lo / kChunk;
  s.c1 = s.hi > s.lo ? (s.hi + kChunk - 1) / kChunk : s.c0;
  return s;
}
template <int kChunk>
__device__ __forceinline__ RowSpan row_span(const AttendParams& p, int row) {
  return row_span<kChunk>(p, p.shared ? group_tokens(p, (int)div_by(row, p.group_div)) : 0, p.kv.len[row]);
}

// A place on the line: unit `unit` of piece (row, kv head h, split), in that order; the first kPieceCost units of a
// piece stand for no chunk.  Divisions are kept out of the walk.
template <int kChunk>
struct Place {
  int row, h, split, unit;
  int group, n, tokens;        // row = group * p.group + n; the group's shared tokens
  int next_len;                // of the next row, fetched long before it is needed
  bool takes, next_takes;      // the row's last token is its new one; the next row's
  RowSpan span;
  static __device__ __forceinline__ bool takes_new(const AttendParams& p, int row) { return p.k_new && has_room(p.kv, row, 1); }
  __device__ __forceinline__ void fetch(const AttendParams& p) {
    if (row + 1 >= p.kv.n_rows) return;
    next_len = p.kv.len[row + 1];
    next_takes = takes_new(p, row + 1);
  }
  __device__ __forceinline__ void next_piece(const AttendParams& p) {
    unit = 0;
    if (++split < p.n_split) return;
    split = 0;
    if (++h < p.kv.n_kv_heads) return;
    h = 0;
    do {
      if (++row >= p.kv.n_rows) return;
      if (++n == p.group) {
        n = 0;
        ++group;
        tokens = p.shared ? group_tokens(p, group) : 0;
      }
      span = row_span<kChunk>(p, tokens, next_len);
      takes = next_takes;
      fetch(p);
    } while (span.c1 == span.c0);
  }
  __device__ __forceinline__ void set(const AttendParams& p, int row_, int piece, int unit_, const RowSpan& span_) {
    row = row_;
    h = piece / p.n_split;
    split = piece - h * p.n_split;
    unit = unit_;
    group = (int)div_by(row_, p.group_div);
    n = row_ - group * p.group;
    takes = takes_new(p, row_);
    tokens = p.shared ? group_tokens(p, group) : 0;
    span = span_;
  }
};

template <typename T, typename Body, int kWarps, int kStages>
struct AttendShared {
  static constexpr int kStageBytes = 2 * Body::kChunk * Body::kRowBytes;
  static constexpr size_t kRing = (size_t)kWarps * kStages * kStageBytes;
  static constexpr size_t kBytes = 1024 + kRing + kWarps * Body::kQBytes;          // the ring starts on 1024 bytes
  static_assert(Body::kRegs * 128 <= kStages * kStageBytes, "a warp's ring takes a dump of its accumulator");
};

// What a warp leaves behind of a piece that it has not seen whole.
struct Left {
  int row, h, split, chunk0;   // the piece, and the first of its chunks in this part
  long long line;              // line unit of the piece's chunk 0
  int chunks;                  // chunks of the whole piece
  int any, goes_on;            // filled; continues in the next warp
};

// The pools as the tensor copies see them: [page][64-element block of the head dimension][kv head, slot][64].
struct PoolMaps {
  CUtensorMap k, v;
};
constexpr int kBoxTokens = 16;       // tokens of a tensor copy

// kBulk: whole chunks (16 tokens of a page at a time) come by bulk copies that one lane issues - tensor
// copies with the 128-byte swizzle in 16 bits, plain ones in fp32 - instead of 16 bytes a lane.  Against the latter the
// walk takes a quarter fewer instructions (29.5 M to 22.3 M, 117 to 98 us for the own tokens of 768 rows of 1..512), which
// a warp with short pieces gains most from.
template <typename T, typename Body, int kWarps, int kStages, bool kBulk>
__global__ void __launch_bounds__(kWarps * 32, 1) attend_kernel(const __grid_constant__ AttendParams p, const __grid_constant__ PoolMaps maps) {
  using S = AttendShared<T, Body, kWarps, kStages>;
  constexpr int kThreads = kWarps * 32;
  constexpr int kChunk = Body::kChunk, kRegs = Body::kRegs;
  constexpr int kPart = kRegs * 32 + 2 * kMaxHeads;
  extern __shared__ char smem_raw[];
  char* smem = smem_raw + (-(int)shared_addr(smem_raw) & 1023);
  __shared__ __align__(8) uint64_t bars[kBulk ? kWarps * kStages : 1];
  __shared__ long long warp_sum_[kWarps];
  __shared__ int warp_max_[kWarps];
  __shared__ Place<kChunk> first[kWarps];
  __shared__ Left left[kWarps][2];                    // [0]: began before the warp's part, [1]: began in it
  __shared__ float2 stat[kWarps][2][kMaxHeads];
  __shared__ float2 sums[kMaxHeads];
  __shared__ float factor[kWarps][kMaxHeads];
  __shared__ int is_last;
  constexpr int kMaxEmpty = 64;
  __shared__ int n_empty, empty[kMaxEmpty];
  const KvView& kv = p.kv;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int pieces = kv.n_kv_heads * p.n_split;

  // Planning: the rows' units are summed, then the rows that hold this CTA's cuts are found.
  const int per = (kv.n_rows + kThreads - 1) / kThreads;
  const int r0 = min((int)threadIdx.x * per, kv.n_rows), r1 = min(r0 + per, kv.n_rows);
  const uint32_t bar = shared_addr(bars) + (kBulk ? warp * kStages * 8 : 0);
  if (kBulk && lane == 0) {
    for (int i = 0; i < kStages; ++i) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bar + 8 * i) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (threadIdx.x == 0) n_empty = 0;
  if (lane < 2) left[warp][lane].any = 0;
  __syncthreads();
  // rows without tokens, dealt round the CTAs, are cleared at the end of the planning
  auto clear_row = [&](int r, int from, int step) {
    T* out = (T*)p.out + r * p.out_stride;
    for (int i = from; i < p.n_q_heads * kv.head_dim; i += step) out[i] = from_float<T>(0.f);
    if (p.lse)
      for (int i = from; i < p.n_q_heads; i += step) p.lse[(int64_t)r * p.n_q_heads + i] = -INFINITY;
  };
  long long mine = 0;
  int longest = 0;
  for (int r = r0; r < r1; ++r) {
    const RowSpan s = row_span<kChunk>(p, r);
    mine += s.units();
    longest = max(longest, s.chunks());
    if (s.c1 == s.c0 && r % gridDim.x == blockIdx.x) {
      const int at = atomicAdd(&n_empty, 1);
      if (at < kMaxEmpty) empty[at] = r;
      else clear_row(r, 0, 1);
    }
  }
  long long upto = mine;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const long long y = __shfl_up_sync(0xFFFFFFFFu, upto, d);
    if (lane >= d) upto += y;
  }
  longest = __reduce_max_sync(0xFFFFFFFFu, longest);
  if (lane == 31) {
    warp_sum_[warp] = upto;
    warp_max_[warp] = longest;
  }
  __syncthreads();
  long long all = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w < warp) upto += warp_sum_[w];
    all += warp_sum_[w];
    longest = max(longest, warp_max_[w]);
  }
  const long long total = all * pieces;
  // Few and short rows: a CTA for every (row, piece), so that nothing is joined across CTAs.
  const bool by_piece = (long long)kv.n_rows * pieces <= gridDim.x && longest <= kWarps * 4;
  long long quota = 0, begin = 0;                     // units of a CTA's part, and its first
  long long wbegin, wend;                             // this warp's units
  if (by_piece) {
    const int r = blockIdx.x / pieces;
    if (r < kv.n_rows) {
      const RowSpan s = row_span<kChunk>(p, r);
      const int share = (s.chunks() + kWarps - 1) / kWarps, from = min(warp * share, s.chunks());
      wbegin = kPieceCost + from;                     // counted from the piece's own start
      wend = kPieceCost + min(from + share, s.chunks());
      if (lane == 0) first[warp].set(p, r, blockIdx.x - r * pieces, (int)wbegin, s);
    } else {
      wbegin = wend = 0;
    }
  } else {
    const long long share = (total + (long long)gridDim.x * kWarps - 1) / ((long long)gridDim.x * kWarps);
    quota = share * kWarps;
    begin = blockIdx.x * quota;
    wbegin = min(begin + warp * share, total);
    wend = min(wbegin + share, total);
    const long long before = (upto - mine) * pieces, end = before + mine * pieces;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const long long cut = begin + w * share;
      if (cut < before || cut >= end) continue;
      long long rest = cut - before;
      for (int r = r0; r < r1; ++r) {
        const RowSpan s = row_span<kChunk>(p, r);
        const long long n = (long long)s.units() * pieces;
        if (rest < n) {
          const int piece = (int)(rest / s.units());
          first[w].set(p, r, piece, (int)(rest - (long long)piece * s.units()), s);
          break;
        }
        rest -= n;
      }
    }
  }
  __syncthreads();
  for (int i = 0; i < min(n_empty, kMaxEmpty); ++i) clear_row(empty[i], threadIdx.x, kThreads);

  // Loads.  A lane looks up the page of one token of the chunk (one chunk ahead of its copies); the
  // copies then go two or more tokens at a time, 16 bytes a lane.
  const uint32_t ring = shared_addr(smem) + warp * kStages * S::kStageBytes;
  char* scratch = smem + S::kRing + warp * Body::kQBytes;
  constexpr int kLanesPerRow = Body::kRowBytes / 16 < 32 ? Body::kRowBytes / 16 : 32;
  constexpr int kRowsPerCopy = 32 / kLanesPerRow;
  constexpr int kPiecesPerLane = Body::kRowBytes / 16 / kLanesPerRow;
  const int row_pieces = kv.head_dim * (int)sizeof(T) / 16;
  Place<kChunk> ahead = first[warp];
  if (wbegin < wend) ahead.fetch(p);
  long long ahead_at = wbegin;                        // line unit of `ahead`, at a chunk or past the end
  if (ahead_at < wend && ahead.unit < kPieceCost) {
    ahead_at += kPieceCost - ahead.unit;
    ahead.unit = kPieceCost;
  }
  constexpr int kBoxes = kBulk && kChunk > kBoxTokens ? kChunk / kBoxTokens : 1;
  int entry[kBoxes];
  bool gave_up = false;
  uint32_t parity = 0;                                // bulk copies: the phase that every stage's next chunk completes
  auto look_up = [&]() {
    if (ahead_at >= wend) return;
    const int t0 = (ahead.span.c0 + ahead.unit - kPieceCost) * kChunk;
    const int32_t* row = kv.table + (int64_t)ahead.row * kv.max_pages;
    if constexpr (kBulk) {
#pragma unroll
      for (int i = 0; i < kBoxes; ++i)
        if (t0 + i * kBoxTokens < ahead.span.hi) entry[i] = row[div_by(t0 + i * kBoxTokens, p.page)];
    } else {
      const int t = t0 + lane;
      if (lane < kChunk && t < ahead.span.hi && t >= ahead.span.lo) entry[0] = row[div_by(t, p.page)];
    }
  };
  look_up();
  auto issue = [&](int stage) {
    if (ahead_at < wend && !gave_up) {
      const int t0 = (ahead.span.c0 + ahead.unit - kPieceCost) * kChunk;
      const uint32_t kb = ring + stage * S::kStageBytes, vb = kb + kChunk * Body::kRowBytes;
      if constexpr (kBulk) {
        // slots past the row's end come along and are cleared when the chunk is used; a bad entry reads page 0
        const int boxes = min(kBoxes, (ahead.span.hi - t0 + kBoxTokens - 1) / kBoxTokens);
        constexpr int kBox = kChunk / kBoxes * Body::kRowBytes;
        if (lane == 0) expect_bytes(bar + 8 * stage, 2 * boxes * kBox);
#pragma unroll
        for (int i = 0; i < kBoxes; ++i) {
          if (i >= boxes) continue;
          const int t = t0 + i * kBoxTokens;
          int page = entry[i];
          if ((unsigned int)page >= (unsigned int)kv.n_pages) {
            flag(kv.status, kStatusIndex);
            page = 0;
          }
          const int at = ahead.h * kv.page_size + t - (int)div_by(t, p.page) * kv.page_size;
          if (lane == 0) {
            if constexpr (sizeof(T) == 2) {
              copy_tensor(kb + i * kBoxTokens * 128, &maps.k, at, page, bar + 8 * stage);
              copy_tensor(vb + i * kBoxTokens * 128, &maps.v, at, page, bar + 8 * stage);
            } else {
              const int64_t e = page * kv.page_stride + (int64_t)at * kv.head_dim;
              copy_bulk(kb, (const T*)kv.k + e, kBox, bar + 8 * stage);
              copy_bulk(vb, (const T*)kv.v + e, kBox, bar + 8 * stage);
            }
          }
        }
      } else {
        const int t = t0 + lane;
        // where the token is: an element offset in the pools, -1 for zeros, -2 - e for element e of the new tokens
        int64_t from = -1;
        if (lane < kChunk && t < ahead.span.hi && t >= ahead.span.lo) {
          if (ahead.takes && t == ahead.span.hi - 1) {
            from = -2 - (ahead.row * p.new_stride + (int64_t)ahead.h * kv.head_dim);
          } else if ((unsigned int)entry[0] < (unsigned int)kv.n_pages) {
            const int slot = t - (int)div_by(t, p.page) * kv.page_size;
            from = entry[0] * kv.page_stride + ((int64_t)ahead.h * kv.page_size + slot) * kv.head_dim;
          } else {
            flag(kv.status, kStatusIndex);
          }
        }
#pragma unroll
        for (int i = 0; i < kChunk; i += kRowsPerCopy) {
          const int tok = i + lane / kLanesPerRow;
          const int64_t e = __shfl_sync(0xFFFFFFFFu, from, tok);
          const T* kp = e >= 0 ? (const T*)kv.k + e : (const T*)p.k_new + (-2 - e);
          const T* vp = e >= 0 ? (const T*)kv.v + e : (const T*)p.v_new + (-2 - e);
#pragma unroll
          for (int j = 0; j < kPiecesPerLane; ++j) {
            const int c = lane % kLanesPerRow + j * kLanesPerRow;
            const bool some = e != -1 && c < row_pieces;
            copy_async(kb + Body::piece_at(tok, c), some ? (const char*)kp + c * 16 : (const char*)kv.k, some);
            copy_async(vb + Body::piece_at(tok, c), some ? (const char*)vp + c * 16 : (const char*)kv.v, some);
          }
        }
      }
      ++ahead_at;
      if (++ahead.unit == ahead.span.units()) {
        if (ahead_at < wend) ahead.next_piece(p);
        ahead_at += kPieceCost;
        ahead.unit = kPieceCost;
      }
      look_up();
    }
    if constexpr (!kBulk) copy_commit();
  };
  // The stage's chunk is in place.  Bulk: a wait that runs out is reported and ends the loads; what is still on its way
  // (this stage's and those after it; one with nothing on its way waits in vain) gets a second, last wait, so that no copy
  // lands in memory that has been given to something else.
  auto arrived = [&](int stage) {
    if constexpr (kBulk) {
      if (!gave_up) {
        const bool there = mbarrier_wait_bounded(bar + 8 * stage, parity >> stage & 1u, wait_limit(p, TokenWait::kChunks, kBulkWaitLimit));
        if (__all_sync(0xFFFFFFFFu, there)) {
          parity ^= 1u << stage;
        } else {
          gave_up = true;
          flag(kv.status, kStatusTimeout);
          for (int i = 0, s = stage; i < kStages - 1; ++i, s = s + 1 == kStages ? 0 : s + 1)
            mbarrier_wait_bounded(bar + 8 * s, parity >> s & 1u, kBulkWaitLimit);
        }
      }
    } else {
      copy_wait<kStages - 2>();
    }
    __syncwarp();
  };
  // What a bulk copy cannot do for a row's last chunk: the new token's row, and zeros past the end (V only: the
  // scores there are masked, but 0 times what a free slot holds need not be 0).
  auto complete = [&](const Place<kChunk>& at, int t0, char* kb, char* vb) {
    if constexpr (kBulk) {
      if (t0 + kChunk < at.span.hi) return;
      for (int i = lane; i < kChunk * row_pieces; i += 32) {
        const int tok = i / row_pieces, c = i - tok * row_pieces;
        if (t0 + tok >= at.span.hi) *(uint4*)(vb + Body::piece_at(tok, c)) = make_uint4(0, 0, 0, 0);
      }
      if (at.takes) {
        const int64_t e = at.row * p.new_stride + (int64_t)at.h * kv.head_dim;
        for (int c = lane; c < row_pieces; c += 32) {
          const uint32_t to = Body::piece_at(at.span.hi - 1 - t0, c);
          *(uint4*)(kb + to) = ((const uint4*)((const T*)p.k_new + e))[c];
          *(uint4*)(vb + to) = ((const uint4*)((const T*)p.v_new + e))[c];
        }
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");        // before the stage's next bulk copy
      __syncwarp();
    }
  };
#pragma unroll
  for (int s = 0; s < kStages - 1; ++s) issue(s);

  // While the first chunks are on their way: the new tokens' keys and values go to their pages, a warp
  // for each row and kv head.
  if (p.k_new) {
    for (int64_t i = (int64_t)blockIdx.x * kWarps + warp; i < (int64_t)kv.n_rows * kv.n_kv_heads; i += (int64_t)gridDim.x * kWarps) {
      const int r = (int)(i / kv.n_kv_heads), h = (int)(i - (int64_t)r * kv.n_kv_heads);
      const int t = checked_len(kv, kv.len[r]) - 1;
      if (t < 0 || !has_room(kv, r, 1)) continue;
      const int pg = (int)div_by(t, p.page), page = kv.table[(int64_t)r * kv.max_pages + pg];
      if ((unsigned int)page >= (unsigned int)kv.n_pages) {
        if (lane == 0) flag(kv.status, kStatusIndex);
        continue;
      }
      const int64_t to = page * kv.page_stride + ((int64_t)h * kv.page_size + t - pg * kv.page_size) * kv.head_dim;
      const int64_t from = r * p.new_stride + (int64_t)h * kv.head_dim;
      for (int c = lane; c < row_pieces; c += 32) {
        const uint4 a = ((const uint4*)((const T*)p.k_new + from))[c], b = ((const uint4*)((const T*)p.v_new + from))[c];
        ((uint4*)((T*)kv.k + to))[c] = a;
        ((uint4*)((T*)kv.v + to))[c] = b;
      }
    }
  }

  Body body;
  Place<kChunk> here = first[warp];
  if (wbegin < wend) here.fetch(p);
  long long pos = wbegin;
  int stage = 0;
  float* dumps = p.dumps + (size_t)blockIdx.x * kWarps * kRegs * 32;
  auto out_at = [&](int row, int head) { return (T*)p.out + row * p.out_stride + (int64_t)head * kv.head_dim; };
  auto lse_of = [&](float m, float l) {
    constexpr float kDown = Body::kLift == 0.f ? 1.f : 1.f / 32768.f;       // 2^-kLift
    static_assert(Body::kLift == 0.f || Body::kLift == 15.f, "kDown");
    return l == 0.f ? -INFINITY : (m == -INFINITY ? 0.f : m + Body::kLift) * 0.6931471805599453f + logf(l * kDown);
  };
  while (pos < wend) {
    const RowSpan span = here.span;
    const int n_units = (int)min((long long)(span.units() - here.unit), wend - pos);
    const int j0 = max(here.unit - kPieceCost, 0), j1 = here.unit + n_units - kPieceCost;
    if (j1 > j0) {
      const int head0 = here.h * p.per_kv + here.split * p.piece_heads;
      const int heads = min(p.piece_heads, p.per_kv - here.split * p.piece_heads);
      body.begin(p, here.row, head0, heads, lane, scratch);
      if (span.lo > 0 && j0 == 0) {
        int column;
        const int unit = shared_unit(p, here.group, here.n, here.h, &column);
        body.join_shared(p, unit, column + here.split * p.piece_heads, heads, lane);
      }
      for (int j = j0; j < j1; ++j) {
        arrived(stage);
        issue(stage == 0 ? kStages - 1 : stage - 1);
        const uint32_t kb = ring + stage * S::kStageBytes;
        char* kp = smem + (size_t)(warp * kStages + stage) * S::kStageBytes;
        complete(here, (span.c0 + j) * kChunk, kp, kp + kChunk * Body::kRowBytes);
        body.step(p, kb, kb + kChunk * Body::kRowBytes, scratch, (span.c0 + j) * kChunk, span.lo, span.hi, lane);
        stage = stage + 1 == kStages ? 0 : stage + 1;
      }
      const int slot = j0 == 0 ? 1 : 0;
      body.stats(stat[warp][slot], lane);
      if (j0 == 0 && j1 == span.chunks()) {            // seen whole: nothing to join
        __syncwarp();
        const float2* st = stat[warp][1];
        body.store(p, st, here.row, head0, heads, lane);
        if (p.lse && lane < heads) p.lse[(int64_t)here.row * p.n_q_heads + head0 + lane] = lse_of(st[lane].x, st[lane].y);
        __syncwarp();
      } else {
        // a piece that goes on past this warp is its last: its loads are done, and the ring is free
        if (!kBulk && j0 == 0) copy_wait<0>();
        __syncwarp();
        float* dump = j0 == 0 ? (float*)(smem + (size_t)warp * kStages * S::kStageBytes) : dumps + warp * kRegs * 32;
#pragma unroll
        for (int i = 0; i < kRegs; i += 4)
          ((float4*)dump)[i * 8 + lane] = make_float4(body.o[i], body.o[i + 1], body.o[i + 2], body.o[i + 3]);
        if (lane == 0) {
          Left& x = left[warp][slot];
          x.row = here.row;
          x.h = here.h;
          x.split = here.split;
          x.chunk0 = j0;
          x.line = pos - here.unit + kPieceCost;
          x.chunks = span.chunks();
          x.goes_on = j1 < span.chunks();
          x.any = 1;
        }
      }
    }
    pos += n_units;
    if (pos < wend) here.next_piece(p);
    else break;
  }
  if constexpr (!kBulk) copy_wait<0>();
  __syncthreads();

  // Pieces that the warps of this CTA, or several CTAs, have shared: a run of dumps is slot s0 of warp w0
  // and then slot 0 of the warps after it, up to w1.
  auto dump_of = [&](int w, int s) {
    return s ? (const float*)(smem + (size_t)w * kStages * S::kStageBytes) : (const float*)dumps + w * kRegs * 32;
  };
  for (int k = 0; k < 2 * kWarps;) {
    const int w0 = k >> 1, s0 = k & 1;
    if (!left[w0][s0].any) {
      ++k;
      continue;
    }
    const Left x = left[w0][s0];
    int w1 = w0;
    bool goes_on = x.goes_on;
    while (goes_on && w1 + 1 < kWarps) goes_on = left[++w1][0].goes_on;
    k = (w1 > w0 ? 2 * w1 : k) + 1;
    const bool whole = x.chunk0 == 0 && !goes_on;
    const int head0 = x.h * p.per_kv + x.split * p.piece_heads;
    const int heads = min(p.piece_heads, p.per_kv - x.split * p.piece_heads);
    const int cta0 = whole ? 0 : (int)(x.line / quota), cta1 = whole ? 0 : (int)((x.line + x.chunks - 1) / quota);
    auto part_of = [&](int c) { return p.parts + (size_t)(2 * c + (c == cta0 ? 1 : 0)) * kPart; };
    float* part = whole ? nullptr : part_of(blockIdx.x);
    // Thread (warp, lane) adds the float4s (registers 4 u .. 4 u + 3 of lane `lane`) of u = warp, warp + kWarps, ...
    auto store_out = [&](int u, const float4& v, float l0, float l1, float l2, float l3) {
      const float vs[4] = {v.x, v.y, v.z, v.w}, ls[4] = {l0, l1, l2, l3};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int head = Body::head_of(4 * u + j, lane), d = Body::dim_of(4 * u + j, lane);
        if (head < heads && d < kv.head_dim) out_at(x.row, head0 + head)[d] = from_float<T>(ls[j] == 0.f ? 0.f : vs[j] / ls[j]);
      }
    };
    // statistics of the run, and its dumps' factors
    if (threadIdx.x < kMaxHeads) {
      const int head = threadIdx.x;
      float m = -INFINITY, l = 0.f;
      for (int w = w0; w <= w1; ++w) m = fmaxf(m, stat[w][w == w0 ? s0 : 0][head].x);
      const float off = m == -INFINITY ? 0.f : m;
      for (int w = w0; w <= w1; ++w) {
        const float2 s = stat[w][w == w0 ? s0 : 0][head];
        factor[w][head] = exp2_fast(s.x - off);
        l = fmaf(factor[w][head], s.y, l);
      }
      sums[head] = make_float2(m, l);
      if (head < heads) {
        if (!whole) __stcg((float2*)&part[kRegs * 32 + 2 * head], make_float2(m, l));
        else if (p.lse) p.lse[(int64_t)x.row * p.n_q_heads + head0 + head] = lse_of(m, l);
      }
    }
    __syncthreads();
#pragma unroll
    for (int u = warp; u < kRegs / 4; u += kWarps) {
      int hd[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) hd[j] = Body::head_of(4 * u + j, lane);
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int w = w0; w <= w1; ++w) {
        const float4 y = ((const float4*)dump_of(w, w == w0 ? s0 : 0))[u * 32 + lane];
        v.x = fmaf(factor[w][hd[0]], y.x, v.x);
        v.y = fmaf(factor[w][hd[1]], y.y, v.y);
        v.z = fmaf(factor[w][hd[2]], y.z, v.z);
        v.w = fmaf(factor[w][hd[3]], y.w, v.w);
      }
      if (!whole) __stcg((float4*)part + u * 32 + lane, v);
      else store_out(u, v, sums[hd[0]].y, sums[hd[1]].y, sums[hd[2]].y, sums[hd[3]].y);
    }
    __syncthreads();
    if (!whole) {
      // the last of the CTAs that hold a part of this piece adds them, in CTA order
      if (threadIdx.x == 0) {
        __threadfence();
        is_last = atomicAdd(&p.tickets[cta0], 1u) == (unsigned int)(cta1 - cta0);
        if (is_last) p.tickets[cta0] = 0;
      }
      __syncthreads();
      if (is_last) {
        __threadfence();
        const int n = cta1 - cta0 + 1;
#pragma unroll 1
        for (int u = warp; u < kRegs / 4; u += kWarps) {
          int hd[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) hd[j] = Body::head_of(4 * u + j, lane);
          float v[4] = {0.f, 0.f, 0.f, 0.f}, m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll 8
          for (int c = 0; c < n; ++c) {
            const float* q = part_of(cta0 + c);
            const float4 y = __ldcg((const float4*)q + u * 32 + lane);
            float f[2], g[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float2 s = __ldcg((const float2*)(q + kRegs * 32) + hd[e * Body::kSecond]);
              const float m2 = fmaxf(m[e], s.x), off = m2 == -INFINITY ? 0.f : m2;
              f[e] = exp2_fast(m[e] - off);
              g[e] = exp2_fast(s.x - off);
              l[e] = l[e] * f[e] + s.y * g[e];
              m[e] = m2;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = v[j] * f[Body::pair_of(j)] + (&y.x)[j] * g[Body::pair_of(j)];
          }
          store_out(u, make_float4(v[0], v[1], v[2], v[3]), l[Body::pair_of(0)], l[Body::pair_of(1)], l[Body::pair_of(2)], l[Body::pair_of(3)]);
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (p.lse && hd[j] < heads && Body::dim_of(4 * u + j, lane) == 0)
              p.lse[(int64_t)x.row * p.n_q_heads + head0 + hd[j]] = lse_of(m[Body::pair_of(j)], l[Body::pair_of(j)]);
        }
        __syncthreads();
      }
    }
  }
}
#endif

// ---------------------------------------------------------------- launch

static std::atomic<uint32_t> lost_waits{0};          // pg_selftest_token_waits

static int attend_check(const pg_kv* kv, int n_q_heads, int group) {
  const int rc = kv_check(kv);
  if (rc != PG_OK) return rc;
  if (n_q_heads < 1 || n_q_heads % kv->n_kv_heads || n_q_heads > 65535) return PG_EINVAL;
  if (group < 1 || kv->n_rows % group) return PG_EINVAL;
  return PG_OK;
}

// Query heads of a kv head beyond kMaxHeads are dealt to several pieces, evenly.
static void split_heads(int per_kv, int* n_split, int* piece_heads) {
  *n_split = (per_kv + kMaxHeads - 1) / kMaxHeads;
  *piece_heads = (per_kv + *n_split - 1) / *n_split;
}

// [n_pages][head_dim / 64][kv heads * page_size][64] 16-bit elements, boxes of 16 tokens and `blocks` blocks.
static bool make_map(CUtensorMap* map, const AttendParams& p, const void* pool, int dtype_bf16, int blocks) {
  using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                              const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
  static Encode encode = [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess)
      f = nullptr;
    return (Encode)f;
  }();
  if (!encode) return false;
  const KvView& kv = p.kv;
  const cuuint64_t size[4] = {64, (cuuint64_t)kv.n_kv_heads * kv.page_size, (cuuint64_t)kv.head_dim / 64, (cuuint64_t)kv.n_pages};
  const cuuint64_t stride[3] = {(cuuint64_t)kv.head_dim * 2, 128, (cuuint64_t)kv.page_stride * 2};
  const cuuint32_t box[4] = {64, (cuuint32_t)kBoxTokens, (cuuint32_t)blocks, 1}, step[4] = {1, 1, 1, 1};
  return encode(map, dtype_bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, (void*)pool, size, stride, box, step,
                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, typename Body, int kWarps, int kStages, bool kBulk>
static int launch_attend(const AttendParams& p, const PoolMaps& maps, cudaStream_t st) {
  using S = AttendShared<T, Body, kWarps, kStages>;
  static_assert(S::kBytes <= 223 * 1024, "shared memory");
  static_assert(kWarps <= kMaxWarps, "workspace");
  auto kernel = attend_kernel<T, Body, kWarps, kStages, kBulk>;
  static std::atomic<uint64_t> done{0};
  if (const int rc = allow_shared(kernel, (int)S::kBytes, done)) return rc;
  const long long most = (long long)p.kv.n_rows * p.kv.n_kv_heads * p.n_split *
                         (((long long)p.kv.max_pages * p.kv.page_size + Body::kChunk - 1) / Body::kChunk);
  kernel<<<(unsigned)(most < kSms ? most : kSms), kWarps * 32, S::kBytes, st>>>(p, maps);
  PG_LAUNCH_CHECK();
  return PG_OK;
}

// Bulk copies where 16 tokens in a row always lie in one page, and no padding has to be filled in between: head
// dim a multiple of 64 (tensor copies, 16 bits; what is past it up to the body's size is outside the map and reads
// as zeros) or the body's own size (fp32).
template <typename T, typename Body, int DP, int kWarps, int kStages>
static int launch_copies(const AttendParams& p, cudaStream_t st) {
  PoolMaps maps;
  bool bulk = p.kv.page_size % kBoxTokens == 0 && p.kv.head_dim % 64 == 0 && (sizeof(T) == 2 || p.kv.head_dim == DP);
  if (bulk && sizeof(T) == 2) {
    const bool bf = std::is_same<T, __nv_bfloat16>::value;
    bulk = make_map(&maps.k, p, p.kv.k, bf, DP / 64) && make_map(&maps.v, p, p.kv.v, bf, DP / 64);
  }
  return bulk ? launch_attend<T, Body, kWarps, kStages, true>(p, maps, st) : launch_attend<T, Body, kWarps, kStages, false>(p, maps, st);
}

// One CTA per SM; its warps' rings take most of the shared memory (three stages of 8 KB for eight warps,
// or of 16 KB for four).
template <typename T, template <int, int> class Body, int DP, int NT>
static int launch_body(const AttendParams& p, cudaStream_t st) {
  constexpr int kStage = 2 * Body<DP, NT>::kChunk * Body<DP, NT>::kRowBytes;
  if constexpr (sizeof(T) == 2 && DP <= 128) return launch_copies<T, Body<DP, NT>, DP, 8, 3>(p, st);
  else return launch_copies<T, Body<DP, NT>, DP, 4, 4 * (3 * kStage + (int)Body<DP, NT>::kQBytes) <= 221 * 1024 ? 3 : 2>(p, st);
}

template <typename T, template <int, int> class Body>
static int launch_type(const AttendParams& p, cudaStream_t st) {
  const int d = p.kv.head_dim;
  if (p.piece_heads <= 8) {
    if (d <= 64) return launch_body<T, Body, 64, 1>(p, st);
    if (d <= 128) return launch_body<T, Body, 128, 1>(p, st);
    return launch_body<T, Body, 256, 1>(p, st);
  }
  if (d <= 64) return launch_body<T, Body, 64, 2>(p, st);
  if (d <= 128) return launch_body<T, Body, 128, 2>(p, st);
  return launch_body<T, Body, 256, 2>(p, st);
}

template <int DP, int NT> using Bf16Body = MmaBody<__nv_bfloat16, DP, NT, DP <= 64 ? 32 : 16>;
template <int DP, int NT> using F16Body = MmaBody<__half, DP, NT, DP <= 64 ? 32 : 16>;

static size_t spans_bytes(const pg_kv* kv, int group, int blocks) {
  return ((size_t)(kv->n_rows / group) * kv->n_kv_heads * blocks * sizeof(int2) + 15) & ~(size_t)15;
}
static size_t shared_bytes(const pg_kv* kv, int n_q_heads, int group) {
  int blocks, rows, queries;
  if (group < 2 || kv->dtype == PG_F32 || !shared_blocks(group, n_q_heads / kv->n_kv_heads, kv->head_dim, &blocks, &rows, &queries))
    return 0;
  const size_t units = (size_t)(kv->n_rows / group) * kv->n_kv_heads * blocks;
  return spans_bytes(kv, group, blocks) + (kSms + units) * queries * (kv->head_dim + 2) * sizeof(float);
}

}  // namespace pg

extern "C" {

size_t pg_kv_attend_workspace_bytes(const pg_kv* kv, int32_t n_q_heads, int32_t group) {
  if (pg::attend_check(kv, n_q_heads, group) != PG_OK) return 0;
  // tickets first, so that their place depends on nothing
  const size_t dp = kv->head_dim <= 64 ? 64 : kv->head_dim <= 128 ? 128 : 256;
  const size_t acc = dp * pg::kMaxHeads;
  return pg::kCounterBytes + pg::kSms * (2 * (acc + 2 * pg::kMaxHeads) + pg::kMaxWarps * acc) * sizeof(float) +
         pg::shared_bytes(kv, n_q_heads, group);
}

int pg_kv_attend(const pg_kv* kv, int32_t layer, int32_t n_q_heads, const void* q, int64_t q_stride,
                 const void* k_new, const void* v_new, int64_t new_stride, float scale, int32_t group,
                 const int32_t* shared, void* out, int64_t out_stride, float* lse, void* workspace,
                 size_t workspace_bytes, int32_t* status, void* stream) {
  pg::TraceRange trace_range("pg_kv_attend");
  const int rc = pg::attend_check(kv, n_q_heads, group);
  if (rc != PG_OK) return rc;
  if (layer < 0 || layer >= kv->n_layers || !(scale == scale) || (!k_new != !v_new)) return PG_EINVAL;
  if (kv->n_rows == 0) return PG_OK;
  const int64_t dense = (int64_t)n_q_heads * kv->head_dim, dense_new = (int64_t)kv->n_kv_heads * kv->head_dim;
  if (q_stride == 0) q_stride = dense;
  if (out_stride == 0) out_stride = dense;
  if (new_stride == 0) new_stride = dense_new;
  const size_t b = pg::dtype_bytes(kv->dtype);
  if (!q || !out || q_stride < dense || out_stride < dense) return PG_EINVAL;
  if (((uintptr_t)q | (uintptr_t)out) & (b - 1)) return PG_EINVAL;
  if (k_new && (new_stride < dense_new || (new_stride * b & 15) || (((uintptr_t)k_new | (uintptr_t)v_new) & 15)))
    return PG_EINVAL;
  if (!workspace || ((uintptr_t)workspace & 15) || workspace_bytes < pg_kv_attend_workspace_bytes(kv, n_q_heads, group))
    return PG_EINVAL;
  if ((int64_t)kv->n_rows * n_q_heads > 0x7FFFFFFFLL) return PG_EINVAL;
  pg::AttendParams p;
  p.kv = pg::kv_view(kv, status);
  p.kv.k = (char*)kv->k + (size_t)layer * p.kv.layer_stride * b;
  p.kv.v = (char*)kv->v + (size_t)layer * p.kv.layer_stride * b;
  p.q = q; p.k_new = k_new; p.v_new = v_new; p.out = out; p.lse = lse;
  p.shared = group > 1 ? shared : nullptr;
  p.q_stride = q_stride; p.new_stride = new_stride; p.out_stride = out_stride;
  p.n_q_heads = n_q_heads; p.per_kv = n_q_heads / kv->n_kv_heads; p.group = group;
  pg::split_heads(p.per_kv, &p.n_split, &p.piece_heads);
  p.q_words = ((((uintptr_t)q) | (uintptr_t)(q_stride * b)) & 3) == 0;
  p.out_words = ((((uintptr_t)out) | (uintptr_t)(out_stride * b)) & 3) == 0;
  p.scale_log2 = (float)((double)scale * 1.4426950408889634);
  p.lost_waits = pg::lost_waits.load(std::memory_order_relaxed);
  p.page = pg::fast_div((uint32_t)kv->page_size);
  p.group_div = pg::fast_div((uint32_t)group);
  p.tickets = (unsigned int*)workspace;
  p.parts = (float*)((char*)workspace + pg::kCounterBytes);
  const size_t dp = kv->head_dim <= 64 ? 64 : kv->head_dim <= 128 ? 128 : 256;
  p.dumps = p.parts + 2 * pg::kSms * (dp + 2) * pg::kMaxHeads;
  cudaStream_t st = (cudaStream_t)stream;
  if (kv->dtype == PG_F32 || (p.shared && !pg::shared_blocks(group, p.per_kv, kv->head_dim, &p.q_blocks, &p.block_rows, &p.block_queries)))
    p.shared = nullptr;
  if (p.shared) {
    p.spans = (int2*)(p.dumps + pg::kSms * pg::kMaxWarps * dp * pg::kMaxHeads);
    p.shared_out = (float*)((char*)p.spans + pg::spans_bytes(kv, group, p.q_blocks));
    const int e = pg::launch_shared(p, kv->dtype, st);
    if (e != PG_OK) return e;
  }
  if (kv->dtype == PG_F32) return pg::launch_type<float, pg::F32Body>(p, st);
  if (kv->dtype == PG_BF16) return pg::launch_type<__nv_bfloat16, pg::Bf16Body>(p, st);
  return pg::launch_type<__half, pg::F16Body>(p, st);
}

int pg_selftest_token_waits(uint32_t kinds) {
  if (kinds >> (int)pg::TokenWait::kKinds) return PG_EINVAL;
  pg::lost_waits.store(kinds, std::memory_order_relaxed);
  return PG_OK;
}

}  // extern "C"
