// Policy update on rows of logits: log-probs of given tokens, entropy, alternatives, divergence from a teacher's list, and their
// gradient (pg_token_forward / _backward / _forward_backward).
//
// Bound: HBM, each logit read once and each gradient written once.  A CTA takes a row, or a part of one, in tiles of eight 16-byte
// units a thread that lie in registers as they came from memory; as a unit is done with, the next tile's is asked for.  In the base-2
// domain, with c = log2(e) / T,
//     y_v = (l_v - m) c,   s0 = sum 2^y,   s1 = sum 2^y y,   m the largest logit that the thread has,
// so one exponential a logit gives lse = m / T + ln s0 and the entropy ln s0 - ln 2 s1 / s0.  The triples (m, s0, s1) of threads and
// warps, and of the CTAs of a cluster through each other's shared memory, are joined in a fixed order.
// The gradient of all terms together is, away from given and listed tokens, e (a + b ln e) with two numbers a row and e a softmax: a
// second pass over the row.  Of its part the CTA has kept a tile in registers and one in shared memory; the others come back from the
// L2 cache, which holds them because all else is read and written with the wish to be evicted first.  Given and listed tokens are
// written over the pass afterwards, one thread each.
// With a bucket for the mass outside a teacher's list that mass is summed by itself (the list's logits are taken out of the registers),
// since the difference 1 - (list's mass) has no digits left where the list has nearly everything.
// Alternatives: bounds from the threads' largest logits leave few tiles of few threads to look at again; what passes is ranked by
// counting.
//
// Masks: logits of -inf leave the sums by themselves.  Where the reference lies far from 0 (a finite mask, a small T) the product l c loses what the
// difference l - m still has; sums take the difference first from kFar on, gradients see Slope2.
//
// Measured (B200; share of the floor at the copy rate, calls back to back, a token and the entropy of each row): 2368 x 131072 bf16 forward 96 us
// (98 %), with gradient 224 us (85 %; without the entropy 217 us), distillation from a list of 64 232 us (82 %), with a bucket 246 us (77 %);
// 2368 x 50001 fp16 50 us (73 %), 104 us (69 %; without 92 us), 101 us (72 %), 112 us (64 %); 2368 x 32000 fp32 52 us (90 %), 112 us (83 %), 121 us
// (76 %), 126 us (74 %); 1024 x 131072 bf16 gradient alone 90 us (91 %).  What is left: the join of a row, about 0.7 us in which its CTA asks for
// nothing, longer with a list (one or two warps sum it, the others wait), and rows that are little longer than whole tiles.
// Tried and left out, against builds of their time in which a list's distillation over 2048 x 131072 took 209 to 237 us (203 us in this one): rows kept
// in the registers or shared memory of clusters (the join of eight CTAs costs more than the second read: 343 and 302 us), CTAs that stay and
// ask for their next row ahead (220 us), bulk prefetches into the L2 cache (233 us), five CTAs an SM with smaller tiles (225 to 234 us); listed
// tokens in a hash table instead of a byte for each unit (1251 x 65536 forward 45 us, not 41).
#pragma once

#include "pg_kv.cuh"
#include "pg_trace.cuh"
#include "pg_units.cuh"

#include <algorithm>
#include <type_traits>

namespace pg {

constexpr int kTokThreads = 256, kTokCtas = 4;  // of a CTA; CTAs of an SM, 64 registers a thread
constexpr int kPartBytes = 128 * 1024;          // of a row that is read twice; 2048 x 131072 bf16 with gradient 197 us, 256 KB: 225 us, 64 KB: 215 us
constexpr int kOnChip = 2;                      // tiles of a part that stay on chip: one in registers, one in shared memory
constexpr int kSavedBytes = 64 << 20;           // of the logits, which pg_token_backward meets first, wanted in the L2 cache with `saved`: both passes
                                                // over 1251 x 65536 bf16 86.0 us; none 89.3 us, 32 MB 87.7 us, 96 MB 87.3 us
constexpr int kBackwardTiles = 2;               // of a CTA that only writes gradients, whose row's numbers serve both: 2368 x 50001 fp16 81 us (1: 90 us, 4: 87 us),
                                                // both passes over 1251 x 65536 86 us (1: 90 us, 4: 88 us); 1024 x 131072 90 us (1: 86 us, 4: 94 us)
constexpr int kTokWarps = kTokThreads / 32;
constexpr int kMostParts = 8;                   // CTAs of a cluster
constexpr int kCandidates = 1024;
constexpr int kMostTiles = 16;                  // of a part with alternatives
constexpr int kMostGroups = 1024;               // threads' tiles that are read again for them
constexpr int kMergeBytes = kMostParts * PG_TOKEN_MAX_TOP * 8;
constexpr float kLn2 = 0.6931471805599453f, kLog2e = 1.4426950408889634f;
constexpr float kMean = 1.f / (2 * PG_TOKEN_MAX_LIST);   // of sums over a list whose mean is wanted: log-probs near the type's end, of masked tokens,
                                                // do not pass it on the way.  A factor of these, not of weights, which may be next to 0
constexpr float kFloorY = -1e4f;                // 2^y = 0 long before; keeps 0 * y from being NaN
constexpr float kFar = 4194304.f;               // 2^22: below it m c is off by 1/8 at most; from there on (finite masks of any size, a
                                                // small T) l - m is taken first, or 2^off would leave 32 bits

enum TokenMode { kForward, kBackward, kBoth };
enum TokenLists { kNoList, kNormalised, kBucket };   // a teacher's list: none, PG_DISTILL_FORWARD, the kinds with a bucket

struct TokenParams {
  pg_token_terms t;
  pg_token_out o;
  pg_token_grads g;
  const void* in;
  void* dl;
  int64_t in_stride, dl_stride;
  int n_rows, vocab;
  int parts, units, tiles;                      // CTAs of a row; units of a part; tiles of a part
};

// What is known of a row when its logits have been read.
struct TokenRow {
  float m, l2, h;                // p_v = 2^((l_v - m) c - l2); entropy
  float mr, l2r, lr;             // the same of the distribution outside the list; ln p_r (-inf: nothing there)
  float loss, lt, w;             // divergence; ln t_r; sum t (+ t_r).  FORWARD: ln of the list's mass is lt + l2r, its largest tl and the rest, since
                                 // the sum has no digits for the rest where raw logits are far from 0
  float some;                    // 0: a row that allows nothing
};
// The gradient away from given and listed tokens: e (a + b ln e), e = 2^((l - ref) c - l2).
struct TokenSlope {
  float a, b, ref, l2;
};

// Sums over a warp's share of a teacher's list.  Reference of e: the largest logit m among them; of t: `tm` (FORWARD), else 0.
struct ListSums {
  float m, s0, s1, etl;                         // sum e, e y, kMean e tl
  float tm, ts, ttl, ty;                        // sum t, t (tl - tm), kMean t (l - m) / T
  double mass;                                  // sum t (the kinds with a bucket)
};

struct TokenShared {
  float4 part[kMostParts * kTokWarps];          // triples of the cluster's warps, written by each
  TokenRow row;
  TokenSlope slope;
  float lp_part;
  ListSums list[PG_TOKEN_MAX_LIST / 32];
  float dsum[PG_TOKEN_MAX_LIST / 32];
  int gid[PG_TOKEN_MAX_LIST];                   // given tokens, -1: padding
  float gdl[PG_TOKEN_MAX_LIST];
  alignas(16) int tid[PG_TOKEN_MAX_LIST];       // listed tokens, -1: unused
  uint32_t edges;                               // bits of the listed ones among the edge tokens
};

typedef unsigned long long f2;                  // two floats for the packed fp32 instructions
__device__ __forceinline__ f2 make2(float a, float b) {
  f2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void split2(f2 v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ f2 add2(f2 a, f2 b) {
  f2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f2 mul2(f2 a, f2 b) {
  f2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c) {
  f2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ float ex2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// Address of `p`, a shared variable of this CTA, in the CTA of rank r.
__device__ __forceinline__ uint32_t peer(const void* p, int r) {
  uint32_t at;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(r));
  return at;
}
__device__ __forceinline__ void peer_store(uint32_t at, float a, float b, float c) {
  asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(at), "f"(a), "f"(b), "f"(c), "f"(0.f) : "memory");
}
__device__ __forceinline__ void peer_store(uint32_t at, unsigned long long v) {
  asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(at), "l"(v) : "memory");
}

__device__ __forceinline__ float warp_total(float v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
  return v;
}
__device__ __forceinline__ double warp_total(double v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
  return v;
}
__device__ __forceinline__ float warp_most(float v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(~0u, v, o));
  return v;
}

// Moves a triple to the reference `to` >= m.
__device__ __forceinline__ void refer(float m, float to, float c, float& s0, float& s1) {
  if (!(to > m)) return;
  const float d = fmaxf((m - to) * c, kFloorY), f = ex2(d);
  s1 = f * fmaf(d, s0, s1);
  s0 *= f;
}
__device__ __forceinline__ float finite_ref(float m) { return m == -INFINITY ? 0.f : m; }

template <typename T> struct Empty8;            // a unit of logits that are -inf
template <> struct Empty8<float> { static constexpr uint32_t word = 0xFF800000u; };
template <> struct Empty8<__nv_bfloat16> { static constexpr uint32_t word = 0xFF80FF80u; };
template <> struct Empty8<__half> { static constexpr uint32_t word = 0xFC00FC00u; };

__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b, __nv_bfloat16) {
  const __nv_bfloat162 r = __hmax2(*reinterpret_cast<__nv_bfloat162*>(&a), *reinterpret_cast<__nv_bfloat162*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b, __half) {
  const __half2 r = __hmax2(*reinterpret_cast<__half2*>(&a), *reinterpret_cast<__half2*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b, float) {
  return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
}
template <typename T>
__device__ __forceinline__ float max_of(uint32_t w) {
  if constexpr (sizeof(T) == 4) return __uint_as_float(w);
  else {
    const uint32_t m = max2(w, w >> 16 | w << 16, T());
    T x;
    *reinterpret_cast<uint16_t*>(&x) = (uint16_t)m;
    return to_float(x);
  }
}
// A unit is 16 bytes of a row: eight or four logits.
template <typename T> constexpr int kPer = 16 / (int)sizeof(T);
template <typename T>
__device__ __forceinline__ uint32_t max_unit(uint32_t w, const uint4& v) {
  return max2(max2(max2(w, v.x, T()), v.y, T()), max2(v.z, v.w, T()), T());
}
// The logits of bits in `listed` replaced by -inf.
template <typename T>
__device__ __forceinline__ void set_empty(uint4& v, uint32_t listed) {
  uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) {
      if (listed >> i & 1) w[i] = Empty8<T>::word;
    } else {
      if (listed >> (2 * i) & 1) w[i] = (w[i] & 0xFFFF0000u) | (Empty8<T>::word & 0xFFFFu);
      if (listed >> (2 * i + 1) & 1) w[i] = (w[i] & 0xFFFFu) | (Empty8<T>::word & 0xFFFF0000u);
    }
  }
  v = make_uint4(w[0], w[1], w[2], w[3]);
}
template <typename T>
__device__ __forceinline__ uint4 empty_unit() { return make_uint4(Empty8<T>::word, Empty8<T>::word, Empty8<T>::word, Empty8<T>::word); }
template <typename T>
__device__ __forceinline__ f2 pair_of(const uint4& v, int i) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  if constexpr (sizeof(T) == 4) return make2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
  else if constexpr (std::is_same<T, __half>::value) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
    return make2(f.x, f.y);
  } else return make2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
}
template <typename T>
__device__ __forceinline__ void store_unit(T* to, const float (&g)[kPer<T>]) {
  if constexpr (sizeof(T) == 4) __stcs((float4*)to, make_float4(g[0], g[1], g[2], g[3]));
  else __stcs((uint4*)to, make_uint4(pack2(g[0], g[1], T()), pack2(g[2], g[3], T()), pack2(g[4], g[5], T()), pack2(g[6], g[7], T())));
}

__device__ __forceinline__ unsigned long long top_key(float x, int id) {
  const uint32_t b = __float_as_uint(x + 0.f);                     // -0 = +0
  return (unsigned long long)(b ^ (b >> 31 ? 0xFFFFFFFFu : 0x80000000u)) << 32 | (0xFFFFFFFFu - (uint32_t)id);
}

__device__ __forceinline__ void save_row(float4* at, const TokenRow& r) {
  at[0] = make_float4(r.m, r.l2, r.h, r.mr);
  at[1] = make_float4(r.l2r, r.lr, r.loss, r.lt);
  at[2] = make_float4(r.w, r.some, 0.f, 0.f);
}
__device__ __forceinline__ TokenRow load_row(const float4* at) {
  const float4 a = at[0], b = at[1], d = at[2];
  return {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w, d.x, d.y};
}

// Joins triples of the lanes of a warp; all lanes get the result.
__device__ __forceinline__ void join_warp(float& m, float& s0, float& s1, float c) {
  const float to = warp_most(m);
  refer(m, to, c, s0, s1);
  m = to;
  s0 = warp_total(s0);
  s1 = warp_total(s1);
}

// By one warp: from the sums over the row, or over the row outside the list (kBucket), and the list's.
template <int kLists>
__device__ __forceinline__ TokenRow finish_row(const TokenShared& s, const float4* triples, int parts, int lists, int kind, float inv) {
  const float c = inv * kLog2e;
  const int lane = threadIdx.x & 31;
  TokenRow r;
  float m = -INFINITY, s0 = 0.f, s1 = 0.f;
  for (int i = lane; i < parts * kTokWarps; i += 32) {
    float4 v = triples[i];
    const float to = fmaxf(m, v.x);
    refer(m, to, c, s0, s1);
    refer(v.x, to, c, v.y, v.z);
    m = to;
    s0 += v.y;
    s1 += v.z;
  }
  ListSums l;
  l.m = l.tm = -INFINITY;
  l.s0 = l.s1 = l.etl = l.ts = l.ttl = l.ty = 0.f;
  l.mass = 0.;
  if (kLists != kNoList && lane < lists) l = s.list[lane];
  bool outside = true;
  r.mr = r.lr = r.l2r = 0.f;
  if (kLists == kBucket) {                                             // outside the list and in all, side by side
    const float to = warp_most(fmaxf(m, l.m));
    r.mr = warp_most(m);
    float r0 = s0, r1 = 0.f, a = l.s0, b = l.s1;
    refer(m, r.mr, c, r0, r1);
    refer(m, to, c, s0, s1);
    refer(l.m, to, c, a, b);
    r0 = warp_total(r0);
    s0 = warp_total(s0 + a);
    s1 = warp_total(s1 + b);
    m = to;
    outside = !(r0 == 0.f);
    r.l2r = outside ? log2f(r0) : 0.f;
  } else {
    join_warp(m, s0, s1, c);
  }
  r.some = s0 == 0.f ? 0.f : 1.f;
  r.m = finite_ref(m);
  r.l2 = r.some != 0.f ? log2f(s0) : 0.f;
  r.h = r.some != 0.f ? kLn2 * (r.l2 - s1 / s0) : 0.f;
  double lr = 0.;
  if (kLists == kBucket) {                                             // in 64 bits: where only tokens of the type's lowest value are left,
    lr = ((double)finite_ref(r.mr) - r.m) * inv + (double)(kLn2 * (r.l2r - r.l2));      // it is finite and its share of the loss may be
    r.lr = !outside ? -INFINITY : lr < -3e38 ? -3e38f : (float)lr;
  }
  r.mr = finite_ref(r.mr);
  r.loss = r.lt = r.w = 0.f;
  if (kLists == kNoList || r.some == 0.f) return r;
  if (kLists == kNormalised) {
    const float tm = warp_most(l.tm);
    float z = l.ts, ttl = 0.f, tlp = 0.f;                              // ts without tm: NaN
    if (l.tm != -INFINITY) {
      const float f = expf(l.tm - tm);
      z = f * l.ts;
      if (f != 0.f) {                                                  // entries of no weight add nothing, whatever p_i is
        ttl = f * (l.ttl + l.ts * (l.tm - tm));
        tlp = f * (l.ty + l.ts * (kMean * (finite_ref(l.m) - r.m)) * inv - l.ts * (kMean * kLn2 * r.l2));
      }
    }
    z = warp_total(z);
    ttl = warp_total(ttl);
    tlp = warp_total(tlp);
    if (z == 0.f) {                                                    // no list
      r.loss = 0.f * r.l2;                                             // NaN in a row with one
      return r;
    }
    r.lt = tm;
    r.l2r = logf(z);
    r.w = 1.f;
    r.loss = ttl / z - r.l2r - tlp / z / kMean;
    return r;
  }
  const double mass = warp_total(l.mass);
  const double tr = fmax(1. - mass, 1. / (1 << 20));
  r.lt = logf((float)tr);
  r.w = (float)(outside ? mass + tr : mass);
  if (mass != mass) r.lt = r.w = NAN;
  if (kind == PG_DISTILL_FORWARD_REST) {
    const float tlp = warp_total(l.ts != 0.f ? l.ty + l.ts * (kMean * (finite_ref(l.m) - r.m)) * inv - l.ts * (kMean * kLn2 * r.l2) : 0.f) / kMean;
    r.loss = warp_total(l.ttl) - tlp + (outside ? r.lr > -1e30f ? (float)tr * (r.lt - r.lr) : (float)(tr * (r.lt - lr)) : 0.f);
  } else {
    float plp = 0.f, ptl = 0.f;
    if (l.s0 != 0.f) {
      const float d = (l.m - r.m) * c, f = ex2(fmaxf(d, kFloorY));
      if (f != 0.f) {
        plp = f * (l.s1 + l.s0 * (d - r.l2));
        ptl = f * l.etl;
      }
    }
    plp = warp_total(plp);
    ptl = warp_total(ptl);
    const float pr = outside ? expf(r.lr) : 0.f;
    r.loss = kLn2 * plp / s0 - ptl / s0 / kMean + (outside ? pr * (r.lr - r.lt) : 0.f);
  }
  return r;
}

__device__ __forceinline__ float key_value(unsigned long long key) {
  const uint32_t b = (uint32_t)(key >> 32);
  return __uint_as_float(b >> 31 ? b ^ 0x80000000u : ~b);
}

// A part of a row.  Units lie on 16-byte boundaries of the row's memory.  The up to 14 tokens before the first and behind the last one,
// the row's edges, are part 0's, one a thread.
template <typename T>
struct RowPart {
  const T* in;
  int head, units, first, last, edges, part;
  __device__ __forceinline__ RowPart(const TokenParams& p, int row, int part_) : part(part_) {
    in = (const T*)p.in + row * p.in_stride;
    head = min((int)((16 - ((uintptr_t)in & 15)) & 15) / (int)sizeof(T), p.vocab);
    units = (p.vocab - head) / kPer<T>;
    first = part * p.units;
    last = min(first + p.units, units);
    edges = part == 0 ? p.vocab - units * kPer<T> : 0;
  }
  __device__ __forceinline__ bool owns(int t) const {
    const int u = (t - head) >> (kPer<T> == 8 ? 3 : 2);
    return u < 0 || u >= units ? part == 0 : u >= first && u < last;
  }
  __device__ __forceinline__ int edge(int i) const { return i < head ? i : i + units * kPer<T>; }
};

constexpr int kTokUnits = 8;                    // units of a thread and tile
constexpr int kTileUnits = kTokUnits * kTokThreads;
constexpr int kTileBytes = kTileUnits * 16;
// Bits of listed tokens: a byte for each unit u of a part, a thread's of a tile side by side.
__device__ __forceinline__ int bits_at(int u) {
  return (u / kTileUnits * kTokThreads + u % kTokThreads) * kTokUnits + u % kTileUnits / kTokThreads;
}

// The n-th largest of the warp's values, 1 <= n <= 32.
__device__ __forceinline__ float nth_largest(float v, int n) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int k = 2; k <= 32; k <<= 1)
#pragma unroll
    for (int j = k >> 1; j; j >>= 1) {
      const float o = __shfl_xor_sync(~0u, v, j);
      v = ((lane & j) == 0) == ((lane & k) == 0) ? fmaxf(v, o) : fminf(v, o);
    }
  return __shfl_sync(~0u, v, n - 1);
}

// For alternatives.  Keys order by (logit, lowest index first); 0 is none.
struct TopShared {
  unsigned long long cand[kCandidates], best[PG_TOKEN_MAX_TOP];
  float bounds[kTokWarps], bound;
  unsigned int hist[256];
  unsigned long long prefix;
  int count, groups, left, shift;
  unsigned int group[kMostGroups];                                  // tiles of threads: largest logit, tile * kTokThreads + thread
  uint16_t most[kMostTiles * kTokThreads];                          // the largest logit of each thread's tile; as many as there are tiles

  __device__ __forceinline__ void push(float x, int id) {
    const int at = atomicAdd(&count, 1);
    if (at < kCandidates) cand[at] = top_key(x, id);
  }
};

__host__ __device__ constexpr int top_bytes(int tiles) { return (int)sizeof(TopShared) - (kMostTiles - tiles) * kTokThreads * 2; }

// The largest of logits in 16 bits, not below it: as it is, or of fp32 ones rounded up to bf16.  Few bytes, since shared memory is
// taken from the cache that loads arrive in (46 KB more a CTA: 63 us, not 55, for 1184 x 131072).
template <typename T>
__device__ __forceinline__ uint32_t most_bits(uint32_t w) {
  if constexpr (sizeof(T) == 4) return (w >> 31 ? w : w + 0xFFFFu) >> 16;
  else return max2(w, w >> 16 | w << 16, T()) & 0xFFFFu;
}
template <typename T>
__device__ __forceinline__ float most_value(uint32_t h) {
  if constexpr (std::is_same<T, __half>::value) return __half2float(__ushort_as_half((unsigned short)h));
  else return __uint_as_float(h << 16);
}
// The n largest keys of the part into `best`, in order; by all threads.  `most` is filled, m a thread's largest logit, edge_x and list_x
// what it has outside the units (-inf: nothing).
// Every warp has as many threads with a logit at or above its own bound, the n / warps-th largest of its threads' largest, that all of
// them make n; so the n-th largest logit is not below the least of these bounds, and few of the threads' tiles reach it.  They are read again.
template <typename T>
__device__ __noinline__ void select_top(TopShared& s, const RowPart<T>& at, int n, int tiles, float m, float edge_x, float list_x, int list_id,
                                        const uint8_t* bits) {
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const float own = nth_largest(m, (n + kTokWarps - 1) / kTokWarps);
  if (lane == 0) s.bounds[warp] = own;
  if (tid == 0) s.count = s.groups = 0;
  __syncthreads();
  float bound = s.bounds[0];
#pragma unroll
  for (int i = 1; i < kTokWarps; ++i) bound = fminf(bound, s.bounds[i]);
  if (m >= bound && m > -INFINITY) {
    for (int tile = 0; tile < tiles; ++tile) {
      const uint32_t h = s.most[tile * kTokThreads + tid];
      const float x = most_value<T>(h);
      if (x >= bound && x > -INFINITY) {
        const int to = atomicAdd(&s.groups, 1);
        if (to < kMostGroups) s.group[to] = (h ^ (h >> 15 ? 0xFFFFu : 0x8000u)) << 16 | (uint32_t)(tile * kTokThreads + tid);
      }
    }
  }
  for (int i = tid; i < n; i += kTokThreads) s.best[i] = 0;
  if (tid == 0) s.bound = bound;
  __syncthreads();
  const int work = s.groups;
  // The n-th largest of these tiles' largest is a better bound, worth its search for long lists (64 of 2368 x 131072 bf16: 134 us, not 140).
  if (n > 32 && work <= kMostGroups && work > n) {
    for (int i = tid; i < work; i += kTokThreads) {
      const unsigned int key = s.group[i];
      int rank = 0;
#pragma unroll 8
      for (int j = 0; j < work; ++j) rank += s.group[j] > key;
      if (rank == n - 1) {
        uint32_t h = key >> 16;
        if (sizeof(T) == 4 && h > 0) --h;                           // what was rounded up may lie below
        h ^= h >> 15 ? 0x8000u : 0xFFFFu;
        s.bound = fmaxf(bound, most_value<T>(h));
      }
    }
    __syncthreads();
    bound = s.bound;
  }
  if (edge_x >= bound && edge_x > -INFINITY) s.push(edge_x, at.edge(tid));
  if (list_x >= bound && list_x > -INFINITY) s.push(list_x, list_id);
#pragma unroll 2
  for (int i = tid; i < work * kTokUnits && work <= kMostGroups; i += kTokThreads) {
    const unsigned int key = s.group[i / kTokUnits];
    uint32_t h = key >> 16;
    h ^= h >> 15 ? 0x8000u : 0xFFFFu;
    if (!(most_value<T>(h) >= bound)) continue;
    const int g = key & 0xFFFFu, u = g / kTokThreads * kTileUnits + i % kTokUnits * kTokThreads + g % kTokThreads;
    if (at.first + u >= at.last) continue;
    const int t0 = at.head + (at.first + u) * kPer<T>;
    const uint4 unit = *(const uint4*)(at.in + t0);
    if (!(most_value<T>(most_bits<T>(max_unit<T>(Empty8<T>::word, unit))) >= bound)) continue;
    const uint32_t listed = bits ? bits[bits_at(u)] : 0u;
#pragma unroll
    for (int k = 0; k < kPer<T> / 2; ++k) {
      float x0, x1;
      split2(pair_of<T>(unit, k), x0, x1);
      if (x0 >= bound && x0 > -INFINITY && !(listed >> (2 * k) & 1)) s.push(x0, t0 + 2 * k);
      if (x1 >= bound && x1 > -INFINITY && !(listed >> (2 * k + 1) & 1)) s.push(x1, t0 + 2 * k + 1);
    }
  }
  __syncthreads();
  int total = work > kMostGroups ? kCandidates + 1 : s.count;
  __syncthreads();
  if (total > kCandidates) {
    // Many equal logits: the n-th largest key of the part, eight bits at a time, until few enough reach it.
    auto each = [&](auto f) {
      for (int t = at.head + at.first * kPer<T> + tid; t < at.head + at.last * kPer<T>; t += kTokThreads) {
        const float x = to_float(at.in[t]);
        if (x > -INFINITY) f(top_key(x, t));
      }
      if (tid < at.edges) {
        const float x = to_float(at.in[at.edge(tid)]);
        if (x > -INFINITY) f(top_key(x, at.edge(tid)));
      }
    };
    if (tid == 0) {
      s.prefix = 0;
      s.left = n;
    }
    __syncthreads();
    for (int by = 56; by >= 0; by -= 8) {
      for (int i = tid; i < 256; i += kTokThreads) s.hist[i] = 0;
      __syncthreads();
      const unsigned long long before = s.prefix;
      each([&](unsigned long long key) {
        if (by == 56 || key >> (by + 8) == before) atomicAdd(&s.hist[key >> by & 255], 1u);
      });
      __syncthreads();
      if (tid == 0) {
        int want = s.left, b = 255;
        while (b > 0 && (int)s.hist[b] < want) want -= s.hist[b--];
        s.prefix = before << 8 | (unsigned)b;
        s.shift = by;
        s.count = n - want + (int)s.hist[b] <= kCandidates ? 0 : -1;
        s.left = want;
      }
      __syncthreads();
      if (s.count == 0) break;
    }
    const unsigned long long from = s.prefix << s.shift;
    __syncthreads();
    each([&](unsigned long long key) {
      if (key >= from) s.cand[atomicAdd(&s.count, 1) & (kCandidates - 1)] = key;
    });
    __syncthreads();
    total = s.count;
  }
  for (int i = tid; i < total; i += kTokThreads) {
    const unsigned long long key = s.cand[i];
    int rank = 0, j = 0;
#pragma unroll 8
    for (; j + 1 < total; j += 2) {
      const ulonglong2 o = *reinterpret_cast<const ulonglong2*>(&s.cand[j]);
      rank += (o.x > key) + (o.y > key);
    }
    if (j < total) rank += s.cand[j] > key;
    if (rank < n) s.best[rank] = key;
  }
  __syncthreads();
}

// What a thread knows of its given token and of its entry of the teacher's list (-1: none, padding, unused).
struct Entry {
  int id, tid;
  float x, tx, tl, dl;
};

// The slope for the stream: y = l c - r in one rounding, with r = ref c + l2 rounded; what the roundings of r leave, up to 1e-6 of
// every p_v, is a factor of a and b.  The steps to `off` are exact as they stand, not as fused products.
// From |ref c| = 2^31 on (rows, or what is outside the list, masked throughout by a finite value; a small T) off could be 128 and the factor
// out of range.  But there logits next to each other are 2^31 2^-24 = 128 apart in y, so e is 0 but for those equal to ref.  Any
// other c that keeps them apart does as well: a power of two with |ref c| in [2^31, 2^32), whose product with ref is exact, and
// y = 0 for those that are equal; their 2^-l2 is the factor.  Short of
// 2^31 e carries 2^off, |off| <= 64, and shares below 2^-62 may come out as 0.  (The difference first, in a loop of its own, costs every row with
// a bucket 8 %.)
struct Slope2 {
  f2 c, nr, a, b;
  __device__ __forceinline__ Slope2(const TokenSlope& k, float c_) {
    const float mc = __fmul_rn(k.ref, c_);
    float r = __fadd_rn(mc, k.l2);
    const float back = __fsub_rn(r, mc);
    float off = __fadd_rn(fmaf(k.ref, c_, -mc), __fadd_rn(__fsub_rn(mc, __fsub_rn(r, back)), __fsub_rn(k.l2, back)));   // ref c + l2 - r
    if (!(fabsf(mc) < 2147483648.f)) {
      c_ = __uint_as_float(min(285u - (__float_as_uint(k.ref) >> 23 & 255u), 254u) << 23);
      r = k.ref * c_;
      off = k.l2;
    }
    const float f = ex2(-off), bl = k.b * kLn2;
    c = make2(c_, c_);
    nr = make2(-r, -r);
    const float af = f * fmaf(-off, bl, k.a), bf = f * bl;
    a = make2(af, af);
    b = make2(bf, bf);
  }
};
template <typename T, bool kEnt>
__device__ __forceinline__ void slope_unit(const uint4& v, const Slope2& k, float (&g)[kPer<T>]) {
#pragma unroll
  for (int i = 0; i < kPer<T> / 2; ++i) {
    float y0, y1;
    split2(fma2(pair_of<T>(v, i), k.c, k.nr), y0, y1);
    const f2 e = make2(ex2(y0), ex2(y1));
    f2 f = k.a;
    if (kEnt) f = fma2(make2(fmaxf(y0, kFloorY), fmaxf(y1, kFloorY)), k.b, k.a);
    split2(mul2(e, f), g[2 * i], g[2 * i + 1]);
  }
}
// A part from memory, logit by logit: whose gradient lies off its logits' 16 bytes, or whose row has an infinite logit (NaN).
template <typename T>
__device__ __noinline__ void slope_single(const RowPart<T>& at, T* dl, const TokenSlope& k, float c) {
  for (int t = at.head + at.first * kPer<T> + threadIdx.x; t < at.head + at.last * kPer<T>; t += kTokThreads) {
    const float y = (to_float(at.in[t]) - k.ref) * c - k.l2;
    dl[t] = from_float<T>(ex2(y) * fmaf(fmaxf(y, kFloorY), k.b * kLn2, k.a));
  }
}
// The part's gradient where a row has no derivatives.
template <typename T>
__device__ __noinline__ void zero_part(const RowPart<T>& at, T* dl) {
  if (((uintptr_t)(dl + at.head) & 15) == 0) {
    for (int u = at.first + (int)threadIdx.x; u < at.last; u += kTokThreads) __stcs((uint4*)(dl + at.head) + u, make_uint4(0u, 0u, 0u, 0u));
  } else {
    for (int t = at.head + at.first * kPer<T> + threadIdx.x; t < at.head + at.last * kPer<T>; t += kTokThreads) dl[t] = from_float<T>(0.f);
  }
  if ((int)threadIdx.x < at.edges) dl[at.edge(threadIdx.x)] = from_float<T>(0.f);
}
template <typename T>
__device__ __forceinline__ void put_edge(T* to, float x, const TokenSlope& k, float c) {
  const float y = (x - k.ref) * c - k.l2;
  *to = from_float<T>(ex2(y) * fmaf(fmaxf(y, kFloorY), k.b * kLn2, k.a));
}

// The divergence's derivative to the logits outside the list, over their shares of what is there (pr = p_r, whose logarithm may be far
// beyond 32 bits).
__device__ __forceinline__ float rest_slope(const TokenRow& r, int kind, float pr) {
  if (kind == PG_DISTILL_FORWARD_REST) return pr * r.w - expf(r.lt);
  return pr == 0.f ? 0.f : pr * (r.lr - r.lt - r.loss);
}

// By one warp: the gradient's slope from what is known of the row.
__device__ __forceinline__ TokenSlope slope_of(const TokenRow& r, bool rest, int kind, float lp_part, float dh, float dd, float inv) {
  TokenSlope k;
  if (rest) {
    const bool outside = r.lr > -INFINITY;
    const float pr = outside || r.lr != r.lr ? expf(r.lr) : 0.f;
    k.a = outside || r.lr != r.lr ? inv * ((pr == 0.f ? 0.f : pr * (lp_part - dh * r.lr)) + (dd == 0.f ? 0.f : dd * rest_slope(r, kind, pr))) : 0.f;
    k.b = -inv * dh * pr;
    k.ref = r.mr;
    k.l2 = r.l2r;
  } else {
    k.a = inv * (lp_part + dd * r.w);
    k.b = -inv * dh;
    k.ref = r.m;
    k.l2 = r.l2;
  }
  if (r.some == 0.f) k.a = k.b = 0.f;
  return k;
}

// Whether the list has `id` from entry j on, a multiple of 4.
__device__ __forceinline__ bool on_list(const TokenShared& s, int id, int j, int n_list) {
  bool on = false;
#pragma unroll 4
  for (; j < n_list; j += 4) {
    const int4 o = *reinterpret_cast<const int4*>(&s.tid[j]);
    on |= o.x == id || o.y == id || o.z == id || o.w == id;
  }
  return on;
}
// By whole warps, an entry a lane: whether a later entry of the list has the same id.  Of those the last one counts.
__device__ __forceinline__ bool again_later(const TokenShared& s, int id, int n_list) {
  const unsigned int same = __match_any_sync(~0u, id);
  return (same >> (threadIdx.x & 31) >> 1) != 0u || on_list(s, id, (threadIdx.x | 31) + 1, n_list);
}

// Given and listed tokens, over what the stream has written.
template <typename T>
__device__ __forceinline__ void fix_tokens(const TokenShared& s, const RowPart<T>& at, const Entry& e, const TokenRow& r, T* dl, int n_ids,
                                           int n_list, bool fix_list, bool rest, int kind, float lp_part, float dh, float dd,
                                           float inv) {
  const int tid = threadIdx.x;
  const float c = inv * kLog2e;
  auto base = [&](float pv, float lp) { return pv == 0.f ? 0.f : pv * (lp_part - dh * lp); };
  if (fix_list && e.tid >= 0 && at.owns(e.tid)) {
    const float y = (e.tx - r.m) * c - r.l2, pv = ex2(y), lp = kLn2 * y;
    float dist;
    if (kind == PG_DISTILL_FORWARD) dist = r.w * pv - expf(e.tl - r.lt - r.l2r);
    else if (kind == PG_DISTILL_FORWARD_REST) dist = r.w * pv - expf(e.tl);
    else dist = pv == 0.f ? 0.f : pv * (lp - e.tl - r.loss);
    float sum = base(pv, lp) + (dd == 0.f ? 0.f : dd * dist);
    for (int j = 0; j < n_ids; ++j)
      if (s.gid[j] == e.tid) sum += s.gdl[j];
    dl[e.tid] = from_float<T>(r.some != 0.f ? inv * sum : 0.f);
  }
  if (e.id >= 0 && at.owns(e.id)) {
    bool mine = true;                                               // the last of its token, and not on the list
    for (int j = tid + 1; j < n_ids; ++j) mine &= s.gid[j] != e.id;
    if (fix_list) mine &= !on_list(s, e.id, 0, n_list);
    if (mine) {
      const float y = (e.x - r.m) * c - r.l2, pv = ex2(y);
      float sum = base(pv, kLn2 * y);
      if (!rest) sum += dd * r.w * pv;
      else if (dd != 0.f) sum += dd * ex2((e.x - r.mr) * c - r.l2r) * rest_slope(r, kind, expf(r.lr));   // outside the list
      for (int j = 0; j <= tid; ++j)
        if (s.gid[j] == e.id) sum += s.gdl[j];
      dl[e.id] = from_float<T>(r.some != 0.f ? inv * sum : 0.f);
    }
  }
}

// How the L2 cache is to keep what a load brings: evicted first if it is not read again, so that it does not drive out what is.
__device__ __forceinline__ uint64_t keep_policy(bool again) {
  uint64_t first, normal;
  asm("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(first));
  asm("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(normal));
  return again ? normal : first;
}
// Unit j of the thread in a tile.
template <typename T>
__device__ __forceinline__ void load_unit(const T* at, int j, uint64_t policy, uint4& v) {
  asm volatile("ld.global.L2::cache_hint.v4.u32 {%0, %1, %2, %3}, [%4], %5;" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(at + j * kTokThreads * kPer<T>), "l"(policy) : "memory");
}
template <typename T>
__device__ __forceinline__ bool whole_tile(const RowPart<T>& at, int tile) { return at.first + (tile + 1) * kTileUnits <= at.last; }
// The thread's place in a tile.
template <typename T>
__device__ __forceinline__ const T* tile_at(const RowPart<T>& at, int tile) {
  return at.in + at.head + (int64_t)(at.first + tile * kTileUnits + (int)threadIdx.x) * kPer<T>;
}
// The thread's units of a tile; -inf where the part has none.
template <typename T>
__device__ __forceinline__ void load_tile(const RowPart<T>& at, int tile, uint64_t policy, uint4 (&raw)[kTokUnits]) {
  const T* from = tile_at(at, tile);
  if (whole_tile(at, tile)) {
#pragma unroll
    for (int j = 0; j < kTokUnits; ++j) load_unit(from, j, policy, raw[j]);
  } else {
    const int u0 = at.first + tile * kTileUnits + (int)threadIdx.x;
#pragma unroll
    for (int j = 0; j < kTokUnits; ++j) {
      raw[j] = empty_unit<T>();
      if (u0 + j * kTokThreads < at.last) load_unit(from, j, policy, raw[j]);
    }
  }
}

// The gradient of a tile in registers; dl: of the row's first unit, its units on 16 bytes.  kAsk: as a unit is done
// with, the next tile's is asked for (from); that tile is whole.
template <typename T, bool kEnt, bool kAsk>
__device__ __forceinline__ void slope_tile(const RowPart<T>& at, int tile, uint4 (&raw)[kTokUnits], const Slope2& k, T* dl, const T* from,
                                            uint64_t policy) {
  const int left = at.last - at.first - tile * kTileUnits - (int)threadIdx.x;   // units from the thread's first on
  T* to = dl + (int64_t)(at.first + tile * kTileUnits + (int)threadIdx.x) * kPer<T>;
#pragma unroll
  for (int j = 0; j < kTokUnits; ++j) {
    float g[kPer<T>];
    slope_unit<T, kEnt>(raw[j], k, g);
    if (kAsk) load_unit(from, j, policy, raw[j]);
    if (j * kTokThreads < left) store_unit<T>(to + j * kTokThreads * kPer<T>, g);
  }
}
// The sums of a tile in registers, against y = l c - by; kFirst: y = (l - by) c, differences first.
template <typename T, bool kEnt, bool kAsk, bool kFirst>
__device__ __forceinline__ void sum_tile(uint4 (&raw)[kTokUnits], float c, float by, float& t0, float& t1, const T* from, uint64_t policy) {
  const f2 nr = make2(-by, -by), c2 = make2(c, c);
  f2 a0 = make2(0.f, 0.f), a1 = a0, b0 = a0, b1 = a0;
#pragma unroll
  for (int j = 0; j < kTokUnits; ++j) {
#pragma unroll
    for (int i = 0; i < kPer<T> / 2; ++i) {
      float y0, y1;
      split2(kFirst ? mul2(add2(pair_of<T>(raw[j], i), nr), c2) : fma2(pair_of<T>(raw[j], i), c2, nr), y0, y1);
      const f2 e = make2(ex2(y0), ex2(y1));
      if (i & 1) b0 = add2(b0, e);
      else a0 = add2(a0, e);
      if (kEnt) {
        const f2 y = make2(fmaxf(y0, kFloorY), fmaxf(y1, kFloorY));
        if (i & 1) b1 = fma2(e, y, b1);
        else a1 = fma2(e, y, a1);
      }
    }
    if (kAsk) load_unit(from, j, policy, raw[j]);
  }
  float u, v;
  split2(add2(a0, b0), u, v);
  t0 = u + v;
  split2(add2(a1, b1), u, v);
  t1 = u + v;
}

// Forward, with the gradient on top (kGrad).
template <typename T, bool kGrad, bool kEnt, int kLists>
__global__ void __launch_bounds__(kTokThreads, kTokCtas)
token_kernel(const __grid_constant__ TokenParams p) {
  constexpr bool kRest = kLists == kBucket;
  constexpr int kUnits = kTokUnits;
  __shared__ TokenShared s;
  extern __shared__ __align__(16) unsigned char more[];             // a tile; TopShared and the parts' lists if there are alternatives; bits (kRest)
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int row = blockIdx.x / p.parts;
  const RowPart<T> at(p, row, blockIdx.x - row * p.parts);
  const bool many = p.parts > 1;
  if (many) cluster_arrive();                                       // all CTAs run before one writes into another's memory
  const int n_ids = p.t.n_ids, n_list = kLists == kNoList ? 0 : p.t.n_teacher, n_top = p.t.n_top;
  const int lists = (n_list + 31) / 32;
  unsigned char* const behind = more + (kGrad && p.tiles > 1 ? kTileBytes : 0);
  TopShared& top = *reinterpret_cast<TopShared*>(behind);
  unsigned long long* const merge = reinterpret_cast<unsigned long long*>(behind + top_bytes(p.tiles));
  uint8_t* const bits = reinterpret_cast<uint8_t*>(behind + (n_top ? top_bytes(p.tiles) + (many ? kMergeBytes : 0) : 0));

  if constexpr (kRest) {
    for (int i = tid; i < p.tiles * kTokThreads; i += kTokThreads) reinterpret_cast<uint2*>(bits)[i] = make_uint2(0u, 0u);
    if (tid == 0) s.edges = 0;
  }
  uint4* const kept = reinterpret_cast<uint4*>(more) + tid;         // a thread's own places: its units of tile 1, those of tile 0 stay in registers
  uint4 raw[kUnits];
  const bool soon = !kGrad && p.o.saved && (int64_t)(p.n_rows - row) * p.vocab * (int)sizeof(T) <= kSavedBytes;
  const uint64_t last_read = keep_policy(soon), read_again = keep_policy(true);
  // the part's cut tile first: the last two, that stay here, are whole
  load_tile(at, p.tiles - 1, kGrad && p.tiles > kOnChip ? read_again : last_read, raw);
  const float inv = p.t.temperature ? 1.f / p.t.temperature[row] : 1.f, c = inv * kLog2e;
  const float dh = kGrad && p.g.dentropy ? p.g.dentropy[row] * p.g.entropy_scale : 0.f;
  const float dd = kGrad && p.g.ddistill ? p.g.ddistill[row] * p.g.distill_scale : 0.f;
  const float edge_x = tid < at.edges ? to_float(at.in[at.edge(tid)]) : -INFINITY;
  // Given and listed tokens, one a thread.  What depends on these loads - the tokens' logits, what others see of them - comes after the first
  // tile, so that the warps that have them do not wait for two of them in turn before the stream.
  const int given = tid < n_ids ? p.t.ids[(int64_t)row * n_ids + tid] : -1;
  const float given_dl = kGrad && tid < n_ids && p.g.dlogp ? p.g.dlogp[(int64_t)row * n_ids + tid] : 0.f;
  const int listed = tid < n_list ? p.t.teacher_ids[(int64_t)row * n_list + tid] : -1;
  const float listed_tl = tid < n_list ? p.t.teacher_logp[(int64_t)row * n_list + tid] : 0.f;
  Entry my = {-1, -1, 0.f, -INFINITY, 0.f, 0.f};
  T given_x = from_float<T>(0.f), listed_x = given_x;
  auto meet = [&] {
    if ((unsigned int)given < (unsigned int)p.vocab) {
      my.id = given;
      my.dl = given_dl;
      given_x = at.in[given];
    }
    my.tl = listed_tl;
    if ((unsigned int)listed < (unsigned int)p.vocab && !(listed_tl == -INFINITY)) {
      my.tid = listed;
      listed_x = at.in[listed];
    }
    if (tid < n_ids) {
      s.gid[tid] = my.id;
      s.gdl[tid] = my.dl;
    }
    if (tid < (n_list + 3 & ~3)) s.tid[tid] = my.tid;
    if (kGrad && warp < (n_ids + 31) / 32) {
      const float d = warp_total(my.dl);
      if (lane == 0) s.dsum[warp] = d;
    }
  };
  if (kGrad) meet();                                                // registers are scarce here: not through the first tile
  if constexpr (kRest) {
    __syncthreads();                                                // the bits are zero
    if ((unsigned int)listed < (unsigned int)p.vocab && !(listed_tl == -INFINITY) && at.owns(listed)) {
      const int t = listed - at.head;
      if (t < 0 || t >= at.units * kPer<T>) {
        atomicOr(&s.edges, 1u << (t < 0 ? listed : listed - at.units * kPer<T>));
      } else {
        const int b = bits_at(t / kPer<T> - at.first);
        atomicOr(reinterpret_cast<uint32_t*>(bits) + (b >> 2), 1u << ((b & 3) * 8 + t % kPer<T>));
      }
    }
    __syncthreads();
  }
  // Takes the listed tokens out of the registers.
  auto mask_tile = [&](int tile) {
    if constexpr (kRest) {
      const uint2 b = reinterpret_cast<const uint2*>(bits)[tile * kTokThreads + tid];
      if (b.x | b.y) {
#pragma unroll
        for (int j = 0; j < kUnits; ++j)
          if (const uint32_t l = (j < 4 ? b.x : b.y) >> (j % 4 * 8) & 255u) set_empty<T>(raw[j], l);
      }
    }
  };
  const int lists_at = max(p.tiles - (kGrad ? 1 : 2), 0);           // the listed tokens' logits were asked for a tile before
  float m = -INFINITY, s0 = 0.f, s1 = 0.f, edge_left = -INFINITY;
  for (int tile = p.tiles - 1; tile >= 0; --tile) {
    mask_tile(tile);
    if (kGrad && tile == kOnChip - 1 && tile > 0) {
#pragma unroll
      for (int j = 0; j < kUnits; ++j) kept[j * kTokThreads] = raw[j];
    }
    uint32_t w = Empty8<T>::word;
#pragma unroll
    for (int j = 0; j < kUnits; ++j) w = max_unit<T>(w, raw[j]);
    if (n_top) top.most[tile * kTokThreads + tid] = (uint16_t)most_bits<T>(w);
    const float tm = max_of<T>(w);
    refer(m, fmaxf(m, tm), c, s0, s1);
    m = fmaxf(m, tm);
    const float ref = finite_ref(m), r = ref * c;
    float t0, t1;
    // as a unit is done with, the next tile's is asked for
    const bool ask = tile > 0 && whole_tile(at, tile - 1);
    const uint64_t policy = kGrad && tile > kOnChip ? read_again : last_read;
    // By warps: a mask's few allowed tokens lie in few threads, and one path is cheaper than two.  Both cost the same where HBM is the
    // bound (2368 x 131072 bf16, all but 64 tokens masked: 97 us as without a mask).
    if (__any_sync(~0u, !(fabsf(r) < kFar))) {
      if (ask) sum_tile<T, kEnt, true, true>(raw, c, ref, t0, t1, tile_at(at, tile - 1), policy);
      else sum_tile<T, kEnt, false, true>(raw, c, ref, t0, t1, nullptr, 0);
      s0 += t0;
      if (kEnt) s1 += t1;
    } else {
      // y = l c - r in one rounding; what r = m c rounded is off by is taken back from the sums
      const float off = fmaf(ref, c, -r), f = ex2(-off);
      if (ask) sum_tile<T, kEnt, true, false>(raw, c, r, t0, t1, tile_at(at, tile - 1), policy);
      else sum_tile<T, kEnt, false, false>(raw, c, r, t0, t1, nullptr, 0);
      s0 += f * t0;
      if (kEnt) s1 += f * fmaf(-off, t0, t1);
    }
    if (!kGrad && tile == p.tiles - 1) meet();
    if (kLists != kNoList && tile == lists_at) {                    // while the next tile is on its way
      if (lists > 1) __syncthreads();                               // the list's ids are there
      else __syncwarp();
      if (warp < lists) {
        if (my.tid >= 0) my.tx = to_float(listed_x);
        if (again_later(s, my.tid, n_list)) my.tid = -1;
        const bool used = my.tid >= 0;
        const float x = used ? my.tx : -INFINITY;
        ListSums l;
        l.m = warp_most(x);
        const float y = (x - finite_ref(l.m)) * c, e = used ? ex2(y) : 0.f;
        l.s0 = warp_total(e);
        l.s1 = warp_total(e * fmaxf(y, kFloorY));
        l.etl = warp_total(e != 0.f ? e * (kMean * my.tl) : 0.f);
        l.tm = !kRest ? warp_most(used ? my.tl : -INFINITY) : 0.f;
        const float t = used ? expf(my.tl - finite_ref(l.tm)) : 0.f;
        l.ts = warp_total(t);
        l.ttl = warp_total(t != 0.f ? t * (my.tl - finite_ref(l.tm)) : 0.f);
        l.ty = warp_total(t != 0.f ? t * (kMean * (x - finite_ref(l.m))) * inv : 0.f);
        l.mass = kRest ? warp_total(used ? exp((double)my.tl) : 0.) : 0.;
        if (lane == 0) s.list[warp] = l;
      }
    }
    if (tile > 0 && !ask) load_tile(at, tile - 1, policy, raw);
  }
  if (at.edges > 0) {
    const float x = kRest && tid < at.edges && s.edges >> tid & 1 ? -INFINITY : edge_x;
    const float to = fmaxf(m, x), y = (x - finite_ref(to)) * c, e = ex2(y);
    refer(m, to, c, s0, s1);
    m = to;
    s0 += e;
    s1 += e * fmaxf(y, kFloorY);
    edge_left = x;
  }
  my.x = to_float(given_x);
  const float own = m;
  m = warp_most(m);
  refer(own, m, c, s0, s1);
  s0 = warp_total(s0);
  if (kEnt) s1 = warp_total(s1);
  if (n_top)
    select_top(top, at, n_top, p.tiles, own, edge_left, kRest && my.tid >= 0 && at.owns(my.tid) ? my.tx : -INFINITY, my.tid,
               kRest ? bits : nullptr);
  // the triples of the parts' warps, to all parts
  float4* const triples = s.part;
  if (many) {
    cluster_wait();
    if (lane < p.parts) peer_store(peer(&triples[at.part * kTokWarps + warp], lane), m, s0, s1);
    for (int i = tid; i < n_top; i += kTokThreads) peer_store(peer(merge + at.part * PG_TOKEN_MAX_TOP + i, 0), top.best[i]);
    __syncwarp();
    cluster_arrive();
    cluster_wait();
  } else {
    if (lane == 0) triples[warp] = make_float4(m, s0, s1, 0.f);
    __syncthreads();
  }
  TokenRow r;
  if (warp == 0) {
    r = finish_row<kLists>(s, triples, p.parts, lists, p.t.kind, inv);
    float lp_part = 0.f;
    TokenSlope k = {};
    if (kGrad) {
      float d = 0.f;
      for (int i = 0; i < (n_ids + 31) / 32; ++i) d += s.dsum[i];
      lp_part = -fmaf(dh, r.h, d);                                // of p_v (.. - dh ln p_v)
      k = slope_of(r, kRest, p.t.kind, lp_part, dh, dd, inv);
    }
    if (lane == 0) {
      s.row = r;
      s.slope = k;
      s.lp_part = lp_part;
    }
  }
  bool quiet = false;
  if (kGrad) quiet = !__syncthreads_or(my.dl != 0.f || dh != 0.f || dd != 0.f);
  else __syncthreads();
  r = s.row;
  if (at.part == 0) {
    if (tid < n_ids && p.o.logp) {
      const float lp = r.some != 0.f ? (my.x - r.m) * inv - kLn2 * r.l2 : -INFINITY;
      p.o.logp[(int64_t)row * n_ids + tid] = my.id >= 0 ? lp : 0.f;
    }
    if (tid == 0) {
      if (p.o.lse) p.o.lse[row] = r.some != 0.f ? r.m * inv + kLn2 * r.l2 : -INFINITY;
      if (p.o.entropy) p.o.entropy[row] = r.h;
      if (p.o.distill) p.o.distill[row] = r.loss;
      if (p.o.saved) save_row((float4*)p.o.saved + (int64_t)row * (PG_TOKEN_SAVED / 4), r);
    }
    if (n_top) {
      auto write = [&](int at, unsigned long long key) {
        const float x = key_value(key);
        p.o.top_ids[(int64_t)row * n_top + at] = key ? (int)(0xFFFFFFFFu - (uint32_t)key) : -1;
        if (p.o.top_logp) p.o.top_logp[(int64_t)row * n_top + at] = key ? (x - r.m) * inv - kLn2 * r.l2 : -INFINITY;
      };
      if (!many) {
        for (int i = tid; i < n_top; i += kTokThreads) write(i, top.best[i]);
      } else {
        // the parts' lists are sorted: a key's rank is its own place and how many of each other list are above it
        const unsigned long long* from = merge;
        auto above = [&](int o, unsigned long long key) {
          int a = 0, b = n_top;
          while (a < b) {
            const int mid = (a + b) >> 1;
            if (from[o * PG_TOKEN_MAX_TOP + mid] > key) a = mid + 1;
            else b = mid;
          }
          return a;
        };
        for (int i = tid; i < n_top * p.parts; i += kTokThreads) {
          const int q = i / n_top, at = i - q * n_top;
          const unsigned long long key = from[q * PG_TOKEN_MAX_TOP + at];
          if (!key) continue;
          int rank = at;
          for (int o = 0; o < p.parts; ++o)
            if (o != q) rank += above(o, key);
          if (rank < n_top) write(rank, key);
        }
        if (tid < n_top) {                                        // places that are left over
          int some = 0;
          for (int o = 0; o < p.parts; ++o) some += above(o, 0);
          if (tid >= some) write(tid, 0);
        }
      }
    }
  }
  if constexpr (kGrad) {
    T* dl = (T*)p.dl + row * p.dl_stride;
    if (quiet) {                                                      // no derivatives: zeros, whatever the row holds
      zero_part(at, dl);
      return;
    }
    const TokenSlope slope = s.slope;
    const Slope2 k(slope, c);
    const bool aligned = ((uintptr_t)(dl + at.head) & 15) == 0;
    // An infinite logit has no product with c.  (Without this condition the compiler lays the loops out with more spills: 236 us, not 226.)
    if (fabsf(slope.ref) == INFINITY || !aligned) {
      slope_single(at, dl, slope, c);
    } else {
      for (int tile = 0; tile < p.tiles; ++tile) {
        const int next = tile + 1;
        const bool ask = next >= kOnChip && next < p.tiles && whole_tile(at, next);
        if (ask) slope_tile<T, kEnt, true>(at, tile, raw, k, dl + at.head, tile_at(at, next), last_read);      // from the L2 cache
        else slope_tile<T, kEnt, false>(at, tile, raw, k, dl + at.head, nullptr, 0);
        if (next < kOnChip && next < p.tiles) {
#pragma unroll
          for (int j = 0; j < kUnits; ++j) raw[j] = kept[j * kTokThreads];
        } else if (next < p.tiles && !ask) {
          load_tile(at, next, last_read, raw);
        }
      }
    }
    if (tid < at.edges) put_edge(dl + at.edge(tid), edge_x, slope, c);
    const bool fix_list = n_list > 0 && (kRest || p.g.ddistill);
    if (n_ids > 0 || fix_list) {
      __syncthreads();
      // the row once more from shared memory, not from registers kept through the stream (2368 x 131072 bf16 with a list: 236 us, not 241)
      fix_tokens(s, at, my, s.row, dl, n_ids, n_list, fix_list, kRest, p.t.kind, s.lp_part, dh, dd, inv);
    }
  }
}

// The gradient alone, from what a forward pass has saved.
template <typename T, bool kEnt>
__global__ void __launch_bounds__(kTokThreads, kTokCtas)
token_backward_kernel(const __grid_constant__ TokenParams p) {
  constexpr int kUnits = kTokUnits;
  __shared__ TokenShared s;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int back = blockIdx.x / p.parts, row = p.n_rows - 1 - back;   // the rows that a forward pass read last are in the L2 cache
  const RowPart<T> at(p, row, blockIdx.x - back * p.parts);
  const int n_ids = p.g.dlogp ? p.t.n_ids : 0, n_list = p.t.n_teacher;
  const bool distill = p.g.ddistill != nullptr && n_list > 0, rest = distill && p.t.kind != PG_DISTILL_FORWARD;
  const float inv = p.t.temperature ? 1.f / p.t.temperature[row] : 1.f, c = inv * kLog2e;
  const float dh = p.g.dentropy ? p.g.dentropy[row] * p.g.entropy_scale : 0.f;
  const float dd = p.g.ddistill ? p.g.ddistill[row] * p.g.distill_scale : 0.f;
  const TokenRow r = load_row((const float4*)p.o.saved + (int64_t)row * (PG_TOKEN_SAVED / 4));
  Entry my = {-1, -1, 0.f, -INFINITY, 0.f, 0.f};
  if (tid < n_ids) {
    const int id = p.t.ids[(int64_t)row * n_ids + tid];
    if ((unsigned int)id < (unsigned int)p.vocab) {
      my.id = id;
      my.dl = p.g.dlogp[(int64_t)row * n_ids + tid];
    }
    s.gid[tid] = my.id;
    s.gdl[tid] = my.dl;
  }
  const bool quiet = !__syncthreads_or(my.dl != 0.f || dh != 0.f || dd != 0.f);
  const uint64_t last_read = keep_policy(false);
  T* dl = (T*)p.dl + row * p.dl_stride;
  if (quiet) {
    zero_part(at, dl);
    return;
  }
  uint4 raw[kUnits];
  load_tile(at, p.tiles - 1, last_read, raw);                       // the cut tile first
  const float edge_x = tid < at.edges ? to_float(at.in[at.edge(tid)]) : -INFINITY;
  if (my.id >= 0 && at.owns(my.id)) my.x = to_float(at.in[my.id]);
  if (distill && tid < n_list) {
    const int id = p.t.teacher_ids[(int64_t)row * n_list + tid];
    my.tl = p.t.teacher_logp[(int64_t)row * n_list + tid];
    if ((unsigned int)id < (unsigned int)p.vocab && !(my.tl == -INFINITY)) my.tid = id;
    if (my.tid >= 0 && at.owns(my.tid)) my.tx = to_float(at.in[my.tid]);
  }
  if (distill && tid < (n_list + 3 & ~3)) s.tid[tid] = my.tid;
  if (warp < (n_ids + 31) / 32) {
    const float d = warp_total(my.dl);
    if (lane == 0) s.dsum[warp] = d;
  }
  if (n_ids > 0 || distill) __syncthreads();
  if (distill && (tid & ~31) < n_list && again_later(s, my.tid, n_list)) my.tid = -1;
  float d = 0.f;
  for (int i = 0; i < (n_ids + 31) / 32; ++i) d += s.dsum[i];
  const float lp_part = -fmaf(dh, r.h, d);
  const TokenSlope slope = slope_of(r, rest, p.t.kind, lp_part, dh, dd, inv);
  const Slope2 k(slope, c);
  const bool aligned = ((uintptr_t)(dl + at.head) & 15) == 0;
  if (fabsf(slope.ref) == INFINITY || !aligned) {
    slope_single(at, dl, slope, c);
  } else {
    for (int tile = p.tiles - 1; tile >= 0; --tile) {
      const bool ask = tile > 0 && whole_tile(at, tile - 1);
      if (ask) slope_tile<T, kEnt, true>(at, tile, raw, k, dl + at.head, tile_at(at, tile - 1), last_read);
      else slope_tile<T, kEnt, false>(at, tile, raw, k, dl + at.head, nullptr, 0);
      if (tile > 0 && !ask) load_tile(at, tile - 1, last_read, raw);
    }
  }
  if (tid < at.edges) put_edge(dl + at.edge(tid), edge_x, slope, c);
  if (n_ids == 0 && !distill) return;
  __syncthreads();
  fix_tokens(s, at, my, r, dl, n_ids, n_list, distill, rest, p.t.kind, lp_part, dh, dd, inv);
}

template <typename T, bool kGrad, bool kEnt, int kLists>
int launch_forward(TokenParams p, cudaStream_t st) {
  constexpr int kTile = kTileUnits;
  constexpr bool kRest = kLists == kBucket;
  const int total = std::max(p.vocab / kPer<T>, 1);
  int parts = 1;
  // Rows that are read twice: parts of 128 KB, so that what all SMs work on stays in the L2 cache.  With a bucket: bits of 16 KB at most.
  if (kGrad) parts = std::min((total * 16 + kPartBytes - 1) / kPartBytes, kMostParts);
  else if (kRest) parts = std::min((total + 16383) / 16384, kMostParts);
  // More while SMs are without work: down to a unit a thread, but whole tiles where lists of alternatives have to be made and joined
  // (12 x 50001 with 100 of them 13 us in parts of a tile, 25 us in eight).
  const int busy = p.t.n_top ? 148 : 2 * 148, least = p.t.n_top ? kTile : kTokThreads;
  while (parts * 2 <= kMostParts && (int64_t)p.n_rows * parts * (p.t.n_top ? 2 : 1) <= busy && total / parts >= 2 * least) parts *= 2;
  if (p.t.n_top) parts = std::max(parts, (total + kMostTiles * kTile - 1) / (kMostTiles * kTile));
  p.parts = parts;
  p.units = (total + parts - 1) / parts;
  p.tiles = (p.units + kTile - 1) / kTile;
  if ((int64_t)p.n_rows * parts > 0x7FFFFFFFLL) return PG_EINVAL;
  const int bytes = (kGrad && p.tiles > 1 ? kTileBytes : 0) + (p.t.n_top ? top_bytes(p.tiles) + (parts > 1 ? kMergeBytes : 0) : 0) +
                    (kRest ? p.tiles * kTileUnits : 0);
  auto kernel = token_kernel<T, kGrad, kEnt, kLists>;
  static std::atomic<uint64_t> done{0};
  constexpr int kMostBytes = kTileBytes + (int)sizeof(TopShared) + kMergeBytes + PG_TOKEN_MAX_VOCAB / 4 / kMostParts + kTileUnits;
  if (bytes > 32 * 1024)
    if (const int rc = allow_shared(kernel, kMostBytes, done)) return rc;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(p.n_rows * parts));
  cfg.blockDim = dim3(kTokThreads);
  cfg.dynamicSmemBytes = bytes;
  cfg.stream = st;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = (unsigned)parts;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = parts > 1 ? 1 : 0;
  PG_CUDA(cudaLaunchKernelEx(&cfg, kernel, p));
  PG_LAUNCH_CHECK();
  return PG_OK;
}

template <typename T, bool kEnt>
int launch_backward(TokenParams p, cudaStream_t st) {
  const int total = std::max(p.vocab / kPer<T>, 1);
  // what a CTA learns of its row serves two tiles, where there are rows enough
  const int tiles = (total + kTileUnits - 1) / kTileUnits;
  const int most = (int)std::min<int64_t>(std::max<int64_t>((int64_t)p.n_rows * tiles / (2 * 148 * kTokCtas), 1), kBackwardTiles);
  p.parts = (tiles + most - 1) / most;
  p.units = (total + p.parts - 1) / p.parts;
  p.tiles = (p.units + kTileUnits - 1) / kTileUnits;
  if ((int64_t)p.n_rows * p.parts > 0x7FFFFFFFLL) return PG_EINVAL;
  token_backward_kernel<T, kEnt><<<(unsigned)(p.n_rows * p.parts), kTokThreads, 0, st>>>(p);
  PG_LAUNCH_CHECK();
  return PG_OK;
}

template <typename T, int kMode>
int token_launch(const TokenParams& p, cudaStream_t st) {
  const bool ent = kMode == kBackward ? p.g.dentropy != nullptr : p.o.entropy || p.o.saved || (kMode == kBoth && p.g.dentropy);
  if constexpr (kMode == kBackward) {
    return ent ? launch_backward<T, true>(p, st) : launch_backward<T, false>(p, st);
  } else {
    constexpr bool kGrad = kMode == kBoth;
    if (p.t.n_teacher == 0) return ent ? launch_forward<T, kGrad, true, kNoList>(p, st) : launch_forward<T, kGrad, false, kNoList>(p, st);
    if (p.t.kind == PG_DISTILL_FORWARD)
      return ent ? launch_forward<T, kGrad, true, kNormalised>(p, st) : launch_forward<T, kGrad, false, kNormalised>(p, st);
    return ent ? launch_forward<T, kGrad, true, kBucket>(p, st) : launch_forward<T, kGrad, false, kBucket>(p, st);
  }
}

}  // namespace pg
