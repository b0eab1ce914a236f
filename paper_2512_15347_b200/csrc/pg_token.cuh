// Policy update on rows of logits: log-probs of given tokens, entropy, alternatives, divergence from a teacher's list, and their
// gradient (pg_token_forward / _backward / _forward_backward).
//
// Bound: HBM.  A row is cut into as many parts as a thread block cluster has CTAs; a part lies in registers as it came from memory
// (64 16-bit or 32 fp32 logits a thread) and longer ones go through them tile by tile.  In the base-2 domain, with c = log2(e) / T,
//     y_v = (l_v - m) c,   s0 = sum 2^y,   s1 = sum 2^y y,   m the largest logit that the thread has,
// so one exponential a logit gives lse = m / T + ln s0 and the entropy ln s0 - ln 2 s1 / s0; the triples (m, s0, s1) of threads, warps and CTAs
// are joined in a fixed order, those of the cluster through each other's shared memory.  The difference is taken before the product with c,
// so that rows masked with the type's lowest value neither overflow nor lose their maximum.
// The gradient of all terms together is, away from given and listed tokens, e_v (A + B ln e_v) with two numbers a row: a second pass over
// the registers.  Given and listed tokens are written over it afterwards, one thread each.
// With a bucket for the mass outside a teacher's list that mass is summed by itself (the list's logits are taken out of the registers),
// since the difference 1 - (list's mass) has no digits left where the list has nearly everything.
// Alternatives: the n-th largest of the threads' maxima bounds the n-th largest logit from below, so only threads that hold one look
// at their logits again; what passes is ranked by counting.
#pragma once

#include "pg_kv.cuh"
#include "pg_trace.cuh"
#include "pg_units.cuh"

#include <algorithm>
#include <type_traits>

namespace pg {


constexpr int kTokThreads = 512;
constexpr int kTokWarps = kTokThreads / 32;
constexpr int kMostParts = 8;                   // CTAs of a cluster
constexpr int kCandidates = 1024;
constexpr float kLn2 = 0.6931471805599453f, kLog2e = 1.4426950408889634f;
constexpr float kFloorY = -1e4f;                // 2^y = 0 long before; keeps 0 * y from being NaN

enum TokenMode { kForward, kBackward, kBoth };

struct TokenParams {
  pg_token_terms t;
  pg_token_out o;
  pg_token_grads g;
  const void* in;
  void* dl;
  int64_t in_stride, dl_stride;
  int vocab, parts, units, tiles;               // CTAs of a row; units of a part; tiles of a part
};

// Sums over a warp's share of a teacher's list.  Reference of e: the largest logit m among them; of t: `tm` (FORWARD), else 0.
struct ListSums {
  float m, s0, s1, etl;                         // sum e, e y, e tl
  float tm, ts, ttl, ty;                        // sum t, t (tl - tm), t (l - m) / T
  double mass;                                  // sum t (the kinds with a bucket)
};

struct TokenShared {
  float wm[kTokWarps], ws0[kTokWarps], ws1[kTokWarps];
  float part[kMostParts][4];                    // triples of the cluster's CTAs, written by each
  ListSums list[PG_TOKEN_MAX_LIST / 32];
  float dsum[PG_TOKEN_MAX_LIST / 32];
  int gid[PG_TOKEN_MAX_LIST];                   // given tokens, -1: padding
  float gdl[PG_TOKEN_MAX_LIST];
  int tid[PG_TOKEN_MAX_LIST];                   // listed tokens, -1: unused
};
// Behind it, for alternatives; keys order by (logit, lowest index first).
struct TopShared {
  unsigned long long cand[kCandidates];
  unsigned long long merge[kMostParts][PG_TOKEN_MAX_TOP];   // the parts' lists, in part 0's
  unsigned long long best[PG_TOKEN_MAX_TOP];
  float tmax[kTokThreads];
  unsigned int hist[256];
  unsigned long long prefix;
  float bound;
  int count, left, shift;
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
__device__ __forceinline__ void peer_store(uint32_t at, float v) {
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at), "f"(v) : "memory");
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
// Word i of a unit; token k of a unit as bits; one token replaced by -inf.
template <typename T>
__device__ __forceinline__ uint32_t& word_of(Raw8<T>& r, int i) { return reinterpret_cast<uint32_t*>(&r)[i]; }
template <typename T>
__device__ __forceinline__ void set_empty(Raw8<T>& r, int k) {
  if constexpr (sizeof(T) == 4) word_of(r, k) = Empty8<T>::word;
  else word_of(r, k >> 1) = k & 1 ? (word_of(r, k >> 1) & 0xFFFFu) | (Empty8<T>::word & 0xFFFF0000u)
                                  : (word_of(r, k >> 1) & 0xFFFF0000u) | (Empty8<T>::word & 0xFFFFu);
}
template <typename T>
__device__ __forceinline__ f2 pair_of(const Raw8<T>& r, int i) {
  const uint32_t* w = reinterpret_cast<const uint32_t*>(&r);
  if constexpr (sizeof(T) == 4) return make2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
  else if constexpr (std::is_same<T, __half>::value) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
    return make2(f.x, f.y);
  } else return make2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
}

__device__ __forceinline__ unsigned long long top_key(float x, int id) {
  const uint32_t b = __float_as_uint(x + 0.f);                     // -0 = +0
  return (unsigned long long)(b ^ (b >> 31 ? 0xFFFFFFFFu : 0x80000000u)) << 32 | (0xFFFFFFFFu - (uint32_t)id);
}

// What is known of a row when its logits have been read.
struct TokenRow {
  float m, l2, h;                // p_v = 2^((l_v - m) c - l2); entropy
  float mr, l2r, lr;             // the same of the distribution outside the list; ln p_r (-inf: nothing there)
  float loss, lt, w;             // divergence; ln t_r, or ln of the list's mass (FORWARD); sum t (+ t_r)
  float some;                    // 0: a row that allows nothing
};
__device__ __forceinline__ void save_row(float4* at, const TokenRow& r) {
  at[0] = make_float4(r.m, r.l2, r.h, r.mr);
  at[1] = make_float4(r.l2r, r.lr, r.loss, r.lt);
  at[2] = make_float4(r.w, r.some, 0.f, 0.f);
}
__device__ __forceinline__ TokenRow load_row(const float4* at) {
  const float4 a = at[0], b = at[1], d = at[2];
  return {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w, d.x, d.y};
}

// From the sums over the row outside the list (`rest`) or over all of it, and the list's.
__device__ __forceinline__ TokenRow finish_row(const TokenShared& s, int parts, int lists, bool rest, int kind, float inv) {
  const float c = inv * kLog2e;
  TokenRow r;
  float m = -INFINITY, s0 = 0.f, s1 = 0.f;
  for (int i = 0; i < parts; ++i) m = fmaxf(m, s.part[i][0]);
  for (int i = 0; i < parts; ++i) {
    float a = s.part[i][1], b = s.part[i][2];
    refer(s.part[i][0], m, c, a, b);
    s0 += a;
    s1 += b;
  }
  r.mr = m;
  const bool outside = !(s0 == 0.f);
  r.l2r = outside ? log2f(s0) : 0.f;
  if (rest) {
    const float sr = s0, sr1 = s1;
    for (int i = 0; i < lists; ++i) m = fmaxf(m, s.list[i].m);
    s0 = sr;
    s1 = sr1;
    refer(r.mr, m, c, s0, s1);
    for (int i = 0; i < lists; ++i) {
      float a = s.list[i].s0, b = s.list[i].s1;
      refer(s.list[i].m, m, c, a, b);
      s0 += a;
      s1 += b;
    }
  }
  r.some = s0 == 0.f ? 0.f : 1.f;
  r.m = finite_ref(m);
  r.l2 = r.some != 0.f ? log2f(s0) : 0.f;
  r.h = r.some != 0.f ? kLn2 * (r.l2 - s1 / s0) : 0.f;
  // in 64 bits: where only tokens of the type's lowest value are left, it is finite and its share of the loss may be
  const double lr = ((double)finite_ref(r.mr) - r.m) * inv + (double)(kLn2 * (r.l2r - r.l2));
  r.lr = !rest ? 0.f : !outside ? -INFINITY : lr < -3e38 ? -3e38f : (float)lr;
  r.mr = finite_ref(r.mr);
  r.loss = r.lt = r.w = 0.f;
  if (lists == 0 || r.some == 0.f) return r;
  if (kind == PG_DISTILL_FORWARD) {
    float tm = -INFINITY, z = 0.f, ttl = 0.f, tlp = 0.f;
    for (int i = 0; i < lists; ++i) tm = fmaxf(tm, s.list[i].tm);
    for (int i = 0; i < lists; ++i) {
      const ListSums& l = s.list[i];
      if (l.tm == -INFINITY) { z += l.ts; continue; }                 // nothing used (or NaN)
      const float f = expf(l.tm - tm);
      z += f * l.ts;
      ttl += f * (l.ttl + l.ts * (l.tm - tm));
      tlp += f * (l.ty + l.ts * ((finite_ref(l.m) - r.m) * inv - kLn2 * r.l2));
    }
    if (z == 0.f) {                                                    // no list
      r.loss = 0.f * r.l2;                                             // NaN in a row with one
      return r;
    }
    r.lt = tm + logf(z);
    r.w = 1.f;
    r.loss = ttl / z - logf(z) - tlp / z;
    return r;
  }
  double mass = 0.;
  for (int i = 0; i < lists; ++i) mass += s.list[i].mass;
  const double tr = fmax(1. - mass, 1. / (1 << 20));
  r.lt = (float)log(tr);
  r.w = (float)(outside ? mass + tr : mass);
  if (mass != mass) r.lt = r.w = NAN;
  if (kind == PG_DISTILL_FORWARD_REST) {
    float ttl = 0.f, tlp = 0.f;
    for (int i = 0; i < lists; ++i) {
      const ListSums& l = s.list[i];
      ttl += l.ttl;
      if (l.ts != 0.f) tlp += l.ty + l.ts * ((finite_ref(l.m) - r.m) * inv - kLn2 * r.l2);
    }
    r.loss = ttl - tlp + (outside ? (float)(tr * (r.lt - lr)) : 0.f);
  } else {
    float plp = 0.f, ptl = 0.f;
    for (int i = 0; i < lists; ++i) {
      const ListSums& l = s.list[i];
      if (l.s0 == 0.f) continue;
      const float d = (l.m - r.m) * c, f = ex2(fmaxf(d, kFloorY));
      if (f == 0.f) continue;
      plp += f * (l.s1 + l.s0 * (d - r.l2));
      ptl += f * l.etl;
    }
    const float pr = outside ? expf(r.lr) : 0.f;
    r.loss = (kLn2 * plp - ptl) / s0 + (outside ? pr * (r.lr - r.lt) : 0.f);
  }
  return r;
}

template <typename T, int kMode, bool kEnt, bool kRest>
__global__ void __launch_bounds__(kTokThreads, 2)
token_kernel(const __grid_constant__ TokenParams p) {
  constexpr int kUnits = sizeof(T) == 4 ? 4 : 8;                    // of a thread and tile
  constexpr int kTile = kUnits * kTokThreads;
  __shared__ TokenShared s;
  extern __shared__ __align__(16) unsigned char more[];             // TopShared if there are alternatives, then bits of listed tokens (kRest)
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int row = blockIdx.x / p.parts, part = blockIdx.x - row * p.parts;
  const bool many = kMode != kBackward && p.parts > 1;
  if (many) cluster_arrive();                                       // all CTAs run before one writes into another's memory
  const int n_ids = p.t.ids ? p.t.n_ids : 0, n_list = p.t.teacher_ids ? p.t.n_teacher : 0;
  const int lists = (n_list + 31) / 32, n_top = kMode != kBackward && p.o.top_ids ? p.t.n_top : 0;
  TopShared& top = *reinterpret_cast<TopShared*>(more);
  uint32_t* bits = reinterpret_cast<uint32_t*>(more + (n_top ? sizeof(TopShared) : 0));

  const T* in = (const T*)p.in + row * p.in_stride;
  // Units of eight tokens lie on 16-byte boundaries of the row's memory: the first begins `lead` tokens before it.
  const int lead = (int)(((uintptr_t)in & 15) / sizeof(T));
  const int first = part * p.units;                                 // the part's first unit
  const int last = min(first + p.units, (p.vocab + lead + kUnit - 1) / kUnit);
  const int lo = max(first * kUnit - lead, 0), hi = min((first + p.units) * kUnit - lead, p.vocab);   // its tokens

  Raw8<T> raw[kUnits];
  auto load_tile = [&](int tile) {
#pragma unroll
    for (int j = 0; j < kUnits; ++j) {
      const int u = first + tile * kTile + j * kTokThreads + tid;
      const int t0 = u * kUnit - lead;
      if (u < last && t0 >= 0 && t0 + kUnit <= p.vocab) {
        load8(in + t0, raw[j]);
      } else {
#pragma unroll
        for (int i = 0; i < (int)sizeof(Raw8<T>) / 4; ++i) word_of(raw[j], i) = Empty8<T>::word;
        if (u < last) {                                             // cut by the row's ends
#pragma unroll
          for (int k = 0; k < kUnit; ++k) {
            if (t0 + k < 0 || t0 + k >= p.vocab) continue;
            const T x = in[t0 + k];
            if constexpr (sizeof(T) == 4) word_of(raw[j], k) = __float_as_uint(x);
            else {
              const uint32_t b = *reinterpret_cast<const uint16_t*>(&x);
              uint32_t& w = word_of(raw[j], k >> 1);
              w = k & 1 ? (w & 0xFFFFu) | b << 16 : (w & 0xFFFF0000u) | b;
            }
          }
        }
      }
    }
  };
  auto mask_tile = [&](int tile) {                                  // takes the listed tokens out
    if constexpr (kRest) {
#pragma unroll
      for (int j = 0; j < kUnits; ++j) {
        const int u = tile * kTile + j * kTokThreads + tid;
        const uint32_t b = u < p.units ? reinterpret_cast<const uint8_t*>(bits)[u] : 0u;
        if (b) {
#pragma unroll
          for (int k = 0; k < kUnit; ++k)
            if (b >> k & 1) set_empty(raw[j], k);
        }
      }
    }
  };

  const float inv = p.t.temperature ? 1.f / p.t.temperature[row] : 1.f, c = inv * kLog2e;
  if constexpr (kMode != kBackward) load_tile(0);

  // given and listed tokens, one a thread
  int my_id = -1, my_tid = -1;
  float my_x = 0.f, my_tx = -INFINITY, my_tl = 0.f, my_dl = 0.f;
  if (tid < n_ids) {
    const int id = p.t.ids[(int64_t)row * n_ids + tid];
    if ((unsigned int)id < (unsigned int)p.vocab) {
      my_id = id;
      if (kMode != kBackward || (id >= lo && id < hi)) my_x = to_float(in[id]);
      if (kMode != kForward && p.g.dlogp) my_dl = p.g.dlogp[(int64_t)row * n_ids + tid];
    }
    s.gid[tid] = my_id;
    s.gdl[tid] = my_dl;
  }
  if (tid < n_list) {
    const int id = p.t.teacher_ids[(int64_t)row * n_list + tid];
    my_tl = p.t.teacher_logp[(int64_t)row * n_list + tid];
    if ((unsigned int)id < (unsigned int)p.vocab && !(my_tl == -INFINITY)) my_tid = id;
    s.tid[tid] = my_tid;
    if (my_tid >= 0 && (kMode != kBackward || (my_tid >= lo && my_tid < hi))) my_tx = to_float(in[my_tid]);
  }
  if (kMode != kForward && warp < PG_TOKEN_MAX_LIST / 32) {
    const float d = warp_total(my_dl);
    if (lane == 0) s.dsum[warp] = d;
  }
  if constexpr (kRest)
    for (int i = tid; i < (p.units + 3) / 4; i += kTokThreads) bits[i] = 0;
  if (n_ids + n_list > 0 || kRest) __syncthreads();
  if (my_tid >= 0) {
    bool later = false;                                             // of entries with the same id the last one counts
    for (int j = tid + 1; j < n_list; ++j) later |= s.tid[j] == my_tid;
    if (later) my_tid = -1;
    else if (kRest && my_tid >= lo && my_tid < hi) {
      const int at = my_tid + lead - first * kUnit;
      atomicOr(&bits[at >> 5], 1u << (at & 31));
    }
  }
  if (kMode != kBackward && warp < lists) {
    const bool used = my_tid >= 0;
    const float x = used ? my_tx : -INFINITY;
    ListSums l;
    l.m = warp_most(x);
    const float y = (x - finite_ref(l.m)) * c, e = used ? ex2(y) : 0.f;
    l.s0 = warp_total(e);
    l.s1 = warp_total(e * fmaxf(y, kFloorY));
    l.etl = warp_total(e != 0.f ? e * my_tl : 0.f);
    l.tm = p.t.kind == PG_DISTILL_FORWARD ? warp_most(used ? my_tl : -INFINITY) : 0.f;
    const float t = used ? expf(my_tl - finite_ref(l.tm)) : 0.f;
    l.ts = warp_total(t);
    l.ttl = warp_total(t != 0.f ? t * (my_tl - finite_ref(l.tm)) : 0.f);
    l.ty = warp_total(t != 0.f ? t * (x - finite_ref(l.m)) * inv : 0.f);
    l.mass = kRest ? warp_total(used ? exp((double)my_tl) : 0.) : 0.;
    if (lane == 0) s.list[warp] = l;
  }
  // the threads' own columns of the list are done with; s.tid keeps the ids that count
  if (n_list > 0) {
    __syncthreads();
    if (tid < n_list) s.tid[tid] = my_tid;
  }

  TokenRow r;
  if constexpr (kMode != kBackward) {
    mask_tile(0);
    float m = -INFINITY, s0 = 0.f, s1 = 0.f;
    for (int tile = 0;;) {
      uint32_t w = Empty8<T>::word;
#pragma unroll
      for (int j = 0; j < kUnits; ++j) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(Raw8<T>) / 4; ++i) w = max2(w, word_of(raw[j], i), T());
      }
      const float tm = max_of<T>(w);
      refer(m, tm, c, s0, s1);
      m = fmaxf(m, tm);
      const float ref = finite_ref(m);
      const f2 nref = make2(-ref, -ref), c2 = make2(c, c);
      f2 a0 = make2(s0, 0.f), a1 = make2(s1, 0.f), b0 = make2(0.f, 0.f), b1 = b0;
#pragma unroll
      for (int j = 0; j < kUnits; ++j) {
        if (tile * kTile + j * kTokThreads >= p.units) break;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float y0, y1;
          split2(mul2(add2(pair_of(raw[j], i), nref), c2), y0, y1);
          const f2 e = make2(ex2(y0), ex2(y1));
          if (i & 1) b0 = add2(b0, e);
          else a0 = add2(a0, e);
          if (kEnt) {
            const f2 y = make2(fmaxf(y0, kFloorY), fmaxf(y1, kFloorY));
            if (i & 1) b1 = fma2(e, y, b1);
            else a1 = fma2(e, y, a1);
          }
        }
      }
      float u, v;
      split2(add2(a0, b0), u, v);
      s0 = u + v;
      split2(add2(a1, b1), u, v);
      s1 = u + v;
      if (++tile == p.tiles) break;
      load_tile(tile);
      mask_tile(tile);
    }
    const float own = m;                                             // the thread's largest
    m = warp_most(m);
    refer(own, m, c, s0, s1);
    s0 = warp_total(s0);
    if (kEnt) s1 = warp_total(s1);
    if (lane == 0) {
      s.wm[warp] = m;
      s.ws0[warp] = s0;
      s.ws1[warp] = s1;
    }
    if (n_top) {
      top.tmax[tid] = own;
      if (tid == 0) {
        top.count = 0;
        top.bound = -INFINITY;
      }
    }
    __syncthreads();
    if (warp == 0) {
      float wm = lane < kTokWarps ? s.wm[lane] : -INFINITY, a = lane < kTokWarps ? s.ws0[lane] : 0.f, b = lane < kTokWarps ? s.ws1[lane] : 0.f;
      const float cm = warp_most(wm);
      refer(wm, cm, c, a, b);
      a = warp_total(a);
      b = warp_total(b);
      if (!many) {
        if (lane == 0) {
          s.part[0][0] = cm;
          s.part[0][1] = a;
          s.part[0][2] = b;
        }
      }
      m = cm;
      s0 = a;
      s1 = b;
    }
    if (n_top) {
      // the n_top-th largest of the threads' maxima
      const float mine = top.tmax[tid];
      int above = 0;
      for (int j = 0; j < kTokThreads; j += 4) {
        const float4 o = *reinterpret_cast<const float4*>(&top.tmax[j]);
        above += (o.x > mine || (o.x == mine && j < tid)) + (o.y > mine || (o.y == mine && j + 1 < tid)) +
                 (o.z > mine || (o.z == mine && j + 2 < tid)) + (o.w > mine || (o.w == mine && j + 3 < tid));
      }
      if (above == n_top - 1) top.bound = mine;
      __syncthreads();
      const float bound = top.bound;
      // f(logit, token) for every logit of the part that is an alternative
      auto each = [&](auto f) {
        for (int tile = p.tiles - 1; tile >= 0; --tile) {
          if (p.tiles > 1) {
            load_tile(tile);
            mask_tile(tile);
          }
#pragma unroll
          for (int j = 0; j < kUnits; ++j) {
            const int t0 = (first + tile * kTile + j * kTokThreads + tid) * kUnit - lead;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              float x0, x1;
              split2(pair_of(raw[j], i), x0, x1);
              if (x0 > -INFINITY) f(x0, t0 + 2 * i);
              if (x1 > -INFINITY) f(x1, t0 + 2 * i + 1);
            }
          }
        }
        if (kRest && my_tid >= lo && my_tid < hi && my_tx > -INFINITY) f(my_tx, my_tid);
      };
      auto each_again = [&](auto f) {                               // from memory, for the rare path below
        for (int t = lo + tid; t < hi; t += kTokThreads) {
          const float x = to_float(in[t]);
          if (x > -INFINITY) f(x, t);
        }
      };
      auto push = [&](unsigned long long key) {
        const int at = atomicAdd(&top.count, 1);
        if (at < kCandidates) top.cand[at] = key;
      };
      if (own >= bound || (kRest && my_tx >= bound))
        each([&](float x, int id) { if (x >= bound) push(top_key(x, id)); });
      __syncthreads();
      if (top.count > kCandidates) {
        // Many equal logits: the n_top-th largest key, eight bits at a time, until few enough reach it.
        __syncthreads();
        if (tid == 0) {
          top.prefix = 0;
          top.left = n_top;
          top.shift = 64;
        }
        __syncthreads();
        for (int shift = 56; shift >= 0; shift -= 8) {
          if (tid < 256) top.hist[tid] = 0;
          __syncthreads();
          const unsigned long long prefix = top.prefix;
          each_again([&](float x, int id) {
            const unsigned long long key = top_key(x, id);
            if (shift == 56 || key >> (shift + 8) == prefix) atomicAdd(&top.hist[key >> shift & 255], 1u);
          });
          __syncthreads();
          if (tid == 0) {
            int left = top.left, b = 255;
            while (b > 0 && (int)top.hist[b] < left) left -= top.hist[b--];
            top.prefix = prefix << 8 | (unsigned)b;
            top.shift = shift;
            const bool few = n_top - left + (int)top.hist[b] <= kCandidates;
            top.left = left;
            top.count = few ? 0 : -1;
          }
          __syncthreads();
          if (top.count == 0) break;
        }
        const unsigned long long from = top.prefix << top.shift;
        __syncthreads();
        each_again([&](float x, int id) {
          const unsigned long long key = top_key(x, id);
          if (key >= from) push(key);
        });
        __syncthreads();
      }
      const int n = min(top.count, kCandidates);
      for (int i = tid; i < n_top; i += kTokThreads)
        if (i >= n) top.best[i] = 0;
      for (int i = tid; i < n; i += kTokThreads) {
        const unsigned long long key = top.cand[i];
        int rank = 0;
        for (int j = 0; j < n; ++j) rank += top.cand[j] > key;
        if (rank < n_top) top.best[rank] = key;
      }
      __syncthreads();
    }
    if (many) {
      cluster_wait();
      if (warp == 0 && lane < p.parts) {
        const uint32_t at = peer(&s.part[part][0], lane);
        peer_store(at, m);
        peer_store(at + 4, s0);
        peer_store(at + 8, s1);
      }
      for (int i = tid; i < n_top; i += kTokThreads) peer_store(peer(&top.merge[part][i], 0), top.best[i]);
      __syncwarp();
      cluster_arrive();
      cluster_wait();
    } else {
      __syncthreads();
    }
    r = finish_row(s, p.parts, lists, kRest, p.t.kind, inv);
    if (part == 0) {
      if (tid < n_ids && p.o.logp) {
        const float lp = r.some != 0.f ? (my_x - r.m) * inv - kLn2 * r.l2 : -INFINITY;
        p.o.logp[(int64_t)row * n_ids + tid] = my_id >= 0 ? lp : 0.f;
      }
      if (tid == 0) {
        if (p.o.lse) p.o.lse[row] = r.some != 0.f ? r.m * inv + kLn2 * r.l2 : -INFINITY;
        if (p.o.entropy) p.o.entropy[row] = r.h;
        if (p.o.distill) p.o.distill[row] = r.loss;
        if (p.o.saved) save_row((float4*)p.o.saved + (int64_t)row * (PG_TOKEN_SAVED / 4), r);
      }
      if (n_top) {
        auto write = [&](int at, unsigned long long key) {
          const uint32_t b = (uint32_t)(key >> 32);
          const float x = __uint_as_float(b >> 31 ? b ^ 0x80000000u : ~b);
          p.o.top_ids[(int64_t)row * n_top + at] = key ? (int)(0xFFFFFFFFu - (uint32_t)key) : -1;
          if (p.o.top_logp) p.o.top_logp[(int64_t)row * n_top + at] = key ? (x - r.m) * inv - kLn2 * r.l2 : -INFINITY;
        };
        if (!many) {
          for (int i = tid; i < n_top; i += kTokThreads) write(i, top.best[i]);
        } else {
          // the parts' lists are sorted: a key's rank is its own place and how many of each other list are above it
          for (int i = tid; i < n_top * p.parts; i += kTokThreads) {
            const int q = i / n_top, at = i - q * n_top;
            const unsigned long long key = top.merge[q][at];
            int rank = at;
            if (key) {
              for (int o = 0; o < p.parts; ++o) {
                if (o == q) continue;
                int a = 0, b = n_top;
                while (a < b) {
                  const int mid = (a + b) >> 1;
                  if (top.merge[o][mid] > key) a = mid + 1;
                  else b = mid;
                }
                rank += a;
              }
              if (rank < n_top) write(rank, key);
            }
          }
          if (tid < n_top) {                                        // places that are left over
            int some = 0;
            for (int o = 0; o < p.parts; ++o) {
              int a = 0, b = n_top;
              while (a < b) {
                const int mid = (a + b) >> 1;
                if (top.merge[o][mid] > 0) a = mid + 1;
                else b = mid;
              }
              some += a;
            }
            if (tid >= some) write(tid, 0);
          }
        }
      }
    }
  } else {
    r = load_row((const float4*)p.o.saved + (int64_t)row * (PG_TOKEN_SAVED / 4));
  }

  if constexpr (kMode != kForward) {
    const float dh = p.g.dentropy ? p.g.dentropy[row] * p.g.entropy_scale : 0.f;
    const float dd = p.g.ddistill ? p.g.ddistill[row] * p.g.distill_scale : 0.f;
    const bool rest = kMode == kBackward ? p.g.ddistill && n_list > 0 && p.t.kind != PG_DISTILL_FORWARD : kRest;
    const bool fix_list = n_list > 0 && (rest || p.g.ddistill);
    float d = 0.f;
    if (n_ids > 0)
      for (int i = 0; i < (n_ids + 31) / 32; ++i) d += s.dsum[i];
    const float lp_part = -fmaf(dh, r.h, d);                        // of p_v (.. - dh ln p_v)
    float a, b, ref, l2;
    if (rest) {
      const bool outside = r.lr > -INFINITY;
      const float pr = outside ? expf(r.lr) : 0.f, lr = outside ? r.lr : 0.f;
      const float dist = p.t.kind == PG_DISTILL_FORWARD_REST ? pr * r.w - expf(r.lt) : pr * (lr - r.lt - r.loss);
      a = outside || r.lr != r.lr ? inv * (pr * (lp_part - dh * lr) + dd * dist) : 0.f;
      b = -inv * dh * pr;
      ref = r.mr;
      l2 = r.l2r;
    } else {
      a = inv * (lp_part + dd * r.w);
      b = -inv * dh;
      ref = r.m;
      l2 = r.l2;
    }
    if (r.some == 0.f) a = b = 0.f;
    bool quiet = false;
    if constexpr (kMode == kBackward) quiet = !__syncthreads_or(my_dl != 0.f || dh != 0.f || dd != 0.f);
    if (quiet) a = b = 0.f;
    T* dl = (T*)p.dl + row * p.dl_stride;
    const bool aligned = ((uintptr_t)(dl - lead) & 15) == 0;
    const f2 nref = make2(-ref, -ref), c2 = make2(c, c), nl2 = make2(-l2, -l2), a2 = make2(a, a), b2 = make2(b * kLn2, b * kLn2);
    const bool kept = p.tiles == 1 || n_top == 0;                   // the last tile, in registers
    for (int tile = p.tiles - 1; tile >= 0; --tile) {
      if (kMode == kBackward ? !quiet : tile != p.tiles - 1 || !kept) load_tile(tile);
      if (kMode == kBackward && quiet) {
#pragma unroll
        for (int j = 0; j < kUnits; ++j)
#pragma unroll
          for (int i = 0; i < (int)sizeof(Raw8<T>) / 4; ++i) word_of(raw[j], i) = Empty8<T>::word;
      }
#pragma unroll
      for (int j = 0; j < kUnits; ++j) {
        if (tile * kTile + j * kTokThreads >= p.units) break;
        const int u = first + tile * kTile + j * kTokThreads + tid;
        const int t0 = u * kUnit - lead;
        float g[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          f2 y = fma2(add2(pair_of(raw[j], i), nref), c2, nl2);
          float y0, y1;
          split2(y, y0, y1);
          const f2 e = make2(ex2(y0), ex2(y1));
          f2 k = a2;
          if (kEnt) k = fma2(make2(fmaxf(y0, kFloorY), fmaxf(y1, kFloorY)), b2, a2);
          split2(mul2(e, k), g[2 * i], g[2 * i + 1]);
        }
        if (u >= last) continue;
        if (aligned && t0 >= 0 && t0 + kUnit <= p.vocab) {
          store8(dl + t0, g);
        } else {
#pragma unroll
          for (int k = 0; k < kUnit; ++k)
            if (t0 + k >= 0 && t0 + k < p.vocab) dl[t0 + k] = from_float<T>(g[k]);
        }
      }
    }
    // given and listed tokens
    if (quiet || (n_ids == 0 && !fix_list)) return;
    __syncthreads();
    auto about = [&](float x, float& pv, float& lp) {
      const float y = (x - r.m) * c - r.l2;
      pv = ex2(y);
      lp = kLn2 * y;
    };
    auto base = [&](float pv, float lp) { return pv == 0.f ? 0.f : pv * (lp_part - dh * lp); };
    if (fix_list && my_tid >= lo && my_tid < hi) {
      float pv, lp, dist;
      about(my_tx, pv, lp);
      if (p.t.kind == PG_DISTILL_FORWARD) dist = r.w * pv - expf(my_tl - r.lt);
      else if (p.t.kind == PG_DISTILL_FORWARD_REST) dist = r.w * pv - expf(my_tl);
      else dist = pv == 0.f ? 0.f : pv * (lp - my_tl - r.loss);
      float sum = base(pv, lp) + dd * dist;
      for (int j = 0; j < n_ids; ++j)
        if (s.gid[j] == my_tid) sum += s.gdl[j];
      dl[my_tid] = from_float<T>(r.some != 0.f ? inv * sum : 0.f);
    }
    if (my_id >= lo && my_id < hi) {
      bool mine = true;                                             // the last of its token, and not on the list
      for (int j = tid + 1; j < n_ids; ++j) mine &= s.gid[j] != my_id;
      if (fix_list)
        for (int j = 0; j < n_list; ++j) mine &= s.tid[j] != my_id;
      if (mine) {
        float pv, lp;
        about(my_x, pv, lp);
        float sum = base(pv, lp);
        if (!rest) sum += dd * r.w * pv;
        else if (p.g.ddistill) {                                    // outside the list
          const float rv = ex2((my_x - r.mr) * c - r.l2r), pr = expf(r.lr);
          sum += dd * rv * (p.t.kind == PG_DISTILL_FORWARD_REST ? pr * r.w - expf(r.lt) : pr * (r.lr - r.lt - r.loss));
        }
        for (int j = 0; j <= tid; ++j)
          if (s.gid[j] == my_id) sum += s.gdl[j];
        dl[my_id] = from_float<T>(r.some != 0.f ? inv * sum : 0.f);
      }
    }
  }
}

template <typename T, int kMode, bool kEnt, bool kRest>
int launch_token(TokenParams p, int n_rows, cudaStream_t st) {
  constexpr int kTile = (sizeof(T) == 4 ? 4 : 8) * kTokThreads;
  // rows that do not all start on 16 bytes may need a unit more (lead)
  const bool aligned = (((uintptr_t)p.in | (uintptr_t)(p.in_stride * sizeof(T))) & 15) == 0;
  const int total = (p.vocab + (aligned ? 0 : 16 / (int)sizeof(T) - 1) + kUnit - 1) / kUnit;
  int parts = 1;
  if (kMode == kBackward) {
    parts = (total + kTile - 1) / kTile;
  } else {
    // a part for each tile, so that the rows stay in registers; more, down to a unit a thread, while that leaves SMs without work
    while (parts < kMostParts && (kMode == kBoth ? (total + parts - 1) / parts > kTile : false)) parts *= 2;
    while (parts < kMostParts && (int64_t)n_rows * parts < 2 * 148 && total / parts >= 2 * kTokThreads) parts *= 2;
  }
  p.parts = parts;
  p.units = (total + parts - 1) / parts;
  p.tiles = (p.units + kTile - 1) / kTile;
  if ((int64_t)n_rows * parts > 0x7FFFFFFFLL) return PG_EINVAL;
  const bool top = kMode != kBackward && p.o.top_ids && p.t.n_top > 0;
  const int bytes = (top ? (int)sizeof(TopShared) : 0) + (kRest ? (p.units + 3) / 4 * 4 : 0);
  auto kernel = token_kernel<T, kMode, kEnt, kRest>;
  static std::atomic<uint64_t> done{0};
  constexpr int kMostBytes = (int)sizeof(TopShared) + PG_TOKEN_MAX_VOCAB / kUnit + 16;
  if (bytes > 40 * 1024)
    if (const int rc = allow_shared(kernel, kMostBytes, done)) return rc;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(n_rows * parts));
  cfg.blockDim = dim3(kTokThreads);
  cfg.dynamicSmemBytes = bytes;
  cfg.stream = st;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = (unsigned)parts;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = kMode != kBackward && parts > 1 ? 1 : 0;
  PG_CUDA(cudaLaunchKernelEx(&cfg, kernel, p));
  PG_LAUNCH_CHECK();
  return PG_OK;
}

template <typename T, int kMode>
int token_launch(const TokenParams& p, int n_rows, cudaStream_t st) {
  const bool ent = kMode == kBackward ? p.g.dentropy != nullptr : p.o.entropy || p.o.saved || (kMode == kBoth && p.g.dentropy);
  const bool teacher = p.t.teacher_ids && p.t.n_teacher > 0;
  if constexpr (kMode != kBackward) {
    if (teacher && p.t.kind != PG_DISTILL_FORWARD)
      return ent ? launch_token<T, kMode, true, true>(p, n_rows, st) : launch_token<T, kMode, false, true>(p, n_rows, st);
  }
  return ent ? launch_token<T, kMode, true, false>(p, n_rows, st) : launch_token<T, kMode, false, false>(p, n_rows, st);
}

}  // namespace pg
