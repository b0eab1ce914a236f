// Sampling rules on logits (pg_logits_process): penalties for repeated tokens, biases, temperature and
// grammar masks in one pass over the logits.
//
// Bound: HBM, each logit read and written once.  A CTA takes a part of a row and works in three steps:
//   1. the tokens of the row's history and the biases that fall into the part go into a table in shared memory
//      (a hash table, or one place per token where that is no larger); their results are computed there;
//   2. the part streams through registers with the temperature and the mask alone;
//   3. the table's results are written over the streamed ones.
// All warps do the first step together (four or eight of sixteen, with the others streaming meanwhile, took 200 and
// 156 us where all take 139: 1024 x 131072, bf16, 1024 tokens of history).
// So the penalties cost what the few tokens cost that have one: testing every logit for a penalty on the way
// (a word or a bit per token of the part) took twice the time of the stream in instructions and barriers.
// Every part scans the row's whole history, so parts are as long as the number of rows allows.
#include "pg_kv.cuh"
#include "pg_trace.cuh"

#include <algorithm>

namespace pg {

struct LogitsParams {
  pg_logits_rules r;
  const void* in;
  void* out;
  int64_t in_stride, out_stride;
  int vocab, parts, part;      // parts of a row, tokens of a part
  int slots, direct;           // of the table; direct: one for each token of the part
};

constexpr int kLogitsThreads = 512;
constexpr int kUnit = 8;                      // tokens that a thread handles at a time
constexpr int kGrain = kLogitsThreads * kUnit;
// A table entry counts in one word: bit 31 seen, bits 20..30 bias entry + 1, bits 0..19 count.
constexpr uint32_t kSeen = 0x80000000u, kCountMask = 0xFFFFFu;
constexpr int kBiasShift = 20;

__device__ __forceinline__ void unpack8(const uint4& a, float (&x)[8], __nv_bfloat16) {
  const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void unpack8(const uint4& a, float (&x)[8], __half) {
  const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
    x[2 * i] = f.x;
    x[2 * i + 1] = f.y;
  }
}
// Eight logits as they lie in memory.
template <typename T> struct Raw8 { uint4 v[sizeof(T) / 2]; };
template <typename T>
__device__ __forceinline__ void load8(const T* at, Raw8<T>& r) {
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 2; ++i) r.v[i] = __ldcs((const uint4*)at + i);
}
template <typename T>
__device__ __forceinline__ void floats8(const Raw8<T>& r, float (&x)[8]) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      x[4 * i] = __uint_as_float(r.v[i].x);
      x[4 * i + 1] = __uint_as_float(r.v[i].y);
      x[4 * i + 2] = __uint_as_float(r.v[i].z);
      x[4 * i + 3] = __uint_as_float(r.v[i].w);
    }
  } else {
    unpack8(r.v[0], x, T());
  }
}
__device__ __forceinline__ uint32_t pack2(float a, float b, __nv_bfloat16) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t pack2(float a, float b, __half) {
  const __half2 v = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}
template <typename T>
__device__ __forceinline__ void store8(T* at, const float (&x)[8]) {
  if constexpr (sizeof(T) == 4) {
    __stcs((float4*)at, make_float4(x[0], x[1], x[2], x[3]));
    __stcs((float4*)at + 1, make_float4(x[4], x[5], x[6], x[7]));
  } else {
    __stcs((uint4*)at, make_uint4(pack2(x[0], x[1], T()), pack2(x[2], x[3], T()), pack2(x[4], x[5], T()), pack2(x[6], x[7], T())));
  }
}

template <typename In, typename Out>
__global__ void __launch_bounds__(kLogitsThreads, 3)
logits_kernel(const __grid_constant__ LogitsParams p) {
  constexpr int kBatch = 4;                                       // units of a thread in flight
  extern __shared__ int32_t table[];                              // [slots] tokens (-1: none), [slots] words, later results
  const pg_logits_rules& r = p.r;
  const int row = blockIdx.x / p.parts;
  const In* in = (const In*)p.in + row * p.in_stride;
  Out* out = (Out*)p.out + row * p.out_stride;
  // Units of eight tokens lie on 16-byte boundaries of the row's memory: the first begins `lead` tokens before it.
  const int lead = (int)(((uintptr_t)in & 15) / sizeof(In));
  const int begin = (blockIdx.x - row * p.parts) * p.part - lead;      // the part's first unit, may be negative
  const int lo = max(begin, 0), hi = (int)min((int64_t)begin + p.part, (int64_t)p.vocab);
  if (lo >= hi) return;
  const bool out_aligned = (((uintptr_t)(out - lead)) & 15) == 0;
  const uint32_t* mask = r.mask ? r.mask + row * r.mask_stride : nullptr;
  const float inv = r.temperature ? 1.f / r.temperature[row] : 1.f;

  // step 1
  int32_t* key = table;
  uint32_t* word = (uint32_t*)table + p.slots;
  if (p.slots) {
    const int32_t* tokens = r.tokens ? r.tokens + row * r.token_stride : nullptr;
    const int n = tokens ? min(max(r.n_tokens ? r.n_tokens[row] : r.max_tokens, 0), r.max_tokens) : 0;
    const int n0 = r.n_prompt ? r.n_prompt[row] : 0;
    const float rho = r.repetition ? r.repetition[row] : 1.f, pi = r.presence ? r.presence[row] : 0.f;
    const float phi = r.frequency ? r.frequency[row] : 0.f;
    constexpr int kAhead = 4;                                     // tokens of the history on their way meanwhile
    int ahead[kAhead];
#pragma unroll
    for (int e = 0; e < kAhead; ++e) {
      const int j = e * kLogitsThreads + (int)threadIdx.x;
      ahead[e] = tokens && j < r.max_tokens ? tokens[j] : -1;
    }
    for (int i = threadIdx.x; i < p.slots; i += kLogitsThreads) {
      key[i] = -1;
      word[i] = 0;
    }
    __syncthreads();
    // place of a token of the part; there are more slots than tokens and biases, so the search ends
    auto place = [&](int id) {
      if (p.direct) {
        key[id - begin] = id;
        return id - begin;
      }
      int at = (int)__umulhi((uint32_t)id * 2654435761u, (uint32_t)p.slots);
      for (;;) {
        const int held = atomicCAS(&key[at], -1, id);
        if (held == -1 || held == id) return at;
        at = at + 1 == p.slots ? 0 : at + 1;
      }
    };
    if (r.bias_ids) {
      for (int j = threadIdx.x; j < r.n_bias; j += kLogitsThreads) {
        const int id = r.bias_ids[(int64_t)row * r.n_bias + j];
        if (id >= lo && id < hi) atomicMax(&word[place(id)], (uint32_t)(j + 1) << kBiasShift);
      }
      __syncthreads();                                            // entries first: the maximum must see no counts
    }
    auto count = [&](int id, int j) {                             // prompt tokens set `seen`, generated ones count
      if (id < lo || id >= hi) return;
      uint32_t* w = &word[place(id)];
      if (j < n0) atomicOr(w, kSeen);
      else atomicAdd(w, 1u);
    };
#pragma unroll
    for (int e = 0; e < kAhead; ++e) {
      const int j = e * kLogitsThreads + (int)threadIdx.x;
      if (j < n) count(ahead[e], j);
    }
#pragma unroll 4
    for (int j = kAhead * kLogitsThreads + (int)threadIdx.x; j < n; j += kLogitsThreads) count(tokens[j], j);
    __syncthreads();
    // four entries at a time: what they need from global memory is asked for together
    constexpr int kEntries = 4;
    for (int i0 = threadIdx.x; i0 < p.slots; i0 += kLogitsThreads * kEntries) {
      int id[kEntries];
      uint32_t w[kEntries], bits[kEntries];
      float x[kEntries], bias[kEntries];
#pragma unroll
      for (int e = 0; e < kEntries; ++e) {
        const int i = i0 + e * kLogitsThreads;
        id[e] = i < p.slots ? key[i] : -1;
        w[e] = i < p.slots ? word[i] : 0;
        const int b = (int)((w[e] & ~kSeen) >> kBiasShift);
        x[e] = id[e] >= 0 ? to_float(in[id[e]]) : 0.f;
        bits[e] = mask && id[e] >= 0 ? mask[id[e] >> 5] : 0xFFFFFFFFu;
        bias[e] = b ? r.bias_values[(int64_t)row * r.n_bias + b - 1] : 0.f;
      }
#pragma unroll
      for (int e = 0; e < kEntries; ++e) {
        if (id[e] < 0) continue;
        const uint32_t c = w[e] & kCountMask;
        if ((w[e] & kSeen) || c) x[e] = x[e] > 0.f ? x[e] / rho : x[e] * rho;
        if (c) x[e] -= phi * (float)c + pi;
        if ((w[e] & ~kSeen) >> kBiasShift) x[e] += bias[e];
        x[e] *= inv;
        word[i0 + e * kLogitsThreads] = __float_as_uint(bits[e] >> (id[e] & 31) & 1 ? x[e] : -INFINITY);
      }
    }
    __syncthreads();                                                       // out = in: all that is read here has been read
  }

  // step 2
  auto finish = [&](int t, float (&x)[8], uint32_t free) {
#pragma unroll
    for (int k = 0; k < kUnit; ++k) x[k] *= inv;
    if ((free & 0xFFu) != 0xFFu) {
#pragma unroll
      for (int k = 0; k < kUnit; ++k)
        if (!(free >> k & 1)) x[k] = -INFINITY;
    }
    if (out_aligned) {
      store8(out + t, x);
    } else {
#pragma unroll
      for (int k = 0; k < kUnit; ++k) out[t + k] = from_float<Out>(x[k]);
    }
  };
  const bool bytes = (begin & 7) == 0;                            // a unit's mask bits are one byte of the row of bits
  auto one_unit = [&](int t) {                                    // whole, or cut by the row's ends
    if (t >= lo && t + kUnit <= hi) {
      Raw8<In> raw;
      load8(in + t, raw);
      float x[8];
      floats8(raw, x);
      finish(t, x, !mask ? 0xFFu : bytes ? ((const uint8_t*)mask)[t >> 3] : __funnelshift_r(mask[t >> 5], mask[(t + kUnit - 1) >> 5], t & 31));
    } else {
#pragma unroll 1
      for (int k = max(0, lo - t); k < min(kUnit, hi - t); ++k) {
        const float x = to_float(in[t + k]) * inv;
        out[t + k] = from_float<Out>(!mask || (mask[(t + k) >> 5] >> ((t + k) & 31) & 1) ? x : -INFINITY);
      }
    }
  };
  // Blocks of kBatch units a lane, a warp each.
  constexpr int kBlock = 32 * kUnit * kBatch;
  const int lane = threadIdx.x & 31;
  for (int first = begin + (int)(threadIdx.x >> 5) * kBlock; first < hi; first += kLogitsThreads / 32 * kBlock) {
    const int t0 = first + lane * kUnit;
    if (first < lo || first + kBlock > hi) {
#pragma unroll 1
      for (int u = 0; u < kBatch; ++u) one_unit(t0 + u * 32 * kUnit);
      continue;
    }
    Raw8<In> raw[kBatch];
    uint32_t allowed[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) load8(in + t0 + u * 32 * kUnit, raw[u]);
    if (!mask) {
#pragma unroll
      for (int u = 0; u < kBatch; ++u) allowed[u] = 0xFFu;
    } else if (bytes) {
#pragma unroll
      for (int u = 0; u < kBatch; ++u) allowed[u] = ((const uint8_t*)mask)[(t0 >> 3) + u * 32];
    } else {
      // the bits may reach into the next word, which exists: all eight tokens do
      const int w = t0 >> 5, w1 = (t0 + kUnit - 1) >> 5;
#pragma unroll
      for (int u = 0; u < kBatch; ++u) allowed[u] = __funnelshift_r(mask[w + u * kUnit], mask[w1 + u * kUnit], t0 & 31);
    }
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      float x[8];
      floats8(raw[u], x);
      finish(t0 + u * 32 * kUnit, x, allowed[u]);
    }
  }

  // step 3
  if (p.slots == 0) return;
  __syncthreads();
  for (int i = threadIdx.x; i < p.slots; i += kLogitsThreads)
    if (const int id = key[i]; id >= 0) out[id] = from_float<Out>(__uint_as_float(word[i]));
}

template <typename In, typename Out>
static int launch_logits(LogitsParams p, int n_rows, cudaStream_t st) {
  // rows that do not all start on 16 bytes may need a unit more (lead)
  const bool aligned = (((uintptr_t)p.in | (uintptr_t)(p.in_stride * sizeof(In))) & 15) == 0;
  const int64_t tokens = (int64_t)p.vocab + (aligned ? 0 : kUnit - 1);
  const int64_t entries = (p.r.tokens ? p.r.max_tokens : 0) + (p.r.bias_ids ? p.r.n_bias : 0);
  const int64_t hashed = entries ? entries + entries / 4 + 32 : 0;
  // Parts for about twelve CTAs per SM - four rounds of three, two of two if the table is large - of whole grains; a part whose
  // tokens would need more than 128 KB of table either way is shortened to 16384 tokens.
  const int64_t ctas = 148 * (hashed * 8 > 48 * 1024 ? 4 : 12);
  int64_t part = (tokens * n_rows + ctas - 1) / ctas;
  part = std::max<int64_t>((part + kGrain - 1) / kGrain * kGrain, kGrain);
  const int64_t whole = (tokens + kGrain - 1) / kGrain * kGrain;
  part = std::min(part, whole);
  if (std::min(hashed, part) > 16384) part = 16384;
  const int64_t parts = (tokens + part - 1) / part;
  if (n_rows * parts > 0x7FFFFFFFLL) return PG_EINVAL;
  p.parts = (int)parts;
  p.part = (int)part;
  p.slots = (int)std::min(hashed, part);
  p.direct = hashed >= part;
  const size_t bytes = (size_t)p.slots * 8;
  auto kernel = logits_kernel<In, Out>;
  static std::atomic<uint64_t> done{0};
  if (bytes > 48 * 1024)
    if (const int rc = allow_shared(kernel, 16384 * 8, done)) return rc;
  kernel<<<(unsigned)(n_rows * parts), kLogitsThreads, bytes, st>>>(p);
  PG_LAUNCH_CHECK();
  return PG_OK;
}

template <typename In>
static int launch_logits_out(int out_dtype, const LogitsParams& p, int n_rows, cudaStream_t st) {
  if (out_dtype == PG_F32) return launch_logits<In, float>(p, n_rows, st);
  if (out_dtype == PG_BF16) return launch_logits<In, __nv_bfloat16>(p, n_rows, st);
  return launch_logits<In, __half>(p, n_rows, st);
}

}  // namespace pg

extern "C" int pg_logits_process(int32_t n_rows, int32_t vocab, int32_t dtype, const void* logits,
                                 int64_t logits_stride, int32_t out_dtype, void* out, int64_t out_stride,
                                 const pg_logits_rules* rules, void* stream) {
  pg::TraceRange trace_range("pg_logits_process");
  if (n_rows < 0 || vocab < 1 || vocab > 0x7FFF0000 || !rules) return PG_EINVAL;
  if (dtype != PG_F32 && dtype != PG_BF16 && dtype != PG_F16) return PG_EINVAL;
  if (out_dtype != PG_F32 && out_dtype != PG_BF16 && out_dtype != PG_F16) return PG_EINVAL;
  if (n_rows == 0) return PG_OK;
  if (logits_stride == 0) logits_stride = vocab;
  if (out_stride == 0) out_stride = vocab;
  const size_t bi = pg::dtype_bytes(dtype), bo = pg::dtype_bytes(out_dtype);
  if (!logits || !out || logits_stride < vocab || out_stride < vocab) return PG_EINVAL;
  if (((uintptr_t)logits & (bi - 1)) || ((uintptr_t)out & (bo - 1))) return PG_EINVAL;
  if (logits == out && (dtype != out_dtype || logits_stride != out_stride)) return PG_EINVAL;
  const pg_logits_rules& r = *rules;
  if (r.tokens && (r.max_tokens < 0 || r.max_tokens > PG_LOGITS_MAX_TOKENS || r.token_stride < 0)) return PG_EINVAL;
  if (r.bias_ids && (!r.bias_values || r.n_bias < 0 || r.n_bias > PG_LOGITS_MAX_BIAS)) return PG_EINVAL;
  if (r.mask && r.mask_stride != 0 && r.mask_stride < ((int64_t)vocab + 31) / 32) return PG_EINVAL;
  pg::LogitsParams p;
  p.r = r;
  p.in = logits; p.out = out;
  p.in_stride = logits_stride; p.out_stride = out_stride;
  p.vocab = vocab;
  cudaStream_t st = (cudaStream_t)stream;
  if (dtype == PG_F32) return pg::launch_logits_out<float>(out_dtype, p, n_rows, st);
  if (dtype == PG_BF16) return pg::launch_logits_out<__nv_bfloat16>(out_dtype, p, n_rows, st);
  return pg::launch_logits_out<__half>(out_dtype, p, n_rows, st);
}
