// Sampling rules on logits (pg_logits_process): penalties for repeated tokens, biases, temperature and
// grammar masks in one pass over the logits.
//
// Bound: HBM, each logit read and written once.  A CTA takes a part of a row and works in three steps:
//   1. the tokens of the row's history and the biases that fall into the part go into a table in shared memory
//      (a hash table, or one place per token where that is no larger); their results are computed there;
//   2. the part streams through registers with the temperature and the mask alone;
//   3. the table's results are written over the streamed ones.
// So the penalties cost what the few tokens cost that have one: testing every logit for a penalty on the way
// (a word or a bit per token of the part) took twice the time of the stream in instructions and barriers.
// Every part scans the row's whole history, so parts are as long as the number of rows allows.
#include "pg_kv.cuh"

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
  const int lo = max(begin, 0), hi = min(begin + p.part, p.vocab);
  if (lo >= hi) return;
  const bool out_aligned = (((uintptr_t)(out - lead)) & 15) == 0;
  const uint32_t* mask = r.mask ? r.mask + row * r.mask_stride : nullptr;
  const int words = (p.vocab + 31) >> 5;
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
#pragma unroll 4
    for (int j = threadIdx.x; j < n; j += kLogitsThreads) {
      const int id = tokens[j];
      if (id < lo || id >= hi) continue;
      uint32_t* w = &word[place(id)];
      if (j < n0) atomicOr(w, kSeen);                             // prompt tokens set `seen`, generated ones count
      else atomicAdd(w, 1u);
    }
    __syncthreads();
#pragma unroll 2
    for (int i = threadIdx.x; i < p.slots; i += kLogitsThreads) {
      const int id = key[i];
      if (id < 0) continue;
      const uint32_t w = word[i], c = w & kCountMask;
      const int b = (int)((w & ~kSeen) >> kBiasShift);
      float x = to_float(in[id]);
      if ((w & kSeen) || c) x = x > 0.f ? x / rho : x * rho;
      if (c) x -= phi * (float)c + pi;
      if (b) x += r.bias_values[(int64_t)row * r.n_bias + b - 1];
      x *= inv;
      if (mask && !(mask[id >> 5] >> (id & 31) & 1)) x = -INFINITY;
      word[i] = __float_as_uint(x);
    }
    __syncthreads();                                              // in may be out: all reads of the part's own logits are
  }                                                               // done, or are the stream's, which writes what it read

  // step 2
  for (int t0 = begin + (int)threadIdx.x * kUnit; t0 < hi; t0 += kBatch * kGrain) {
    Raw8<In> raw[kBatch];
    uint32_t allowed[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int t = t0 + u * kGrain;
      if (t >= lo && t + kUnit <= hi) load8(in + t, raw[u]);
      allowed[u] = 0xFFu;
      if (mask && t < hi) {
        const int w0 = t >> 5;                                    // rounds down for negative t too
        const uint32_t a = w0 >= 0 ? mask[w0] : 0, b = (t & 31) > 32 - kUnit && w0 + 1 < words ? mask[w0 + 1] : 0;
        allowed[u] = __funnelshift_r(a, b, t & 31);
      }
    }
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int t = t0 + u * kGrain;
      const uint32_t free = allowed[u];
      if (t >= lo && t + kUnit <= hi) {
        float x[8];
        floats8(raw[u], x);
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
      } else if (t < hi) {                                        // the row begins or ends inside the unit
        for (int k = max(0, lo - t); k < min(kUnit, hi - t); ++k) {
          const float x = to_float(in[t + k]) * inv;
          out[t + k] = from_float<Out>(free >> k & 1 ? x : -INFINITY);
        }
      }
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
  // Parts for about eight CTAs per SM - four if the table leaves room for less - of whole grains; a part whose
  // tokens would need more than 128 KB of table either way is shortened to 16384 tokens.
  const int64_t ctas = 148 * (hashed * 8 > 48 * 1024 ? 4 : 8);
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
  if (bytes > 48 * 1024) PG_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 16384 * 8));
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
