// Sampling rules on logits (pg_logits_process): penalties for repeated tokens, biases, temperature and
// grammar masks in one pass over the logits.
//
// Bound: HBM, each logit read and written once.  A row is cut into slices of 2048 * kUnits tokens, one CTA
// each: it starts its loads, counts the row's history into one word per token of its slice in shared
// memory (every slice scans the whole history - 4 bytes a token from L2, against 4 to 8 bytes a token of
// the vocabulary from HBM - which needs neither a count array in global memory nor a second launch),
// then applies the rules from registers.  A bit per token says whether its word has to be read at all.
// Slices are 8192 tokens where that fills the GPU several times over, else shorter ones (latency).
#include "pg_kv.cuh"

namespace pg {

struct LogitsParams {
  pg_logits_rules r;
  const void* in;
  void* out;
  int64_t in_stride, out_stride;
  int vocab, slices;
};

constexpr int kLogitsThreads = 256;
constexpr int kUnit = 8;                      // tokens that a thread handles at a time
// Per token of the slice one word: bit 31 seen, bits 20..30 bias entry + 1, bits 0..19 count.
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

template <typename In, typename Out, int kUnits>
__global__ void __launch_bounds__(kLogitsThreads, 4)
logits_kernel(const __grid_constant__ LogitsParams p) {
  constexpr int kSlice = kLogitsThreads * kUnits * kUnit;
  __shared__ __align__(16) uint32_t word[kSlice];
  __shared__ uint32_t touched[kSlice / 32];
  const pg_logits_rules& r = p.r;
  const int row = blockIdx.x / p.slices, slice = blockIdx.x - row * p.slices;
  const In* in = (const In*)p.in + row * p.in_stride;
  Out* out = (Out*)p.out + row * p.out_stride;
  // Units of eight tokens lie on 16-byte boundaries of the row's memory: the first begins `lead` tokens before it.
  const int lead = (int)(((uintptr_t)in & 15) / sizeof(In));
  const int first = slice * kSlice - lead;                        // token of the slice's word 0, may be negative
  const bool out_aligned = (((uintptr_t)(out - lead)) & 15) == 0;

  Raw8<In> raw[kUnits];
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    const int t = first + (u * kLogitsThreads + (int)threadIdx.x) * kUnit;
    if (t >= 0 && t + kUnit <= p.vocab) load8(in + t, raw[u]);
  }
  const float rho = r.repetition ? r.repetition[row] : 1.f, pi = r.presence ? r.presence[row] : 0.f;
  const float phi = r.frequency ? r.frequency[row] : 0.f, tau = r.temperature ? r.temperature[row] : 1.f;
  const uint32_t* mask = r.mask ? r.mask + row * r.mask_stride : nullptr;
  const int words = (p.vocab + 31) >> 5;

  const bool any = r.tokens || r.bias_ids;
  if (any) {
    for (int i = threadIdx.x; i < kSlice / 4; i += kLogitsThreads) ((uint4*)word)[i] = make_uint4(0, 0, 0, 0);
    for (int i = threadIdx.x; i < kSlice / 32; i += kLogitsThreads) touched[i] = 0;
    __syncthreads();
    if (r.bias_ids) {
      for (int j = threadIdx.x; j < r.n_bias; j += kLogitsThreads) {
        const int id = r.bias_ids[(int64_t)row * r.n_bias + j];
        const unsigned int at = (unsigned int)(id - first);
        if ((unsigned int)id < (unsigned int)p.vocab && at < (unsigned int)kSlice) {
          atomicMax(&word[at], (uint32_t)(j + 1) << kBiasShift);
          atomicOr(&touched[at >> 5], 1u << (at & 31));
        }
      }
      __syncthreads();                                            // entries first: the maximum must see no counts
    }
    if (r.tokens) {
      const int n = min(max(r.n_tokens ? r.n_tokens[row] : r.max_tokens, 0), r.max_tokens);
      const int n0 = r.n_prompt ? r.n_prompt[row] : 0;
      const int32_t* tokens = r.tokens + row * r.token_stride;
#pragma unroll 4
      for (int j = threadIdx.x; j < n; j += kLogitsThreads) {
        const int id = tokens[j];
        const unsigned int at = (unsigned int)(id - first);
        if ((unsigned int)id < (unsigned int)p.vocab && at < (unsigned int)kSlice) {
          atomicOr(&word[at], kSeen);
          atomicOr(&touched[at >> 5], 1u << (at & 31));
          if (j >= n0) atomicAdd(&word[at], 1u);
        }
      }
    }
    __syncthreads();
  }
  // x / tau as a product with 1 / tau (one rounding more); a tau whose inverse is no number divides
  const float inv = 1.f / tau;
  const bool divide = !(fabsf(inv) < INFINITY);
  auto rules = [&](float x, uint32_t w) {
    if (w & kSeen) x = x > 0.f ? x / rho : x * rho;
    const uint32_t c = w & kCountMask;
    if (c) x -= phi * (float)c + pi;
    const int b = (int)((w & ~kSeen) >> kBiasShift);
    if (b) x += r.bias_values[(int64_t)row * r.n_bias + b - 1];
    return x;
  };
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    const int i = u * kLogitsThreads + (int)threadIdx.x, t = first + i * kUnit;
    if (t >= p.vocab || t + kUnit <= 0) continue;
    uint32_t hit = any ? touched[i >> 2] >> (i & 3) * 8 & 0xFFu : 0;
    uint32_t allowed = 0xFFu;
    if (mask) {
      const int w0 = t >> 5;                                      // rounds down for negative t too
      const uint32_t lo = w0 >= 0 ? mask[w0] : 0, hi = (t & 31) > 32 - kUnit && w0 + 1 < words ? mask[w0 + 1] : 0;
      allowed = __funnelshift_r(lo, hi, t & 31) & 0xFFu;
    }
    if (t >= 0 && t + kUnit <= p.vocab) {
      float x[8];
      floats8(raw[u], x);
      if (hit) {
#pragma unroll
        for (int k = 0; k < kUnit; ++k)
          if (hit >> k & 1) x[k] = rules(x[k], word[i * kUnit + k]);
      }
#pragma unroll
      for (int k = 0; k < kUnit; ++k) {
        x[k] = divide ? x[k] / tau : x[k] * inv;
        if (!(allowed >> k & 1)) x[k] = -INFINITY;
      }
      if (out_aligned) {
        store8(out + t, x);
      } else {
#pragma unroll
        for (int k = 0; k < kUnit; ++k) out[t + k] = from_float<Out>(x[k]);
      }
    } else {                                                      // the row begins or ends inside the unit
      for (int k = max(0, -t); k < min(kUnit, p.vocab - t); ++k) {
        float x = to_float(in[t + k]);
        if (hit >> k & 1) x = rules(x, word[i * kUnit + k]);
        x = divide ? x / tau : x * inv;
        out[t + k] = from_float<Out>(allowed >> k & 1 ? x : -INFINITY);
      }
    }
  }
}

template <typename In, typename Out>
static int launch_logits(LogitsParams p, int n_rows, cudaStream_t st) {
  // the last unit may begin up to seven tokens later than the row's length says (lead)
  auto slices = [&](int units) {
    const int64_t slice = (int64_t)kLogitsThreads * units * kUnit;
    return ((int64_t)p.vocab + kUnit - 1 + slice - 1) / slice;
  };
  const int64_t wanted = 148 * 12;                                // CTAs that fill the GPU twice
  const int units = n_rows * slices(4) >= wanted ? 4 : n_rows * slices(2) >= wanted ? 2 : 1;
  const int64_t grid = n_rows * slices(units);
  if (grid > 0x7FFFFFFFLL) return PG_EINVAL;
  p.slices = (int)slices(units);
  if (units == 4) logits_kernel<In, Out, 4><<<(unsigned)grid, kLogitsThreads, 0, st>>>(p);
  else if (units == 2) logits_kernel<In, Out, 2><<<(unsigned)grid, kLogitsThreads, 0, st>>>(p);
  else logits_kernel<In, Out, 1><<<(unsigned)grid, kLogitsThreads, 0, st>>>(p);
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
