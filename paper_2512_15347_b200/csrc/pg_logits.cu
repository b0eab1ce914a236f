// Sampling rules on logits (pg_logits_process): penalties for repeated tokens, biases, temperature
// and grammar masks, one pass over the logits.
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
constexpr int kLogitsSlice = 8192;            // tokens per CTA
// Per token of the slice one word: bit 31 seen, bits 20..30 bias entry + 1, bits 0..19 count.
constexpr uint32_t kSeen = 0x80000000u, kCountMask = 0xFFFFFu;
constexpr int kBiasShift = 20;

template <typename In, typename Out>
__global__ void __launch_bounds__(kLogitsThreads)
logits_kernel(const __grid_constant__ LogitsParams p) {
  __shared__ uint32_t word[kLogitsSlice];
  const pg_logits_rules& r = p.r;
  const int row = blockIdx.x / p.slices, slice = blockIdx.x - row * p.slices;
  const int v0 = slice * kLogitsSlice, nv = min(kLogitsSlice, p.vocab - v0);
  const In* in = (const In*)p.in + row * p.in_stride + v0;
  Out* out = (Out*)p.out + row * p.out_stride + v0;
  for (int i = threadIdx.x; i < kLogitsSlice; i += kLogitsThreads) word[i] = 0;
  __syncthreads();
  if (r.bias_ids)
    for (int j = threadIdx.x; j < r.n_bias; j += kLogitsThreads) {
      const unsigned int at = (unsigned int)r.bias_ids[(int64_t)row * r.n_bias + j] - (unsigned int)v0;
      if (at < (unsigned int)nv) atomicMax(&word[at], (uint32_t)(j + 1) << kBiasShift);
    }
  __syncthreads();
  if (r.tokens) {
    const int n = min(max(r.n_tokens ? r.n_tokens[row] : r.max_tokens, 0), r.max_tokens);
    const int n0 = r.n_prompt ? r.n_prompt[row] : 0;
    for (int j = threadIdx.x; j < n; j += kLogitsThreads) {
      const unsigned int at = (unsigned int)r.tokens[row * r.token_stride + j] - (unsigned int)v0;
      if (at < (unsigned int)nv) {
        atomicOr(&word[at], kSeen);
        if (j >= n0) atomicAdd(&word[at], 1u);
      }
    }
  }
  __syncthreads();
  const float rho = r.repetition ? r.repetition[row] : 1.f, pi = r.presence ? r.presence[row] : 0.f;
  const float phi = r.frequency ? r.frequency[row] : 0.f, tau = r.temperature ? r.temperature[row] : 1.f;
  for (int i = threadIdx.x; i < nv; i += kLogitsThreads) {
    float x = to_float(in[i]);
    const uint32_t w = word[i];
    if (w & kSeen) x = x > 0.f ? x / rho : x * rho;
    const uint32_t c = w & kCountMask;
    if (c) x -= phi * (float)c + pi;
    const int b = (int)((w & ~kSeen) >> kBiasShift);
    if (b) x += r.bias_values[(int64_t)row * r.n_bias + b - 1];
    x = x / tau;
    if (r.mask && !((r.mask[row * r.mask_stride + ((v0 + i) >> 5)] >> ((v0 + i) & 31)) & 1)) x = -INFINITY;
    out[i] = from_float<Out>(x);
  }
}

template <typename In>
static void launch_logits(int out_dtype, unsigned grid, const LogitsParams& p, cudaStream_t st) {
  if (out_dtype == PG_F32) logits_kernel<In, float><<<grid, kLogitsThreads, 0, st>>>(p);
  else if (out_dtype == PG_BF16) logits_kernel<In, __nv_bfloat16><<<grid, kLogitsThreads, 0, st>>>(p);
  else logits_kernel<In, __half><<<grid, kLogitsThreads, 0, st>>>(p);
}

}  // namespace pg

extern "C" int pg_logits_process(int32_t n_rows, int32_t vocab, int32_t dtype, const void* logits,
                                 int64_t logits_stride, int32_t out_dtype, void* out, int64_t out_stride,
                                 const pg_logits_rules* rules, void* stream) {
  if (n_rows < 0 || vocab < 1 || !rules) return PG_EINVAL;
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
  p.slices = (int)(((int64_t)vocab + pg::kLogitsSlice - 1) / pg::kLogitsSlice);
  const int64_t grid = (int64_t)n_rows * p.slices;
  if (grid > 0x7FFFFFFFLL) return PG_EINVAL;
  cudaStream_t st = (cudaStream_t)stream;
  if (dtype == PG_F32) pg::launch_logits<float>(out_dtype, (unsigned)grid, p, st);
  else if (dtype == PG_BF16) pg::launch_logits<__nv_bfloat16>(out_dtype, (unsigned)grid, p, st);
  else pg::launch_logits<__half>(out_dtype, (unsigned)grid, p, st);
  PG_LAUNCH_CHECK();
  return PG_OK;
}
