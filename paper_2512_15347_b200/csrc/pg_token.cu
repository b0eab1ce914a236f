// Entry points of the policy update on rows of logits: argument checks, choice of the kernel (pg_token.cuh).
#include "pg_token.cuh"

namespace pg {

extern template int token_launch<float, kForward>(const TokenParams&, cudaStream_t);
extern template int token_launch<float, kBackward>(const TokenParams&, cudaStream_t);
extern template int token_launch<float, kBoth>(const TokenParams&, cudaStream_t);
extern template int token_launch<__nv_bfloat16, kForward>(const TokenParams&, cudaStream_t);
extern template int token_launch<__nv_bfloat16, kBackward>(const TokenParams&, cudaStream_t);
extern template int token_launch<__nv_bfloat16, kBoth>(const TokenParams&, cudaStream_t);
extern template int token_launch<__half, kForward>(const TokenParams&, cudaStream_t);
extern template int token_launch<__half, kBackward>(const TokenParams&, cudaStream_t);
extern template int token_launch<__half, kBoth>(const TokenParams&, cudaStream_t);

template <int kMode>
static int token_call(int32_t n_rows, int32_t vocab, int32_t dtype, const void* logits, int64_t logits_stride, const pg_token_terms* terms,
                      const pg_token_out* out, const pg_token_grads* grads, void* dlogits, int64_t dlogits_stride, void* stream) {
  if (n_rows < 0 || vocab < 1 || vocab > PG_TOKEN_MAX_VOCAB || !terms) return PG_EINVAL;
  if (dtype != PG_F32 && dtype != PG_BF16 && dtype != PG_F16) return PG_EINVAL;
  if (n_rows == 0) return PG_OK;
  TokenParams p = {};
  p.t = *terms;
  if (out) p.o = *out;
  if (grads) p.g = *grads;
  if (logits_stride == 0) logits_stride = vocab;
  if (dlogits_stride == 0) dlogits_stride = vocab;
  const size_t b = dtype_bytes(dtype);
  if (!logits || logits_stride < vocab || ((uintptr_t)logits & (b - 1))) return PG_EINVAL;
  if (logits_stride > ((int64_t)1 << 60) / n_rows || dlogits_stride > ((int64_t)1 << 60) / n_rows) return PG_EINVAL;
  if (p.t.ids && (p.t.n_ids < 0 || p.t.n_ids > PG_TOKEN_MAX_LIST)) return PG_EINVAL;
  if (p.t.teacher_ids && (!p.t.teacher_logp || p.t.n_teacher < 0 || p.t.n_teacher > PG_TOKEN_MAX_LIST)) return PG_EINVAL;
  if (p.t.kind < PG_DISTILL_FORWARD || p.t.kind > PG_DISTILL_REVERSE_REST) return PG_EINVAL;
  if (p.t.n_top < 0 || p.t.n_top > PG_TOKEN_MAX_TOP || p.t.n_top > vocab) return PG_EINVAL;
  if (p.o.top_logp && !p.o.top_ids) return PG_EINVAL;
  if ((uintptr_t)p.o.saved & 15) return PG_EINVAL;
  if (kMode != kForward) {
    if (!dlogits || dlogits_stride < vocab || ((uintptr_t)dlogits & (b - 1))) return PG_EINVAL;
    if (dlogits == logits && dlogits_stride != logits_stride) return PG_EINVAL;
    if (kMode == kBackward && !p.o.saved) return PG_EINVAL;
    if ((p.g.dlogp && !(p.t.ids)) || (p.g.ddistill && !p.t.teacher_ids)) return PG_EINVAL;
  }
  p.in = logits;
  p.dl = dlogits;
  p.n_rows = n_rows;
  p.vocab = vocab;
  if (!p.t.ids) p.t.n_ids = 0;
  if (!p.t.teacher_ids) p.t.n_teacher = 0;
  if (!p.o.top_ids) p.t.n_top = 0;
  p.in_stride = logits_stride;
  p.dl_stride = dlogits_stride;
  cudaStream_t st = (cudaStream_t)stream;
  if (dtype == PG_F32) return token_launch<float, kMode>(p, st);
  if (dtype == PG_BF16) return token_launch<__nv_bfloat16, kMode>(p, st);
  return token_launch<__half, kMode>(p, st);
}

}  // namespace pg

extern "C" int pg_token_forward(int32_t n_rows, int32_t vocab, int32_t dtype, const void* logits, int64_t logits_stride,
                                const pg_token_terms* terms, const pg_token_out* out, void* stream) {
  pg::TraceRange trace_range("pg_token_forward");
  if (!out) return PG_EINVAL;
  return pg::token_call<pg::kForward>(n_rows, vocab, dtype, logits, logits_stride, terms, out, nullptr, nullptr, 0, stream);
}

extern "C" int pg_token_backward(int32_t n_rows, int32_t vocab, int32_t dtype, const void* logits, int64_t logits_stride,
                                 const pg_token_terms* terms, const float* saved, const pg_token_grads* grads, void* dlogits,
                                 int64_t dlogits_stride, void* stream) {
  pg::TraceRange trace_range("pg_token_backward");
  if (!grads) return PG_EINVAL;
  pg_token_out out = {};
  out.saved = const_cast<float*>(saved);
  return pg::token_call<pg::kBackward>(n_rows, vocab, dtype, logits, logits_stride, terms, &out, grads, dlogits, dlogits_stride, stream);
}

extern "C" int pg_token_forward_backward(int32_t n_rows, int32_t vocab, int32_t dtype, const void* logits, int64_t logits_stride,
                                         const pg_token_terms* terms, const pg_token_out* out, const pg_token_grads* grads,
                                         void* dlogits, int64_t dlogits_stride, void* stream) {
  pg::TraceRange trace_range("pg_token_forward_backward");
  if (!out || !grads) return PG_EINVAL;
  return pg::token_call<pg::kBoth>(n_rows, vocab, dtype, logits, logits_stride, terms, out, grads, dlogits, dlogits_stride, stream);
}
