// Clipped objective over ragged rows of tokens and its derivatives (pg_token_objective).
//
// Bound: latency; one launch, a token a thread at a time: what the token needs is asked for first, while the warp finds the row of
// its first token by a search of `start` 32 ways at a time, and its other lanes walk on from there.  A CTA leaves its sums in a slot of
// the workspace; the one that draws the last ticket adds the slots in their order; up to 1024 tokens are one CTA's, which spares that.
// Measured (B200, calls back to back): 768 rows of up to 4096 tokens 12.3 us, 64 rows of up to 16 tokens 10 us (4 us as a graph: the
// rest is the call on the host).
// fp64 throughout: differences of log-probs lie next to 0, where exp(d) - d - 1 has no digits left in 32 bits.  Results are rounded to 32
// bits, so exponentials are Taylor polynomials good to 1e-11: exp(x) = 2^n exp(x - n ln 2), and below 0.35 exp(d) - d - 1 by its own series.
#include "pg_kv.cuh"
#include "pg_trace.cuh"

#include <algorithm>

namespace pg {

constexpr int kObjectiveFew = 1024, kObjectiveThreads = 512;   // threads of a CTA, for few tokens and for many
constexpr int kObjectiveMostCtas = 2 * 148;                 // two an SM: more in turn would wait for one another's joins (17 us, not 13)
constexpr int kObjectiveWalk = 8;                           // rows that a lane walks before it searches
constexpr int kSums = PG_TOKEN_STATS;                       // weighted surr, kl, entropy, distill; clipped tokens

struct ObjectiveParams {
  pg_token_batch b;
  float *objective, *dlogp, *weight, *ratio, *stats;
  double* slots;
  unsigned int* ticket;
  int32_t* status;
  int n_rows, n_tokens, chunks;                             // runs of as many tokens as threads that a CTA takes
};

// (exp(r) - 1 - r) / r^2 for |r| <= 0.35, relative error below 1e-11.
__device__ __forceinline__ double second_part(double r) {
  double q = 1. / 39916800.;
  q = fma(q, r, 1. / 3628800.);
  q = fma(q, r, 1. / 362880.);
  q = fma(q, r, 1. / 40320.);
  q = fma(q, r, 1. / 5040.);
  q = fma(q, r, 1. / 720.);
  q = fma(q, r, 1. / 120.);
  q = fma(q, r, 1. / 24.);
  q = fma(q, r, 1. / 6.);
  return fma(q, r, .5);
}
// exp(x); exp(x) - x - 1 in *rest and exp(x) - 1 in *less, each of its own: from the other by x they would lose all digits where x is far
// from 0.  Outside +-87 exp(x) is 0 or infinite in 32 bits or near it, and so it is from +-700 on.
__device__ __forceinline__ double exp_rest(double x, double* rest, double* less) {
  const float f = (float)x;
  const float n = rintf(fminf(fmaxf(f, -700.f), 700.f) * 1.44269504f);
  const double r = fma((double)n, -0.693147180559945309417, x);         // off by n 2.3e-17
  const double k = second_part(r) * r * r;
  double y = (1. + (r + k)) * __hiloint2double((1023 + (int)n) << 20, 0);
  if (fabsf(f) > 700.f) y = f > 0.f ? INFINITY : 0.;
  if (rest) {
    *rest = n == 0.f ? k : f > 700.f ? INFINITY : y - x - 1.;
    *less = n == 0.f ? k + r : y - 1.;
  }
  return y;
}
// 1 / n for a whole number n >= 1: Newton's iteration r + r (1 - n r), from 2^-23 over 2^-46 to the last bits.
__device__ __forceinline__ double reciprocal(int n) {
  double r = (double)__frcp_rn((float)n);
  r = fma(r, fma(-(double)n, r, 1.), r);
  return fma(r, fma(-(double)n, r, 1.), r);
}

__device__ __forceinline__ double sum_warp(double v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
  return v;
}

// Sums of every thread's `v`, the same in all threads of warp 0.
__device__ __forceinline__ void sum_cta(double (&v)[kSums], double (&part)[kSums][kObjectiveFew / 32]) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
#pragma unroll
  for (int k = 0; k < kSums; ++k) v[k] = sum_warp(v[k]);
  if (lane == 0)
#pragma unroll
    for (int k = 0; k < kSums; ++k) part[k][warp] = v[k];
  __syncthreads();
  if (warp == 0) {
#pragma unroll
    for (int k = 0; k < kSums; ++k) v[k] = sum_warp(lane < warps ? part[k][lane] : 0.);
  }
}

__global__ void __launch_bounds__(kObjectiveFew)
token_objective_kernel(const __grid_constant__ ObjectiveParams p) {
  __shared__ double part[kSums][kObjectiveFew / 32];
  __shared__ bool is_last;
  const pg_token_batch& b = p.b;
  const int* start = b.start;
  const int lane = threadIdx.x & 31, threads = blockDim.x;
  for (int64_t i = (int64_t)blockIdx.x * threads + threadIdx.x; i <= p.n_rows; i += (int64_t)gridDim.x * threads)
    if (start[i] < 0 || start[i] > p.n_tokens || (i < p.n_rows && start[i] > start[i + 1])) flag(p.status, kStatusIndex);
  const int in_rows = start[p.n_rows] - start[0];
  const double lo = 1. - (double)b.clip_low, hi = 1. + (double)b.clip_high;
  const double scale = b.norm == PG_NORM_ROWS  ? (double)b.scale / p.n_rows
                       : b.norm == PG_NORM_SUM ? (double)b.scale
                       : in_rows > 0           ? (double)b.scale / in_rows
                                               : 0.;
  double sums[kSums] = {};
  for (int chunk = 0; chunk < p.chunks; ++chunk) {
    const int64_t first = ((int64_t)blockIdx.x * p.chunks + chunk) * threads + (threadIdx.x & ~31);   // the warp's first token
    if (first >= p.n_tokens) break;
    const int j = (int)first + lane;
    const bool in = first + lane < p.n_tokens;
    const float fresh = in ? b.logp_new[j] : 0.f;
    const float old = in && b.logp_old ? b.logp_old[j] : fresh, ref = in && b.logp_ref ? b.logp_ref[j] : fresh;
    const float ent = in && b.entropy ? b.entropy[j] : 0.f, div = in && b.distill ? b.distill[j] : 0.f;
    // how many rows end at the first token or before
    int row = 0, most = p.n_rows;
    while (row < most) {
      const int step = (most - row + 31) / 32, at = row + (lane + 1) * step;
      const int ended = __popc(__ballot_sync(~0u, at <= most && start[min(at, most)] <= (int)first));
      most = min(row + (ended + 1) * step - 1, most);
      row = min(row + ended * step, most);
    }
    // a lane's token: the rows that end between them
    for (int walked = 0; in && row < p.n_rows && start[row + 1] <= j; ++row) {
      if (++walked < kObjectiveWalk) continue;
      int h = p.n_rows;
      while (row < h) {
        const int mid = row + (h - row) / 2;
        if (start[mid + 1] <= j) row = mid + 1;
        else h = mid;
      }
      break;
    }
    if (!in) continue;
    const int from = row < p.n_rows ? start[row] : 0, to = row < p.n_rows ? start[row + 1] : 0;
    if (j < from || j >= to) {                                // a token of no row
      p.dlogp[j] = 0.f;
      if (p.weight) p.weight[j] = 0.f;
      if (p.ratio) p.ratio[j] = 1.f;
      continue;
    }
    const double a = b.adv[row];
    double w = scale;
    if (b.norm == PG_NORM_ROWS) w *= reciprocal(to - from);
    const double r = b.logp_old ? exp_rest((double)fresh - (double)old, nullptr, nullptr) : 1.;
    const double free = a == 0. && r == INFINITY ? 0. : r * a;      // e^x times 0 for any x, also where e^x has no number
    const double held = (r < lo ? lo : r > hi ? hi : r) * a;
    const bool clipped = held < free;
    double g = clipped ? 0. : free;
    sums[0] += w * (clipped ? held : free);
    if (b.logp_ref) {
      const double d = (double)ref - (double)fresh;
      double kl, slope;
      exp_rest(d, &kl, &slope);
      sums[1] += w * kl;
      if (b.beta != 0.f) g += (double)b.beta * slope;         // a reference that is only watched may be infinitely far
    }
    sums[2] += w * (double)ent;
    sums[3] += w * (double)div;
    sums[4] += clipped;
    p.dlogp[j] = (float)(w * g);
    if (p.weight) p.weight[j] = (float)w;
    if (p.ratio) p.ratio[j] = (float)r;
  }
  sum_cta(sums, part);
  if (gridDim.x > 1) {
    if (threadIdx.x == 0) {
#pragma unroll
      for (int k = 0; k < kSums; ++k) p.slots[(int64_t)blockIdx.x * kSums + k] = sums[k];
      __threadfence();
      is_last = atomicAdd(p.ticket, 1u) == gridDim.x - 1;
    }
    __syncthreads();
    if (!is_last) return;
    __threadfence();
#pragma unroll
    for (int k = 0; k < kSums; ++k) sums[k] = 0.;
#pragma unroll 2
    for (int i = threadIdx.x; i < (int)gridDim.x; i += threads)
#pragma unroll
      for (int k = 0; k < kSums; ++k) sums[k] += __ldcg(p.slots + (int64_t)i * kSums + k);
    sum_cta(sums, part);
    if (threadIdx.x == 0) *p.ticket = 0u;                     // ready for the next call
  }
  if (threadIdx.x == 0) {
    // a term without weight is left out: what is only watched may be infinite
    double j = sums[0];
    if (b.beta != 0.f) j -= (double)b.beta * sums[1];
    if (b.entropy_coef != 0.f) j += (double)b.entropy_coef * sums[2];
    if (b.distill_coef != 0.f) j -= (double)b.distill_coef * sums[3];
    p.objective[0] = (float)j;
    if (p.stats) {
#pragma unroll
      for (int k = 0; k < 4; ++k) p.stats[k] = (float)sums[k];
      p.stats[4] = in_rows > 0 ? (float)(sums[4] / in_rows) : 0.f;
    }
  }
}

static void objective_shape(int n_tokens, int* threads, int* chunks, int* ctas) {
  *threads = n_tokens <= kObjectiveFew ? kObjectiveFew : kObjectiveThreads;
  const int64_t runs = ((int64_t)n_tokens + *threads - 1) / *threads;
  *chunks = (int)std::max<int64_t>((runs + kObjectiveMostCtas - 1) / kObjectiveMostCtas, 1);
  *ctas = (int)std::max<int64_t>((runs + *chunks - 1) / *chunks, 1);
}

}  // namespace pg

extern "C" size_t pg_token_objective_workspace_bytes(int32_t n_tokens) {
  if (n_tokens < 0) return 0;
  int threads, chunks, ctas;
  pg::objective_shape(n_tokens, &threads, &chunks, &ctas);
  // never less than a shorter batch needs: the slots of as many CTAs as any has
  ctas = (int)std::min<int64_t>((int64_t)n_tokens / pg::kObjectiveThreads + 1, pg::kObjectiveMostCtas);
  return pg::kCounterBytes + (size_t)ctas * pg::kSums * sizeof(double);
}

extern "C" int pg_token_objective(int32_t n_rows, int32_t n_tokens, const pg_token_batch* batch, float* objective, float* dlogp,
                                  float* weight, float* ratio, float* stats, void* workspace, size_t workspace_bytes, int32_t* status,
                                  void* stream) {
  pg::TraceRange trace_range("pg_token_objective");
  if (n_rows < 0 || n_rows > pg::kMostItems || n_tokens < 0 || n_tokens > pg::kMostItems || !batch || !objective) return PG_EINVAL;
  const pg_token_batch& b = *batch;
  if (b.norm < PG_NORM_ROWS || b.norm > PG_NORM_SUM) return PG_EINVAL;
  if (!(b.clip_low >= 0.f && b.clip_low <= 1.f && b.clip_high >= 0.f)) return PG_EINVAL;
  if (!b.start || (n_rows > 0 && !b.adv) || (n_tokens > 0 && (!b.logp_new || !dlogp))) return PG_EINVAL;
  if (!workspace || ((uintptr_t)workspace & 15) || workspace_bytes < pg_token_objective_workspace_bytes(n_tokens)) return PG_EINVAL;
  pg::ObjectiveParams p;
  p.b = b;
  p.objective = objective;
  p.dlogp = dlogp;
  p.weight = weight;
  p.ratio = ratio;
  p.stats = stats;
  p.ticket = (unsigned int*)workspace;
  p.slots = (double*)((char*)workspace + pg::kCounterBytes);
  p.status = status;
  p.n_rows = n_rows;
  p.n_tokens = n_tokens;
  int threads, ctas;
  pg::objective_shape(n_tokens, &threads, &p.chunks, &ctas);
  pg::token_objective_kernel<<<ctas, threads, 0, (cudaStream_t)stream>>>(p);
  PG_LAUNCH_CHECK();
  return PG_OK;
}
