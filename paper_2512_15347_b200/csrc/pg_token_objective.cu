// Clipped objective over ragged rows of tokens and its derivatives (pg_token_objective).
//
// Bound: latency for a few thousand tokens, HBM (three to five floats read and two or three written a token) beyond.  One launch: a CTA
// takes a run of tokens, asks for all that a thread needs at once, brings the rows' starts into shared memory meanwhile, finds each token's row by bisection
// and leaves its sums in a slot of the workspace; the CTA that draws the last ticket adds the slots in their order.  fp64 throughout:
// differences of log-probs lie next to 0, where exp(d) - d - 1 has no digits left in 32 bits.
#include "pg_kv.cuh"
#include "pg_trace.cuh"

#include <algorithm>

namespace pg {

constexpr int kObjectiveThreads = 256;
constexpr int kObjectiveRun = 4;                            // tokens of a thread that are asked for together
constexpr int kObjectiveChunk = kObjectiveThreads * kObjectiveRun;
constexpr int kObjectiveMostCtas = 4096;
constexpr int kObjectiveRows = 1024;                        // rows whose starts and advantages fit into shared memory
constexpr int kSums = PG_TOKEN_STATS;                       // weighted surr, kl, entropy, distill; clipped tokens

struct ObjectiveParams {
  pg_token_batch b;
  float *objective, *dlogp, *weight, *ratio, *stats;
  double* slots;
  unsigned int* ticket;
  int32_t* status;
  int n_rows, n_tokens, per_cta;                            // tokens of a CTA, a multiple of kObjectiveThreads
};

__device__ __forceinline__ double sum_warp(double v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
  return v;
}

// Sums of every thread's `v`, the same in all threads of warp 0.
__device__ __forceinline__ void sum_cta(double (&v)[kSums], double (&part)[kSums][kObjectiveThreads / 32]) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll
  for (int k = 0; k < kSums; ++k) {
    v[k] = sum_warp(v[k]);
    if (lane == 0) part[k][warp] = v[k];
  }
  __syncthreads();
  if (warp == 0) {
#pragma unroll
    for (int k = 0; k < kSums; ++k) v[k] = sum_warp(lane < kObjectiveThreads / 32 ? part[k][lane] : 0.);
  }
}

__global__ void __launch_bounds__(kObjectiveThreads)
token_objective_kernel(const __grid_constant__ ObjectiveParams p) {
  __shared__ double part[kSums][kObjectiveThreads / 32];
  __shared__ bool is_last;
  __shared__ int starts[kObjectiveRows + 1];
  __shared__ float advs[kObjectiveRows];
  const pg_token_batch& b = p.b;
  const int* start = b.start;
  const float* adv = b.adv;
  auto bad = [&](int i) { return start[i] < 0 || start[i] > p.n_tokens || (i < p.n_rows && start[i] > start[i + 1]); };
  for (int64_t i = (int64_t)blockIdx.x * kObjectiveThreads + threadIdx.x; i <= p.n_rows; i += (int64_t)gridDim.x * kObjectiveThreads)
    if (bad((int)i)) flag(p.status, kStatusIndex);
  const int in_rows = start[p.n_rows] - start[0];
  const double lo = 1. - (double)b.clip_low, hi = 1. + (double)b.clip_high;
  double sums[kSums] = {};
  const int64_t first = (int64_t)blockIdx.x * p.per_cta, last = min(first + p.per_cta, (int64_t)p.n_tokens);
  const bool shared = p.n_rows <= kObjectiveRows;
  for (int64_t base = first + threadIdx.x; base - threadIdx.x < last; base += kObjectiveChunk) {
    float fresh[kObjectiveRun], old[kObjectiveRun], ref[kObjectiveRun], ent[kObjectiveRun], div[kObjectiveRun];
#pragma unroll
    for (int e = 0; e < kObjectiveRun; ++e) {
      const int64_t j = base + e * kObjectiveThreads;
      const bool in = j < last;
      fresh[e] = in ? b.logp_new[j] : 0.f;
      old[e] = in && b.logp_old ? b.logp_old[j] : fresh[e];
      ref[e] = in && b.logp_ref ? b.logp_ref[j] : fresh[e];
      ent[e] = in && b.entropy ? b.entropy[j] : 0.f;
      div[e] = in && b.distill ? b.distill[j] : 0.f;
    }
    if (shared && base - threadIdx.x == first) {              // while they are on their way
      for (int i = threadIdx.x; i <= p.n_rows; i += kObjectiveThreads) {
        starts[i] = start[i];
        if (i < p.n_rows) advs[i] = adv[i];
      }
      __syncthreads();
      start = starts;
      adv = advs;
    }
#pragma unroll
    for (int e = 0; e < kObjectiveRun; ++e) {
      const int64_t j64 = base + e * kObjectiveThreads;
      if (j64 >= last) break;
      const int j = (int)j64;
      int l = 0, h = p.n_rows;                                // how many rows end at j or before
      while (l < h) {
        const int mid = l + (h - l) / 2;
        if (start[mid + 1] <= j) l = mid + 1;
        else h = mid;
      }
      const int from = l < p.n_rows ? start[l] : 0, to = l < p.n_rows ? start[l + 1] : 0;
      if (j < from || j >= to) {                              // a token of no row
        p.dlogp[j] = 0.f;
        if (p.weight) p.weight[j] = 0.f;
        if (p.ratio) p.ratio[j] = 1.f;
        continue;
      }
      double w = b.scale;
      if (b.norm == PG_NORM_ROWS) w /= (double)(to - from) * p.n_rows;
      if (b.norm == PG_NORM_TOKENS) w = in_rows > 0 ? w / in_rows : 0.;
      const double a = adv[l];
      const double r = b.logp_old ? exp((double)fresh[e] - (double)old[e]) : 1.;
      const double free = r * a, held = (r < lo ? lo : r > hi ? hi : r) * a;
      const bool clipped = held < free;
      double g = clipped ? 0. : free;
      sums[0] += w * (clipped ? held : free);
      if (b.logp_ref) {
        const double d = (double)ref[e] - (double)fresh[e], em = expm1(d);
        sums[1] += w * (em - d);
        g += (double)b.beta * em;
      }
      sums[2] += w * (double)ent[e];
      sums[3] += w * (double)div[e];
      sums[4] += clipped;
      p.dlogp[j] = (float)(w * g);
      if (p.weight) p.weight[j] = (float)w;
      if (p.ratio) p.ratio[j] = (float)r;
    }
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
    for (int i = threadIdx.x; i < (int)gridDim.x; i += kObjectiveThreads)
#pragma unroll
      for (int k = 0; k < kSums; ++k) sums[k] += __ldcg(p.slots + (int64_t)i * kSums + k);
    sum_cta(sums, part);
    if (threadIdx.x == 0) *p.ticket = 0u;                     // ready for the next call
  }
  if (threadIdx.x == 0) {
    p.objective[0] = (float)(sums[0] - (double)b.beta * sums[1] + (double)b.entropy_coef * sums[2] - (double)b.distill_coef * sums[3]);
    if (p.stats) {
#pragma unroll
      for (int k = 0; k < 4; ++k) p.stats[k] = (float)sums[k];
      p.stats[4] = in_rows > 0 ? (float)(sums[4] / in_rows) : 0.f;
    }
  }
}

// One CTA for what it takes in one go, which spares the join; else a token a thread while there are few, for latency, and
// kObjectiveRun a thread and more from there on.
static void objective_shape(int n_tokens, int* ctas, int* per_cta) {
  int64_t per = n_tokens <= kObjectiveChunk ? kObjectiveChunk : kObjectiveThreads;
  if (n_tokens > 148 * 2 * kObjectiveThreads) per = kObjectiveChunk;
  const int64_t least = ((int64_t)n_tokens + kObjectiveMostCtas - 1) / kObjectiveMostCtas;
  if (per < least) per = (least + kObjectiveChunk - 1) / kObjectiveChunk * kObjectiveChunk;
  *per_cta = (int)per;
  *ctas = (int)std::max<int64_t>(((int64_t)n_tokens + per - 1) / per, 1);
}

}  // namespace pg

extern "C" size_t pg_token_objective_workspace_bytes(int32_t n_tokens) {
  if (n_tokens < 0) return 0;
  return pg::kCounterBytes + (size_t)std::min<int64_t>((int64_t)n_tokens / pg::kObjectiveThreads + 1, pg::kObjectiveMostCtas) * pg::kSums * sizeof(double);
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
  int ctas;
  pg::objective_shape(n_tokens, &ctas, &p.per_cta);
  pg::token_objective_kernel<<<ctas, pg::kObjectiveThreads, 0, (cudaStream_t)stream>>>(p);
  PG_LAUNCH_CHECK();
  return PG_OK;
}
