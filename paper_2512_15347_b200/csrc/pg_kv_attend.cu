// Attention of one new token per row over the paged cache (pg_kv_attend).
//   out = sum_t p_t v_t,  p = softmax(scale q.k_t) over the row's tokens, lse = ln sum exp.
#include "pg_kv.cuh"

namespace pg {

struct AttendParams {
  KvView kv;
  const void* q;
  const void *k_new, *v_new;
  void* out;
  float* lse;
  const int32_t* shared;
  int64_t q_stride, new_stride, out_stride;   // elements
  int n_q_heads, per_kv, group;
  float scale;
};

constexpr int kAttendWarps = 4;

// One CTA per (row, query head): each warp takes every fourth token with a running maximum m and sum
// l of its own, lanes hold the elements lane, lane + 32, ...; the warps are joined at the end.
template <typename T>
__global__ void __launch_bounds__(kAttendWarps * 32)
attend_kernel(const __grid_constant__ AttendParams p) {
  constexpr int kPer = 256 / 32;
  __shared__ float part[kAttendWarps][256];
  __shared__ float stat[kAttendWarps][2];
  const KvView& kv = p.kv;
  const int row = blockIdx.x / p.n_q_heads, head = blockIdx.x - row * p.n_q_heads;
  const int h = head / p.per_kv, D = kv.head_dim;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int n = row_len(kv, row);
  const T* q = (const T*)p.q + row * p.q_stride + (int64_t)head * D;
  float qr[kPer], acc[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    qr[i] = lane + 32 * i < D ? to_float(q[lane + 32 * i]) * p.scale : 0.f;
    acc[i] = 0.f;
  }
  float m = -INFINITY, l = 0.f;
  for (int t = warp; t < n; t += kAttendWarps) {
    const int page = kv.table[(int64_t)row * kv.max_pages + t / kv.page_size];
    const bool ok = (unsigned int)page < (unsigned int)kv.n_pages;
    if (!ok) flag(kv.status, kStatusIndex);
    const int64_t at = (ok ? page : 0) * kv.page_stride + ((int64_t)h * kv.page_size + t % kv.page_size) * D;
    T* kp = (T*)kv.k + at;
    T* vp = (T*)kv.v + at;
    const bool fresh = p.k_new && t == n - 1;
    const T* ks = fresh ? (const T*)p.k_new + row * p.new_stride + (int64_t)h * D : kp;
    const T* vs = fresh ? (const T*)p.v_new + row * p.new_stride + (int64_t)h * D : vp;
    float s = 0.f, vr[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int d = lane + 32 * i;
      vr[i] = 0.f;
      if (d < D && (ok || fresh)) {
        const T a = ks[d], b = vs[d];
        s = fmaf(qr[i], to_float(a), s);
        vr[i] = to_float(b);
        if (fresh && ok && head % p.per_kv == 0) { kp[d] = a; vp[d] = b; }
      }
    }
    s = warp_sum(s);
    const float m2 = fmaxf(m, s), safe = fmaxf(m2, -3e38f);
    const float keep = expf(m - safe), w = expf(s - safe);
    l = l * keep + w;
#pragma unroll
    for (int i = 0; i < kPer; ++i) acc[i] = acc[i] * keep + w * vr[i];
    m = m2;
  }
  if (lane == 0) { stat[warp][0] = m; stat[warp][1] = l; }
#pragma unroll
  for (int i = 0; i < kPer; ++i) part[warp][lane + 32 * i] = acc[i];
  __syncthreads();
  float top = -3e38f, total = 0.f, f[kAttendWarps];
  for (int w = 0; w < kAttendWarps; ++w) top = fmaxf(top, stat[w][0]);
  for (int w = 0; w < kAttendWarps; ++w) {
    f[w] = expf(stat[w][0] - top);
    total += f[w] * stat[w][1];
  }
  for (int d = threadIdx.x; d < D; d += blockDim.x) {
    float o = 0.f;
    for (int w = 0; w < kAttendWarps; ++w) o += f[w] * part[w][d];
    ((T*)p.out)[row * p.out_stride + (int64_t)head * D + d] = from_float<T>(total == 0.f ? 0.f : o / total);
  }
  if (threadIdx.x == 0 && p.lse) p.lse[(int64_t)row * p.n_q_heads + head] = total == 0.f ? -INFINITY : top + logf(total);
}

static int attend_check(const pg_kv* kv, int n_q_heads, int group) {
  const int rc = kv_check(kv);
  if (rc != PG_OK) return rc;
  if (n_q_heads < 1 || n_q_heads % kv->n_kv_heads || n_q_heads > 65535) return PG_EINVAL;
  if (group < 1 || kv->n_rows % group) return PG_EINVAL;
  return PG_OK;
}

}  // namespace pg

extern "C" {

size_t pg_kv_attend_workspace_bytes(const pg_kv* kv, int32_t n_q_heads, int32_t group) {
  if (pg::attend_check(kv, n_q_heads, group) != PG_OK) return 0;
  return 16;
}

int pg_kv_attend(const pg_kv* kv, int32_t layer, int32_t n_q_heads, const void* q, int64_t q_stride,
                 const void* k_new, const void* v_new, int64_t new_stride, float scale, int32_t group,
                 const int32_t* shared, void* out, int64_t out_stride, float* lse, void* workspace,
                 size_t workspace_bytes, int32_t* status, void* stream) {
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
  p.scale = scale;
  const unsigned grid = (unsigned)(kv->n_rows * n_q_heads);
  cudaStream_t st = (cudaStream_t)stream;
  if (kv->dtype == PG_F32) pg::attend_kernel<float><<<grid, pg::kAttendWarps * 32, 0, st>>>(p);
  else if (kv->dtype == PG_BF16) pg::attend_kernel<__nv_bfloat16><<<grid, pg::kAttendWarps * 32, 0, st>>>(p);
  else pg::attend_kernel<__half><<<grid, pg::kAttendWarps * 32, 0, st>>>(p);
  PG_LAUNCH_CHECK();
  return PG_OK;
}

}  // extern "C"
