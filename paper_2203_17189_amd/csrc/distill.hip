// Loss of a student against a teacher's top logits, with its gradient.  Per counted row, with student logits x, teacher
// entries (t_k, id_k), temperature tau and soft weight a:
//   p = softmax_k(t_k / tau) over the entries with an id in [0, V),   log q_v = x_v / tau - lse(x / tau)
//   row = (1 - a) (lse(x) - x_target) + z lse(x)^2 + a tau^2 sum_k p_k (log p_k - log q_{id_k})
//   d row / d x_v = softmax(x)_v (1 - a + 2 z lse(x)) - (1 - a) [v = target] + a tau (q_v - sum_{k: id_k = v} p_k)
// Bound by bytes: every logit is read once and its gradient written once.
#include "kernels.h"
#include <algorithm>

namespace t5mi {

namespace {

constexpr float kLog2e = 1.4426950408889634f;

template <int NW>
__device__ __forceinline__ float block_max_of(float v, float* red) {
  v = wave_max(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  float m = red[0];
#pragma unroll
  for (int i = 1; i < NW; ++i) m = fmaxf(m, red[i]);
  return m;
}

// Counted rows, as a float, by one workgroup.
__global__ __launch_bounds__(1024) void distill_count_kernel(const int32_t* __restrict__ targets, int64_t rows, int V,
                                                             float* __restrict__ n_counted) {
  __shared__ int red[16];
  int c = 0;
  for (int64_t r = threadIdx.x; r < rows; r += 1024) c += !targets || (targets[r] >= 0 && targets[r] < V) ? 1 : 0;
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) c += __shfl_xor(c, off, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = c;
  __syncthreads();
  if (threadIdx.x == 0) {
    int t = 0;
    for (int i = 0; i < 16; ++i) t += red[i];
    *n_counted = (float)t;
  }
}

// One workgroup per row; the row is read again for each pass.  `out` may be the logits themselves.
template <typename T>
__global__ __launch_bounds__(256) void distill_rows_kernel(DistillArgs a, const T* logits, T* out) {
  __shared__ float red[4];
  __shared__ int s_id[256];
  __shared__ float s_p[256];
  const int tid = threadIdx.x, V = a.V;
  const int64_t row = blockIdx.x;
  const T* x = logits + row * a.ld;
  T* g = out ? out + row * a.ld : nullptr;
  const int tgt = a.targets ? a.targets[row] : -1;
  const bool hard = tgt >= 0 && tgt < V, counted = !a.targets || hard;
  if (!counted) {
    if (tid == 0) a.row_loss[row] = 0.f;
    if (g)
      for (int c = tid; c < V; c += 256) g[c] = from_f32<T>(0.f);
    return;
  }
  float m = -INFINITY;
  for (int c = tid; c < V; c += 256) m = fmaxf(m, to_f32(x[c]));
  m = block_max_of<4>(m, red);
  const float c1 = kLog2e, ct = kLog2e * a.inv_tau;
  float s1 = 0.f, stau = 0.f;
  for (int c = tid; c < V; c += 256) {
    const float d = to_f32(x[c]) - m;
    s1 += __builtin_amdgcn_exp2f(d * c1);
    stau += __builtin_amdgcn_exp2f(d * ct);
  }
  s1 = block_sum<4>(s1, red);
  stau = block_sum<4>(stau, red);
  const float log_s1 = logf(s1), log_st = logf(stau), lse = m + log_s1;
  // teacher: thread k holds entry k
  int id = -1;
  float t = -INFINITY, xk = 0.f;
  if (tid < a.K) {
    id = a.teacher_ids[row * a.K + tid];
    if (id < 0 || id >= V) id = -1;
    if (id >= 0) {
      t = a.teacher_logits[row * a.K + tid];
      xk = to_f32(x[id]);
    }
  }
  // (fmax passes a NaN over: it counts as +inf here and comes back in the sum)
  const float tm = block_max_of<4>(t != t ? INFINITY : t, red);
  const bool any = tm != -INFINITY;
  const float w = id >= 0 && any ? __builtin_amdgcn_exp2f((t - tm) * ct) : 0.f;
  const float total = block_sum<4>(w, red);
  const float p = any ? w / total : 0.f;
  const float log_p = (t - tm) * a.inv_tau - logf(total);
  const float kl = block_sum<4>(id >= 0 && p != 0.f ? p * (log_p - ((xk - m) * a.inv_tau - log_st)) : 0.f, red);
  s_id[tid] = id;
  s_p[tid] = p;
  const float x_t = hard ? to_f32(x[tgt]) : 0.f;
  if (tid == 0) {
    float r = a.z_loss * lse * lse;
    if (a.soft > 0.f) r += a.soft * a.tau * a.tau * kl;
    if (a.soft < 1.f) r += (1.f - a.soft) * (log_s1 - (x_t - m));
    a.row_loss[row] = r;
  }
  if (!g) return;
  const float inv_n = 1.f / fmaxf(*a.n_counted, 1.f);
  const float h = 1.f - a.soft;
  const float k1 = (h + 2.f * a.z_loss * lse) * inv_n / s1, ktau = any ? a.soft * a.tau * inv_n / stau : 0.f;
  const float kp = a.soft * a.tau * inv_n;
  auto grad = [&](float xv) {
    const float d = xv - m;
    return __builtin_amdgcn_exp2f(d * c1) * k1 + __builtin_amdgcn_exp2f(d * ct) * ktau;
  };
  __syncthreads();
  for (int c = tid; c < V; c += 256) g[c] = from_f32<T>(grad(to_f32(x[c])));
  __syncthreads();  // the entries' own elements are written again, whole
  auto whole = [&](int v, float xv) {
    float ps = 0.f;
    for (int k = 0; k < a.K; ++k) ps += s_id[k] == v ? s_p[k] : 0.f;
    float r = grad(xv) - kp * ps;
    if (v == tgt) r -= h * inv_n;
    g[v] = from_f32<T>(r);
  };
  if (id >= 0) whole(id, xk);
  if (hard && tid == 0) whole(tgt, x_t);
}

__global__ __launch_bounds__(1024) void distill_mean_kernel(const float* __restrict__ row_loss, int64_t rows,
                                                            const float* __restrict__ n_counted, float* __restrict__ loss) {
  __shared__ float red[16];
  float s = 0.f;
  for (int64_t r = threadIdx.x; r < rows; r += 1024) s += row_loss[r];
  s = block_sum<16>(s, red);
  if (threadIdx.x == 0) *loss = s / fmaxf(*n_counted, 1.f);
}

}  // namespace

hipError_t launch_distill_count(const int32_t* targets, int64_t rows, int V, float* n_counted, hipStream_t st) {
  distill_count_kernel<<<1, 1024, 0, st>>>(targets, rows, V, n_counted);
  return hipGetLastError();
}

hipError_t launch_distill_rows(const DistillArgs& a, const void* logits, void* out, int type, int64_t rows, hipStream_t st) {
  if (rows <= 0) return hipSuccess;
  if (type == IN_BF16) distill_rows_kernel<bf16><<<(unsigned)rows, 256, 0, st>>>(a, (const bf16*)logits, (bf16*)out);
  else distill_rows_kernel<float><<<(unsigned)rows, 256, 0, st>>>(a, (const float*)logits, (float*)out);
  return hipGetLastError();
}

hipError_t launch_distill_mean(const float* row_loss, int64_t rows, const float* n_counted, float* loss, hipStream_t st) {
  distill_mean_kernel<<<1, 1024, 0, st>>>(row_loss, rows, n_counted, loss);
  return hipGetLastError();
}

}  // namespace t5mi
