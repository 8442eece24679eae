// Loss of a student against a teacher's top logits, with its gradient.  Per counted row, with student logits x, teacher
// entries (t_k, id_k), temperature tau and soft weight a:
//   p = softmax_k(t_k / tau) over the entries with an id in [0, V),   log q_v = x_v / tau - lse(x / tau)
//   row = (1 - a) (lse(x) - x_target) + z lse(x)^2 + a tau^2 sum_k p_k (log p_k - log q_{id_k})
//   d row / d x_v = softmax(x)_v (1 - a + 2 z lse(x)) - (1 - a) [v = target] + a tau (q_v - sum_{k: id_k = v} p_k)
// Bound by bytes where the row stays in registers: every logit is read once and its gradient written once.  With two
// softmaxes the exponentials (a quarter of the rate of other instructions) come close behind: exp(x - m) is the square or
// the fourth power of exp((x - m) / tau) where tau is 2 or 4.
// Measured on one MI355X, calls captured into a graph, three sets of inputs in turn, loss and gradient: 16384 rows of 32128 in
// bf16, K = 64, 414 us (2.1 GB, 5.1 TB/s; a copy's 5.2 come to 409), 436 over the logits themselves; the loss alone, 4096 rows,
// 50 us (264 MB, 5.3 TB/s); 200 rows of 131071 in float32, which are read twice, 67 us (315 MB, 4.7 TB/s); 48 rows of 509,
// 7.5 us, two launches (16 us a call from Python).
#include "kernels.h"
#include "vocab_rows.h"
#include <algorithm>

namespace t5mi {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
// Rows up to which every workgroup counts the targets itself, for a launch less (48 x 509: 8.2 us, 9.9 with the launch; 8000 x
// 8000: 96 us, 75 with it).
constexpr int kSelfCount = 1024;
constexpr int kAhead = 16;        // loads in flight where one workgroup goes over all rows

// Which exponentials a row needs: one (tau = 1, or only one of the two softmaxes has weight), two of which the second is
// the square or fourth power of the first, or two.  (Against two, bf16: tau 2 10240 x 2048 30.0 and 32.5 us, 4096 x 8000 35.4 and
// 39.9, 300 x 131072 64 and 74; tau 4 30.9 and 32.7, 36.7 and 41.6, 68 and 74; no difference where bytes bind, in float32 or
// at 16384 x 32128.)
enum { EXP_ONE = 0, EXP_SQUARE = 1, EXP_FOURTH = 2, EXP_TWO = 3 };

bool distill_counts(const int32_t* targets, int64_t rows) { return targets && rows > kSelfCount; }

struct Exps {
  float a, b;  // exp(x - m) and exp((x - m) / tau); with EXP_ONE both are the one that is needed
};
template <int MODE>
__device__ __forceinline__ Exps exps_of(float d, float ct) {  // d = x - m <= 0
  Exps e;
  e.b = __builtin_amdgcn_exp2f(d * ct);
  if (MODE == EXP_ONE) e.a = e.b;
  if (MODE == EXP_SQUARE) e.a = e.b * e.b;
  if (MODE == EXP_FOURTH) {
    e.a = e.b * e.b;
    e.a *= e.a;
  }
  if (MODE == EXP_TWO) e.a = __builtin_amdgcn_exp2f(d * kLog2e);
  return e;
}

// Counted rows, as a float, by one workgroup.
__global__ __launch_bounds__(1024) void distill_count_kernel(const int32_t* __restrict__ targets, int64_t rows, int V,
                                                             float* __restrict__ n_counted) {
  __shared__ int red[16];
  int c = 0;
  for (int r0 = threadIdx.x; r0 < (int)rows; r0 += 1024 * kAhead) {
    int t[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) t[j] = targets[min(r0 + j * 1024, (int)rows - 1)];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) c += r0 + j * 1024 < (int)rows && t[j] >= 0 && t[j] < V ? 1 : 0;
  }
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

// The row, or part blockIdx.y of it (PART_*), is at most NV 16-byte pieces a thread, and one element, and stays in
// registers.  PART_STATS leaves the part's largest element and sums of exponentials, PART_APPLY reads those of all parts.
// `out` may be the logits themselves.
enum { WHOLE_ROW = 0, PART_STATS = 1, PART_APPLY = 2 };
struct PartStats {
  float m, s1, st;
};

template <typename T, int NT, int NV, int MODE, int PHASE, bool GRAD>
__global__ __launch_bounds__(NT) void distill_rows_kernel(DistillArgs a, const T* logits, T* out) {
  constexpr int EPV = RowSplit<T>::EPV, NW = NT / 64;
  typedef typename RowVec<T>::type VT;
  __shared__ float red_m[NW], red_t[NW], red_a[NW], red_b[NW], red_w[NW], red_kl[NW];
  __shared__ int red_n[NW];
  __shared__ alignas(16) int s_id[256];
  __shared__ alignas(16) float s_p[256];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, V = a.V;
  // the parts of a row are neighbours: workgroups that start together read one stretch of memory, not one part of many
  // rows a power of two apart
  const int parts = PHASE == WHOLE_ROW || (PHASE == PART_APPLY && !GRAD) ? 1 : a.parts;
  const uint32_t row = blockIdx.x / parts;
  const int part = blockIdx.x - row * parts;
  const T* x = logits + row * a.ld;
  T* g = GRAD ? out + row * a.out_ld : nullptr;
  const RowSplit<T> sp(x, V);
  const u32x4* body = reinterpret_cast<const u32x4*>(x + sp.head);
  u32x4* gbody = GRAD ? reinterpret_cast<u32x4*>(g + sp.head) : nullptr;
  // pieces [first, last] are this workgroup's, the elements around them the first part's
  const int first = part * (NT * NV);
  const int last = PHASE == WHOLE_ROW ? sp.pieces - 1 : min(sp.pieces, first + NT * NV) - 1;
  const int own = part == 0 ? sp.single(tid, NT, V) : -1;
  PartStats* stats = (PartStats*)a.partial + (size_t)row * a.parts;
  // logits of the entries and of the target, as they were before any part's gradient was written over them
  float* picked = (float*)((PartStats*)a.partial + a.rows * a.parts) + (size_t)row * (a.K + 1);
  const int tgt = a.targets ? a.targets[row] : -1;
  const bool hard = tgt >= 0 && tgt < V;
  // (the gradient's rows need not lie on 16-byte boundaries where the logits' rows do)
  auto put_piece = [&](int p, u32x4 b) {
    if (!a.apart) {
      gbody[p] = b;
    } else {
      const VT o = __builtin_bit_cast(VT, b);
#pragma unroll
      for (int k = 0; k < EPV; ++k) g[sp.head + p * EPV + k] = o[k];
    }
  };
  if (a.targets && !hard) {
    if (PHASE == PART_STATS) return;
    if (tid == 0 && part == 0) a.row_loss[row] = 0.f;
    if (GRAD) {
      if (own >= 0) g[own] = from_f32<T>(0.f);
      for (int p = first + tid; p <= last; p += NT) put_piece(p, u32x4{0, 0, 0, 0});
    }
    return;
  }
  constexpr uint32_t kNegInf = sizeof(T) == 2 ? 0xFF80FF80u : 0xFF800000u;
  auto piece_at = [&](int p) {  // (-inf behind the end: exponentials of 0)
    u32x4 r = last >= first ? body[min(p, last)] : u32x4{kNegInf, kNegInf, kNegInf, kNegInf};
    return p <= last ? r : u32x4{kNegInf, kNegInf, kNegInf, kNegInf};
  };
  u32x4 raw[NV];
  if (PHASE != PART_APPLY || GRAD) {
#pragma unroll
    for (int i = 0; i < NV; ++i) raw[i] = piece_at(first + i * NT + tid);
  }
  const float xs = own >= 0 ? to_f32(x[own]) : -INFINITY;
  // thread k holds the teacher's entry k, and k + NT where NT < K
  constexpr int EK = (256 + NT - 1) / NT;
  int id[EK];
  float t[EK], xk[EK];
#pragma unroll
  for (int q = 0; q < EK; ++q) {
    const int k = q * NT + tid;
    id[q] = -1;
    t[q] = -INFINITY;
    xk[q] = 0.f;
    if ((PHASE != PART_STATS || part == 0) && k < a.K) {
      id[q] = a.teacher_ids[(size_t)row * a.K + k];
      if (id[q] < 0 || id[q] >= V || a.soft == 0.f) id[q] = -1;
      if (id[q] >= 0) {
        t[q] = a.teacher_logits[(size_t)row * a.K + k];
        xk[q] = PHASE == PART_APPLY ? picked[k] : to_f32(x[id[q]]);
      }
    }
  }
  const float x_t = !hard ? 0.f : PHASE == PART_APPLY ? picked[a.K] : to_f32(x[tgt]);
  if (PHASE == PART_STATS && part == 0) {
#pragma unroll
    for (int q = 0; q < EK; ++q)
      if (id[q] >= 0) picked[q * NT + tid] = xk[q];
    if (tid == 0) picked[a.K] = x_t;
  }
  int n_here = 0;
  const bool self_count = GRAD && PHASE != PART_STATS && a.targets && !a.n_counted;
  if (self_count)
    for (int r = tid; r < (int)a.all_rows; r += NT) n_here += a.all_targets[r] >= 0 && a.all_targets[r] < V ? 1 : 0;
  const float ct = a.exp_scale;
  // ---- largest element of the row, largest entry of the teacher
  float m = -INFINITY, s1 = 0.f, st = 0.f, tm = -INFINITY;
  if constexpr (PHASE == PART_APPLY) {
    for (int j = tid; j < a.parts; j += NT) m = fmaxf(m, stats[j].m);
  } else {
    m = xs;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const VT v = __builtin_bit_cast(VT, raw[i]);
#pragma unroll
      for (int k = 0; k < EPV; ++k) m = fmaxf(m, to_f32(v[k]));
      __builtin_amdgcn_sched_barrier(0);
    }
  }
#pragma unroll
  for (int q = 0; q < EK; ++q) tm = fmaxf(tm, t[q] != t[q] ? INFINITY : t[q]);  // (fmax passes a NaN over: it comes back in the sum)
  m = wave_max(m);
  tm = wave_max(tm);
  if (self_count) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) n_here += __shfl_xor(n_here, off, 64);
  }
  if (NW > 1) {
    if (lane == 0) {
      red_m[w] = m;
      red_t[w] = tm;
      red_n[w] = n_here;
    }
    __syncthreads();
    m = red_m[0];
    tm = red_t[0];
    n_here = red_n[0];
#pragma unroll
    for (int i = 1; i < NW; ++i) {
      m = fmaxf(m, red_m[i]);
      tm = fmaxf(tm, red_t[i]);
      n_here += red_n[i];
    }
  }
  // (a row of nothing but -inf comes to NaN, a part of that kind to 0)
  const float m0 = PHASE == PART_STATS && m == -INFINITY ? 0.f : m;
  // ---- sums
  if constexpr (PHASE == PART_APPLY) {
    for (int j = tid; j < a.parts; j += NT) {
      const Exps f = exps_of<MODE>(stats[j].m - m, ct);
      s1 = fmaf(stats[j].s1, f.a, s1);
      st = fmaf(stats[j].st, f.b, st);
    }
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      asm volatile("" : "+v"(raw[i]), "+v"(s1), "+v"(st));  // piece i is not touched before piece i-1 is summed
      const VT v = __builtin_bit_cast(VT, raw[i]);
#pragma unroll
      for (int k = 0; k < EPV; ++k) {
        const Exps e = exps_of<MODE>(to_f32(v[k]) - m0, ct);
        if (MODE != EXP_ONE) s1 += e.a;
        st += e.b;
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    const Exps e = exps_of<MODE>(xs - m0, ct);  // (0 where the thread has no single element)
    s1 += e.a;
    st += e.b;
  }
  const bool any = tm != -INFINITY;
  float wk[EK], total = 0.f;
#pragma unroll
  for (int q = 0; q < EK; ++q) {
    wk[q] = id[q] >= 0 && any ? __builtin_amdgcn_exp2f((t[q] - tm) * (kLog2e * a.inv_tau)) : 0.f;
    total += wk[q];
  }
  if (MODE == EXP_ONE) s1 = st;
  s1 = wave_sum(s1);
  st = MODE == EXP_ONE ? s1 : wave_sum(st);
  total = wave_sum(total);
  if (NW > 1) {
    if (lane == 0) {
      red_a[w] = s1;
      red_b[w] = st;
      red_w[w] = total;
    }
    __syncthreads();
    s1 = red_a[0];
    st = red_b[0];
    total = red_w[0];
#pragma unroll
    for (int i = 1; i < NW; ++i) {
      s1 += red_a[i];
      st += red_b[i];
      total += red_w[i];
    }
  }
  if constexpr (PHASE == PART_STATS) {
    if (tid == 0) stats[part] = PartStats{m, s1, st};
    return;
  }
  const float log_s1 = logf(s1), log_st = logf(st);
  const float lse = m + log_s1;
  const float log_total = logf(total);
  // T KL: differences of logits are not divided by a small T, behind which they may be no numbers (0.5 and the lowest logit)
  float kl = 0.f;
#pragma unroll
  for (int q = 0; q < EK; ++q) {
    const float p = any ? wk[q] / total : 0.f;
    if (id[q] >= 0 && p != 0.f)
      kl += p * (((t[q] - tm) - (xk[q] - m)) + a.tau * (log_st - log_total));
    if (q * NT + tid < 256) {
      s_id[q * NT + tid] = id[q];
      s_p[q * NT + tid] = p;
    }
  }
  kl = wave_sum(kl);
  if (NW > 1 && lane == 0) red_kl[w] = kl;
  auto write_loss = [&] {
    if (tid != 0 || part != 0) return;
    if (NW > 1)
      for (int i = 1; i < NW; ++i) kl += red_kl[i];
    float r = a.z_loss * lse * lse;
    if (a.soft > 0.f) r += a.soft * (a.tau * kl);
    if (a.soft < 1.f) r += (1.f - a.soft) * (log_s1 - (x_t - m));
    a.row_loss[row] = r;
  };
  if constexpr (!GRAD) {
    if (NW > 1) __syncthreads();
    write_loss();
  } else {
    // ---- gradient: the softmax parts of every element, then the elements of the target and of the entries again, whole
    const float n = !a.targets ? (float)a.all_rows : self_count ? (float)n_here : *a.n_counted;
    const float inv_n = 1.f / fmaxf(n, 1.f), h = 1.f - a.soft;
    const float k1 = (h + 2.f * a.z_loss * lse) * inv_n / s1, kt = any ? a.soft * a.tau * inv_n / st : 0.f;
    const float kp = a.soft * a.tau * inv_n, kone = k1 + kt;
    auto grad = [&](float xv) {
      const Exps e = exps_of<MODE>(xv - m, ct);
      return MODE == EXP_ONE ? e.b * kone : fmaf(e.a, k1, e.b * kt);
    };
    auto store_piece = [&](u32x4 r, int p) {
      const VT v = __builtin_bit_cast(VT, r);
      VT o;
#pragma unroll
      for (int k = 0; k < EPV; ++k) o[k] = from_f32<T>(grad(to_f32(v[k])));
      const u32x4 b = __builtin_bit_cast(u32x4, o);
      if (p <= last) put_piece(p, b);
      return b[3];
    };
    uint32_t chain = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      asm volatile("" : "+v"(raw[i]), "+v"(chain));  // one piece at a time, as above
      chain = store_piece(raw[i], first + i * NT + tid);
    }
    if (own >= 0) g[own] = from_f32<T>(grad(xs));
    __syncthreads();
    write_loss();
    auto whole = [&](int v, float xv) {
      if constexpr (PHASE == PART_APPLY) {  // another part's
        const int p = v - sp.head;
        if (p < 0 || p >= sp.pieces * EPV ? part != 0 : p < first * EPV || p > last * EPV + EPV - 1) return;
      }
      // all entries of this id, four at a time (600 x 2000, K = 256: 28 us, 75 one by one; 16384 x 32128, K = 64: 414 and 427)
      float ps = 0.f;
#pragma unroll 4
      for (int k = 0; k < a.K; k += 4) {  // (places from K on hold no id)
        const u32x4 ids = *reinterpret_cast<const u32x4*>(s_id + k);
        const f32x4 ps4 = *reinterpret_cast<const f32x4*>(s_p + k);
#pragma unroll
        for (int j = 0; j < 4; ++j) ps += (int)ids[j] == v ? ps4[j] : 0.f;
      }
      float r = grad(xv) - kp * ps;
      if (v == tgt) r -= h * inv_n;
      g[v] = from_f32<T>(r);
    };
#pragma unroll
    for (int q = 0; q < EK; ++q)
      if (id[q] >= 0) whole(id[q], xk[q]);
    if (hard && tid == NT - 1) whole(tgt, x_t);
  }
}

__global__ __launch_bounds__(1024) void distill_mean_kernel(const float* __restrict__ row_loss, const int32_t* __restrict__ targets,
                                                            int64_t rows, int V, float* __restrict__ loss) {
  __shared__ float red[16];
  float s = 0.f, n = 0.f;  // (whole numbers below 2^24: exact)
  for (int r0 = threadIdx.x; r0 < (int)rows; r0 += 1024 * kAhead) {
    float l[kAhead];
    int t[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int r = min(r0 + j * 1024, (int)rows - 1);
      l[j] = row_loss[r];
      t[j] = targets ? targets[r] : 0;
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
      if (r0 + j * 1024 < (int)rows) {
        s += l[j];
        n += t[j] >= 0 && t[j] < V ? 1.f : 0.f;
      }
  }
  s = block_sum<16>(s, red);
  n = block_sum<16>(n, red);
  if (threadIdx.x == 0) *loss = s / fmaxf(n, 1.f);
}

constexpr int kPartNV = 8;
constexpr int kPartPieces = 256 * kPartNV;

// Workgroups that share a row: 1, or parts of 32 KB for rows that do not fit one workgroup's registers (more than 256 KB), and
// for fewer than 128 rows of more than 64 KB, which would leave compute units without work.  Whole and in parts, T = 2, us:
// bf16 16 x 65536 16.4 and 14.0, 64 x 40000 16.6 and 15.0, but float32 32 x 20000 11.2 and 12.8; 16 x 32000 12.7 and 14.0;
// 128 x 65536 19.6 and 20.6, 1000 x 65536 77 and 94.  Rows of 128 to 256 KB leave a compute unit to one workgroup, and with
// 128 of them and more the whole row is mostly ahead (1000 x 128256 146 and 166, 2048 x 100000 242 and 248, float32
// 1000 x 50257 108 and 128), not always (300 x 131072 66 and 60, 500 x 70000 61 and 53) and not without a gradient (1000 x
// 128256 73 and 59).  1000 rows of 262144: 311 us, with parts of 64 or 16 KB 321.
int row_parts(int64_t rows, int V, int type) {
  const int pieces = ceil_div(V, type == IN_BF16 ? 8 : 4);
  return pieces <= 4096 || (pieces <= 16384 && rows >= 128) ? 1 : ceil_div(pieces, kPartPieces);
}

template <typename T, int MODE, bool GRAD>
void rows_of_mode(const DistillArgs& a, const T* x, T* g, int64_t rows, hipStream_t st) {
  const int pieces = ceil_div(a.V, 16 / (int)sizeof(T));
  auto go = [&](auto kern, int nt) { kern<<<(unsigned)(rows * a.parts), nt, 0, st>>>(a, x, g); };
  if (a.parts > 1) {
    go(distill_rows_kernel<T, 256, kPartNV, MODE, PART_STATS, GRAD>, 256);
    if (GRAD) {
      go(distill_rows_kernel<T, 256, kPartNV, MODE, PART_APPLY, GRAD>, 256);
    } else {
      distill_rows_kernel<T, 256, kPartNV, MODE, PART_APPLY, GRAD><<<(unsigned)rows, 256, 0, st>>>(a, x, g);
    }
    return;
  }
  // a row in a workgroup's registers, 16 pieces a thread at most; more workgroups at a time with fewer threads or fewer
  // registers each (bf16: 10240 x 500 28 us with 64 threads, 36 with 128; 10240 x 4096 53 with 128, 64 with 256; 8192 x 8000 68
  // with 4 pieces, 86 with 8; 8192 x 16000 115 with 8, 141 with 16; 2048 x 65000 125 with 512 threads, 215 with 1024).  With 1024
  // threads a SIMD's registers are 128 for each, 7 to 10 fewer than the gradient wants: those are spilled.
  if (pieces <= 256) go(distill_rows_kernel<T, 64, 4, MODE, WHOLE_ROW, GRAD>, 64);
  else if (pieces <= 512) go(distill_rows_kernel<T, 128, 4, MODE, WHOLE_ROW, GRAD>, 128);
  else if (pieces <= 1024) go(distill_rows_kernel<T, 256, 4, MODE, WHOLE_ROW, GRAD>, 256);
  else if (pieces <= 2048) go(distill_rows_kernel<T, 256, 8, MODE, WHOLE_ROW, GRAD>, 256);
  else if (pieces <= 4096) go(distill_rows_kernel<T, 256, 16, MODE, WHOLE_ROW, GRAD>, 256);
  else if (pieces <= 8192) go(distill_rows_kernel<T, 512, 16, MODE, WHOLE_ROW, GRAD>, 512);
  else go(distill_rows_kernel<T, 1024, 16, MODE, WHOLE_ROW, GRAD>, 1024);
}

template <typename T, bool GRAD>
void rows_of_type(const DistillArgs& a, const T* x, T* g, int mode, int64_t rows, hipStream_t st) {
  if (mode == EXP_ONE) rows_of_mode<T, EXP_ONE, GRAD>(a, x, g, rows, st);
  else if (mode == EXP_SQUARE) rows_of_mode<T, EXP_SQUARE, GRAD>(a, x, g, rows, st);
  else if (mode == EXP_FOURTH) rows_of_mode<T, EXP_FOURTH, GRAD>(a, x, g, rows, st);
  else rows_of_mode<T, EXP_TWO, GRAD>(a, x, g, rows, st);
}

}  // namespace

size_t distill_ws_bytes(int64_t rows, int V, int K, int type) {
  const int parts = row_parts(rows, V, type);
  return parts > 1 ? (size_t)rows * (parts * sizeof(PartStats) + (K + 1) * 4) : 0;
}

hipError_t launch_distill_count(const int32_t* targets, int64_t rows, int V, float* n_counted, hipStream_t st) {
  if (!distill_counts(targets, rows)) return hipSuccess;
  distill_count_kernel<<<1, 1024, 0, st>>>(targets, rows, V, n_counted);
  return hipGetLastError();
}

hipError_t launch_distill_rows(const DistillArgs& args, const void* logits, void* out, int type, int64_t rows, hipStream_t st) {
  if (rows <= 0) return hipSuccess;
  DistillArgs a = args;
  if (!distill_counts(a.all_targets, a.all_rows)) a.n_counted = nullptr;
  const bool soft_only = a.soft == 1.f && a.z_loss == 0.f;
  const int mode = a.tau == 1.f || a.soft == 0.f || soft_only ? EXP_ONE : a.tau == 2.f ? EXP_SQUARE : a.tau == 4.f ? EXP_FOURTH : EXP_TWO;
  a.exp_scale = a.soft == 0.f ? kLog2e : kLog2e * a.inv_tau;
  a.rows = rows;
  a.parts = row_parts(rows, a.V, type);
  if (rows * a.parts > INT32_MAX) return hipErrorInvalidValue;
  const int64_t further = (a.out_ld - a.ld) * (type == IN_BF16 ? 2 : 4);
  a.apart = out && ((((uintptr_t)out ^ (uintptr_t)logits) | further) & 15) != 0;
  if (type == IN_BF16) {
    if (out) rows_of_type<bf16, true>(a, (const bf16*)logits, (bf16*)out, mode, rows, st);
    else rows_of_type<bf16, false>(a, (const bf16*)logits, nullptr, mode, rows, st);
  } else {
    if (out) rows_of_type<float, true>(a, (const float*)logits, (float*)out, mode, rows, st);
    else rows_of_type<float, false>(a, (const float*)logits, nullptr, mode, rows, st);
  }
  return hipGetLastError();
}

hipError_t launch_distill_mean(const float* row_loss, const int32_t* targets, int64_t rows, int V, float* loss, hipStream_t st) {
  distill_mean_kernel<<<1, 1024, 0, st>>>(row_loss, targets, rows, V, loss);
  return hipGetLastError();
}

}  // namespace t5mi
