// AdamW over many tensors in one launch, states in 32 bits or in 8 (see include/t5mi.h).
//
// One pass: parameter, gradient and states are read once and written once; nothing else moves.  A workgroup takes a chunk of
// one tensor; which one it finds in the launch's list of first chunks.  The list travels as the kernel's argument (4 KB hold
// kAdamTensors entries): no table in device memory, nothing to allocate, and a captured launch keeps it.
#include "fp8.h"
#include "kernels.h"
#include <cmath>
#include <cstring>

namespace t5mi {
namespace {

constexpr int kThreads = 256, kChunk = kThreads * 8;  // threads of a workgroup, 8 elements each

enum { AW_8BIT = 1, AW_BF16_GRAD = 2, AW_VEC = 4 };
struct AdamItem {
  float* p;
  const void* g;
  void *m, *v;
  uint8_t *ms, *vs;
  bf16* lp;
  int64_t n;
  float keep;     // 1 - lr * weight_decay
  uint32_t key;   // of the tensor's random bits
  int32_t flags, pad;
};
struct AdamBatch {
  int32_t count;
  uint32_t seed_hi;
  float b1, one_b1, b2, one_b2, root_b2, root_one_b2, root_factor, eps, step_size;
  const float* grad_scale;
  int32_t start[kAdamTensors + 1];
  AdamItem it[kAdamTensors];
};
static_assert(sizeof(AdamBatch) <= 4096, "kernel arguments");

// Up to 8 elements from p + i on (n of them exist), in 16-byte pieces where VEC and all 8 exist.
template <bool VEC>
__device__ __forceinline__ void load8(const float* p, int n, float (&v)[8]) {
  if (VEC && n >= 8) {
    const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
    for (int j = 0; j < 4; ++j) { v[j] = a[j]; v[j + 4] = b[j]; }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = j < n ? p[j] : 0.f;
  }
}
template <bool VEC>
__device__ __forceinline__ void load8(const bf16* p, int n, float (&v)[8]) {
  if (VEC && n >= 8) {
    const bf16x8 a = *reinterpret_cast<const bf16x8*>(p);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (float)a[j];
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = j < n ? (float)p[j] : 0.f;
  }
}
template <bool VEC>
__device__ __forceinline__ void store8(float* p, int n, const float (&v)[8]) {
  if (VEC && n >= 8) {
    *reinterpret_cast<f32x4*>(p) = f32x4{v[0], v[1], v[2], v[3]};
    *reinterpret_cast<f32x4*>(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < n) p[j] = v[j];
  }
}
template <bool VEC>
__device__ __forceinline__ void store8(bf16* p, int n, const float (&v)[8]) {
  if (VEC && n >= 8) {
    *reinterpret_cast<u32x4*>(p) = u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < n) p[j] = (bf16)v[j];
  }
}
template <bool VEC>
__device__ __forceinline__ u32x2 load_codes(const uint8_t* p, int n) {
  if (VEC && n >= 8) return *reinterpret_cast<const u32x2*>(p);
  u32x2 r = {0, 0};
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (j < n) r[j >> 2] |= (uint32_t)p[j] << ((j & 3) * 8);
  return r;
}
template <bool VEC>
__device__ __forceinline__ void store_codes(uint8_t* p, int n, u32x2 c) {
  if (VEC && n >= 8) {
    *reinterpret_cast<u32x2*>(p) = c;
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < n) p[j] = (uint8_t)(c[j >> 2] >> ((j & 3) * 8));
  }
}

typedef __attribute__((ext_vector_type(2))) float f32x2;
__device__ __forceinline__ void decode8(u32x2 c, float scale, float (&v)[8]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const f32x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8((int)c[h], scale, false), hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8((int)c[h], scale, true);
    v[h * 4] = lo[0]; v[h * 4 + 1] = lo[1]; v[h * 4 + 2] = hi[0]; v[h * 4 + 3] = hi[1];
  }
}

// Four codes of x / scale, each floor(t + u) steps: the conversion with a random word adds the word's top bits below the
// type's last place, in its subnormal range too, and cuts off; u is `bits` / 2^16 where the word is bits << 16.
__device__ __forceinline__ uint32_t round_at_random4(const float* x, const uint32_t* word, float scale) {
  int r = __builtin_amdgcn_cvt_scalef32_sr_fp8_f32(0, x[0], word[0], scale, 0);
  r = __builtin_amdgcn_cvt_scalef32_sr_fp8_f32(r, x[1], word[1], scale, 1);
  r = __builtin_amdgcn_cvt_scalef32_sr_fp8_f32(r, x[2], word[2], scale, 2);
  return (uint32_t)__builtin_amdgcn_cvt_scalef32_sr_fp8_f32(r, x[3], word[3], scale, 3);
}

// Bits of the largest finite |x| of a thread's eight.
__device__ __forceinline__ uint32_t largest8(const float (&x)[8]) {
  uint32_t b = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) b = max(b, __float_as_uint(x[j]) & 0x7FFFFFFFu);
  if (b >= 0x7F800000u) {
    b = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) b = max(b, finite_bits(x[j]));
  }
  return b;
}

// v_sqrt_f32 takes subnormal numbers as zero: those, and what else is small, are scaled.
__device__ __forceinline__ float root_of(float v) {
  const bool small = v < 0x1p-96f;
  const float r = __builtin_amdgcn_sqrtf(small ? v * 0x1p32f : v);
  return small ? r * 0x1p-16f : r;
}
// sqrt(x^2 + y^2) where the squares may leave float32, by the power of two of the larger.
__device__ __forceinline__ float root_of_squares(float x, float y) {
  const int e = __builtin_amdgcn_frexp_expf(fmaxf(fabsf(x), fabsf(y)));
  x = ldexpf(x, -e);
  y = ldexpf(y, -e);
  return ldexpf(__builtin_amdgcn_sqrtf(fmaf(x, x, y * y)), e);
}

struct Step {
  float b1, one_b1, b2, one_b2, root_b2, root_one_b2, root_factor, eps, step_size, keep;
  __device__ __forceinline__ void moments(float g, float& m, float& v) const {
    m = fmaf(b1, m, one_b1 * g);
    v = fmaf(b2, v, one_b2 * g * g);
  }
  // Whether the root cannot be had from the sum v = b2 r^2 + one_b2 g^2: it, or what counts of its parts, is below float32's
  // normal range, or it is above.  (Zeros of both are ordinary: tables have many.)
  __device__ __forceinline__ bool far(float v, float r, float g) const {
    return !(v >= 0x1p-96f && v < __builtin_inff()) && (r != 0.f || g != 0.f);
  }
  // (v_sqrt_f32 and v_rcp_f32 are within one unit of the last place; the divisor is eps or more, 1e-30 at least)
  __device__ __forceinline__ float update(float p, float m, float root) const {
    return fmaf(p, keep, -step_size * (m * __builtin_amdgcn_rcpf(fmaf(root, root_factor, eps))));
  }
};

template <bool VEC, bool EIGHT>
__device__ __forceinline__ void adam_chunk(const AdamItem& it, const Step& s, const float* gs, uint32_t seed_hi, int64_t i) {
  const int64_t left = it.n - i;
  const int n = left >= 8 ? 8 : left > 0 ? (int)left : 0;
  float p[8], g[8], m[8], v[8], root[8];
  if (it.flags & AW_BF16_GRAD) load8<VEC>((const bf16*)it.g + i, n, g);
  else load8<VEC>((const float*)it.g + i, n, g);
  load8<VEC>(it.p + i, n, p);
  const int64_t block = i >> 7;
  if constexpr (EIGHT) {
    const u32x2 cm = load_codes<VEC>((const uint8_t*)it.m + i, n), cv = load_codes<VEC>((const uint8_t*)it.v + i, n);
    decode8(cm, n > 0 ? scale_operand8(it.ms[block]) : 0.f, m);
    decode8(cv, n > 0 ? scale_operand8(it.vs[block]) : 0.f, root);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = root[j] * root[j];
  } else {
    load8<VEC>((const float*)it.m + i, n, m);
    load8<VEC>((const float*)it.v + i, n, v);
  }
  if (gs) {
    const float f = *gs;
#pragma unroll
    for (int j = 0; j < 8; ++j) g[j] *= f;
  }
  if constexpr (EIGHT) {
    // The root is held, over all of float32's range; its square has half of that range.
    float r[8];
    bool far = false;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      r[j] = root[j];
      s.moments(g[j], m[j], v[j]);
      root[j] = __builtin_amdgcn_sqrtf(v[j]);
      far |= s.far(v[j], r[j], g[j]);
    }
    if (far) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (s.far(v[j], r[j], g[j])) root[j] = root_of_squares(s.root_b2 * r[j], s.root_one_b2 * g[j]);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      s.moments(g[j], m[j], v[j]);
      root[j] = root_of(v[j]);
    }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) p[j] = s.update(p[j], m[j], root[j]);
  store8<VEC>(it.p + i, n, p);
  if (it.lp) store8<VEC>(it.lp + i, n, p);
  if constexpr (EIGHT) {
    if (n < 8) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j >= n) m[j] = root[j] = 0.f;
    }
    const int em = block_exponent<T5_E4M3>(max16(largest8(m))), er = block_exponent<T5_E4M3>(max16(largest8(root)));
    const float sm = scale_of(em), sr = scale_of(er), least = scale_value((uint32_t)(er + 127)) * (1.f / 512.f);
    const uint32_t row = mix32(it.key ^ (uint32_t)block ^ seed_hi), pre = row ^ (row >> 16);
    const int c0 = (int)(i & 127);
    uint32_t wm[8], wr[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      // mix32(row ^ column): the first step's x >> 16 holds none of the column's seven bits
      uint32_t h = (pre ^ (uint32_t)(c0 + j)) * 0x7FEB352Du;
      h = (h ^ (h >> 15)) * 0x846CA68Bu;
      h ^= h >> 16;
      wm[j] = h << 16;
      wr[j] = h & 0xFFFF0000u;
      root[j] = root[j] > 0.f ? fmaxf(root[j], least) : root[j];  // at least the smallest code
    }
    store_codes<VEC>((uint8_t*)it.m + i, n, u32x2{round_at_random4(m, wm, sm), round_at_random4(m + 4, wm + 4, sm)});
    store_codes<VEC>((uint8_t*)it.v + i, n, u32x2{round_at_random4(root, wr, sr), round_at_random4(root + 4, wr + 4, sr)});
    if (n > 0 && c0 == 0) {
      it.ms[block] = (uint8_t)(em + 127);
      it.vs[block] = (uint8_t)(er + 127);
    }
  } else {
    store8<VEC>((float*)it.m + i, n, m);
    store8<VEC>((float*)it.v + i, n, v);
  }
}

__global__ __launch_bounds__(kThreads) void adamw_kernel(AdamBatch b) {
  // The tensor: how many start at or before this workgroup, but for the first (one load; in turn, each waits for the one before).
  const int lane = threadIdx.x & 63;
  const int t = __popcll(__ballot(lane < b.count - 1 && (int)blockIdx.x >= b.start[min(lane + 1, kAdamTensors)]));
  const AdamItem& it = b.it[t];
  const int64_t i = (int64_t)((int)blockIdx.x - b.start[t]) * kChunk + threadIdx.x * 8;
  const float* gs = b.grad_scale;
  const Step s{b.b1, b.one_b1, b.b2, b.one_b2, b.root_b2, b.root_one_b2, b.root_factor, b.eps, b.step_size, it.keep};
  if (it.flags & AW_8BIT) {
    if (it.flags & AW_VEC) adam_chunk<true, true>(it, s, gs, b.seed_hi, i);
    else adam_chunk<false, true>(it, s, gs, b.seed_hi, i);
  } else {
    if (it.flags & AW_VEC) adam_chunk<true, false>(it, s, gs, b.seed_hi, i);
    else adam_chunk<false, false>(it, s, gs, b.seed_hi, i);
  }
}

}  // namespace

hipError_t launch_adamw(const adamw_tensor* t, int n, int first, const adamw_cfg& c, hipStream_t st) {
  if (n < 1 || n > kAdamTensors) return hipErrorInvalidValue;
  AdamBatch b;
  std::memset(&b, 0, sizeof(b));
  b.count = n;
  b.seed_hi = c.seed_hi;
  b.b1 = (float)c.beta1; b.one_b1 = (float)(1.0 - c.beta1);
  b.b2 = (float)c.beta2; b.one_b2 = (float)(1.0 - c.beta2);
  b.root_b2 = (float)std::sqrt(c.beta2); b.root_one_b2 = (float)std::sqrt(1.0 - c.beta2);
  b.root_factor = (float)(1.0 / std::sqrt(1.0 - std::pow(c.beta2, (double)c.step)));
  b.eps = (float)c.eps;
  b.step_size = (float)(c.lr / (1.0 - std::pow(c.beta1, (double)c.step)));
  b.grad_scale = c.grad_scale;
  const uint32_t k0 = mix32(c.seed_lo ^ (uint32_t)c.step);
  int64_t chunks = 0;
  for (int i = 0; i < n; ++i) {
    AdamItem& it = b.it[i];
    it.p = t[i].param; it.g = t[i].grad; it.m = t[i].m; it.v = t[i].v;
    it.ms = t[i].m_scale; it.vs = t[i].v_scale; it.lp = (bf16*)t[i].bf16_copy_out; it.n = t[i].n;
    it.keep = (float)(1.0 - c.lr * t[i].weight_decay);
    it.key = mix32(k0 ^ (uint32_t)(first + i) * 0x9E3779B9u);
    const uintptr_t code_mask = t[i].state_bits == 8 ? 7 : 15;
    const uintptr_t odd = ((uintptr_t)it.p & 15) | ((uintptr_t)it.g & 15) | ((uintptr_t)it.m & code_mask) |
                          ((uintptr_t)it.v & code_mask) | ((uintptr_t)it.lp & 15);
    it.flags = (t[i].state_bits == 8 ? AW_8BIT : 0) | (t[i].grad_dtype == T5_BF16 ? AW_BF16_GRAD : 0) | (odd == 0 ? AW_VEC : 0);
    b.start[i] = (int32_t)chunks;
    chunks += (t[i].n + kChunk - 1) / kChunk;
    if (chunks >= (1 << 24)) return hipErrorInvalidValue;
  }
  b.start[n] = (int32_t)chunks;
  adamw_kernel<<<(unsigned)chunks, kThreads, 0, st>>>(b);
  return hipGetLastError();
}

}  // namespace t5mi
