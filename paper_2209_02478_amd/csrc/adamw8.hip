// AdamW over many tensors in one launch, moments held in 8 bits.
//
//   m = b1 m + (1-b1) g;  v = b2 v + (1-b2) g^2;  p = p - lr ((m / c1) / (sqrt(v / c2) + eps) + wd p)
//
// Held are m and sqrt(v), not v: its square root has half the range in powers of two.  kAdamBlock neighbouring elements
// of a tensor share an fp32 scale, which puts their largest value at 448, the largest of e4m3 (four bits of exponent,
// three of mantissa).  Values down to 2^-14.8 of the largest (2^-6 of 448) lie within 1/8 of the next code; below that codes
// are 2^-17.8 of the largest apart, so that a value at 2^-16 is held to a third and one below 2^-17.8 as nothing or as
// the smallest code.  Rounded to the nearest code a slow moment would stand still (with b2 = 0.999 an update moves sqrt(v)
// by a twentieth of a per cent, codes lie 6 to 12 per cent apart), so codes are rounded with a dither: a 20-bit number added
// below the last bit that is kept.  It is the Weyl sequence (a element + b update) mod 2^32, b the golden ratio's: over the
// updates every element meets evenly spread numbers, the rounding averages out, and nothing random has to be kept.
// A second moment above zero is never held as zero, which would make the next step one of m / eps.  That is the one bias: a
// root below 2^-17.8 of its block's largest is held as the smallest code and does not decay below it, so that such an
// element's steps are smaller than the formula's, by the root's share of that code, as long as the block's largest stays.
// Values that are not finite are held as NaN and do not enter their block's scale.
//
// Bound by memory: 18 bytes an element where a bf16 copy is written (30 with fp32 moments), 16 where not (28).  Nothing is
// touched again before it has left the caches but the low-precision copy, so all else goes past them: 355 M elements in
// bf16 1187 -> 1106 us (5.8 TB/s), 109 M 339 -> 328 (6.0; with fp32 moments 623).  Each operation of the formula is rounded
// by itself (no fused multiply-adds), so that what is held can be reproduced by any other program.
#include "device_common.h"

namespace mk {

struct Adam8Hyper { float lr, beta1, beta2, eps, weight_decay, inv_c1, root_inv_c2; uint32_t dither; };

// code of |x| / scale, dither in the low 20 bits
__device__ __forceinline__ uint32_t to_e4m3(float x, float inv_scale, uint32_t dither) {
  const float y = fminf(fabsf(x) * inv_scale, 448.f);
  const uint32_t normal = ((__float_as_uint(y) + dither) >> 20) - 960u;
  const uint32_t small = ((uint32_t)(fminf(y, 0x1p-6f) * 0x1p29f) + dither) >> 20;   // below 2^-6 codes are 2^-9 apart
  uint32_t code = y >= 0x1p-6f ? normal : small;
  if (!(fabsf(x) < INFINITY)) code = 127u;
  return code | (x < 0.f ? 128u : 0u);
}
__device__ __forceinline__ void from_e4m3(uint32_t codes, float scale, float (&x)[4]) {
  const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
  x[0] = a[0] * scale; x[1] = a[1] * scale; x[2] = b[0] * scale; x[3] = b[1] * scale;
}
__device__ __forceinline__ float finite_abs(float x) { return fabsf(x) < INFINITY ? fabsf(x) : 0.f; }
__device__ __forceinline__ float block_scale(float top) { return fmaxf(top, 0x1p-100f) * (1.f / 448.f); }

// a wave for a block of 256 elements, four a lane
constexpr int kAdam8Threads = 256, kAdam8Blocks = kAdamChunk / (4 * kAdam8Threads);
__global__ __launch_bounds__(kAdam8Threads) void adamw8_kernel(const Adam8Tensor* __restrict__ tensors, const AdamChunk* __restrict__ chunks,
                                                               Adam8Hyper h) {
#pragma clang fp contract(off)
  typedef float f32x4 __attribute__((ext_vector_type(4)));
  const AdamChunk ck = chunks[blockIdx.x / kAdam8Blocks];
  const Adam8Tensor t = tensors[ck.tensor];
  const float wd = t.decay ? h.weight_decay : 0.f;
  const int64_t i = ck.start + 4 * ((int64_t)(blockIdx.x % kAdam8Blocks) * kAdam8Threads + threadIdx.x);
  const int64_t block = i / kAdamBlock;                 // the same for a wave
  if (block * kAdamBlock >= t.n) return;
  const int count = (int)max((int64_t)0, min((int64_t)4, t.n - i));
  float g[4] = {}, p[4] = {}, m[4] = {}, v[4] = {};
  uint32_t mc = 0, vc = 0;
  if (count == 4) {
    const f32x4 g4 = __builtin_nontemporal_load(in_global((const f32x4*)(t.grad + i))),
                p4 = __builtin_nontemporal_load(in_global((const f32x4*)(t.master + i)));
    g[0] = g4[0]; g[1] = g4[1]; g[2] = g4[2]; g[3] = g4[3];
    p[0] = p4[0]; p[1] = p4[1]; p[2] = p4[2]; p[3] = p4[3];
    mc = __builtin_nontemporal_load(in_global((const uint32_t*)(t.m + i)));
    vc = __builtin_nontemporal_load(in_global((const uint32_t*)(t.v + i)));
  } else {
    for (int e = 0; e < count; ++e) {
      g[e] = t.grad[i + e]; p[e] = t.master[i + e];
      mc |= (uint32_t)t.m[i + e] << (8 * e);
      vc |= (uint32_t)t.v[i + e] << (8 * e);
    }
  }
  from_e4m3(mc, in_global(t.m_scale)[block], m);
  from_e4m3(vc, in_global(t.v_scale)[block], v);
  float root[4], top_m = 0.f, top_v = 0.f;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    m[e] = h.beta1 * m[e] + (1.f - h.beta1) * g[e];
    v[e] = h.beta2 * (v[e] * v[e]) + (1.f - h.beta2) * g[e] * g[e];
    root[e] = sqrtf(v[e]);
    p[e] -= h.lr * ((m[e] * h.inv_c1) / (root[e] * h.root_inv_c2 + h.eps) + wd * p[e]);
    top_m = fmaxf(top_m, finite_abs(m[e]));
    top_v = fmaxf(top_v, finite_abs(root[e]));
  }
  const float m_scale = block_scale(wave_max(top_m)), v_scale = block_scale(wave_max(top_v));
  const float m_inv = 1.f / m_scale, v_inv = 1.f / v_scale;
  mc = vc = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t at = (uint32_t)(i + e);
    mc |= to_e4m3(m[e], m_inv, (at * 0xC13FA9A9u + h.dither) >> 12) << (8 * e);
    const uint32_t c = to_e4m3(root[e], v_inv, (at * 0x91E10DA5u + h.dither) >> 12);
    vc |= (c == 0u && root[e] > 0.f ? 1u : c) << (8 * e);
  }
  if (count == 4) {
    f32x4 p4 = {p[0], p[1], p[2], p[3]};
    __builtin_nontemporal_store(mc, in_global((uint32_t*)(t.m + i)));
    __builtin_nontemporal_store(vc, in_global((uint32_t*)(t.v + i)));
    if (t.lowp) {
      __builtin_nontemporal_store(p4, in_global((f32x4*)(t.master + i)));
      typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
      *in_global((u32x2*)((bf16_t*)t.lowp + i)) = u32x2{pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3])};
    } else {
      asm volatile("" : "+v"(p4));                      // (else the compiler makes one ordinary store of the two)
      *in_global((f32x4*)(t.master + i)) = p4;          // fp32: the master is what the next forward reads
    }
  } else {
    for (int e = 0; e < count; ++e) {
      t.master[i + e] = p[e];
      t.m[i + e] = (uint8_t)(mc >> (8 * e));
      t.v[i + e] = (uint8_t)(vc >> (8 * e));
      if (t.lowp) ((bf16_t*)t.lowp)[i + e] = f32_to_bf16(p[e]);
    }
  }
  if (threadIdx.x % 64 == 0) { in_global(t.m_scale)[block] = m_scale; in_global(t.v_scale)[block] = v_scale; }
}

void adamw8_update(const Adam8Tensor* tensors, const AdamChunk* chunks, int n_chunks, AdamHyper h, int64_t step, hipStream_t st) {
  if (n_chunks <= 0) return;
  const float root_inv_c2 = (float)std::sqrt(1.0 / (1.0 - std::pow((double)h.beta2, (double)step)));
  const Adam8Hyper h8{h.lr, h.beta1, h.beta2, h.eps, h.weight_decay, h.inv_c1, root_inv_c2, (uint32_t)step * 0x9E3779B9u};
  hipLaunchKernelGGL(adamw8_kernel, dim3((unsigned)n_chunks * kAdam8Blocks), dim3(kAdam8Threads), 0, st, tensors, chunks, h8);
}

}  // namespace mk
