// Fused attention over packed sequences with grouped heads in fp32, head sizes 32, 64 and 128, on the fp32 matrix
// instruction (v_mfma_f32_32x32x2_f32); formulas as in packed_attention.hip.
//
// Bound by the matrix instruction: 64 clocks for 4096 operations, two (forward), three (dQ) and four (dK/dV) times D / 2 of
// them for 32 x 32 scores.  So everything else may take its time: 32 own rows belong to W waves, which take the 32-row
// tiles of the opposite rows in turn and add their results in wave order at the end.  A wave loads a tile's rows from
// memory straight into operands of the products along the head, the next tile's while it works, and passes them through LDS
// of its own for the product that needs them by columns, without a barrier.
//
// MFMA 32x32x2: A, B: lane holds row / column lane % 32, index lane / 32 of the pair; D: lane holds column lane % 32,
// register r holds row 8 * (r / 4) + 4 * (lane / 32) + r % 4.  Score tiles have the own rows as columns, so that register r
// is, as it stands, the B operand of the next product for the index pair (8 * (r / 4) + r % 4, the same + 4).
#include "gemm_device.h"
#include "packed_device.h"

namespace mk {
namespace {

constexpr int TR = 32;                 // own rows of a block, and rows of a streamed tile
constexpr float LOG2E = 1.44269504088896340736f;
__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }   // 1 unit in the last place; -inf gives 0

template <int D> using Rows4 = float4[D / 8];

// row l32 of the tile from r0 on (rows past `last` are read as `last`): element j of group g is column 8 g + 4 h + j
template <int D>
__device__ __forceinline__ void fetch_rows(const float* src, int64_t ld, int r0, int last, int l32, int h, Rows4<D>& f) {
  const float* p = src + (int64_t)min(r0 + l32, last) * ld + 4 * h;
#pragma unroll
  for (int g = 0; g < D / 8; ++g) f[g] = *(const float4*)(p + 8 * g);
}
// the same rows as they lie, [row][D + 4], to be read by columns
template <int D>
__device__ __forceinline__ void stash(float* tile, int l32, int h, const Rows4<D>& f) {
#pragma unroll
  for (int g = 0; g < D / 8; ++g) *(float4*)&tile[l32 * (D + 4) + 8 * g + 4 * h] = f[g];
}
__device__ __forceinline__ void clear(f32x16& v) {
#pragma unroll
  for (int r = 0; r < 16; ++r) v[r] = 0.f;
}
// s = tile rows (A) x own rows (B), which lie in LDS, over the D columns
template <int D>
__device__ __forceinline__ void scores(const Rows4<D>& rows, const float* own, int l32, int h, f32x16& s) {
  clear(s);
#pragma unroll
  for (int g = 0; g < D / 8; ++g) {
    const float4 a = rows[g], b = *(const float4*)&own[l32 * (D + 4) + 8 * g + 4 * h];
    s = __builtin_amdgcn_mfma_f32_32x32x2f32(a.x, b.x, s, 0, 0, 0);
    s = __builtin_amdgcn_mfma_f32_32x32x2f32(a.y, b.y, s, 0, 0, 0);
    s = __builtin_amdgcn_mfma_f32_32x32x2f32(a.z, b.z, s, 0, 0, 0);
    s = __builtin_amdgcn_mfma_f32_32x32x2f32(a.w, b.w, s, 0, 0, 0);
  }
}
// acc (rows = head columns, columns = own rows) += tile^T x s
template <int D>
__device__ __forceinline__ void accumulate(const float* tile, int l32, int h, const f32x16& s, f32x16 (&acc)[D / 32]) {
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const float* row = &tile[(8 * (r >> 2) + 4 * h + (r & 3)) * (D + 4) + l32];
#pragma unroll
    for (int db = 0; db < D / 32; ++db) acc[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(row[32 * db], s[r], acc[db], 0, 0, 0);
  }
}
// What the lanes of a wave have stored to LDS before, the others read after: the hardware keeps a wave's accesses in order,
// the compiler has to be told.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
  __builtin_amdgcn_wave_barrier();
}
__device__ __forceinline__ float other_half(float v) {
  const uint32_t u = __float_as_uint(v);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __uint_as_float((threadIdx.x & 32) ? r[0] : r[1]);
}
// A wave's part of a sum over the tiles goes into its own part of LDS (TR * (D + 4) floats) ...
template <int D>
__device__ __forceinline__ void put_part(float* part, int lane, const f32x16 (&acc)[D / 32]) {
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *(float4*)&part[((4 * db + g) * 64 + lane) * 4] = make_float4(acc[db][4 * g], acc[db][4 * g + 1], acc[db][4 * g + 2], acc[db][4 * g + 3]);
}
// ... and behind a barrier wave w adds the waves' parts of head columns 8 q + 4 h .., q = w, w + W, ..., in wave order,
// each times a factor of its own.  dst: the lane's row.
template <int D, int W>
__device__ __forceinline__ void store_sum(float* dst, const float* parts, int stride, int wave, int lane, const float (&factor)[W]) {
#pragma unroll
  for (int i = 0; i < D / 8 / W; ++i) {
    const int q = wave + W * i;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float4 v = *(const float4*)&parts[w * stride + (q * 64 + lane) * 4];
      s.x = fmaf(v.x, factor[w], s.x); s.y = fmaf(v.y, factor[w], s.y);
      s.z = fmaf(v.z, factor[w], s.z); s.w = fmaf(v.w, factor[w], s.w);
    }
    if (dst) *(float4*)(dst + 8 * q + 4 * (lane >> 5)) = s;
  }
}

template <int D> constexpr int tile_floats() { return TR * (D + 4); }

}  // namespace

// ------------------------------------------------------------------ forward
// 12 sequences of 153-397 rows without mask, 12 heads of 64: 71 us, 42 TFLOP/s (heads of 32 35, of 128 165); 64 causal ones of 512: 595, 43
// TFLOP/s of the pairs that see each other (a diagonal tile makes twice those), heads of 128 1665, 31: there LDS has room for three blocks of
// two waves on a compute unit, with heads of 64 for five.
template <int D, bool CAUSAL, int W>
__global__ __launch_bounds__(64 * W) void packed_f32_fwd_kernel(PackedAttention p, int slots) {
  constexpr int TILE = tile_floats<D>();
  extern __shared__ __attribute__((aligned(16))) float f_smem[];
  float* const own = f_smem;                          // [TR][D + 4]
  float* const stat = own + TILE;                     // [W][2][64]: maxima, sums
  float* const mine = stat + W * 128;                 // a wave's tile, and its part of the sum afterwards
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, h = lane >> 5;
  PackedPlace w;
  if (!packed_place<TR, CAUSAL>(p, slots, blockIdx.x, w)) return;
  const int qi = w.row + l32, last = w.n - 1;
  const float c2 = p.scale * LOG2E;
  const float* kb = (const float*)p.k + w.first * p.ldk + w.kv * D;
  const float* vb = (const float*)p.v + w.first * p.ldv + w.kv * D;
  Rows4<D> kf, vf;
  if (wave == 0) {
    fetch_rows<D>((const float*)p.q + w.first * p.ldq + w.head * D, p.ldq, w.row, last, l32, h, kf);
    stash<D>(own, l32, h, kf);
  }
  const int kend = CAUSAL ? min(w.n, w.row + TR) : w.n;
  int k0 = wave * TR;
  fetch_rows<D>(kb, p.ldk, k0, last, l32, h, kf);
  fetch_rows<D>(vb, p.ldv, k0, last, l32, h, vf);
  __syncthreads();
  f32x16 o[D / 32];
#pragma unroll
  for (int db = 0; db < D / 32; ++db) clear(o[db]);
  float m = -INFINITY, l = 0.f;
  float* const tile = mine + wave * TILE;
  for (; k0 < kend; k0 += W * TR) {
    f32x16 s;
    scores<D>(kf, own, l32, h, s);
    wave_sync();
    stash<D>(tile, l32, h, vf);
    wave_sync();
    if (k0 + W * TR < kend) {
      fetch_rows<D>(kb, p.ldk, k0 + W * TR, last, l32, h, kf);
      fetch_rows<D>(vb, p.ldv, k0 + W * TR, last, l32, h, vf);
    }
    float mx = -INFINITY;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int key = k0 + 8 * (r >> 2) + 4 * h + (r & 3);
      if (key >= w.n || (CAUSAL && key > qi)) s[r] = -INFINITY;
      mx = fmaxf(mx, s[r]);
    }
    mx = fmaxf(mx, other_half(mx));
    const float mnew = fmaxf(m, mx), base = mnew == -INFINITY ? 0.f : mnew;   // a wave's tile may lie behind all that a row sees
    const float alpha = fast_exp2((m - base) * c2);
    m = mnew;
    float rs = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[r] = fast_exp2((s[r] - base) * c2);
      rs += s[r];
    }
    rs += other_half(rs);
    l = fmaf(l, alpha, rs);
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[db][r] *= alpha;
    accumulate<D>(tile, l32, h, s, o);
  }
  wave_sync();
  put_part<D>(tile, lane, o);
  stat[wave * 128 + lane] = m;
  stat[wave * 128 + 64 + lane] = l;
  __syncthreads();
  float top = -INFINITY, total = 0.f, factor[W];
#pragma unroll
  for (int i = 0; i < W; ++i) top = fmaxf(top, stat[i * 128 + lane]);
#pragma unroll
  for (int i = 0; i < W; ++i) {
    factor[i] = fast_exp2((stat[i * 128 + lane] - top) * c2);
    total = fmaf(stat[i * 128 + 64 + lane], factor[i], total);
  }
#pragma unroll
  for (int i = 0; i < W; ++i) factor[i] /= total;
  const bool real = qi < w.n;
  store_sum<D, W>(real ? (float*)p.out + (w.first + qi) * p.ldo + w.head * D : nullptr, mine, TILE, wave, lane, factor);
  if (real && wave == 0 && h == 0) p.lse[(int64_t)w.head * p.T + w.first + qi] = fmaf(top, p.scale, logf(total));
}

// ------------------------------------------------------------------ dQ
// 12 sequences of 153-397 rows without mask, 12 heads of 64: 75 us, 60 TFLOP/s, the matrix units 60 % busy while a unit has work.
// TELL: delta is written out for the keys' gradients, which are made after.
template <int D, bool CAUSAL, int W, bool TELL>
__device__ __forceinline__ void f32_bwd_dq(const PackedAttention& p, int slots, int block, float* f_smem) {
  constexpr int TILE = tile_floats<D>();
  float *const own_q = f_smem, *const own_g = own_q + TILE, *const mine = own_g + TILE;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, h = lane >> 5;
  PackedPlace w;
  if (!packed_place<TR, CAUSAL>(p, slots, block, w)) return;
  const int qi = w.row + l32, last = w.n - 1;
  const int64_t stats = (int64_t)w.head * p.T + w.first;
  const float* kb = (const float*)p.k + w.first * p.ldk + w.kv * D;
  const float* vb = (const float*)p.v + w.first * p.ldv + w.kv * D;
  Rows4<D> kf, vf;
  fetch_rows<D>((const float*)p.dout + w.first * p.lddo + w.head * D, p.lddo, w.row, last, l32, h, kf);
  fetch_rows<D>((const float*)p.out + w.first * p.ldo + w.head * D, p.ldo, w.row, last, l32, h, vf);
  float delta = 0.f;
#pragma unroll
  for (int g = 0; g < D / 8; ++g) {
    delta = fmaf(kf[g].x, vf[g].x, delta); delta = fmaf(kf[g].y, vf[g].y, delta);
    delta = fmaf(kf[g].z, vf[g].z, delta); delta = fmaf(kf[g].w, vf[g].w, delta);
  }
  delta += other_half(delta);
  if (wave == 0) {
    stash<D>(own_g, l32, h, kf);
    fetch_rows<D>((const float*)p.q + w.first * p.ldq + w.head * D, p.ldq, w.row, last, l32, h, kf);
    stash<D>(own_q, l32, h, kf);
    if (TELL && h == 0 && qi < w.n) p.delta[stats + qi] = delta;
  }
  const float lse = p.lse[stats + min(qi, last)];
  const int kend = CAUSAL ? min(w.n, w.row + TR) : w.n;
  int k0 = wave * TR;
  fetch_rows<D>(kb, p.ldk, k0, last, l32, h, kf);
  fetch_rows<D>(vb, p.ldv, k0, last, l32, h, vf);
  __syncthreads();
  f32x16 dq[D / 32];
#pragma unroll
  for (int db = 0; db < D / 32; ++db) clear(dq[db]);
  float* const tile = mine + wave * TILE;
  for (; k0 < kend; k0 += W * TR) {
    f32x16 s, dp;
    scores<D>(kf, own_q, l32, h, s);
    wave_sync();
    stash<D>(tile, l32, h, kf);
    wave_sync();
    scores<D>(vf, own_g, l32, h, dp);
    if (k0 + W * TR < kend) {
      fetch_rows<D>(kb, p.ldk, k0 + W * TR, last, l32, h, kf);
      fetch_rows<D>(vb, p.ldv, k0 + W * TR, last, l32, h, vf);
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int key = k0 + 8 * (r >> 2) + 4 * h + (r & 3);
      const float pr = fast_exp2(fmaf(s[r], p.scale, -lse) * LOG2E);
      s[r] = key >= w.n || (CAUSAL && key > qi) ? 0.f : pr * (dp[r] - delta);
    }
    accumulate<D>(tile, l32, h, s, dq);
  }
  wave_sync();
  put_part<D>(tile, lane, dq);
  __syncthreads();
  float factor[W];
#pragma unroll
  for (int i = 0; i < W; ++i) factor[i] = p.scale;
  store_sum<D, W>(qi < w.n ? (float*)p.dq + (w.first + qi) * p.lddq + w.head * D : nullptr, mine, TILE, wave, lane, factor);
}

template <int D, bool CAUSAL, int W>
__global__ __launch_bounds__(64 * W) void packed_f32_bwd_dq_kernel(PackedAttention p, int slots) {
  extern __shared__ __attribute__((aligned(16))) float f_smem[];
  f32_bwd_dq<D, CAUSAL, W, true>(p, slots, blockIdx.x, f_smem);
}

// ------------------------------------------------------------------ dK, dV
// A wave has one tile of LDS, for the rows of dO and then for those of Q: with a tile for each, a compute unit holds six waves with heads of
// 64 and two with 128, instead of eight and four (12 sequences of 153-397 rows without mask, 12 heads of 64: 100 us, now 94, 64 TFLOP/s, the matrix
// units 67 % busy while a unit has work, a product of 4096^3 of the library 139; heads of 128, the whole backward pass 410 and 278).
// TOLD: delta is there; else it is made of dO and O.
template <int D, bool CAUSAL, int W, bool TOLD>
__device__ __forceinline__ void f32_bwd_dkv(const PackedAttention& p, int slots, int block, float* f_smem) {
  constexpr int TILE = tile_floats<D>();
  float *const own_k = f_smem, *const own_v = own_k + TILE, *const rowstat = own_v + TILE;   // rowstat [W][2][TR]: lse, delta of a tile
  float* const mine = rowstat + W * 2 * TR;           // a tile of dO, then of Q, to each wave
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, h = lane >> 5;
  PackedPlace w;
  if (!packed_place_kv<TR, CAUSAL>(p, slots, block, w)) return;
  const int ki = w.row + l32, last = w.n - 1, group = p.n_heads / p.n_kv_heads;
  const float* qb = (const float*)p.q + w.first * p.ldq + w.kv * group * D;
  const float* gb = (const float*)p.dout + w.first * p.lddo + w.kv * group * D;
  const int64_t stats = (int64_t)w.kv * group * p.T + w.first;
  Rows4<D> qf, gf;
  if (wave == 0) {
    fetch_rows<D>((const float*)p.k + w.first * p.ldk + w.kv * D, p.ldk, w.row, last, l32, h, qf);
    fetch_rows<D>((const float*)p.v + w.first * p.ldv + w.kv * D, p.ldv, w.row, last, l32, h, gf);
    stash<D>(own_k, l32, h, qf);
    stash<D>(own_v, l32, h, gf);
  }
  // the tiles of all heads that share these keys, one head after the other; a wave takes every W-th
  const int qstart = CAUSAL ? w.row : 0, per_head = (w.n - qstart + TR - 1) / TR, tiles = per_head * group;
  float pre = 0.f;                                    // lse (lanes 0 ..) and delta (lanes 32 ..) of the tile's rows
  auto fetch_q = [&](int t) {
    const int head = t / per_head, q0 = qstart + (t - head * per_head) * TR;
    fetch_rows<D>(qb + head * D, p.ldq, q0, last, l32, h, qf);
  };
  auto fetch_g = [&](int t) {
    const int head = t / per_head, q0 = qstart + (t - head * per_head) * TR;
    fetch_rows<D>(gb + head * D, p.lddo, q0, last, l32, h, gf);
    const int64_t at = stats + (int64_t)head * p.T + min(q0 + l32, last);
    if (TOLD) {
      pre = (h ? p.delta : p.lse)[at];
    } else {
      Rows4<D> of;
      fetch_rows<D>((const float*)p.out + w.first * p.ldo + (w.kv * group + head) * D, p.ldo, q0, last, l32, h, of);
      float delta = 0.f;
#pragma unroll
      for (int g = 0; g < D / 8; ++g) {
        delta = fmaf(gf[g].x, of[g].x, delta); delta = fmaf(gf[g].y, of[g].y, delta);
        delta = fmaf(gf[g].z, of[g].z, delta); delta = fmaf(gf[g].w, of[g].w, delta);
      }
      delta += other_half(delta);
      pre = h ? delta : p.lse[at];
    }
  };
  int t = wave;
  if (t < tiles) {
    fetch_q(t);
    fetch_g(t);
  }
  __syncthreads();
  f32x16 dk[D / 32], dv[D / 32];
#pragma unroll
  for (int db = 0; db < D / 32; ++db) { clear(dk[db]); clear(dv[db]); }
  float *const tile = mine + wave * TILE, *const st = rowstat + wave * 2 * TR;
  for (; t < tiles; t += W) {
    const int q0 = qstart + t % per_head * TR;
    f32x16 s, dp;
    scores<D>(qf, own_k, l32, h, s);
    scores<D>(gf, own_v, l32, h, dp);
    wave_sync();
    stash<D>(tile, l32, h, gf);
    st[lane] = pre;
    wave_sync();
    if (t + W < tiles) fetch_g(t + W);
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const float4 nl = *(const float4*)&st[8 * g + 4 * h], dl = *(const float4*)&st[TR + 8 * g + 4 * h];
      const float ls[4] = {nl.x, nl.y, nl.z, nl.w}, ds[4] = {dl.x, dl.y, dl.z, dl.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int r = 4 * g + e, q = q0 + 8 * g + 4 * h + e;
        const float pr = q >= w.n || (CAUSAL && ki > q) ? 0.f : fast_exp2(fmaf(s[r], p.scale, -ls[e]) * LOG2E);
        s[r] = pr;
        dp[r] = pr * (dp[r] - ds[e]);
      }
    }
    accumulate<D>(tile, l32, h, s, dv);
    wave_sync();
    stash<D>(tile, l32, h, qf);
    wave_sync();
    if (t + W < tiles) fetch_q(t + W);
    accumulate<D>(tile, l32, h, dp, dk);
  }
  wave_sync();
  put_part<D>(tile, lane, dk);
  __syncthreads();
  float factor[W], one[W];
#pragma unroll
  for (int i = 0; i < W; ++i) { factor[i] = p.scale; one[i] = 1.f; }
  const bool real = ki < w.n;
  store_sum<D, W>(real ? (float*)p.dk + (w.first + ki) * p.lddk + w.kv * D : nullptr, mine, TILE, wave, lane, factor);
  __syncthreads();
  put_part<D>(tile, lane, dv);
  __syncthreads();
  store_sum<D, W>(real ? (float*)p.dv + (w.first + ki) * p.lddv + w.kv * D : nullptr, mine, TILE, wave, lane, one);
}

template <int D, bool CAUSAL, int W>
__global__ __launch_bounds__(64 * W) void packed_f32_bwd_dkv_kernel(PackedAttention p, int slots) {
  extern __shared__ __attribute__((aligned(16))) float f_smem[];
  f32_bwd_dkv<D, CAUSAL, W, true>(p, slots, blockIdx.x, f_smem);
}

// Both in one launch, for few rows: the first `queries` blocks make dQ, the others dK and dV with a delta of their own.
template <int D, bool CAUSAL, int W>
__global__ __launch_bounds__(64 * W) void packed_f32_bwd_small_kernel(PackedAttention p, int slots, int queries) {
  extern __shared__ __attribute__((aligned(16))) float f_smem[];
  if ((int)blockIdx.x < queries) f32_bwd_dq<D, CAUSAL, W, false>(p, slots, blockIdx.x, f_smem);
  else f32_bwd_dkv<D, CAUSAL, W, false>(p, slots, blockIdx.x - queries, f_smem);
}

namespace {
template <auto K, int W, int FLOATS, typename... A>
void launch(unsigned blocks, hipStream_t st, A... a) {
  static const bool configured = [] {
    (void)hipFuncSetAttribute((const void*)K, hipFuncAttributeMaxDynamicSharedMemorySize, FLOATS * 4);
    return true;
  }();
  (void)configured;
  hipLaunchKernelGGL(K, dim3(blocks), dim3(64 * W), FLOATS * 4, st, a...);
}
template <int D, bool CAUSAL>
void fwd(const PackedAttention& p, hipStream_t st) {
  constexpr int T = tile_floats<D>();
  const int slots = packed_slots(p.T, p.n_seq, TR);
  const unsigned blocks = packed_blocks(slots, p.n_kv_heads, p.n_heads / p.n_kv_heads);
  // Four waves to 32 rows while blocks are few (and, with heads of 128, rows have tiles for all of them).  Four and two, us, sequences x
  // rows, query heads: heads of 64 behind a mask, 12: 4x64 9.8 and 9.2, 4x128 11.3 and 14.5, 1x1024 59 and 89, 8x128 (480 blocks) 16.5 and
  // 16.8, 8x256 (864) 31 and 33, 8x512 (1632) 76 and 71; heads of 128, 12: 4x64 15.4 and 13.1, 1x1024 (396) 94 and 147, 8x128 35 and 28.
  const bool four = D == 128 ? blocks <= 400 && p.T > (int64_t)p.n_seq * 96 : blocks <= 640;
  if (four) launch<packed_f32_fwd_kernel<D, CAUSAL, 4>, 4, T + 4 * 128 + 4 * T>(blocks, st, p, slots);
  else launch<packed_f32_fwd_kernel<D, CAUSAL, 2>, 2, T + 2 * 128 + 2 * T>(blocks, st, p, slots);
}
template <int D, bool CAUSAL>
void bwd(const PackedAttention& p, hipStream_t st) {
  constexpr int W = 2, T = tile_floats<D>(), WS = 4;
  const int slots = packed_slots(p.T, p.n_seq, TR);
  const unsigned queries = packed_blocks(slots, p.n_kv_heads, p.n_heads / p.n_kv_heads), keys = packed_blocks(slots, p.n_kv_heads, 1);
  const int group = p.n_heads / p.n_kv_heads;
  // One launch, of four waves to 32 rows, while its blocks are few enough to leave compute units for so many.  One launch and two, us,
  // sequences x rows, query heads / heads of keys (blocks of queries), behind a mask: heads of 64, 12 / 12: 4x64 11.8 and 18.6, 8x256 (864) 64
  // and 68, 8x512 (1632) 159 and 140; 16 / 4: 4x128 (320) 37 and 37, 8x256 (1152) 87 and 78; 2 / 1: 1x1024 (66) 93 and 139, 16x512 (544)
  // 98 and 91; heads of 32, 12 / 12: 8x512 81 and 99, 16x512 (3264) 151 and 137; 16 / 4: 8x128 (640) 25 and 28, 8x256 60 and 47; heads of
  // 128, 12 / 12: 8x128 (480) 54 and 58, 8x256 134 and 100; 16 / 4: 2x256 (288) 109 and 115, 8x128 (640) 88 and 74.
  const unsigned most = D == 128 ? 480 : group == 1 ? (D == 32 ? 1700 : 900) : (D == 32 ? 700 : 500);
  if (queries <= most) {
    launch<packed_f32_bwd_small_kernel<D, CAUSAL, WS>, WS, 2 * T + WS * 2 * TR + WS * T>(queries + keys, st, p, slots, (int)queries);
    return;
  }
  launch<packed_f32_bwd_dq_kernel<D, CAUSAL, W>, W, 2 * T + W * T>(queries, st, p, slots);
  // Four waves to 32 keys where these have tiles for all of them, or blocks are few.  Two and four, us, the whole pass, (blocks of keys): heads
  // of 64, 12 / 12 without mask: 64x128 (3840) 183 and 201, 16x512 (3264) 449 and 430, 2x2048 (1560) 879 and 731; behind a mask 122 and
  // 142, 252 and 267, 456 and 432; 16 / 4 behind a mask: 32x512 (2176) 594 and 581; heads of 128, 16 / 4: 8x512 (544) 439 and 333,
  // 16x512 (1088) 627 and 649; 12 / 12: 8x256 (864) 101 and 114.
  const bool four = D == 128 ? keys <= 640 : keys <= 1024 || (int64_t)p.T * group >= (int64_t)p.n_seq * (CAUSAL ? 640 : 320);
  if (four) launch<packed_f32_bwd_dkv_kernel<D, CAUSAL, 4>, 4, 2 * T + 4 * 2 * TR + 4 * T>(keys, st, p, slots);
  else launch<packed_f32_bwd_dkv_kernel<D, CAUSAL, 2>, 2, 2 * T + 2 * 2 * TR + 2 * T>(keys, st, p, slots);
}
}  // namespace

void packed_attention_fwd_bf16(const PackedAttention& p, int d, int causal, hipStream_t st);
void packed_attention_bwd_bf16(const PackedAttention& p, int d, int causal, hipStream_t st);

bool packed_attention_fits(int64_t T, int64_t n_seq, int64_t n_heads) {
  return (packed_slots64(T, n_seq, TR) + 8) * n_heads < (int64_t)1 << 23;   // a grid's threads are counted in 32 bits
}

size_t packed_attention_bwd_workspace_bytes(int64_t T, int n_heads, int n_kv_heads, int d) {
  (void)n_kv_heads; (void)d;
  return ((size_t)T * n_heads * sizeof(float) + 255) / 256 * 256;
}

#define BY_HEAD_(CALL, D, CAUSAL)                                                                       \
  do {                                                                                                  \
    if (D == 32) { if (CAUSAL) CALL(32, true); else CALL(32, false); }                                  \
    else if (D == 64) { if (CAUSAL) CALL(64, true); else CALL(64, false); }                             \
    else { if (CAUSAL) CALL(128, true); else CALL(128, false); }                                        \
  } while (0)

void packed_attention_fwd(int dtype, const PackedAttention& p, int d, int causal, hipStream_t st) {
  if (p.T == 0 || p.n_seq == 0) return;
  if (dtype == BF16) { packed_attention_fwd_bf16(p, d, causal, st); return; }
#define FWD_(D_, C_) fwd<D_, C_>(p, st)
  BY_HEAD_(FWD_, d, causal);
#undef FWD_
}

void packed_attention_bwd(int dtype, PackedAttention p, int d, int causal, void* workspace, hipStream_t st) {
  if (p.T == 0 || p.n_seq == 0) return;
  p.delta = (float*)workspace;
  if (dtype == BF16) { packed_attention_bwd_bf16(p, d, causal, st); return; }
#define BWD_(D_, C_) bwd<D_, C_>(p, st)
  BY_HEAD_(BWD_, d, causal);
#undef BWD_
}

}  // namespace mk
