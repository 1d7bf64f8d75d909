// Update of a model's matrices with an orthogonalised step (Muon), all matrices of a list in a handful of launches.
//
//   m <- mu m + g,   u = g + mu m (nesterov) or m,   X = u / (|u|_F + eps), transposed where it has more rows than columns
//   n times:  A = X X^T,  B = b A + c A A,  X <- a X + B X       (Newton-Schulz; a, b, c = 3.4445, -4.7750, 2.0315)
//   w <- w - lr (rms sqrt(max(rows, cols)) X + weight_decay w)
//
// The polynomial takes every singular value of X from (0, 1] near 1 and keeps it below 1.21, so that no element of X, A or B
// is above 1.21, 1.47 and 11.  The products' operands are therefore held in fp16 times 2^10: as many bits as any 16-bit type has
// (values from 6e-8 of the largest on keep all eleven; bf16 keeps eight, and the step is then 1 to 5 % off instead of 0.1 to
// 0.6), at the same rate of the matrix units.  Sums are fp32, the norm's fp64 (squares of gradients of 1e-20 are numbers there).
// A and A A are symmetric: only tiles on and above the diagonal are multiplied, and stored twice.
#include "gemm_large.h"
#include "muon.h"

namespace mk {
namespace {

typedef _Float16 f16;
typedef f16 f16x4 __attribute__((ext_vector_type(4)));
typedef f16 f16x8 __attribute__((ext_vector_type(8)));
using large::f32x4;

constexpr float kHeld = 1024.f, kBack = 1.f / 1024.f;        // operands are held times 2^10
constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
constexpr int BK = 64;

__device__ __forceinline__ f16* in_scratch(char* ws, uint64_t at) { return (f16*)(ws + at); }

// sum over the block's 256 threads, in every one of them; the order is fixed
__device__ __forceinline__ double block_sum(double v, double* lds) {
  const int tid = threadIdx.x;
  lds[tid] = v;
  __syncthreads();
  for (int s = 128; s > 0; s >>= 1) {
    if (tid < s) lds[tid] += lds[tid + s];
    __syncthreads();
  }
  return lds[0];
}

}  // namespace

// Momentum, and each chunk's sum of u^2.
__global__ __launch_bounds__(256) void muon_momentum_kernel(const MuonMatrix* mats, const MuonChunk* chunks, char* ws, MuonHyper h) {
  __shared__ double lds[256];
  const MuonChunk c = chunks[blockIdx.x];
  const MuonMatrix& t = mats[c.matrix];
  const int64_t n = (int64_t)t.rows * t.cols, end = min(n, c.start + t.chunk);
  const float* g = t.grad;
  float* m = t.momentum;
  double sum = 0.0;
  auto one = [&](float gi, float mi, float& out) {
    out = fmaf(h.momentum, mi, gi);
    const float u = h.nesterov ? fmaf(h.momentum, out, gi) : out;
    sum += (double)u * u;
  };
  int64_t i = c.start + 4 * threadIdx.x;                     // chunks begin on multiples of 4, tensors on 16 bytes
  for (; i + 4 <= end; i += 1024) {
    const float4 gv = *(const float4*)(g + i), mv = *(const float4*)(m + i);
    float4 o;
    one(gv.x, mv.x, o.x); one(gv.y, mv.y, o.y); one(gv.z, mv.z, o.z); one(gv.w, mv.w, o.w);
    *(float4*)(m + i) = o;
  }
  for (int64_t j = i; j < end && j < i + 4; ++j) {
    float o;
    one(g[j], m[j], o);
    m[j] = o;
  }
  sum = block_sum(sum, lds);
  if (threadIdx.x == 0) ((double*)(ws + t.partial))[c.start / t.chunk] = sum;
}

// X = u / (|u| + eps), 128 x 128 of it a block, zeros behind the matrix' last row and column.
__global__ __launch_bounds__(256) void muon_start_kernel(const MuonMatrix* mats, const MuonTile* tiles, char* ws, MuonHyper h) {
  __shared__ double lds[256];
  __shared__ f16 turn[32][kMuonTile + 2];
  const MuonTile tile = tiles[blockIdx.x];
  const MuonMatrix& t = mats[tile.matrix];
  const int64_t n = (int64_t)t.rows * t.cols;
  const int parts = (int)((n + t.chunk - 1) / t.chunk), tid = threadIdx.x;
  double sum = 0.0;
  for (int i = tid; i < parts; i += 256) sum += ((const double*)(ws + t.partial))[i];
  const double norm = sqrt(block_sum(sum, lds)) + (double)h.eps;
  const float inv = (float)((double)kHeld / norm);           // (eps above 0: finite)
  const bool tall = t.rows > t.cols;
  f16* x = in_scratch(ws, t.x[0]) + (int64_t)tile.i * kMuonTile * t.np + (int64_t)tile.j * kMuonTile;
  auto u = [&](int64_t at) {
    const float g = t.grad[at], m = t.momentum[at];
    return (h.nesterov ? fmaf(h.momentum, m, g) : m) * inv;
  };
  const int col = tid & 127, row0 = tid >> 7;
  if (!tall) {
    const int c = tile.j * kMuonTile + col;
    for (int r = row0; r < kMuonTile; r += 2) {
      const int row = tile.i * kMuonTile + r;
      x[(int64_t)r * t.np + col] = row < t.rows && c < t.cols ? (f16)u((int64_t)row * t.cols + c) : (f16)0.f;
    }
    return;
  }
  // X[i][j] = u[j][i]: 32 rows of u at a time through LDS
  for (int j0 = 0; j0 < kMuonTile; j0 += 32) {
    const int c = tile.i * kMuonTile + col;
    for (int r = row0; r < 32; r += 2) {
      const int row = tile.j * kMuonTile + j0 + r;
      turn[r][col] = row < t.rows && c < t.cols ? (f16)u((int64_t)row * t.cols + c) : (f16)0.f;
    }
    __syncthreads();
    for (int i = tid >> 5; i < kMuonTile; i += 8) x[(int64_t)i * t.np + j0 + (tid & 31)] = turn[tid & 31][i];
    __syncthreads();
  }
}

// STAGE 1: A = X X^T.  2: B = b A + c A A.  3: X' = a X + B X.  A block makes 128 x 128.
template <int STAGE>
__global__ __launch_bounds__(256, 2) void muon_product_kernel(const MuonMatrix* mats, const MuonTile* tiles, char* ws, int from) {
  using namespace large;
  constexpr int R = kMuonTile, SIZE = R * BK;                // elements of an operand tile
  constexpr bool KM = STAGE != 3;
  typedef LTileOf<true, R> TA;
  typedef LTileOf<KM, R> TB;
  __shared__ __attribute__((aligned(1024))) f16 smem[2][2][SIZE];
  const MuonTile tile = tiles[blockIdx.x];
  const MuonMatrix& t = mats[tile.matrix];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave >> 1, wn = wave & 1;
  const int mp = __builtin_amdgcn_readfirstlane(t.mp), np = __builtin_amdgcn_readfirstlane(t.np);
  const int ti = __builtin_amdgcn_readfirstlane(tile.i), tj = __builtin_amdgcn_readfirstlane(tile.j);
  const f16 *x = in_scratch(ws, t.x[from]), *a = in_scratch(ws, t.a), *b = in_scratch(ws, t.b);
  const int lda = STAGE == 1 ? np : mp, ldb = STAGE == 2 ? mp : np, K = STAGE == 1 ? np : mp;
  const f16* pa = (STAGE == 1 ? x : STAGE == 2 ? a : b) + (int64_t)ti * R * lda;
  const f16* pb = STAGE == 3 ? x + tj * R : (STAGE == 1 ? x : a) + (int64_t)tj * R * ldb;
  uint64_t base_a, base_b;
  uint32_t bytes_a, bytes_b, off_a[4], off_b[4];
  l_descriptor(pa, TA::bytes(lda, R), base_a, bytes_a);
  l_descriptor(pb, TB::bytes(ldb, R), base_b, bytes_b);      // (columns of X: no bound, every row is whole)
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    off_a[j] = TA::src(lda, R, wave * 4 + j, lane);
    off_b[j] = TB::src(ldb, R, wave * 4 + j, lane);
  }
  const uint64_t step_a = BK * 2, step_b = KM ? BK * 2 : (uint64_t)BK * 2 * ldb;
  const uint32_t lds = l_lds_address(&smem[0][0][0]) + (uint32_t)wave * 4096u;
  auto fetch = [&](int buf) {
#pragma unroll
    for (int j = 0; j < 4; ++j) l_direct_load(base_a, bytes_a, off_a[j], lds + (uint32_t)buf * (4u * SIZE) + j * 1024u);
#pragma unroll
    for (int j = 0; j < 4; ++j) l_direct_load(base_b, bytes_b, off_b[j], lds + (uint32_t)buf * (4u * SIZE) + 2u * SIZE + j * 1024u);
    base_a += step_a;
    base_b += step_b;
  };
  TA fa;
  TB fb;
  fa.init(wm * 4, lane);
  fb.init(wn * 4, lane);
  f32x4 acc[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int steps = K / BK;
  fetch(0);
  for (int k = 0, buf = 0; k < steps; ++k, buf ^= 1) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (k + 1 < steps) fetch(buf ^ 1);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      f16x8 af[4], bf[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) af[i] = __builtin_bit_cast(f16x8, fa.read((const bf16_t*)&smem[buf][0][0], 0, i, h));
#pragma unroll
      for (int j = 0; j < 4; ++j) bf[j] = __builtin_bit_cast(f16x8, fb.read((const bf16_t*)&smem[buf][1][0], 0, j, h));
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(bf[j], af[i], acc[i][j], 0, 0, 0);
    }
  }
  __syncthreads();
  // through LDS: row i of the tile in a row of 128 columns, 8-byte pieces permuted by the row
  f16* const out = &smem[0][0][0];
  const int lr = lane & 15, lq = lane >> 4;
  auto at = [](int row, int piece) { return row * R + ((piece ^ (row & 31)) << 2); };
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int row = wm * 64 + i * 16 + lr, piece = wn * 16 + j * 4 + lq;
      f32x4 v = acc[i][j];
      if (STAGE != 1) {                                      // the operand itself, at the same place
        const f16x4 s = *(const f16x4*)((STAGE == 2 ? a + ((int64_t)ti * R + row) * mp : x + ((int64_t)ti * R + row) * np) + tj * R + piece * 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = STAGE == 2 ? fmaf(kB, (float)s[e], kC * kBack * v[e]) : fmaf(kA, (float)s[e], kBack * v[e]);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] *= kBack;
      }
      f16x4 o;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = (f16)v[e];
      *(f16x4*)(out + at(row, piece)) = o;
    }
  __syncthreads();
  f16* const c = in_scratch(ws, STAGE == 1 ? t.a : STAGE == 2 ? t.b : t.x[from ^ 1]);
  const int ldc = STAGE == 3 ? np : mp;
  for (int s = 0; s < R * R / 4 / 256; ++s) {
    const int row = s * 8 + (tid >> 5), piece = tid & 31;
    *(f16x4*)(c + ((int64_t)ti * R + row) * ldc + tj * R + piece * 4) = *(const f16x4*)(out + at(row, piece));
  }
  if (STAGE != 3 && ti != tj) {
    for (int s = 0; s < R * R / 4 / 256; ++s) {              // the same below the diagonal
      const int col = s * 8 + (tid >> 5), row = (tid & 31) * 4;
      f16x4 o;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = out[at(row + e, col >> 2) + (col & 3)];
      *(f16x4*)(c + ((int64_t)tj * R + col) * ldc + ti * R + row) = o;
    }
  }
}

// The weights' step from the finished X.
__global__ __launch_bounds__(256) void muon_apply_kernel(const MuonMatrix* mats, const MuonTile* tiles, const char* ws, MuonHyper h, int from) {
  __shared__ f16 turn[32][kMuonTile + 2];
  const MuonTile tile = tiles[blockIdx.x];
  const MuonMatrix& t = mats[tile.matrix];
  const bool tall = t.rows > t.cols;
  const f16* x = (const f16*)(ws + t.x[from]) + (int64_t)tile.i * kMuonTile * t.np + (int64_t)tile.j * kMuonTile;
  const float step = h.rms * sqrtf((float)max(t.rows, t.cols)) * kBack;
  auto apply = [&](int64_t at, f16 v) {
    const float w = t.master[at], n = w - h.lr * fmaf(h.weight_decay, w, step * (float)v);
    t.master[at] = n;
    if (t.lowp) t.lowp[at] = f32_to_bf16(n);
  };
  const int tid = threadIdx.x, col = tid & 127, row0 = tid >> 7;
  if (!tall) {
    const int c = tile.j * kMuonTile + col;
    for (int r = row0; r < kMuonTile; r += 2) {
      const int row = tile.i * kMuonTile + r;
      if (row < t.rows && c < t.cols) apply((int64_t)row * t.cols + c, x[(int64_t)r * t.np + col]);
    }
    return;
  }
  for (int j0 = 0; j0 < kMuonTile; j0 += 32) {
    for (int i = tid >> 5; i < kMuonTile; i += 8) turn[tid & 31][i] = x[(int64_t)i * t.np + j0 + (tid & 31)];
    __syncthreads();
    const int c = tile.i * kMuonTile + col;
    for (int r = row0; r < 32; r += 2) {
      const int row = tile.j * kMuonTile + j0 + r;
      if (row < t.rows && c < t.cols) apply((int64_t)row * t.cols + c, turn[r][col]);
    }
    __syncthreads();
  }
}

void muon_update(const MuonMatrix* mats, const MuonChunk* chunks, int n_chunks, const MuonTile* tri, int n_tri, const MuonTile* full, int n_full,
                 void* workspace, const MuonHyper& h, hipStream_t st) {
  if (n_chunks < 1) return;
  char* const ws = (char*)workspace;
  hipLaunchKernelGGL(muon_momentum_kernel, dim3(n_chunks), dim3(256), 0, st, mats, chunks, ws, h);
  hipLaunchKernelGGL(muon_start_kernel, dim3(n_full), dim3(256), 0, st, mats, full, ws, h);
  int from = 0;
  for (int i = 0; i < h.iterations; ++i, from ^= 1) {
    hipLaunchKernelGGL((muon_product_kernel<1>), dim3(n_tri), dim3(256), 0, st, mats, tri, ws, from);
    hipLaunchKernelGGL((muon_product_kernel<2>), dim3(n_tri), dim3(256), 0, st, mats, tri, ws, from);
    hipLaunchKernelGGL((muon_product_kernel<3>), dim3(n_full), dim3(256), 0, st, mats, full, ws, from);
  }
  hipLaunchKernelGGL(muon_apply_kernel, dim3(n_full), dim3(256), 0, st, mats, full, ws, h, from);
}

}  // namespace mk
