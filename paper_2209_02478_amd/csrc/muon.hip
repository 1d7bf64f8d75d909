// Update of a model's matrices with an orthogonalised step (Muon), all matrices of a list in a handful of launches.
//
//   m <- mu m + g,   u = g + mu m (nesterov) or m,   X = u / (|u|_F + eps), transposed where it has more rows than columns
//   n times:  A = X X^T,  B = b A + c A A,  X <- a X + B X       (Newton-Schulz; a, b, c = 3.4445, -4.7750, 2.0315)
//   w <- w - lr (rms sqrt(max(rows, cols)) X + weight_decay w)
//
// The polynomial takes every singular value of X from (0, 1] near 1 and keeps it below 1.21, so that no element of X, A or B
// is above 1.21, 1.47 and 11.  The products' operands are therefore held in fp16 times 2^10: as many bits as any 16-bit type has
// (values from 6e-8 of the largest on keep all eleven; bf16 keeps eight, and the step is then 1 to 5 % off instead of 0.1 to
// 0.6), at the same rate of the matrix units.  That is of full rank: a rounding's part outside of X's singular directions grows 3.44-fold in an
// iteration, five of them make it 0.01 to 0.03 large there, and X of rank 64, 17 or 1 (768 x 768) is 2.3, 4.5 or 15 % off.
// Sums are fp32, the norm's fp64 (squares of gradients of 1e-20 are numbers there).
// A and A A are symmetric: only tiles on and above the diagonal are multiplied, and stored twice.  What is held of an iteration's
// factor is B = a I + b A + c A A, so that X' = B X: a X beside the product would be read again, and the error is the same
// (0.13 and 0.64 % either way for gradients of 768 x 768 from a normal distribution and with few large directions).
#include "muon_device.h"

namespace mk {

using namespace muon;

namespace {

// sum over the block's waves, in every thread; the order is fixed
template <int WAVES>
__device__ __forceinline__ double block_sum(double v, double* lds) {
#pragma unroll
  for (int s = 32; s > 0; s >>= 1) v += __shfl_xor(v, s);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0.0;
#pragma unroll
  for (int i = 0; i < WAVES; ++i) v += lds[i];
  return v;
}

// four elements of a row, which may begin at any of them
typedef float f32x4_at4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x2_at2 __attribute__((ext_vector_type(2), aligned(2)));
__device__ __forceinline__ f32x4 load_row4(const float* row, int c, int cols) {
  if (c + 4 <= cols) return *(const f32x4_at4*)(row + c);
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int e = 0; e < 3; ++e)
    if (c + e < cols) v[e] = row[c + e];
  return v;
}
// the same where rows are asked for together: no branch between the loads.  whole: the four elements exist in every lane.
// PAST: past the caches
template <bool PAST>
__device__ __forceinline__ f32x4 load_edge4(const float* row, int c, int cols, bool whole) {
  if (whole) return PAST ? __builtin_nontemporal_load((const f32x4_at4*)(row + c)) : *(const f32x4_at4*)(row + c);
  f32x4 v;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float x = row[min(c + e, cols - 1)];
    v[e] = c + e < cols ? x : 0.f;
  }
  return v;
}
__device__ __forceinline__ void store_row4(float* row, uint16_t* low, int c, int cols, const f32x4& v) {
  if (c + 4 <= cols) {
    *(f32x4_at4*)(row + c) = v;
    if (low) *(u32x2_at2*)(low + c) = u32x2_at2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
    return;
  }
#pragma unroll
  for (int e = 0; e < 3; ++e)
    if (c + e < cols) {
      row[c + e] = v[e];
      if (low) low[c + e] = f32_to_bf16(v[e]);
    }
}
// the weights' step, of four elements
__device__ __forceinline__ f32x4 stepped(const MuonHyper& h, const f32x4& w, const f32x4& x, float step) {
  f32x4 n;
#pragma unroll
  for (int e = 0; e < 4; ++e) n[e] = w[e] - h.lr * fmaf(h.weight_decay, w[e], step * x[e]);
  return n;
}
__device__ __forceinline__ f32x4 direction(const MuonHyper& h, const f32x4& g, const f32x4& m) {
  f32x4 u;
#pragma unroll
  for (int e = 0; e < 4; ++e) u[e] = h.nesterov ? fmaf(h.momentum, m[e], g[e]) : m[e];
  return u;
}
__device__ __forceinline__ float step_size(const MuonMatrix& t, const MuonHyper& h) { return h.rms * sqrtf((float)max(t.rows, t.cols)) * kBack; }

// A tile that is turned passes through LDS in pieces of four elements: piece p of row i lies at p ^ (i / 4), so that 32 lanes that
// write one piece of rows four apart, or read one row's pieces, meet all banks once.
__device__ __forceinline__ int turn_at(int row, int piece) { return row * kMuonTile + ((piece ^ ((row >> 2) & 31)) << 2); }

}  // namespace

// Momentum, and each chunk's sum of u^2.  Bound by HBM: 264 M elements in 540 us, 5.9 TB/s of the 12 bytes each; through the caches, of which
// the next kernel finds nothing again in a list as large as that, 640.
template <bool PAST>
__global__ __launch_bounds__(256) void muon_momentum_kernel(const MuonMatrix* mats, const MuonChunk* chunks, char* ws, MuonHyper h) {
  __shared__ double lds[4];
  const MuonChunk c = chunks[blockIdx.x];
  const MuonMatrix& t = mats[c.matrix];
  const int64_t chunk = t.chunk, n = min((int64_t)t.rows * t.cols - c.start, chunk);
  const float* g = t.grad + c.start;                         // chunks begin on multiples of 4, tensors on 16 bytes
  float* m = t.momentum + c.start;
  double sum = 0.0;
  auto four = [&](int64_t i, const f32x4& gv, f32x4 mv) {
#pragma unroll
    for (int e = 0; e < 4; ++e) mv[e] = fmaf(h.momentum, mv[e], gv[e]);
    if (PAST) __builtin_nontemporal_store(mv, (f32x4*)(m + i));
    else *(f32x4*)(m + i) = mv;
    const f32x4 u = direction(h, gv, mv);
#pragma unroll
    for (int e = 0; e < 4; ++e) sum += (double)u[e] * u[e];
  };
  int64_t i = 4 * threadIdx.x;
  for (; i + 3 * 1024 + 4 <= n; i += 4 * 1024) {
    f32x4 gv[4], mv[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const f32x4 *const gp = (const f32x4*)(g + i + q * 1024), *const mp = (const f32x4*)(m + i + q * 1024);
      gv[q] = PAST ? __builtin_nontemporal_load(gp) : *gp;
      mv[q] = PAST ? __builtin_nontemporal_load(mp) : *mp;
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) four(i + q * 1024, gv[q], mv[q]);
  }
  for (; i + 4 <= n; i += 1024) four(i, *(const f32x4*)(g + i), *(const f32x4*)(m + i));
  for (int64_t j = i; j < n && j < i + 4; ++j) {
    const float o = fmaf(h.momentum, m[j], g[j]), u = h.nesterov ? fmaf(h.momentum, o, g[j]) : o;
    m[j] = o;
    sum += (double)u * u;
  }
  sum = block_sum<4>(sum, lds);
  if (threadIdx.x == 0) ((double*)(ws + t.partial))[c.start / chunk] = sum;
}

// X = u / (|u| + eps), 128 x 128 of it to STRIPS blocks, zeros behind the matrix' last row and column.  A thread takes 4 x 4 elements at a
// time, eight loads in flight, and turns them in registers where X is the matrix turned.  Four strips of 32 rows where the tiles are too few
// to keep the memory busy.  Bound by HBM: 264 M elements in 511 us, 5.2 TB/s of 10 bytes each (u through the caches 540).
template <int STRIPS>
__global__ __launch_bounds__(256) void muon_start_kernel(const MuonMatrix* mats, const MuonTile* tiles, char* ws, MuonHyper h) {
  __shared__ double lds[4];
  __shared__ __attribute__((aligned(16))) f16 turn[kMuonTile * kMuonTile];
  const MuonTile tile = tiles[blockIdx.x / STRIPS];
  if (tile.matrix < 0) return;
  const MuonMatrix& t = mats[tile.matrix];
  const int rows = t.rows, cols = t.cols, np = t.np, tid = threadIdx.x;
  const int64_t n = (int64_t)rows * cols;
  const int parts = (int)((n + t.chunk - 1) / t.chunk);
  double sum = 0.0;
  for (int i = tid; i < parts; i += 256) sum += ((const double*)(ws + t.partial))[i];
  const double norm = sqrt(block_sum<4>(sum, lds)) + (double)h.eps;
  const float inv = (float)((double)kHeld / norm);           // (eps is 1e-30 or more: finite)
  const bool tall = rows > cols;
  f16* x = in_scratch(ws, t.x[0]) + (int64_t)tile.i * kMuonTile * np + (int64_t)tile.j * kMuonTile;
  const int r0 = (tall ? tile.j : tile.i) * kMuonTile, c = (tid & 31) * 4, at = (tall ? tile.i : tile.j) * kMuonTile + c;   // of u
  const float *const grad = t.grad, *const mom = t.momentum;
  const bool whole = at - c + kMuonTile <= cols;
  const int strip = blockIdx.x % STRIPS * (4 / STRIPS);        // the block's first 32 rows of four
  for (int k = strip; k < strip + 4 / STRIPS; ++k) {
    const int r = k * 32 + (tid >> 5) * 4;
    f32x4 g[4], m[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int64_t row = (int64_t)min(r0 + r + q, rows - 1) * cols;
      g[q] = load_edge4<STRIPS == 1>(grad + row, at, cols, whole);
      m[q] = load_edge4<STRIPS == 1>(mom + row, at, cols, whole);
    }
    f16 o[4][4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const f32x4 u = direction(h, g[q], m[q]);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[q][e] = r0 + r + q < rows ? (f16)(u[e] * inv) : (f16)0.f;
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if (tall) *(f16x4*)&turn[turn_at(c + q, r >> 2)] = f16x4{o[0][q], o[1][q], o[2][q], o[3][q]};
      else *(f16x4*)(x + (int64_t)(r + q) * np + c) = f16x4{o[q][0], o[q][1], o[q][2], o[q][3]};
    }
  }
  if (!tall) return;
  __syncthreads();
  constexpr int PIECES = 32 / STRIPS;                          // of four elements, of a row of X
#pragma unroll 4
  for (int k = 0; k < 16 / STRIPS; ++k) {
    const int i = k * (256 / PIECES) + tid / PIECES, piece = strip * 8 + tid % PIECES;
    *(f16x4*)(x + (int64_t)i * np + 4 * piece) = *(const f16x4*)&turn[turn_at(i, piece)];
  }
}

// STAGE 1: A = X X^T.  2: B = a I + b A + c A A.  3: X' = B X.  A block makes R x R, 128 or 64; for matrices of which larger tiles would
// be mostly padding, or too few.  R of 128: two slots of 64 reduction indices, two blocks to a compute unit; bound by the LDS, through which
// 96 KB go for 64 indices, 0.5 us of a unit with the meetings; a ring of four slots changes nothing, nor do eight waves.  R of 64: 48 KB
// for a quarter of the product, but blocks for four times as many units, and four slots, so that a load may take three rounds.  5 layers
// of 301, 77 and 999: the products take 14.4, 10.3 and 10.0 us on tiles of 128, 8.6, 6.4 and 11.5 on those of 64; one matrix of 301: a step of
// 17 launches on tiles of 64 77 us, little more than the launches by themselves.
template <int STAGE, int R>
__global__ __launch_bounds__(256, 2) void muon_product_kernel(const MuonMatrix* mats, const MuonTile* tiles, char* ws, int from) {
  using namespace large;
  constexpr int SIZE = R * BK, SLOTS = R == 64 ? 4 : 2;       // elements of an operand tile
  constexpr int N = R / 32, LOADS = R / 32;                  // blocks of 16 x 16 of a wave, and its loads of a tile
  constexpr bool KM = STAGE != 3;
  typedef LTileOf<true, R> TA;
  typedef LTileOf<KM, R> TB;
  __shared__ __attribute__((aligned(1024))) f16 smem[SLOTS * 2 * SIZE];   // [slot][A, B]
  const MuonTile tile = tiles[blockIdx.x];
  if (tile.matrix < 0) return;
  const MuonMatrix& t = mats[tile.matrix];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave >> 1, wn = wave & 1;
  const int mp = __builtin_amdgcn_readfirstlane(t.mp), np = __builtin_amdgcn_readfirstlane(t.np);
  const int ti = __builtin_amdgcn_readfirstlane(tile.i), tj = __builtin_amdgcn_readfirstlane(tile.j);
  const f16 *x = in_scratch(ws, t.x[from]), *a = in_scratch(ws, t.a), *b = in_scratch(ws, t.b);
  // (zeros behind the last index need no product)
  const int lda = STAGE == 1 ? np : mp, ldb = STAGE == 2 ? mp : np;
  const int K = __builtin_amdgcn_readfirstlane(STAGE == 1 ? max(t.rows, t.cols) : min(t.rows, t.cols));
  const f16* pa = (STAGE == 1 ? x : STAGE == 2 ? a : b) + (int64_t)ti * R * lda;
  const f16* pb = STAGE == 3 ? x + tj * R : (STAGE == 1 ? x : a) + (int64_t)tj * R * ldb;
  uint64_t base_a, base_b;
  uint32_t bytes_a, bytes_b, off_a[LOADS], off_b[LOADS];
  l_descriptor(pa, TA::bytes(lda, R), base_a, bytes_a);
  l_descriptor(pb, TB::bytes(ldb, R), base_b, bytes_b);      // (columns of X: no bound, every row is whole)
#pragma unroll
  for (int j = 0; j < LOADS; ++j) {
    off_a[j] = TA::src(lda, R, wave * LOADS + j, lane);
    off_b[j] = TB::src(ldb, R, wave * LOADS + j, lane);
  }
  const uint64_t step_a = BK * 2, step_b = KM ? BK * 2 : (uint64_t)BK * 2 * ldb;
  const uint32_t lds = l_lds_address(smem) + (uint32_t)wave * (LOADS * 1024u);
  const int steps = (K + BK - 1) / BK;
  auto fetch = [&](int slot) {
    const uint32_t to = lds + (uint32_t)slot * (4u * SIZE);
#pragma unroll
    for (int j = 0; j < LOADS; ++j) l_direct_load(base_a, bytes_a, off_a[j], to + j * 1024u);
#pragma unroll
    for (int j = 0; j < LOADS; ++j) l_direct_load(base_b, bytes_b, off_b[j], to + 2u * SIZE + j * 1024u);
    base_a += step_a;
    base_b += step_b;
  };
  TA fa;
  TB fb;
  fa.init(wm * N, lane);
  fb.init(wn * N, lane);
  f32x4 acc[N][N];
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int j = 0; j < N; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int k = 0; k < SLOTS - 1 && k < steps; ++k) fetch(k);
  for (int k = 0; k < steps; ++k) {
    if (SLOTS == 4 && k + 2 < steps) __builtin_amdgcn_s_waitcnt(in_flight(4 * LOADS));
    else if (SLOTS == 4 && k + 1 < steps) __builtin_amdgcn_s_waitcnt(in_flight(2 * LOADS));
    else __builtin_amdgcn_s_waitcnt(in_flight(0));
    __syncthreads();                                         // (every wave is done reading the slot that is filled next)
    if (k + SLOTS - 1 < steps) fetch(k + SLOTS - 1 & SLOTS - 1);
    const bf16_t* const sa = (const bf16_t*)(smem + (k & SLOTS - 1) * 2 * SIZE);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      f16x8 af[N], bf[N];
#pragma unroll
      for (int i = 0; i < N; ++i) af[i] = __builtin_bit_cast(f16x8, fa.read(sa, 0, i, h));
#pragma unroll
      for (int j = 0; j < N; ++j) bf[j] = __builtin_bit_cast(f16x8, fb.read(sa + SIZE, 0, j, h));
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(bf[j], af[i], acc[i][j], 0, 0, 0);
    }
  }
  __syncthreads();
  // through LDS: row i of the tile in a row of R columns, 8-byte pieces permuted by the row
  f16* const out = smem;
  const int lr = lane & 15, lq = lane >> 4;
  auto at = [](int row, int piece) { return row * R + ((piece ^ (row & R / 4 - 1)) << 2); };
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int row = wm * (R / 2) + i * 16 + lr, piece = wn * (R / 8) + j * 4 + lq;
      f32x4 v = acc[i][j];
      if (STAGE == 2) {
        const f16x4 s = *(const f16x4*)(a + ((int64_t)ti * R + row) * mp + tj * R + piece * 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = fmaf(kB, (float)s[e], kC * kBack * v[e]) + (ti == tj && row == piece * 4 + e ? kA * kHeld : 0.f);
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
#pragma unroll 4
  for (int s = 0; s < R * R / 4 / 256; ++s) {
    const int row = s * (1024 / R) + tid / (R / 4), piece = tid % (R / 4);
    *(f16x4*)(c + ((int64_t)ti * R + row) * ldc + tj * R + piece * 4) = *(const f16x4*)(out + at(row, piece));
  }
  if (STAGE != 3 && ti != tj) {
#pragma unroll 4
    for (int s = 0; s < R * R / 4 / 256; ++s) {              // the same below the diagonal
      const int col = s * (1024 / R) + tid / (R / 4), row = tid % (R / 4) * 4;
      f16x4 o;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = out[at(row + e, col >> 2) + (col & 3)];
      *(f16x4*)(c + ((int64_t)tj * R + col) * ldc + ti * R + row) = o;
    }
  }
}

// The weights' step from the finished X, in the same blocks of 4 x 4 elements as the start.  Bound by HBM: 264 M elements in 588 us,
// 5.4 TB/s of 12 bytes each (weights through the caches 645; written past them too 620).
template <int STRIPS>
__global__ __launch_bounds__(256) void muon_apply_kernel(const MuonMatrix* mats, const MuonTile* tiles, const char* ws, MuonHyper h, int from) {
  __shared__ __attribute__((aligned(16))) f16 turn[kMuonTile * kMuonTile];
  const MuonTile tile = tiles[blockIdx.x / STRIPS];
  if (tile.matrix < 0) return;
  const MuonMatrix& t = mats[tile.matrix];
  const int rows = t.rows, cols = t.cols, np = t.np, tid = threadIdx.x, c = (tid & 31) * 4;
  const bool tall = rows > cols;
  const f16* x = (const f16*)(ws + t.x[from]) + (int64_t)tile.i * kMuonTile * np + (int64_t)tile.j * kMuonTile;
  const float step = step_size(t, h);
  const int r0 = (tall ? tile.j : tile.i) * kMuonTile, at = (tall ? tile.i : tile.j) * kMuonTile + c;   // of the weights
  float* const master = t.master;
  uint16_t* const lowp = t.lowp;
  const bool whole = at - c + kMuonTile <= cols;
  const int strip = blockIdx.x % STRIPS * (4 / STRIPS);        // the block's first 32 rows of four
  if (tall) {
    constexpr int PIECES = 32 / STRIPS;                        // of four elements, of a row of X
#pragma unroll 4
    for (int k = 0; k < 16 / STRIPS; ++k) {
      const int i = k * (256 / PIECES) + tid / PIECES, piece = strip * 8 + tid % PIECES;
      *(f16x4*)&turn[turn_at(i, piece)] = *(const f16x4*)(x + (int64_t)i * np + 4 * piece);
    }
    __syncthreads();
  }
  for (int k = strip; k < strip + 4 / STRIPS; ++k) {
    const int r = k * 32 + (tid >> 5) * 4;
    f32x4 w[4];
    f16x4 s[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      w[q] = load_edge4<STRIPS == 1>(master + (int64_t)min(r0 + r + q, rows - 1) * cols, at, cols, whole);
      s[q] = tall ? *(const f16x4*)&turn[turn_at(c + q, r >> 2)] : *(const f16x4*)(x + (int64_t)(r + q) * np + c);
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      f32x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = tall ? (float)s[e][q] : (float)s[q][e];
      if (r0 + r + q >= rows) continue;
      const int64_t row = (int64_t)(r0 + r + q) * cols;
      store_row4(master + row, lowp ? lowp + row : nullptr, at, cols, stepped(h, w[q], v, step));
    }
  }
}

constexpr int kSmallThreads = 1024;
// A matrix of at most 128 x 256 (or turned) in one block: X, A and B stay in LDS, and the whole update is one launch.  Rows of X, A
// and B are 16 bytes longer than their elements, so that neither the fragments' rows nor their columns meet in a bank.  What
// the norm is taken of stays in registers until it is known, and the weights are asked for before the products.  Bound by the chain of
// 15 products and their meetings: 12 matrices of 64 x 64 to 64 x 256, 16 waves each, 22.8 us (all read again where they are used 23.1, by
// eight waves 26.9), one of 5 x 5 13.9, four of 100 x 77 37.
__global__ __launch_bounds__(kSmallThreads) void muon_small_kernel(const MuonMatrix* mats, MuonHyper h) {
  extern __shared__ __attribute__((aligned(16))) f16 s_smem[];
  constexpr int WAVES = kSmallThreads / 64;
  __shared__ double lds[WAVES];
  constexpr int PX = kMuonSmallLong + 8, PA = kMuonSmallShort + 8;
  f16 *const X = s_smem, *const A = X + kMuonSmallShort * PX, *const B = A + kMuonSmallShort * PA;
  const MuonMatrix& t = mats[blockIdx.x];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lr = lane & 15, lq = lane >> 4;
  const int rows = t.rows, cols = t.cols;
  const bool tall = rows > cols;
  const int m64 = (min(rows, cols) + 63) / 64 * 64, n64 = (max(rows, cols) + 63) / 64 * 64;   // what there is of X, with zeros behind
  // a lane takes four elements of a row, as many lanes as the row needs (a power of two), rows `apart` apart four at a time
  const int lanes = cols <= 16 ? 2 : cols <= 32 ? 3 : cols <= 64 ? 4 : cols <= 128 ? 5 : 6, apart = kSmallThreads >> lanes;
  const int c = 4 * (tid & ((1 << lanes) - 1)), mine = tid >> lanes, many = min(max(cols - c, 0), 4);
  const float *const grad = t.grad;
  float *const mom = t.momentum, *const master = t.master;
  constexpr int AGAIN = kMuonSmallShort * kMuonSmallLong / 16 / kSmallThreads;   // a lane's fours of rows, at most
  double sum = 0.0;
  f32x4 u[AGAIN][4];
#pragma unroll
  for (int a = 0; a < AGAIN; ++a) {
    const int r0 = mine + a * 4 * apart;
    if (!many || r0 >= rows) continue;
    f32x4 g[4], m[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int r = min(r0 + apart * q, rows - 1) * cols;
      g[q] = load_row4(grad + r, c, cols);
      m[q] = load_row4(mom + r, c, cols);
    }
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (r0 + apart * q < rows) {
#pragma unroll
        for (int e = 0; e < 4; ++e) m[q][e] = fmaf(h.momentum, m[q][e], g[q][e]);
        store_row4(mom + (r0 + apart * q) * cols, nullptr, c, cols, m[q]);
        u[a][q] = direction(h, g[q], m[q]);                  // (zeros behind the row)
#pragma unroll
        for (int e = 0; e < 4; ++e) sum += (double)u[a][q][e] * u[a][q][e];
      }
  }
  f32x4 w[AGAIN][4];                                         // asked for here, used behind the products
#pragma unroll
  for (int a = 0; a < AGAIN; ++a)
    if (many && mine + a * 4 * apart < rows)
#pragma unroll
      for (int q = 0; q < 4; ++q) w[a][q] = load_row4(master + min(mine + (4 * a + q) * apart, rows - 1) * cols, c, cols);
  for (int i = tid; i < m64 * PX / 8; i += kSmallThreads) ((f16x8*)X)[i] = f16x8{};
  const float inv = (float)((double)kHeld / (sqrt(block_sum<WAVES>(sum, lds)) + (double)h.eps));
#pragma unroll
  for (int a = 0; a < AGAIN; ++a)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int r = mine + (4 * a + q) * apart;
      if (r >= rows) continue;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (e < many) X[tall ? (c + e) * PX + r : r * PX + c + e] = (f16)(u[a][q][e] * inv);
    }
  __syncthreads();
  const int mt = m64 / 16, nt = n64 / 16;
  auto row_frag = [&](const f16* s, int pitch, int block, int k) { return *(const f16x8*)(s + (block * 16 + lr) * pitch + k + 8 * lq); };
  // a symmetric product of S's rows with themselves (A: of X's, K = n64; B: of A's, K = m64), tiles on and above the diagonal
  auto symmetric = [&](const f16* S, int pitch, int K, f16* to, bool second) {
    for (int q = wave; q < mt * (mt + 1) / 2; q += WAVES) {
      int i = 0, left = q;
      while (left >= mt - i) { left -= mt - i; ++i; }
      const int j = i + left;
      f32x4 acc = {0.f, 0.f, 0.f, 0.f}, odd = acc;             // (two sums: the one's product need not wait for the other's)
      for (int k = 0; k < K; k += 64) {
        acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(row_frag(S, pitch, j, k), row_frag(S, pitch, i, k), acc, 0, 0, 0);
        odd = __builtin_amdgcn_mfma_f32_16x16x32_f16(row_frag(S, pitch, j, k + 32), row_frag(S, pitch, i, k + 32), odd, 0, 0, 0);
      }
      acc += odd;
      // row 16 i + lr, columns 16 j + 4 lq .. + 3
      f16x4 o;
      f16x4 s = {};
      if (second) s = *(const f16x4*)(A + (16 * i + lr) * PA + 16 * j + 4 * lq);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float v = second ? fmaf(kB, (float)s[e], kC * kBack * acc[e]) + (i == j && lr == 4 * lq + e ? kA * kHeld : 0.f) : kBack * acc[e];
        o[e] = (f16)v;
        if (i != j) to[(16 * j + 4 * lq + e) * PA + 16 * i + lr] = o[e];
      }
      *(f16x4*)(to + (16 * i + lr) * PA + 16 * j + 4 * lq) = o;
    }
  };
  for (int it = 0; it < h.iterations; ++it) {
    symmetric(X, PX, n64, A, false);
    __syncthreads();
    symmetric(A, PA, m64, B, true);
    __syncthreads();
    // X' = B X: 16 columns of X' come from the same 16 of X, which only their wave reads and writes
    for (int j = wave; j < nt; j += WAVES) {
      f32x4 acc[kMuonSmallShort / 16];
#pragma unroll
      for (int i = 0; i < kMuonSmallShort / 16; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
      for (int k = 0; k < m64; k += 32) {
        const f16* p = X + (k + 8 * lq + (lr >> 2)) * PX + 16 * j + 4 * (lr & 3);
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_l*)p), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_l*)(p + 4 * PX));
        typedef short s16x8 __attribute__((ext_vector_type(8)));
        const f16x8 xf = __builtin_bit_cast(f16x8, (s16x8)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
        for (int i = 0; i < kMuonSmallShort / 16; ++i)
          if (i < mt) acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(xf, row_frag(B, PA, i, k), acc[i], 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < kMuonSmallShort / 16; ++i)
        if (i < mt) {
          f16x4 o;
#pragma unroll
          for (int e = 0; e < 4; ++e) o[e] = (f16)(kBack * acc[i][e]);
          *(f16x4*)(X + (16 * i + lr) * PX + 16 * j + 4 * lq) = o;
        }
    }
    __syncthreads();
  }
  const float step = step_size(t, h);
#pragma unroll
  for (int a = 0; a < AGAIN; ++a)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int r = mine + (4 * a + q) * apart;
      if (!many || r >= rows) continue;
      f32x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = (float)X[tall ? min(c + e, cols - 1) * PX + r : r * PX + c + e];
      store_row4(master + r * cols, t.lowp ? t.lowp + r * cols : nullptr, c, cols, stepped(h, w[a][q], v, step));
    }
}

void muon_update_small(const MuonMatrix* mats, int count, const MuonHyper& h, hipStream_t st) {
  if (count < 1) return;
  constexpr int LDS = (kMuonSmallShort * (kMuonSmallLong + 8) + 2 * kMuonSmallShort * (kMuonSmallShort + 8)) * 2;
  static const bool configured = [] {
    (void)hipFuncSetAttribute((const void*)muon_small_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
    return true;
  }();
  (void)configured;
  hipLaunchKernelGGL(muon_small_kernel, dim3(count), dim3(kSmallThreads), LDS, st, mats, h);
}

template <int STAGE>
static void product(const MuonMatrix* mats, const MuonUnits& u, char* ws, int from, hipStream_t st) {
  if (u.large[STAGE - 1]) muon_large_product(STAGE, mats, u.large_tiles[STAGE - 1], u.large[STAGE - 1], ws, from, st);
  const int n = STAGE == 3 ? u.n_full : u.n_tri;
  if (n < 1) return;
  const MuonTile* const list = STAGE == 3 ? u.full : u.tri;
  if (STAGE == 3 ? u.fine_full : u.fine_tri) hipLaunchKernelGGL((muon_product_kernel<STAGE, kMuonFine>), dim3(n), dim3(256), 0, st, mats, list, ws, from);
  else hipLaunchKernelGGL((muon_product_kernel<STAGE, kMuonTile>), dim3(n), dim3(256), 0, st, mats, list, ws, from);
}

void muon_update(const MuonMatrix* mats, const MuonUnits& u, void* workspace, const MuonHyper& h, hipStream_t st) {
  if (u.n_chunks < 1) return;
  char* const ws = (char*)workspace;
  // Few tiles: in strips, and through the caches, which keep what the next kernel reads.  A step with strips and without, us: 9 cells 74
  // and 90, 360 152 and 163, 720 452 and 447; past the caches and through them: 720 430 and 427, 1728 818 and 839, 5184 1960 and 2010.
  const bool few = u.n_cells < 512;
  if (few) hipLaunchKernelGGL((muon_momentum_kernel<false>), dim3(u.n_chunks), dim3(256), 0, st, mats, u.chunks, ws, h);
  else hipLaunchKernelGGL((muon_momentum_kernel<true>), dim3(u.n_chunks), dim3(256), 0, st, mats, u.chunks, ws, h);
  if (few) hipLaunchKernelGGL((muon_start_kernel<4>), dim3(4 * u.n_cells), dim3(256), 0, st, mats, u.cells, ws, h);
  else hipLaunchKernelGGL((muon_start_kernel<1>), dim3(u.n_cells), dim3(256), 0, st, mats, u.cells, ws, h);
  int from = 0;
  for (int i = 0; i < h.iterations; ++i, from ^= 1) {
    product<1>(mats, u, ws, from, st);
    product<2>(mats, u, ws, from, st);
    product<3>(mats, u, ws, from, st);
  }
  if (few) hipLaunchKernelGGL((muon_apply_kernel<4>), dim3(4 * u.n_cells), dim3(256), 0, st, mats, u.cells, ws, h, from);
  else hipLaunchKernelGGL((muon_apply_kernel<1>), dim3(u.n_cells), dim3(256), 0, st, mats, u.cells, ws, h, from);
}

}  // namespace mk
