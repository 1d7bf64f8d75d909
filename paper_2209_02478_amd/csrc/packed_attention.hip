// Fused attention over packed sequences with grouped heads, bf16, head sizes 32, 64 and 128, on the MFMA units
// (v_mfma_f32_32x32x16_bf16).
//
//   forward   s_ij = scale q_i k_j over the rows j of i's sequence (causal: j <= i),
//             lse_i = log sum_j exp(s_ij),  o_i = sum_j exp(s_ij - lse_i) v_j
//   backward  delta_i = do_i o_i,  P_ij = exp(s_ij - lse_i),  dS_ij = P_ij (do_i v_j - delta_i),
//             dq_i = scale sum_j dS_ij k_j,  dk_j = scale sum dS_ij q_i,  dv_j = sum P_ij do_i,
//             the last two over the rows i and the query heads that share the head of keys
//
// Score tiles are computed transposed, S^T = K Q^T, so that a lane's accumulator registers belong to one query (forward,
// dQ) or one key (dK/dV): softmax statistics are reductions over a lane's own registers and one exchange with lane ^ 32,
// and the probabilities, rounded to bf16 (they multiply bf16 rows: the same relative step as the other factor's; sums stay
// in fp32), are the B operand of the next product as they stand.  The operand that multiplies them is read out of LDS by the
// transposing reads, so that a tile is there once, brought by direct loads into one of two buffers while the other is
// multiplied, one barrier to a tile.
//
// MFMA 32x32x16 (A: 32 x 16, B: 16 x 32, D: 32 x 32):
//   A, B: lane holds row / column lane % 32 and reduction indices 8 * (lane / 32) .. + 7
//   D:    lane holds column lane % 32; register r holds row 8 * (r / 4) + 4 * (lane / 32) + r % 4
//
// Rows of other sequences are never read: a tile's buffer ends with the sequence, and what lies behind is zeros in LDS.
// No atomics: dQ comes from a kernel that owns query rows, dK/dV from one that owns key rows, both in a fixed order.
#include "gemm_device.h"
#include "packed_device.h"

#include <algorithm>
#include <type_traits>

namespace mk {
namespace {

constexpr int TK = 64;                 // rows of a streamed tile
constexpr int BM = 128;                // own rows of a block: 32 to a wave
constexpr float LOG2E = 1.44269504088896340736f;

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }   // -inf gives 0

// registers 8c .. 8c+7 of an accumulator as a bf16 operand
__device__ __forceinline__ bf16x8 regs_to_frag(const f32x16& v, int c) {
  uint4 u;
  u.x = pack_bf16x2(v[8 * c + 0], v[8 * c + 1]);
  u.y = pack_bf16x2(v[8 * c + 2], v[8 * c + 3]);
  u.z = pack_bf16x2(v[8 * c + 4], v[8 * c + 5]);
  u.w = pack_bf16x2(v[8 * c + 6], v[8 * c + 7]);
  return __builtin_bit_cast(bf16x8, u);
}
__device__ __forceinline__ void zero(f32x16& v) {
#pragma unroll
  for (int r = 0; r < 16; ++r) v[r] = 0.f;
}
// the value of lane ^ 32
__device__ __forceinline__ float other_half(float v) {
  const uint32_t u = __float_as_uint(v);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __uint_as_float((threadIdx.x & 32) ? r[0] : r[1]);
}

// 16-byte chunk c of a tile's row r lies at position c ^ swizzle(r), so that a plain read (16 rows, one chunk) and a
// transposing one (4 rows, 4 chunks in 32 lanes) both meet all 64 banks once: rows of 64, 128 and 256 bytes begin on
// every fourth, second and the same bank, and the rest of the row number has to move the chunk.
template <int D>
__device__ __forceinline__ int swizzle(int r) {
  return ((r >> 2) & 3) | (D == 64 ? (r & 2) << 1 : D == 128 ? (r & 3) << 2 : 0);
}

// One wave-level direct load of 4 bytes a lane, as l_direct_load.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"      // m0 is a reserved register: named as clobbered on purpose
__device__ __forceinline__ void direct_load4(uint64_t base, uint32_t bytes, uint32_t offset, uint32_t lds_byte_address) {
  const u32x4 r = {(uint32_t)base, (uint32_t)(base >> 32), bytes, 0x00020000u};                 // raw buffer
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dword %0, %1, 0 offen lds" : : "v"(offset), "s"(r), "s"(lds_byte_address) : "memory", "m0");
}
#pragma clang diagnostic pop

// A tile of ROWS rows in LDS: its direct loads by WAVES waves, and a wave's fragments of it.
template <int D, int WAVES = 4, int ROWS = TK>
struct Tile {
  static constexpr int SIZE = ROWS * D;                  // elements
  static constexpr int LOADS = SIZE / 512 / WAVES;       // 1 KB direct loads of each wave
  uint32_t from[LOADS];                            // byte offset of the lane's chunk from the tile's first row
  int plain, turned;
  __device__ __forceinline__ void init(int wave, int lane, int ld) {
    constexpr int NC = D / 8;
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      const int row = ROWS / WAVES * wave + j * (64 / NC) + lane / NC;
      from[j] = (uint32_t)(row * ld + (((lane % NC) ^ swizzle<D>(row)) << 3)) * 2u;
    }
    const int h = lane >> 5, r = lane & 31, q = 4 * h + ((lane & 15) >> 2);
    plain = r * D + ((h ^ swizzle<D>(r)) << 3);
    turned = q * D + (((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ swizzle<D>(q)) << 3) + 4 * (lane & 1);
  }
  // base, bytes: the tile's rows that exist
  __device__ __forceinline__ void load(uint64_t base, uint32_t bytes, int wave, uint32_t lds) const {
#pragma unroll
    for (int j = 0; j < LOADS; ++j) l_direct_load(base, bytes, from[j], lds + (uint32_t)(wave * LOADS + j) * 1024u);
  }
  // row 32 * block + lane % 32, columns 16 kk + 8 h .. + 7
  __device__ __forceinline__ bf16x8 row(const bf16_t* tile, int block, int kk) const {
    return *(const bf16x8*)(tile + block * 32 * D + (plain ^ (kk << 4)));
  }
  // column 32 db + lane % 32, rows base + 4 h + {0..3}, base + 8 + 4 h + {0..3} (base % 16 == 0): within 16 lanes of a
  // transposing read, lane i gets column i of the 4 x 16 block whose row k lies at the four lanes 4k ..; 8 rows on, bit 1
  // of swizzle() flips
  __device__ __forceinline__ bf16x8 column(const bf16_t* tile, int db, int base) const {
    const int at = turned ^ (db << 5);
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_l*)(tile + base * D + at));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_l*)(tile + (base + 8) * D + (at ^ 16)));
    typedef short s16x8 __attribute__((ext_vector_type(8)));
    return __builtin_bit_cast(bf16x8, (s16x8)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }
};

// The rows of an operand from one row on, tile after tile: scalar registers alone.
struct Stream {
  uint64_t base;
  uint32_t pitch;                                  // bytes of a row
  __device__ __forceinline__ void init(const bf16_t* first, int ld) { l_descriptor(first, (uint32_t)ld * 2u, base, pitch); }
  __device__ __forceinline__ uint64_t at(int row) const { return base + (uint64_t)row * pitch; }
  __device__ __forceinline__ uint32_t bytes(int rows) const { return (uint32_t)min(rows, TK) * pitch; }
};

// Every wave's LDS accesses so far are done.
__device__ __forceinline__ void meet() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
// Every wave's direct loads so far are in LDS, and every wave is done reading what it read before.
__device__ __forceinline__ void landed() {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
}

// store a transposed accumulator (rows = head columns, lane column = token) as bf16
template <int D>
__device__ __forceinline__ void store_rows(bf16_t* dst, const f32x16 (&acc)[D / 32], int h, float mul) {
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      uint2 o;
      o.x = pack_bf16x2(acc[db][4 * g] * mul, acc[db][4 * g + 1] * mul);
      o.y = pack_bf16x2(acc[db][4 * g + 2] * mul, acc[db][4 * g + 3] * mul);
      *(uint2*)(dst + 32 * db + 8 * g + 4 * h) = o;
    }
}

}  // namespace

// ------------------------------------------------------------------ forward
// 32 queries to a wave, which holds its part of Q in registers; the scores of a tile are made while the exponentials of the one before are
// taken.  With heads of 64 exponentials and their neighbours need two issue slots for each of the matrix units', with heads of 128 as many.
// 6 causal sequences of 1000-4096 rows, 16 heads of 128, 4 of keys: 215 to 227 us by card, 0.87 to 0.83 PFLOP/s of the pairs that see each
// other (scores not made ahead: 229 beside 215); 32 sequences of 153-512 without mask, 12 heads of 64: 33 to 34 us; 16 causal ones of 128-661, 16
// heads of 64, 4 of keys: 21.  Neither pipe is full: of a wave's cycles 41 % (16 sequences), 35 % (32) and 20 % (6) go by in waits for loads and
// meetings, 28, 30 and 39 % in waits for its turn to issue, 30, 35 and 41 % in instructions.  Nor is it the longest sequence's chain alone: that
// sequence by itself takes 12, 11 and 91 us.
// G groups of four waves have the same queries and every G-th tile of keys, in tiles of their own; their parts are joined at the end.
template <int D, bool CAUSAL, int G>
__global__ __launch_bounds__(256 * G, 2) void packed_fwd_kernel(PackedAttention p, int slots) {
  constexpr int KK = D / 16, DB = D / 32;
  __shared__ __attribute__((aligned(1024))) bf16_t all_tiles[G][2][2][Tile<D>::SIZE];   // [group][buffer][K, V]
  const int tid = threadIdx.x, lane = tid & 63, all = __builtin_amdgcn_readfirstlane(tid >> 6), ql = lane & 31, h = lane >> 5;
  const int g = all >> 2, wave = all & 3;
  auto& tiles = all_tiles[g];
  PackedPlace w;
  if (!packed_place<BM, CAUSAL>(p, slots, blockIdx.x, w)) return;
  const int w0 = w.row + wave * 32, qi = w0 + ql, qc = min(qi, w.n - 1);
  const float c2 = p.scale * LOG2E;                   // exp(scale * s - x) == exp2(c2 * s - LOG2E * x)

  const bf16_t* qrow = (const bf16_t*)p.q + (w.first + qc) * p.ldq + w.head * D + 8 * h;
  bf16x8 qf[KK];
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) qf[kk] = *(const bf16x8*)(qrow + 16 * kk);
  f32x16 o[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) zero(o[db]);
  float m = -INFINITY, l = 0.f;                       // running maximum of the raw (unscaled) scores, sum of exps
  const int kend = CAUSAL ? min(w.n, w.row + BM) : w.n;

  Tile<D> tk, tv;
  tk.init(wave, lane, (int)p.ldk);
  tv.init(wave, lane, (int)p.ldv);
  Stream ks, vs;
  ks.init((const bf16_t*)p.k + w.first * p.ldk + w.kv * D, (int)p.ldk);
  vs.init((const bf16_t*)p.v + w.first * p.ldv + w.kv * D, (int)p.ldv);
  const uint32_t lds = l_lds_address(&tiles[0][0][0]);
  auto fetch_k = [&](int k0, int buf) { tk.load(ks.at(k0), ks.bytes(w.n - k0), wave, lds + (uint32_t)buf * (4u * Tile<D>::SIZE)); };
  auto fetch_v = [&](int k0, int buf) { tv.load(vs.at(k0), vs.bytes(w.n - k0), wave, lds + (uint32_t)buf * (4u * Tile<D>::SIZE) + 2u * Tile<D>::SIZE); };
  f32x16 s[2];                                        // the tile's scores
  auto scores = [&](int buf, f32x16 (&to)[2]) __attribute__((always_inline)) {
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      zero(to[kb]);
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) to[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tk.row(tiles[buf][0], kb, kk), qf[kk], to[kb], 0, 0, 0);
    }
  };
  // A tile's scores are made while the exponentials of the one before are: a wave's products and its vector instructions then run side
  // by side, and not only those of the other wave on its SIMD.
  auto step = [&](int k0, int buf) __attribute__((always_inline)) {
    const bool edge = k0 + TK > w.n || (CAUSAL && k0 + TK - 1 > w0);
    if (edge) {                                       // the tile touches the mask
      const int end = (CAUSAL ? min(w.n, qi + 1) : w.n) - k0 - 4 * h;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (32 * kb + 8 * (r >> 2) + (r & 3) >= end) s[kb][r] = -INFINITY;
    }
    float mx = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[kb][r]);
    mx = fmaxf(mx, other_half(mx));
    const float mnew = fmaxf(m, mx);                  // finite: a sequence's first row is visible to all of them
    float alpha = 1.f;
    if (__any(mx > m)) {                              // else alpha is 1 in every lane: nothing to scale
      alpha = fast_exp2((m - mnew) * c2);
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[db][r] *= alpha;
      m = mnew;
    }
    f32x16 next[2];
    scores(buf ^ 1, next);                            // (behind the last tile: of whatever is there, unused)
    const float off = -mnew * c2;
    float rs = 0.f;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float e = fast_exp2(fmaf(s[kb][r], c2, off));
        s[kb][r] = e;
        rs += e;
      }
    rs += other_half(rs);
    l = fmaf(l, alpha, rs);
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const bf16x8 pf = regs_to_frag(s[kb], c);
#pragma unroll
        for (int db = 0; db < DB; ++db)
          o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tv.column(tiles[buf][1], db, 32 * kb + 16 * c), pf, o[db], 0, 0, 0);
      }
    s[0] = next[0];
    s[1] = next[1];
  };
  constexpr int NEXT = G * TK;                        // from a tile of the group to its next one
  int k0 = g * TK, buf = 0;
  if (k0 < kend) {
    fetch_k(k0, 0);
    fetch_v(k0, 0);
  }
  if (k0 + NEXT < kend) fetch_k(k0 + NEXT, 1);
  landed();
  if (w0 < w.n) scores(0, s);                         // (of a group without a tile: unused)
  meet();                                             // the first tile of K is used up
  // the tiles that this wave's queries see, then those that only other waves' do, as many turns for each group
  const int seen = w0 >= w.n ? 0 : CAUSAL ? min(kend, w0 + 32) : kend;
  const int turns = (kend + NEXT - 1) / NEXT;
  int done = 0;
  auto turn = [&]() __attribute__((always_inline)) {
    if (done > 0) landed();
    if (k0 + 2 * NEXT < kend) fetch_k(k0 + 2 * NEXT, buf);
    if (k0 + NEXT < kend) fetch_v(k0 + NEXT, buf ^ 1);
  };
  for (; k0 < seen; k0 += NEXT, buf ^= 1, ++done) {
    turn();
    step(k0, buf);
  }
  for (; done < turns; k0 += NEXT, buf ^= 1, ++done) turn();
  if constexpr (G == 2) {                             // the other group's part
    float* const part = (float*)&all_tiles[0] + (wave * (16 * DB + 2)) * 64 + lane;
    static_assert((16 * DB + 2) * 4 * 64 * sizeof(float) <= sizeof(all_tiles));
    __syncthreads();
    if (g == 1) {
#pragma unroll
      for (int i = 0; i < 16 * DB; ++i) part[i * 64] = o[i / 16][i & 15];
      part[16 * DB * 64] = m;
      part[(16 * DB + 1) * 64] = l;
    }
    __syncthreads();
    if (g == 1) return;
    const float m1 = part[16 * DB * 64], top = fmaxf(m, m1), f0 = fast_exp2((m - top) * c2), f1 = fast_exp2((m1 - top) * c2);
#pragma unroll
    for (int i = 0; i < 16 * DB; ++i) o[i / 16][i & 15] = fmaf(part[i * 64], f1, o[i / 16][i & 15] * f0);
    l = fmaf(part[(16 * DB + 1) * 64], f1, l * f0);
    m = top;
  }
  if (qi < w.n) {
    store_rows<D>((bf16_t*)p.out + (w.first + qi) * p.ldo + w.head * D, o, h, 1.f / l);
    if (h == 0) p.lse[(int64_t)w.head * p.T + w.first + qi] = m * p.scale + __logf(l);
  }
}

// ------------------------------------------------------------------ dQ
// 32 queries to a wave, as in the forward pass; three products of a tile.  6 causal sequences of 1000-4096 rows, 16 heads of 128: 272 to
// 320 us (the clock falls under it), 1.03 to 0.88 PFLOP/s, the matrix units 49 % busy; 16 of 128-661, heads of 64: 24.8 us.  Two loops, whole tiles
// and those at the mask's edge, gain less than 1 %.
// smem: [buffer][K, V].  TELL: delta is written out for the keys' gradients, which are made after.
template <int D, bool CAUSAL, bool TELL>
__device__ __forceinline__ void bwd_dq(const PackedAttention& p, int slots, int block, bf16_t* smem) {
  constexpr int KK = D / 16, DB = D / 32, SIZE = Tile<D>::SIZE;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), ql = lane & 31, h = lane >> 5;
  PackedPlace w;
  if (!packed_place<BM, CAUSAL>(p, slots, block, w)) return;
  const int w0 = w.row + wave * 32, qi = w0 + ql, qc = min(qi, w.n - 1);
  const float c2 = p.scale * LOG2E;

  // delta: each half of the wave holds half of the head's columns
  bf16x8 qf[KK], gf[KK];
  float delta = 0.f;
  {
    const int64_t r = w.first + qc;
    const bf16_t* qrow = (const bf16_t*)p.q + r * p.ldq + w.head * D + 8 * h;
    const bf16_t* grow = (const bf16_t*)p.dout + r * p.lddo + w.head * D + 8 * h;
    const bf16_t* orow = (const bf16_t*)p.out + r * p.ldo + w.head * D + 8 * h;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      qf[kk] = *(const bf16x8*)(qrow + 16 * kk);
      gf[kk] = *(const bf16x8*)(grow + 16 * kk);
      const bf16x8 of = *(const bf16x8*)(orow + 16 * kk);
#pragma unroll
      for (int e = 0; e < 8; ++e) delta = fmaf((float)of[e], (float)gf[kk][e], delta);
    }
  }
  delta += other_half(delta);
  const int64_t stat = (int64_t)w.head * p.T + w.first;
  if (TELL && h == 0 && qi < w.n) p.delta[stat + qi] = delta;
  const float nlse = -LOG2E * p.lse[stat + qc];
  f32x16 dq[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) zero(dq[db]);
  const int kend = CAUSAL ? min(w.n, w.row + BM) : w.n;

  Tile<D> tk, tv;
  tk.init(wave, lane, (int)p.ldk);
  tv.init(wave, lane, (int)p.ldv);
  Stream ks, vs;
  ks.init((const bf16_t*)p.k + w.first * p.ldk + w.kv * D, (int)p.ldk);
  vs.init((const bf16_t*)p.v + w.first * p.ldv + w.kv * D, (int)p.ldv);
  const uint32_t lds = l_lds_address(smem);
  auto fetch = [&](int k0, int buf) {
    tk.load(ks.at(k0), ks.bytes(w.n - k0), wave, lds + (uint32_t)buf * (4u * SIZE));
    tv.load(vs.at(k0), vs.bytes(w.n - k0), wave, lds + (uint32_t)buf * (4u * SIZE) + 2u * SIZE);
  };
  auto step = [&](int k0, int buf) __attribute__((always_inline)) {
    const bool edge = k0 + TK > w.n || (CAUSAL && k0 + TK - 1 > w0);
    const bf16_t *Ks = smem + buf * 2 * SIZE, *Vs = Ks + SIZE;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      f32x16 s, dp;
      zero(s); zero(dp);
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tk.row(Ks, kb, kk), qf[kk], s, 0, 0, 0);
        dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tv.row(Vs, kb, kk), gf[kk], dp, 0, 0, 0);
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = fast_exp2(fmaf(s[r], c2, nlse)) * (dp[r] - delta);
      if (edge) {
        const int end = (CAUSAL ? min(w.n, qi + 1) : w.n) - k0 - 32 * kb - 4 * h;
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (8 * (r >> 2) + (r & 3) >= end) s[r] = 0.f;
      }
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const bf16x8 dsf = regs_to_frag(s, c);
#pragma unroll
        for (int db = 0; db < DB; ++db)
          dq[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tk.column(Ks, db, 32 * kb + 16 * c), dsf, dq[db], 0, 0, 0);
      }
    }
  };
  fetch(0, 0);
  for (int k0 = 0, buf = 0; k0 < kend; k0 += TK, buf ^= 1) {
    landed();
    if (k0 + TK < kend) fetch(k0 + TK, buf ^ 1);
    if (w0 < w.n && !(CAUSAL && k0 > w0 + 31)) step(k0, buf);   // else none of this wave's queries sees the tile
  }
  if (qi < w.n) store_rows<D>((bf16_t*)p.dq + (w.first + qi) * p.lddq + w.head * D, dq, h, p.scale);
}
template <int D, bool CAUSAL>
__global__ __launch_bounds__(256, 2) void packed_bwd_dq_kernel(PackedAttention p, int slots) {
  __shared__ __attribute__((aligned(1024))) bf16_t tiles[4 * Tile<D>::SIZE];
  bwd_dq<D, CAUSAL, true>(p, slots, blockIdx.x, tiles);
}

// ------------------------------------------------------------------ dK, dV
// A block takes its keys through the query rows of every head that shares them.  G groups of KW waves, 32 keys to a wave: each
// group has the same keys and every G-th tile of those rows, in tiles of its own, and their sums are added at the end in the groups' order.
// 16 causal sequences of 128-661 rows, 16 heads of 64, 4 of keys: 32.4 us, the matrix units 25 % busy: bound by a tile's chain of steps.
// smem: [group][buffer][Q, dO], and behind it lse and delta of the tiles' rows.  TOLD: delta is there; else the block makes it of dO and O.
template <int D, int G> constexpr int dkv_elements() { return G * 4 * TK * D + G * 2 * 2 * TK * 2; }
template <int D, bool CAUSAL, int KW, int G, bool TOLD>
__device__ __forceinline__ void bwd_dkv(const PackedAttention& p, int slots, int block, bf16_t* smem) {
  constexpr int KK = D / 16, DB = D / 32, BN = 32 * KW;
  typedef Tile<D, KW> T;
  const int tid = threadIdx.x, lane = tid & 63, all = __builtin_amdgcn_readfirstlane(tid >> 6), kl = lane & 31, h = lane >> 5;
  const int g = all / KW, wave = all - g * KW;
  PackedPlace w;
  if (!packed_place_kv<BN, CAUSAL>(p, slots, block, w)) return;
  bf16_t* const tiles = smem + g * (4 * T::SIZE);
  float *const lse_s = (float*)(smem + G * 4 * T::SIZE) + g * (4 * TK), *const delta_s = lse_s + 2 * TK;   // [buffer][row]
  const int w0 = w.row + wave * 32, ki = w0 + kl, kc = min(ki, w.n - 1);
  const float c2 = p.scale * LOG2E;

  bf16x8 kf[KK], vf[KK];
  {
    const bf16_t* krow = (const bf16_t*)p.k + (w.first + kc) * p.ldk + w.kv * D + 8 * h;
    const bf16_t* vrow = (const bf16_t*)p.v + (w.first + kc) * p.ldv + w.kv * D + 8 * h;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      kf[kk] = *(const bf16x8*)(krow + 16 * kk);
      vf[kk] = *(const bf16x8*)(vrow + 16 * kk);
    }
  }
  f32x16 dk[DB], dv[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) { zero(dk[db]); zero(dv[db]); }
  const int qstart = CAUSAL ? w.row / TK * TK : 0;    // earlier queries never see these keys
  const int group = p.n_heads / p.n_kv_heads, per_head = (w.n - qstart + TK - 1) / TK, steps = (per_head * group + G - 1) / G;

  T tq, tg;
  tq.init(wave, lane, (int)p.ldq);
  tg.init(wave, lane, (int)p.lddo);
  Stream qs, gs;
  qs.init((const bf16_t*)p.q + w.first * p.ldq + w.kv * group * D, (int)p.ldq);
  gs.init((const bf16_t*)p.dout + w.first * p.lddo + w.kv * group * D, (int)p.lddo);
  const uint32_t lds = l_lds_address(tiles);
  const int64_t stats = (int64_t)w.kv * group * p.T + w.first;
  const int mine = tid - g * (64 * KW);               // thread of the group
  float pre_lse = 0.f, pre_delta = 0.f;
  int head = 0, q0 = qstart + g * TK;                 // the tile to fetch
  auto settle = [&]() {
    while (q0 >= w.n && head < group) { q0 -= per_head * TK; ++head; }
  };
  auto fetch = [&](int buf) {                         // behind the last head: nothing
    if (head < group) {
      const uint64_t at = (uint64_t)head * (D * 2u);
      tq.load(qs.at(q0) + at, qs.bytes(w.n - q0), wave, lds + (uint32_t)buf * (4u * T::SIZE));
      tg.load(gs.at(q0) + at, gs.bytes(w.n - q0), wave, lds + (uint32_t)buf * (4u * T::SIZE) + 2u * T::SIZE);
      if (TOLD) {
        if (mine < TK) {
          const int64_t q = stats + (int64_t)head * p.T + min(q0 + mine, w.n - 1);
          pre_lse = p.lse[q];
          pre_delta = p.delta[q];
        }
      } else {                                        // KW threads to a row
        const int64_t q = min(q0 + mine / KW, w.n - 1);
        const int column = (w.kv * group + head) * D + mine % KW * (D / KW);
        const bf16_t* grow = (const bf16_t*)p.dout + (w.first + q) * p.lddo + column;
        const bf16_t* orow = (const bf16_t*)p.out + (w.first + q) * p.ldo + column;
        pre_lse = p.lse[stats + (int64_t)head * p.T + q];
        pre_delta = 0.f;
#pragma unroll
        for (int i = 0; i < D / KW / 8; ++i) {
          const bf16x8 gv = *(const bf16x8*)(grow + 8 * i), ov = *(const bf16x8*)(orow + 8 * i);
#pragma unroll
          for (int e = 0; e < 8; ++e) pre_delta = fmaf((float)ov[e], (float)gv[e], pre_delta);
        }
#pragma unroll
        for (int s = 1; s < KW; s <<= 1) pre_delta += __shfl_xor(pre_delta, s);
      }
    }
  };
  auto step = [&](int at, int buf) __attribute__((always_inline)) {   // at: the tile's first row
    const bf16_t *Qs = tiles + buf * 2 * T::SIZE, *Gs = Qs + T::SIZE;
#pragma unroll
    for (int qb = 0; qb < 2; ++qb) {
      f32x16 s, dp;
      zero(s); zero(dp);
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tq.row(Qs, qb, kk), kf[kk], s, 0, 0, 0);
        dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tg.row(Gs, qb, kk), vf[kk], dp, 0, 0, 0);
      }
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) {
        const int qq = 32 * qb + 8 * q4 + 4 * h;
        const float4 nl = *(const float4*)&lse_s[buf * TK + qq], dl = *(const float4*)&delta_s[buf * TK + qq];
        const float nls[4] = {nl.x, nl.y, nl.z, nl.w}, dls[4] = {dl.x, dl.y, dl.z, dl.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = 4 * q4 + e;
          const float pr = fast_exp2(fmaf(s[r], c2, nls[e]));
          s[r] = pr;
          dp[r] = pr * (dp[r] - dls[e]);
        }
      }
      if (CAUSAL && at < w0 + 31) {                   // the tile touches the mask
        const int first = ki - at - 32 * qb - 4 * h;
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (8 * (r >> 2) + (r & 3) < first) { s[r] = 0.f; dp[r] = 0.f; }
      }
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const bf16x8 pf = regs_to_frag(s, c), dsf = regs_to_frag(dp, c);
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          dv[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tg.column(Gs, db, 32 * qb + 16 * c), pf, dv[db], 0, 0, 0);
          dk[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tq.column(Qs, db, 32 * qb + 16 * c), dsf, dk[db], 0, 0, 0);
        }
      }
    }
  };
  settle();
  fetch(0);
  for (int turn = 0, buf = 0; turn < steps; ++turn, buf ^= 1) {
    const bool some = head < group && w0 < w.n;
    const int at = q0;
    // lse_s: ready for exp2, and minus infinity behind the sequence: probabilities of zero there.  This buffer was last
    // read two tiles ago, before the last barrier.
    const int r = TOLD ? mine : mine / KW;
    if (r < TK && (TOLD || mine % KW == 0)) { lse_s[buf * TK + r] = at + r < w.n ? -LOG2E * pre_lse : -INFINITY; delta_s[buf * TK + r] = pre_delta; }
    landed();
    q0 += G * TK;
    settle();
    fetch(buf ^ 1);
    if (some && !(CAUSAL && at + TK <= w0)) step(at, buf);   // else no query of the tile sees this wave's keys
  }
  bf16_t* const dk_row = (bf16_t*)p.dk + (w.first + ki) * p.lddk + w.kv * D;
  bf16_t* const dv_row = (bf16_t*)p.dv + (w.first + ki) * p.lddv + w.kv * D;
  if (G == 1) {
    if (ki < w.n) {
      store_rows<D>(dk_row, dk, h, p.scale);
      store_rows<D>(dv_row, dv, h, 1.f);
    }
    return;
  }
  // Four registers at a time are a part: rows 8 (part % 4) + 4 h .. of 32 head columns.  Group g adds all groups' parts
  // of its share of them.
  constexpr int PARTS = 8 * DB, SHARE = PARTS / G;
  float4* const parts = (float4*)smem;  // [group][wave][part][lane], as large as the tiles
  __syncthreads();
#pragma unroll
  for (int i = 0; i < PARTS; ++i) {
    const f32x16& v = i < PARTS / 2 ? dk[i / 4] : dv[i / 4 - DB];
    parts[((g * KW + wave) * PARTS + i) * 64 + lane] = make_float4(v[4 * (i & 3)], v[4 * (i & 3) + 1], v[4 * (i & 3) + 2], v[4 * (i & 3) + 3]);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < SHARE; ++i) {
    const int part = g * SHARE + i;
    float4 s = parts[(wave * PARTS + part) * 64 + lane];
#pragma unroll
    for (int o = 1; o < G; ++o) {
      const float4 v = parts[((o * KW + wave) * PARTS + part) * 64 + lane];
      s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
    }
    const bool keys = part < PARTS / 2;
    const float mul = keys ? p.scale : 1.f;
    const int column = (part % (PARTS / 2)) / 4 * 32 + 8 * (part & 3) + 4 * h;
    if (ki < w.n) *(uint2*)((keys ? dk_row : dv_row) + column) = make_uint2(pack_bf16x2(s.x * mul, s.y * mul), pack_bf16x2(s.z * mul, s.w * mul));
  }
}
template <int D, bool CAUSAL, int KW, int G>
__global__ __launch_bounds__(64 * KW * G, KW * G == 4 ? 2 : 1) void packed_bwd_dkv_kernel(PackedAttention p, int slots) {
  __shared__ __attribute__((aligned(1024))) bf16_t smem[dkv_elements<D, G>()];
  bwd_dkv<D, CAUSAL, KW, G, true>(p, slots, blockIdx.x, smem);
}

// Both in one launch, for few rows: the first `queries` blocks make dQ, the others dK and dV with a delta of their own.
template <int D, bool CAUSAL>
__global__ __launch_bounds__(256) void packed_bwd_small_kernel(PackedAttention p, int slots, int slots_kv, int queries) {
  extern __shared__ __attribute__((aligned(1024))) bf16_t small_smem[];
  if ((int)blockIdx.x < queries) bwd_dq<D, CAUSAL, false>(p, slots, blockIdx.x, small_smem);
  else bwd_dkv<D, CAUSAL, 2, 2, false>(p, slots_kv, blockIdx.x - queries, small_smem);
}

// Heads of 128: a wave with both gradients of 32 keys would need more registers than let two waves run on a SIMD.  So a pair of waves
// has the same 32 keys: the first makes S and P and holds dV, the second makes dP and dS and holds dK.  P passes from the one to the other
// through LDS in fp32, and the second works a tile of 32 rows behind the first, so that they meet once for each tile.  Each makes its
// product S or dP a tile ahead, so that the matrix units have it while the exponentials or differences of this one are taken.
// Bound by the chain of a tile's steps in the block of the longest sequence's first keys: 64 keys to a block, not 128, halve what that
// block has to do alone.  6 causal sequences of 1000-4096 rows, 16 heads, 4 of keys, the median of six runs (the fastest): 577 us (457);
// blocks of 64 keys without the products ahead 595 (491), of 128 keys 605 (522), of 128 with both waves on the same tile and a second
// barrier in it 645 (577), both gradients in one wave, one wave on a SIMD, 860.
template <bool CAUSAL>
__global__ __launch_bounds__(256, 2) void packed_bwd_dkv_pair_kernel(PackedAttention p, int slots) {
  constexpr int D = 128, KK = D / 16, DB = D / 32, BN = 64, ROWS = 32;
  typedef Tile<D, 4, ROWS> T;
  __shared__ __attribute__((aligned(1024))) bf16_t q_tiles[4][T::SIZE], g_tiles[2][T::SIZE];     // of Q and dO: [tile % 4], [tile % 2]
  __shared__ __attribute__((aligned(16))) float4 passed[2][2][4][64];            // P: [tile % 2][keys' wave][registers / 4][lane]
  __shared__ __attribute__((aligned(256))) float stat[4][2][64];                 // [tile % 4][lse, delta][row]
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), kl = lane & 31, h = lane >> 5;
  const int kw = wave & 1;
  const bool values = wave < 2;                       // holds dV
  PackedPlace w;
  if (!packed_place_kv<BN, CAUSAL>(p, slots, blockIdx.x, w)) return;
  const int w0 = w.row + kw * 32, ki = w0 + kl, kc = min(ki, w.n - 1);
  const float c2 = p.scale * LOG2E;

  bf16x8 own[KK];                                     // the keys' rows of K, or of V
  {
    const bf16_t* row = values ? (const bf16_t*)p.k + (w.first + kc) * p.ldk : (const bf16_t*)p.v + (w.first + kc) * p.ldv;
    row += w.kv * D + 8 * h;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) own[kk] = *(const bf16x8*)(row + 16 * kk);
  }
  f32x16 acc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) zero(acc[db]);
  const int qstart = CAUSAL ? w.row : 0;              // earlier queries never see these keys (a multiple of ROWS)
  const int group = p.n_heads / p.n_kv_heads, per_head = (w.n - qstart + ROWS - 1) / ROWS, count = per_head * group;

  T tq, tg;
  tq.init(wave, lane, (int)p.ldq);
  tg.init(wave, lane, (int)p.lddo);
  Stream qs, gs;
  qs.init((const bf16_t*)p.q + w.first * p.ldq + w.kv * group * D, (int)p.ldq);
  gs.init((const bf16_t*)p.dout + w.first * p.lddo + w.kv * group * D, (int)p.lddo);
  uint64_t stat_base;
  uint32_t stat_pitch;                                // bytes from a head's lse, or delta, to the next one's
  l_descriptor((values ? p.lse : p.delta) + (int64_t)w.kv * group * p.T + w.first, (uint32_t)p.T * 4u, stat_base, stat_pitch);
  const uint32_t lds_q = l_lds_address(&q_tiles[0][0]), lds_g = l_lds_address(&g_tiles[0][0]), lds_stat = l_lds_address(&stat[0][0][0]);
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) asm volatile("" : "+v"(own[kk]));     // waited for here: in the loop it would be a wait for every load
  // the tiles of all heads that share these keys, one head after the other.  Behind a sequence's last row and behind the last tile
  // everything is zeros: P is one there, and multiplies dO, or dP - delta, of zero.
  struct At { int head, row; };
  At ahead = {0, qstart}, next = ahead;               // of the next tiles to fetch, of Q and of the rest
  auto fetch_q = [&](int tile) {
    const int left = ahead.head < group ? w.n - ahead.row : 0;
    tq.load(qs.at(ahead.row) + (uint64_t)ahead.head * (D * 2u), qs.bytes(left), wave, lds_q + (uint32_t)(tile & 3) * (2u * T::SIZE));
    ahead.row += ROWS;
    if (ahead.row >= w.n) { ahead.row = qstart; ++ahead.head; }
  };
  auto fetch = [&](int tile) {                        // this tile of dO and of lse or delta, and the one after it of Q
    const int left = next.head < group ? w.n - next.row : 0;
    tg.load(gs.at(next.row) + (uint64_t)next.head * (D * 2u), gs.bytes(left), wave, lds_g + (uint32_t)(tile & 1) * (2u * T::SIZE));
    // (each of a role's waves: the same numbers to the same place)
    direct_load4(stat_base + (uint64_t)next.head * stat_pitch + (uint64_t)next.row * 4u, (uint32_t)left * 4u, (uint32_t)lane * 4u,
                 lds_stat + (uint32_t)(tile & 3) * 512u + (values ? 0u : 256u));
    next = ahead;
    fetch_q(tile + 1);
  };
  auto turn = [&](int tile) {                         // what was fetched has landed, and every wave is done with the tile before
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    fetch(tile + 1);
  };
  auto product = [&](const T& t, const bf16_t* rows) {
    f32x16 s;
    zero(s);
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(t.row(rows, 0, kk), own[kk], s, 0, 0, 0);
    return s;
  };
  auto add = [&](const T& t, const bf16_t* rows, const f32x16& s) {
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const bf16x8 f = regs_to_frag(s, c);
#pragma unroll
      for (int db = 0; db < DB; ++db) acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(t.column(rows, db, 16 * c), f, acc[db], 0, 0, 0);
    }
  };
  fetch_q(0);
  fetch(0);
  turn(0);
  if (values) {
    f32x16 s = product(tq, q_tiles[0]);
    int at = qstart, tile = 0;                        // the tile's first row
    do {
      const f32x16 following = product(tq, q_tiles[(tile + 1) & 3]);
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) {
        const float4 z = *(const float4*)&stat[tile & 3][0][8 * q4 + 4 * h];
        s[4 * q4] = fast_exp2(fmaf(s[4 * q4], c2, -LOG2E * z.x));
        s[4 * q4 + 1] = fast_exp2(fmaf(s[4 * q4 + 1], c2, -LOG2E * z.y));
        s[4 * q4 + 2] = fast_exp2(fmaf(s[4 * q4 + 2], c2, -LOG2E * z.z));
        s[4 * q4 + 3] = fast_exp2(fmaf(s[4 * q4 + 3], c2, -LOG2E * z.w));
      }
      if (CAUSAL && at < w0 + 31) {                   // the tile touches the mask, or lies behind it
        const int from = ki - at - 4 * h;
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (8 * (r >> 2) + (r & 3) < from) s[r] = 0.f;
      }
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4)
        passed[tile & 1][kw][q4][lane] = make_float4(s[4 * q4], s[4 * q4 + 1], s[4 * q4 + 2], s[4 * q4 + 3]);
      add(tg, g_tiles[tile & 1], s);
      s = following;
      at += ROWS;
      if (at >= w.n) at = qstart;
      turn(++tile);
    } while (tile < count);
  } else {
    f32x16 s = product(tg, g_tiles[0]);
    int tile = 0;
    do {
      turn(++tile);
      const f32x16 following = product(tg, g_tiles[tile & 1]);
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) {
        const float4 pr = passed[(tile - 1) & 1][kw][q4][lane], z = *(const float4*)&stat[(tile - 1) & 3][1][8 * q4 + 4 * h];
        s[4 * q4] = pr.x * (s[4 * q4] - z.x);
        s[4 * q4 + 1] = pr.y * (s[4 * q4 + 1] - z.y);
        s[4 * q4 + 2] = pr.z * (s[4 * q4 + 2] - z.z);
        s[4 * q4 + 3] = pr.w * (s[4 * q4 + 3] - z.w);
      }
      add(tq, q_tiles[(tile - 1) & 3], s);
      s = following;
    } while (tile < count);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");    // no direct load may land in LDS that is another block's by then
  if (ki < w.n) {
    if (values) store_rows<D>((bf16_t*)p.dv + (w.first + ki) * p.lddv + w.kv * D, acc, h, 1.f);
    else store_rows<D>((bf16_t*)p.dk + (w.first + ki) * p.lddk + w.kv * D, acc, h, p.scale);
  }
}

namespace {
template <int D>
void launch_fwd(const PackedAttention& p, int causal, hipStream_t st) {
  const int slots = packed_slots(p.T, p.n_seq, BM);
  const dim3 grid(packed_blocks(slots, p.n_kv_heads, p.n_heads / p.n_kv_heads));
  // Few blocks of long rows: two groups of waves to the same queries.  One and two, us, sequences x rows, query heads (blocks), heads of 64:
  // behind a mask 1x1024, 12 (108) 19.3 and 17.0, 2x2048, 12 (408) 34.0 and 28.9, 16 (544) 35.5 and 34.4, 8x512, 12 (480) 14.4 and 17.6, 2 (80)
  // 12.6 and 12.1, 2x256, 2 (12) 9.0 and 9.4; without 1x1024, 16 (144) 19.3 and 17.2, 2x2048, 12 46.9 and 50.1; heads of 128: 1x1024 26.9 and 25.2.
  // The rows of a sequence are taken to be T / n_seq, since lengths are the device's: of one long sequence among short ones this keeps one
  // group where two would be faster (4 heads of 64, 4096 beside 15 of 16 rows 54 and 43, 1024 beside 15 17.8 and 15.7).
  if (grid.x <= (causal ? 448u : 256u) && p.T >= (int64_t)p.n_seq * 640) {
    if (causal) hipLaunchKernelGGL((packed_fwd_kernel<D, true, 2>), grid, dim3(512), 0, st, p, slots);
    else hipLaunchKernelGGL((packed_fwd_kernel<D, false, 2>), grid, dim3(512), 0, st, p, slots);
    return;
  }
  if (causal) hipLaunchKernelGGL((packed_fwd_kernel<D, true, 1>), grid, dim3(256), 0, st, p, slots);
  else hipLaunchKernelGGL((packed_fwd_kernel<D, false, 1>), grid, dim3(256), 0, st, p, slots);
}
template <int D, bool CAUSAL>
void launch_bwd(const PackedAttention& p, hipStream_t st) {
  const int slots = packed_slots(p.T, p.n_seq, BM), kv = p.n_kv_heads, small = packed_slots(p.T, p.n_seq, 64);
  const int group = p.n_heads / kv;
  const unsigned queries = packed_blocks(slots, kv, group), keys = packed_blocks(small, kv, 1);
  // One launch where launches cost more than the shorter chain of tiles that four groups of waves have, or pairs: rows to a block
  // of keys, and few blocks.  One launch and two, us, sequences x rows, query heads / heads of keys: heads of 64, 12 / 12: 4x64 7.7 and
  // 12.7, 1x1024 26.6 and 35.3, 8x256 23.5 and 25.0, 8x512 49.8 and 42.9; 16 / 4: 4x64 10.8 and 13.8, 8x128 17.4 and 18.0, 2x256 25.9
  // and 22.9, 1x1024 82.7 and 57.3; heads of 128, 12 / 12: 2x256 19.4 and 24.5, 8x128 23.1 and 20.3; 16 / 4: 1x16 15.1 and 12.8.
  // Rows to a sequence are taken to be T / n_seq.  One long sequence among short ones, one launch and two, heads of 64, 4 / 4: 4096 beside 15 of
  // 16 rows 83 and 102 (one is taken), 1024 beside 15 25.4 and 34.4 (one); 4 / 2: 160 and 132 (two), 44.1 and 41.6 (one); heads of 128, 2 / 2: 179
  // and 183 (one).  A buffer of eight times the rows, and four times the sequences, all empty: 12 / 12 2x512 29.3 instead of 17.1, 8x256 21.3
  // instead of 23.8, 16 / 4 8x128 18.6 instead of 17.3.
  const bool few = (int64_t)p.T * group <= (int64_t)p.n_seq * (group == 1 ? 1024 : 512) &&
                   (D == 128 ? group <= 2 && queries + keys <= 320 : queries + keys <= 1024);
  if (few) {
    constexpr int LDS = std::max(4 * Tile<D>::SIZE, dkv_elements<D, 2>()) * 2;
    static const bool configured = [] {
      (void)hipFuncSetAttribute((const void*)packed_bwd_small_kernel<D, CAUSAL>, hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
      return true;
    }();
    (void)configured;
    hipLaunchKernelGGL((packed_bwd_small_kernel<D, CAUSAL>), dim3(queries + keys), dim3(256), LDS, st, p, slots, small, (int)queries);
    return;
  }
  hipLaunchKernelGGL((packed_bwd_dq_kernel<D, CAUSAL>), dim3(queries), dim3(256), 0, st, p, slots);
  if constexpr (D == 128) {
    hipLaunchKernelGGL((packed_bwd_dkv_pair_kernel<CAUSAL>), dim3(keys), dim3(256), 0, st, p, small);
  } else if ((int64_t)slots * kv >= (D == 32 ? 224 : 160) + 96 * group) {
    // Blocks of 128 keys enough to fill the device; the longer their chain of tiles, that of all heads that share the keys, the more of
    // them.  128 keys in one group and 64 keys in four, us, behind a mask, heads of 64: 12 / 12 192 blocks 17.0 and 16.9, 288 23.1 and
    // 27.1, 1728 139 and 195; 16 / 4 320 78 and 62, 576 182 and 174, 640 112 and 120, 1280 209 and 252; heads of 32, 12 / 12: 288 18.0 and
    // 17.7, 396 25.7 and 26.8, 1368 25 and 36.
    hipLaunchKernelGGL((packed_bwd_dkv_kernel<D, CAUSAL, 4, 1>), dim3(packed_blocks(slots, kv, 1)), dim3(256), 0, st, p, slots);
  } else {
    hipLaunchKernelGGL((packed_bwd_dkv_kernel<D, CAUSAL, 2, 4>), dim3(keys), dim3(512), 0, st, p, small);
  }
}
}  // namespace

void packed_attention_fwd_bf16(const PackedAttention& p, int d, int causal, hipStream_t st) {
  if (d == 32) launch_fwd<32>(p, causal, st);
  else if (d == 64) launch_fwd<64>(p, causal, st);
  else launch_fwd<128>(p, causal, st);
}
void packed_attention_bwd_bf16(const PackedAttention& p, int d, int causal, hipStream_t st) {
  if (d == 32) causal ? launch_bwd<32, true>(p, st) : launch_bwd<32, false>(p, st);
  else if (d == 64) causal ? launch_bwd<64, true>(p, st) : launch_bwd<64, false>(p, st);
  else causal ? launch_bwd<128, true>(p, st) : launch_bwd<128, false>(p, st);
}

}  // namespace mk
