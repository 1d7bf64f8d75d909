// The products of the update with orthogonalised steps on tiles of 256 x 256 (see muon.hip), by blocks that take one tile after the
// other: the loop of gemm_large.h on fp16 operands, over the tiles of many matrices.
//
// A block of eight waves on a compute unit; a wave owns 128 x 64 of a tile as MFMA tiles of 16 x 16 x 32.  Operand tiles of 64
// reduction indices go to LDS directly, into rings of three (A) and two slots (B), and the loads run through the tile
// boundary.  Why 256 x 256: a compute unit draws about 54 bytes per clock from the L2, tiles of 128 need 64 of it at full rate, of
// 256 half as much.  Tiles differ in their number of k tiles, by matrix: the host deals them out to the blocks once, the longest first,
// a matrix' neighbouring tiles to one XCD (see ops_abi.cpp).
//
// 48 matrices each of 1024 x 1024, 256 x 1024 and 1024 x 4096: the three products take 284, 162 and 500 us, 0.92, 0.64 and 1.04 PFLOP/s of
// what is needed (of the symmetric ones the half above the diagonal; tiles of 256 make 5/8 of 1024 x 1024); a product of 8192^3 of the
// library runs at 1.20.  Bound by the matrix units and, in the shorter second one, by whole rounds of tiles and their stores: with the
// second factor asked for as it is stored and the tile below the diagonal written 16 bytes to a row, it took 175, the first 292.
#include "muon_device.h"

namespace mk {

using namespace muon;

template <int STAGE>
__global__ __launch_bounds__(512) void muon_large_kernel(const MuonMatrix* mats, const MuonTile* tiles, char* ws, int from, const int32_t* starts) {
  using namespace large;
  typedef Sizes<8> Z;
  constexpr bool KM = STAGE != 3;
  typedef LTileOf<true, 256> TA;
  typedef LTileOf<KM, 256> TB;
  constexpr int FM = 8, LA = Z::A_LOADS, LB = Z::B_LOADS, MEET = Z::MEET;
  extern __shared__ __attribute__((aligned(1024))) unsigned char m_smem[];
  bf16_t* const ring = (bf16_t*)m_smem;
  bf16_t* const ring_b = ring + Z::NA * Z::A_TILE;
  typedef const __attribute__((address_space(4))) int32_t* StartPtr;
  const StartPtr sp = (StartPtr)(uintptr_t)(starts + blockIdx.x);
  int unit = sp[0];
  const int u_end = sp[1];
  if (unit >= u_end) return;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave >> 2, wn = wave & 3;

  // What a tile needs of its table entries, by scalar loads: vector loads would wait for the direct loads before them.
  typedef const __attribute__((address_space(4))) uint32_t* TilePtr;
  typedef const __attribute__((address_space(4))) MuonMatrix* MatPtr;
  struct Place { f16* c; const f16* s; int ldc, i, j, steps, m_left, n_left; } cur, ahead;   // s: the second stage's A
  int c_unit = unit, c_left;
  uint64_t base_a, base_b, step_b;
  uint32_t off_a[2], off_b[2], bytes_a, bytes_b, two_a, two_b;
  uint64_t step_a;
  auto enter = [&]() __attribute__((always_inline)) {
    const TilePtr tp = (TilePtr)(uintptr_t)(tiles + c_unit);
    const int which = (int)tp[0], i = (int)(tp[1] & 0xFFFFu), j = (int)(tp[1] >> 16);
    const MatPtr t = (MatPtr)(uintptr_t)(mats + which);
    const int mp = t->mp, np = t->np, small = min(t->rows, t->cols), big = max(t->rows, t->cols);
    const int lda = STAGE == 1 ? np : mp, ldb = STAGE == 2 ? mp : np, K = STAGE == 1 ? big : small;
    f16* const x = (f16*)(ws + t->x[from]);
    f16 *const a = (f16*)(ws + t->a), *const b = (f16*)(ws + t->b);
    ahead.c = STAGE == 1 ? a : STAGE == 2 ? b : (f16*)(ws + t->x[from ^ 1]);
    ahead.s = a;
    ahead.ldc = STAGE == 3 ? np : mp;
    ahead.i = i * 256;
    ahead.j = j * 256;
    ahead.m_left = mp - i * 256;
    ahead.n_left = ahead.ldc - j * 256;
    ahead.steps = c_left = (K + LBK - 1) / LBK;
    const f16* pa = (STAGE == 1 ? x : STAGE == 2 ? a : b) + (int64_t)i * 256 * lda;
    const f16* pb = STAGE == 3 ? x + j * 256 : (STAGE == 1 ? x : a) + (int64_t)j * 256 * ldb;
    l_descriptor(pa, TA::bytes(lda, ahead.m_left), base_a, bytes_a);
    l_descriptor(pb, TB::bytes(ldb, ahead.n_left), base_b, bytes_b);
    step_a = LBK * 2;
    step_b = KM ? LBK * 2 : (uint64_t)LBK * 2 * ldb;
    two_a = TA::two(lda);
    two_b = TB::two(ldb);
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      off_a[q] = TA::src(lda, ahead.m_left, wave * LA + q, lane);
      off_b[q] = TB::src(ldb, ahead.n_left, wave * LB + q, lane);
    }
  };
  enter();
  cur = ahead;
  const uint32_t lds_a = l_lds_address(ring) + (uint32_t)wave * LA * 1024u;
  const uint32_t lds_b = l_lds_address(ring_b) + (uint32_t)wave * LB * 1024u;
  uint32_t fill_a = 0, fill_b = 0;                                // slots to fill, in bytes
  auto load_a = [&](int j) __attribute__((always_inline)) {
    l_direct_load(base_a, bytes_a, off_a[j & 1] + (j >> 1) * two_a, lds_a + fill_a + j * 1024u);
  };
  auto load_b = [&](int j) __attribute__((always_inline)) {
    l_direct_load(base_b, bytes_b, off_b[j & 1] + (j >> 1) * two_b, lds_b + fill_b + j * 1024u);
  };
  // On to the next k tile, or the next tile's first.  Behind the block's last the same k tile is requested again, into slots that
  // are not read any more.
  auto advance = [&]() __attribute__((always_inline)) {
    fill_a = fill_a == (Z::NA - 1) * Z::A_TILE * 2u ? 0 : fill_a + Z::A_TILE * 2u;
    fill_b = fill_b == (Z::NB - 1) * Z::B_TILE * 2u ? 0 : fill_b + Z::B_TILE * 2u;
    base_a += step_a; base_b += step_b;
    if (--c_left == 0) {
      const bool more = c_unit + 1 < u_end;
      base_a -= more ? 0 : step_a; base_b -= more ? 0 : step_b;
      step_a = more ? step_a : 0; step_b = more ? step_b : 0;
      c_left = 1 << 30;
      if (more) {
        ++c_unit;
        enter();
      }
    }
  };

  TA fa;
  TB fb;
  fa.init(wm * FM, lane);
  fb.init(wn * FN, lane);
  int slot_a = 0, slot_b = 0;                                     // in elements
  bf16x8 af[FM], bfr[2][FN];
  auto read_a = [&](int i, int h) __attribute__((always_inline)) { af[i] = fa.read(ring, slot_a, i, h); };
  auto read_b = [&](int j, int h) __attribute__((always_inline)) { bfr[h][j] = fb.read(ring_b, slot_b, j, h); };
  f32x4 acc[FM][FN];
  int stored = 0;                                                 // stores of the tile before
  auto k_tile = [&](auto first_) __attribute__((always_inline)) {
    constexpr bool FIRST = decltype(first_)::value;
    auto row = [&](int i, int h) __attribute__((always_inline)) {
#pragma unroll
      for (int j = 0; j < FN; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, bfr[h][j]), __builtin_bit_cast(f16x8, af[i]),
                                                           FIRST && h == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : acc[i][j], 0, 0, 0);
    };
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      row(i, 0);
      read_a(i, 1);
      if (i < FN) read_b(i, 1);
      if (!FIRST && i % (FM / LA) == 0) {
        __builtin_amdgcn_sched_barrier(0);
        load_a(i / (FM / LA));
        __builtin_amdgcn_sched_barrier(0);
      }
    }
#pragma unroll
    for (int i = 0; i < MEET; ++i) row(i, 1);
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(kLdsDone);
    // all but the loads of later k tiles and, in a tile's first turn, which has issued none yet, the stores of the tile before
    if (!FIRST) __builtin_amdgcn_s_waitcnt(in_flight(Z::YOUNGER));
    else if (stored == 2 * Z::STORES) __builtin_amdgcn_s_waitcnt(in_flight(Z::YOUNGER - LA + 2 * Z::STORES));
    else if (stored == Z::STORES) __builtin_amdgcn_s_waitcnt(in_flight(Z::YOUNGER - LA + Z::STORES));
    else __builtin_amdgcn_s_waitcnt(in_flight(Z::YOUNGER - LA));
    l_meet();
    slot_a = slot_a == (Z::NA - 1) * Z::A_TILE ? 0 : slot_a + Z::A_TILE;
    slot_b = slot_b == (Z::NB - 1) * Z::B_TILE ? 0 : slot_b + Z::B_TILE;
#pragma unroll
    for (int i = 0; i < MEET; ++i) read_a(i, 0);
#pragma unroll
    for (int i = MEET; i < FM; ++i) {
      row(i, 1);
      read_a(i, 0);
#pragma unroll
      for (int j = 0; j < FN; ++j)
        if (j * (FM - MEET) / FN == i - MEET) {
          read_b(j, 0);
          if (!FIRST) {
            __builtin_amdgcn_sched_barrier(0);
            load_b(j);
            __builtin_amdgcn_sched_barrier(0);
          }
        }
    }
    if (FIRST) {                                                  // behind the stores of the tile before
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 0; j < LA; ++j) load_a(j);
#pragma unroll
      for (int j = 0; j < LB; ++j) load_b(j);
      __builtin_amdgcn_sched_barrier(0);
    }
    advance();
  };

  // A finished tile: 16 rows of 64 columns at a time through 2 KB of LDS, the part of the free slot of A that this wave's next loads
  // fill; out along the rows, and for a tile above the diagonal by columns too (transposing reads), to its place below: of two times 16
  // rows the four lanes of a quad hand each other their pieces of 16 bytes, so that they write 64 bytes of one row, not of four.
  // What the second stage adds is asked for before the first store: a load behind stores has to wait for them.
  auto store = [&]() __attribute__((always_inline)) {
    // (padding ends on 128 rows and columns: a wave's part exists or does not)
    stored = 0;
    if (wm * 128 >= cur.m_left || wn * 64 >= cur.n_left) return;
    stored = STAGE != 3 && cur.i != cur.j ? 2 * Z::STORES : Z::STORES;
    int l = lane;                                                 // what the store computes from it is not held through the loop
    asm volatile("" : "+v"(l));
    const int lr = l & 15, lq = l >> 4, sr = l >> 3, sc = l & 7;
    unsigned char* const turn = m_smem;
    const uint32_t own = fill_a + (uint32_t)wave * LA * 1024u;
    const uint32_t in16 = own + lr * 128 + (((lq >> 1) ^ (lr >> 1)) << 4) + (lq & 1) * 8;      // column tile j: ^ 32 j
    const uint32_t out = own + sr * 128 + ((sc ^ (sr >> 1)) << 4);                            // rows 8 .. 15: + 1024 and ^ 64
    auto fence = [&]() __attribute__((always_inline)) { asm volatile("" ::: "memory"); };
    const int m0 = cur.i + wm * 128, n0 = cur.j + wn * 64;
    f16* const rows = cur.c + (int64_t)(m0 + sr) * cur.ldc + n0 + sc * 8;
    f16* const below = cur.c + (int64_t)(n0 + (l & ~3)) * cur.ldc + m0 + 8 * (l & 3);
    const f16* const self = cur.s + (int64_t)(m0 + lr) * cur.ldc + n0 + 4 * lq;
    // transposing reads: within 16 lanes, lane i gets column i of 4 rows; its own address is 4 columns of one of the rows
    const int tr = lr >> 2, tc = 16 * lq + 4 * (lr & 3);
    f16x4 s[STAGE == 2 ? FM : 1][FN];
    if (STAGE == 2) {
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) s[i][j] = *(const f16x4*)(self + (int64_t)i * 16 * cur.ldc + 16 * j);
    }
    u32x4 z[4];                                                   // of two times 16 rows: eight each, of the column of this lane
    // across a quad's lanes: z[k] of lane v becomes z[v] of lane k
    auto swap = [&](u32x4& even, u32x4& odd, auto lanes, bool upper) __attribute__((always_inline)) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t got = __builtin_amdgcn_update_dpp(0, upper ? even[e] : odd[e], decltype(lanes)::value, 0xF, 0xF, false);
        even[e] = upper ? got : even[e];
        odd[e] = upper ? odd[e] : got;
      }
    };
#pragma unroll
    for (int i = 0; i < FM; ++i) {
#pragma unroll
      for (int j = 0; j < FN; ++j) {
        f16x4 o;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float v = acc[i][j][e];
          if (STAGE == 2) v = fmaf(kB, (float)s[i][j][e], kC * kBack * v) + (m0 + 16 * i + lr == n0 + 16 * j + 4 * lq + e ? kA * kHeld : 0.f);
          else v *= kBack;
          o[e] = (f16)v;
        }
        *(f16x4*)(turn + (in16 ^ (j * 32))) = o;
      }
      fence();
      const f16x8 w0 = *(const f16x8*)(turn + out), w1 = *(const f16x8*)(turn + ((out + 1024) ^ 64));
      *(f16x8*)(rows + (int64_t)i * 16 * cur.ldc) = w0;
      *(f16x8*)(rows + (int64_t)(i * 16 + 8) * cur.ldc) = w1;
      if (STAGE != 3 && cur.i != cur.j) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          s16x4 part[2];
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            const int r = 8 * half + 4 * q + tr;
            part[q] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_l*)(turn + own + r * 128 + (((tc >> 3) ^ (r >> 1)) << 4) + (tc & 7) * 2));
          }
          typedef short s16x8 __attribute__((ext_vector_type(8)));
          z[2 * (i & 1) + half] = __builtin_bit_cast(u32x4, (s16x8)__builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7));
        }
        if (i & 1) {
          typedef std::integral_constant<int, 0xB1> NextLane;     // quad_perm 1 0 3 2
          typedef std::integral_constant<int, 0x4E> NextPair;     // quad_perm 2 3 0 1
          swap(z[0], z[1], NextLane(), l & 1);
          swap(z[2], z[3], NextLane(), l & 1);
          swap(z[0], z[2], NextPair(), l & 2);
          swap(z[1], z[3], NextPair(), l & 2);
#pragma unroll
          for (int k = 0; k < 4; ++k) *(u32x4*)(below + (int64_t)k * cur.ldc + (i - 1) * 16) = z[k];
        }
      }
      fence();
      __builtin_amdgcn_sched_barrier(0);
    }
  };

#pragma unroll
  for (int t = 0; t < Z::NB; ++t) {
#pragma unroll
    for (int j = 0; j < LA; ++j) load_a(j);
#pragma unroll
    for (int j = 0; j < LB; ++j) load_b(j);
    advance();
  }
  __builtin_amdgcn_s_waitcnt(in_flight((Z::NB - 1) * (LA + LB)));
  l_meet();
  for (;;) {
#pragma unroll
    for (int j = 0; j < FN; ++j) read_b(j, 0);
#pragma unroll
    for (int i = 0; i < FM; ++i) read_a(i, 0);
    k_tile(std::true_type());
    for (int kt = 1; kt < cur.steps; ++kt) k_tile(std::false_type());
    store();
    if (++unit >= u_end) break;
    cur = ahead;
  }
  __builtin_amdgcn_s_waitcnt(in_flight(0));           // no direct load may land in LDS that is another block's by then
}

void muon_large_product(int stage, const MuonMatrix* mats, const MuonTile* tiles, const int32_t* starts, char* ws, int from, hipStream_t st) {
  constexpr int LDS = large::Sizes<8>::SMEM;
  static const bool configured = [] {
    for (const void* k : {(const void*)muon_large_kernel<1>, (const void*)muon_large_kernel<2>, (const void*)muon_large_kernel<3>})
      (void)hipFuncSetAttribute(k, hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
    return true;
  }();
  (void)configured;
  const dim3 grid(kMuonBlocks), block(512);
  if (stage == 1) hipLaunchKernelGGL((muon_large_kernel<1>), grid, block, LDS, st, mats, tiles, ws, from, starts);
  else if (stage == 2) hipLaunchKernelGGL((muon_large_kernel<2>), grid, block, LDS, st, mats, tiles, ws, from, starts);
  else hipLaunchKernelGGL((muon_large_kernel<3>), grid, block, LDS, st, mats, tiles, ws, from, starts);
}

}  // namespace mk
