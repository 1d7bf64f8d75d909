// Pieces that the kernels of the update with orthogonalised steps share.
#pragma once
#include "gemm_large.h"
#include "muon.h"

namespace mk {
namespace muon {

typedef _Float16 f16;
typedef f16 f16x4 __attribute__((ext_vector_type(4)));
typedef f16 f16x8 __attribute__((ext_vector_type(8)));
using large::f32x4;

constexpr float kHeld = 1024.f, kBack = 1.f / 1024.f;        // operands are held times 2^10
constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
constexpr int BK = 64;

__device__ __forceinline__ f16* in_scratch(char* ws, uint64_t at) { return (f16*)(ws + at); }

}  // namespace muon

// The three products on tiles of 256 x 256 (muon_large.hip): block b of kMuonBlocks takes tiles[starts[b]] .. tiles[starts[b + 1] - 1].
void muon_large_product(int stage, const MuonMatrix* mats, const MuonTile* tiles, const int32_t* starts, char* ws, int from, hipStream_t st);

}  // namespace mk
