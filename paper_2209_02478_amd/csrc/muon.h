// Tables of the update with orthogonalised steps (muon.hip), laid out by the host.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cmath>
#include <vector>

namespace mk {

constexpr int kMuonTile = 128;          // rows and columns of a block's tile; X, A and B are padded to whole tiles of zeros
constexpr int kMuonFine = 64;           // a product's tiles where those are few or mostly padding
constexpr int kMuonSmallShort = 128, kMuonSmallLong = 256;   // sides of the largest matrix that one block updates by itself, in LDS
constexpr int64_t kMuonSide = 1 << 20;  // most rows or columns of a matrix

struct MuonMatrix {
  float* master; uint16_t* lowp; const float* grad; float* momentum;
  uint64_t x[2], a, b, partial;         // bytes into the scratch: X before and after an iteration, A, B, the chunks' sums
  int64_t chunk;                        // elements of a chunk, a multiple of 4
  int32_t rows, cols;
  int32_t mp, np;                       // the smaller side and the larger, rounded up to whole tiles
};
struct MuonChunk { int32_t matrix, pad; int64_t start; };
struct MuonTile { int32_t matrix; uint16_t i, j; };          // row and column of tiles; matrix below 0: none
struct MuonHyper { float lr, momentum, weight_decay, rms, eps; int nesterov, iterations; };

inline const char* bad_muon(float lr, float momentum, float weight_decay, float rms, float eps, int iterations) {
  if (!(lr >= 0.f) || !(momentum >= 0.f && momentum < 1.f) || !(weight_decay >= 0.f) || !(rms >= 0.f) || !(eps >= 1e-30f) || !std::isfinite(lr) ||
      !std::isfinite(weight_decay) || !std::isfinite(rms) || !std::isfinite(eps))
    return "hyper-parameters out of range";
  return iterations < 1 || iterations > 64 ? "1 to 64 iterations required" : nullptr;
}

inline bool muon_small(int64_t rows, int64_t cols) {
  return (rows < cols ? rows : cols) <= kMuonSmallShort && (rows < cols ? cols : rows) <= kMuonSmallLong;
}
// The first `count` matrices of a table, small ones, which need no scratch.
void muon_update_small(const MuonMatrix* mats, int count, const MuonHyper& h, hipStream_t st);
constexpr int kMuonBlocks = 256;        // blocks of a product on large tiles: one to a compute unit, ids go to the 8 XCDs in turn
// The units of work of one part of a list: elements in chunks, X in tiles, and the tiles of the products: of the symmetric ones on and
// above the diagonal (tri) and of X (full), for matrices that take tiles of 128 or 64; for those that take 256 each product's tiles
// block by block, and where each block's begin (null: none).
struct MuonUnits {
  const MuonChunk* chunks = nullptr;
  const MuonTile *cells = nullptr, *tri = nullptr, *full = nullptr, *large_tiles[3] = {nullptr, nullptr, nullptr};
  const int32_t* large[3] = {nullptr, nullptr, nullptr};
  int n_chunks = 0, n_cells = 0, n_tri = 0, n_full = 0;
  bool fine_tri = false, fine_full = false;   // those are tiles of 64
};
// One part of a list after the other uses the scratch.
void muon_update(const MuonMatrix* mats, const MuonUnits& u, void* workspace, const MuonHyper& h, hipStream_t st);

}  // namespace mk
