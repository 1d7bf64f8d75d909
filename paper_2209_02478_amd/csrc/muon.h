// Tables of the update with orthogonalised steps (muon.hip), laid out by the host.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cmath>
#include <vector>

namespace mk {

constexpr int kMuonTile = 128;          // rows and columns of a block's tile; X, A and B are padded to whole tiles of zeros
constexpr int64_t kMuonSide = 1 << 20;  // most rows or columns of a matrix

struct MuonMatrix {
  float* master; uint16_t* lowp; const float* grad; float* momentum;
  uint64_t x[2], a, b, partial;         // bytes into the scratch: X before and after an iteration, A, B, the chunks' sums
  int64_t chunk;                        // elements of a chunk, a multiple of 4
  int32_t rows, cols;
  int32_t mp, np;                       // the smaller side and the larger, rounded up to whole tiles
};
struct MuonChunk { int32_t matrix, pad; int64_t start; };
struct MuonTile { int32_t matrix; uint16_t i, j; };          // row and column of tiles
struct MuonHyper { float lr, momentum, weight_decay, rms, eps; int nesterov, iterations; };

inline const char* bad_muon(float lr, float momentum, float weight_decay, float rms, float eps, int iterations) {
  if (!(lr >= 0.f) || !(momentum >= 0.f && momentum < 1.f) || !(weight_decay >= 0.f) || !(rms >= 0.f) || !(eps >= 1e-30f) || !std::isfinite(lr) ||
      !std::isfinite(weight_decay) || !std::isfinite(rms) || !std::isfinite(eps))
    return "hyper-parameters out of range";
  return iterations < 1 || iterations > 64 ? "1 to 64 iterations required" : nullptr;
}

// One part of a list after the other uses the scratch.
void muon_update(const MuonMatrix* mats, const MuonChunk* chunks, int n_chunks, const MuonTile* tri, int n_tri, const MuonTile* full, int n_full,
                 void* workspace, const MuonHyper& h, hipStream_t st);

}  // namespace mk
