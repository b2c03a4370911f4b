// The GEMM as the library's own callers use it: chorus_gemm_bf16 with optional scratch, with which a gated-residual
// product that would leave most compute units idle is cut into slices of K.
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace chorus {

// Two pieces of scratch (16-byte aligned device memory, either may be empty), used only by the kernels of the call.
// Every slice but the last puts its fp32 [M, N] result there: the first one into `first`, the others into `rest`.
struct GemmParts {
  void* first;
  size_t first_bytes;
  void* rest;
  size_t rest_bytes;
  // kGemmCounts words that are zero when the product starts, or null: the slices may then add to the residual one behind the other instead
  uint32_t* counts;
};
constexpr int kGemmCounts = 256;
// Whether a gated-residual product of that size uses the counts: if not, nothing has to clear them.
bool gemm_bf16_chained(int64_t M, int32_t N, int32_t K, const GemmParts& parts);

// chorus_gemm_bf16 with scratch; the number of slices depends on the sizes given here and on nothing else
int32_t gemm_bf16_parts(const uint16_t* A, const uint16_t* W, int64_t M, int32_t N, int32_t K, int32_t epilogue, void* out,
                        const float* bias, const float* gate0, const float* gate1, float scale, const GemmParts& parts,
                        void* stream);

// out = A W^T + bias and out2 = A2 W2^T + bias2, bf16, the same K: in one launch where that does not fill the chip
int32_t gemm_bf16_two(const uint16_t* A, const uint16_t* W, int64_t M, int32_t N, int32_t K, uint16_t* out, const float* bias,
                      const uint16_t* A2, const uint16_t* W2, int64_t M2, int32_t N2, uint16_t* out2, const float* bias2,
                      void* stream);

// a tile's bytes, 256 rows of 2 K, within the 32-bit offsets of its loads; longer rows are 64 x 64 tiles' alone
constexpr int kMaxOffsetK = (1 << 22) - 64;

// the tile kernels by their shapes
enum Tile { kTile256, kTileWide, kTile128, kTile128Deep, kTile64, kTiles };
constexpr int kTileNumber[kTiles] = {3, 2, 4, 5, 1};  // as chorus_gemm_bf16_kernel names them
constexpr int kTileRows[kTiles] = {256, 128, 128, 128, 64};
constexpr int kTileCols[kTiles] = {256, 256, 128, 128, 64};
// half steps in LDS of the deep 128 x 128 and of the 64 x 64 tiles
constexpr int kHalvesDeep = 7, kHalves64 = 9;

// On which tiles a whole product (no slices) is the fastest by the estimates for bf16: the first head_rows rows on kTile256 in a launch
// of their own (0: none), the others on `tile`. What is estimated is the operands' way into the compute units, so that products of other
// types go by it too, with K in units of 2 bytes and N the rows of all weight matrices.
struct TileCut {
  long head_rows;
  int tile;
};
TileCut gemm_tiles(int64_t M, int32_t N, int32_t K, int32_t epilogue);

}  // namespace chorus
