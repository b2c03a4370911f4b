// bf16 MFMA GEMM with fused epilogues: C = epi(A W^T + bias), A [M,K], W [N,K], both K-contiguous, fp32 accumulation.
//
// One kernel, `gemm_w16_kernel`, that copies its tiles straight from global memory to LDS, in five tile shapes; which shape a
// product is run on, and whether K is cut into slices, is decided by `plan_gemm` at the end of the file.
#include <cmath>

#include "chorus_ops.h"
#include "common.h"
#include "gemm.h"
#include "gemm_tile.h"

namespace chorus {
namespace {

// where the slices of K but the last leave their [M, N] results
struct PartPtrs {
  float* first;
  float* rest;
  __device__ __forceinline__ float* of(int slice, long M, int N) const {
    return slice == 0 ? first : rest + (size_t)(slice - 1) * M * N;
  }
};

// A second product of a launch with bf16 outputs, with the same K: its tiles follow the first one's `first` tiles.
struct Twin {
  const uint16_t* A;
  const uint16_t* W;
  uint16_t* out;
  const float* bias;
  long M;
  int N, tiles_m, tiles_n, first;
  static constexpr bool kTwo = true, kChain = false;
};
struct Alone {  // no second product
  static constexpr bool kTwo = false, kChain = false;
};
// The gated residual in slices of K without scratch: every slice adds its part to the residual itself, in the order of the slices. A
// slice waits until its tile's count has reached its number. Workgroups are dealt out by each XCD for itself, so that a workgroup's
// number says nothing of what has started elsewhere; what a workgroup does is given out by ticket instead. The workgroups
// whose number leaves the same rest by `groups` (8: they share an XCD and its L2) take tickets of one counter for a range of tiles of their
// own, all of its tiles of the first slice first. So a slice only ever waits for a lower ticket of its group, whose workgroup
// has taken it and is running; that one waits for a still lower ticket or for nothing: every wait ends, whatever else runs on the GPU.
// The ticket is a round trip to memory ahead of the first load, about 1 us (by workgroup number / by ticket, us: 3271 x 1536 x 8960 84.4 /
// 86.8, 2000 59.1 / 59.5, 1100 39.3 / 40.7, 300 21.5 / 22.6, 960 x 5120 x 5120 60.3 / 61.2, 200 x 2048 x 4096 13.8 / 15.2, operands warm).
// A word a tile, zero at the start: the slices that have been added in its low four bits and, in the word of a group's first
// tile, the tickets taken in the others.
// Slices of equal length would all end together and then wait for each other's updates: each is a few steps longer than the one in
// front of it instead (3271 x 1536 x 8960, three slices of 256 x 256 tiles: 100 us with equal ones, 87 with five steps more each).
struct Chain {
  uint32_t* count;  // [tiles]
  int stagger;      // steps that a slice is longer than the one in front of it
  int tiles, groups;
  static constexpr bool kTwo = false, kChain = true;
  static constexpr uint32_t kTicket = 16, kAdded = 15;  // one ticket; the bits of the slices that have been added
};

// The 128 x 256 shape takes three quarters of the operand bytes per product of 128 x 128 tiles: for products of about 400 to
// 512 such tiles with a long K, which run two to a unit, half as many wide ones finish earlier (N = 1536, K = 8960: 5000 rows
// 132 -> 117 us; N = 5120, K = 13824, 1200 rows: 202 -> 172; with 312 tiles, 3271 rows of the former, 109 and 112).
// FAR: rows so long that a tile's last byte is out of reach of the 32-bit offsets; loads by 64-bit addresses.
template <int EPI, int WBM, int WBN, int C, bool FAR, class SECOND>
__global__ __launch_bounds__(256, 1) void gemm_w16_kernel(const uint16_t* __restrict__ A, const uint16_t* __restrict__ W,
                                                          long M, int N, int K, EpiArgs ep, PartPtrs parts, int tiles_m,
                                                          int tiles_n, SECOND twin) {
#if defined(__HIP_DEVICE_COMPILE__)  // the buffer descriptors below are types of the device compiler's alone
  static_assert((WBM == 8 || WBM == 4 || WBM == 2) && (WBN == WBM || (WBM == 4 && WBN == 8)), "quadrants of 8 x 8, 4 x 4, 2 x 2 or 4 x 8 blocks");
  static_assert(C >= 5 && (WBM + WBN) / 2 * (C - 1) < 64, "two steps and a half in LDS at least, and the loads in flight must fit the wait counter");
  constexpr int BM = 32 * WBM, BN = 32 * WBN;
  constexpr int WTM = 16 * WBM, WTN = 16 * WBN;  // rows and columns of a wave's quadrant
  constexpr int HA = WTM * BK;  // elements of half a step's rows of A
  extern __shared__ __attribute__((aligned(1024))) uint8_t smem_raw[];
  uint16_t* smem = reinterpret_cast<uint16_t*>(smem_raw);  // [C][HA], [C][HB]

  // The grid's rows are the slices of K, their steps shared out as evenly as can be (never none: the host asks for no more
  // slices than steps). The last slice runs the epilogue, the others leave their plain fp32 result in `parts`. Without a
  // split there is one, and the divisions, a tenth of a microsecond of a product of one to four steps, are left out.
  int block = blockIdx.x, ntiles = gridDim.x;
  if constexpr (SECOND::kTwo) {
    ntiles = twin.first;
    if (block >= twin.first) {
      block -= twin.first;
      ntiles = gridDim.x - twin.first;
      A = twin.A;
      W = twin.W;
      M = twin.M;
      N = twin.N;
      ep.out = twin.out;
      ep.bias = twin.bias;
      tiles_m = twin.tiles_m;
      tiles_n = twin.tiles_n;
    }
  }
  const int nslices = gridDim.y;
  int slice = blockIdx.y, tile;
  if constexpr (SECOND::kChain) {
    const int g = block % twin.groups, q = twin.tiles / twin.groups, r = twin.tiles % twin.groups;
    const int of_group = q + (g < r), first_tile = g * q + (g < r ? g : r);
    if ((slice * (int)gridDim.x + block) / twin.groups >= of_group * nslices) return;  // the grid's x is a multiple of the groups
    // one of the ring's places that nothing is requested into before every wave has read it
    uint32_t* const mine = reinterpret_cast<uint32_t*>(smem + (C - 1) * HA);
    if (threadIdx.x == 0)
      mine[0] = __hip_atomic_fetch_add(twin.count + first_tile, Chain::kTicket, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) / Chain::kTicket;
    __syncthreads();
    const int ticket = __builtin_amdgcn_readfirstlane((int)mine[0]);
    slice = ticket / of_group;
    tile = ticket - slice * of_group;
    tile += first_tile;
  } else {
    tile = xcd_remap(block, ntiles);
  }
  int KTN = K / BK, k_first = 0;
  if (nslices > 1) {
    auto start = [&](int i) {
      if constexpr (SECOND::kChain)
        return i * KTN / nslices - twin.stagger * i * (nslices - i) / 2;
      else
        return i * KTN / nslices;
    };
    k_first = __builtin_amdgcn_readfirstlane(start(slice));
    KTN = __builtin_amdgcn_readfirstlane(start(slice + 1)) - k_first;
    A += (long)k_first * BK;
    W += (long)k_first * BK;
  }
  const TilePlace at = tile_place(tile, tiles_m, tiles_n, K);
  const long m0 = (long)at.m * BM;
  const int n0 = at.n * BN;

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  const int rows_a = M - m0 < BM ? (int)(M - m0) : BM, rows_b = N - n0 < BN ? N - n0 : BN;
  f32x4 acc[8][8];  // [n block][m block]; the WBN x WBM corner is used
  gemm16_loop<MmaBf16, OneMatrix, WBM, WBN, C, FAR>(acc, smem, A + m0 * K, W + (long)n0 * K, OneMatrix{}, rows_a, rows_b, K, k_first, KTN,
                                                    wave, lane);
  const auto sums = [&](int nb, int mb) { return acc[nb][mb]; };
  if constexpr (SECOND::kChain) {
    static_assert(EPI == CHORUS_EPI_RESID, "slices of the gated residual");
    uint32_t* const count = twin.count + tile;
    if (slice > 0) {
      if (tid == 0)
        while ((__hip_atomic_load(count, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) & Chain::kAdded) != (uint32_t)slice) __builtin_amdgcn_s_sleep(1);
      __syncthreads();
      asm volatile("" ::: "memory");  // the residual is read behind the count
      ep.bias = nullptr;              // went in with the first slice
    }
    gemm16_epilogue_resid<WBM, WBN, true>(sums, ep, reinterpret_cast<float*>(smem_raw) + wave * e16_f32_wave<WBN>(), m0 + wm * WTM,
                                          n0 + wn * WTN, M, N, lane);
    if (slice + 1 < nslices) {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the wave's stores have completed, past the L2
      __syncthreads();
      if (tid == 0) __hip_atomic_fetch_add(count, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    return;
  }
  if constexpr (EPI == CHORUS_EPI_RESID) {
    if (slice + 1 < nslices) {
      const EpiArgs plain{parts.of(slice, M, N), nullptr, nullptr, nullptr, 1.f};
      gemm16_finish<CHORUS_EPI_F32, WBM, WBN>(sums, plain, smem_raw, wave, wm, wn, m0, n0, M, N, lane);
      return;
    }
  }
  gemm16_finish<EPI, WBM, WBN>(sums, ep, smem_raw, wave, wm, wn, m0, n0, M, N, lane);
#endif
}

template <int WBM, int WBN, int C, bool FAR = false>
int32_t launch_gemm_w16(const uint16_t* A, const uint16_t* W, long M, int N, int K, int epi, EpiArgs ep, hipStream_t s,
                        int slices, const PartPtrs& parts) {
  constexpr int BM = 32 * WBM, BN = 32 * WBN;
  long tm = (M + BM - 1) / BM;
  int tn = (N + BN - 1) / BN;
  if (tm * tn * slices > 0x7fffffffL) return CHORUS_E_SHAPE;
  dim3 grid((unsigned)(tm * tn), (unsigned)slices), block(256);
  const size_t smem = (size_t)C * (BM + BN) / 2 * BK * sizeof(uint16_t);
#define GEMM_W16(E)                                                                           \
  {                                                                                           \
    auto kern = gemm_w16_kernel<E, WBM, WBN, C, FAR, Alone>;                                  \
    static DynLdsOnce once;                                                                   \
    CHK_STATUS(once.ensure(reinterpret_cast<const void*>(kern), (int)smem));                  \
    hipLaunchKernelGGL(kern, grid, block, smem, s, A, W, M, N, K, ep, parts, (int)tm, tn, Alone{});   \
  }
  switch (epi) {
    case CHORUS_EPI_BF16: GEMM_W16(CHORUS_EPI_BF16); break;
    case CHORUS_EPI_GELU_BF16: GEMM_W16(CHORUS_EPI_GELU_BF16); break;
    case CHORUS_EPI_F32: GEMM_W16(CHORUS_EPI_F32); break;
    case CHORUS_EPI_RESID: GEMM_W16(CHORUS_EPI_RESID); break;
    default: return CHORUS_E_ARG;
  }
#undef GEMM_W16
  CHORUS_LAUNCH_CHECK();
  return CHORUS_OK;
}

// What the last slice of K left out: out[m][n] += gate[n] scale sum_s part_s[m][n], P parts in ascending order (the bias
// went in with the last slice).
template <int P>
__global__ __launch_bounds__(256) void gemm_add_parts_kernel(PartPtrs parts, long M, int N, EpiArgs ep) {
  const long n4 = N / 4, i = (long)blockIdx.x * 256 + threadIdx.x;
  if (i >= M * n4) return;
  const int n = (int)(i % n4) * 4;
  f32x4 p[P];
#pragma unroll
  for (int k = 0; k < P; ++k) p[k] = *reinterpret_cast<const f32x4*>(parts.of(k, M, N) + i * 4);
  f32x4* o = reinterpret_cast<f32x4*>(reinterpret_cast<float*>(ep.out) + i * 4);
  const f32x4 cur = *o;
  f32x4 gate = {1.f, 1.f, 1.f, 1.f};
  if (ep.gate0 || ep.gate1) {
    gate = f32x4{0.f, 0.f, 0.f, 0.f};
    if (ep.gate0) gate += *reinterpret_cast<const f32x4*>(ep.gate0 + n);
    if (ep.gate1) gate += *reinterpret_cast<const f32x4*>(ep.gate1 + n);
  }
  gate *= ep.scale;
#pragma unroll
  for (int k = 1; k < P; ++k) p[0] += p[k];
  *o = cur + gate * p[0];
}

int32_t launch_add_parts(const PartPtrs& parts, int slices, long M, int N, const EpiArgs& ep, hipStream_t s) {
  const dim3 grid((unsigned)((M * (N / 4) + 255) / 256));
  switch (slices) {
    case 2: hipLaunchKernelGGL(gemm_add_parts_kernel<1>, grid, dim3(256), 0, s, parts, M, N, ep); break;
    case 3: hipLaunchKernelGGL(gemm_add_parts_kernel<2>, grid, dim3(256), 0, s, parts, M, N, ep); break;
    case 4: hipLaunchKernelGGL(gemm_add_parts_kernel<3>, grid, dim3(256), 0, s, parts, M, N, ep); break;
    default: return CHORUS_E_ARG;
  }
  CHORUS_LAUNCH_CHECK();
  return CHORUS_OK;
}

// ---------------------------------------------------------------------------
// Which tile, and in how many slices of K. The estimated time of each tile in microseconds, fitted to 3600 measurements
// on this chip with activations in the last-level cache and weights cold, as a request finds them (K from 256 to 13824, N
// from 256 to 15360, M from 64 to 13104; figures in brackets: gated residual, K = 1536 / K = 8960 where N = 1536). What is fitted is the
// choice: over those products the tile and slices taken cost 0.7 % more than the fastest (geometric mean).
// What bounds a launch that does not fill the chip is the rate at which ONE compute unit gets operands: its L1 holds
// 256 lines in flight, 32 KB, so a unit takes in about 60 KB per microsecond whatever the kernel does, and the launch
// that spreads the same problem over more units wins: smaller tiles, or slices of K.
//   256 x 256  one workgroup per unit, rounds of 256; a partly filled round is up to a quarter faster [38 / 161 us, full 54 / 215]
//   128 x 256  one workgroup per unit: up to 256 tiles [23 / 116 few, 32 / 128 all units busy], then a second round
//   128 x 128  two workgroups per unit: one round of up to 256 tiles [18 / 96], then rounds of 512 [31 / 135]
//   128 x 128  three steps and a half in LDS, one workgroup per unit: up to 256 tiles [14 / 75 few, 19 / 82 all units busy]
//   64 x 64    two workgroups per unit: up to 256 tiles [8.2 / 36], growing with the tiles up to 512 [14 / 69]
// ---------------------------------------------------------------------------
constexpr int kMaxSlices = 4;  // more slices than this were never the fastest

long tile_count(int tile, long m, int N) {
  const long rows = kTileRows[tile], cols = kTileCols[tile];
  return ((m + rows - 1) / rows) * ((N + cols - 1) / cols);
}

double tiles_time(int tile, long tiles, int K, int epi, int slices) {
  const double steps = (double)((K / BK + slices - 1) / slices);
  const double w = (double)(tiles * slices), fill = w / 256.0;
  const bool gelu = epi == CHORUS_EPI_GELU_BF16, f32 = slices == 1 && (epi == CHORUS_EPI_F32 || epi == CHORUS_EPI_RESID);
  auto by_epilogue = [&](double bf16, double with_gelu, double resid) { return f32 ? resid : gelu ? with_gelu : bf16; };
  switch (tile) {
    case kTile256: {
      const double full = by_epilogue(2.2, 3.59, 10.87) + 1.583 * steps;
      const double rounds = floor(fill), rest = fill - rounds;
      return full * (rounds + (rest > 0.0 ? 0.76 + 0.253 * rest * rest : 0.0));
    }
    case kTileWide: {
      if (w > 512.0) return INFINITY;
      const double c = by_epilogue(3.58, 3.83, 9.17);
      if (w <= 256.0) return c + (0.72 + 0.141 * fill * fill * fill) * steps;
      return (c + 0.861 * steps) * (1.6 + 0.4 * (fill - 1.0));
    }
    case kTile128: {
      const double one = by_epilogue(1.71, 3.67, 4.97) + 0.74 * steps, round512 = by_epilogue(0.48, 0.57, 5.67) + 1.001 * steps;
      if (w <= 256.0) return one;
      // With bf16 outputs half as many second workgroups cost the whole of it: over 115 products of 257 to 512 tiles (N 768 to 15360,
      // K 256 to 5120) the choice is 0.7 % slower than the fastest tile, 1.5 % with a straight line (1210 x 4608 x 1536, 360 tiles: 27.5
      // us, 128 x 256 24.8; 1956 x 2560 x 2560, 320 tiles: 41.2 and 36.8; the other way 746 x 6144 x 3072, 288 tiles: 40.7 and 45.6).
      const double second = f32 || epi == CHORUS_EPI_RESID ? fill - 1.0 : fmin(2.0 * (fill - 1.0), 1.0);
      if (w <= 512.0) return one + second * fmax(round512 - one, 0.0);
      return (0.784 * ceil(w / 512.0) + 0.216 * w / 512.0) * round512;
    }
    case kTile128Deep: {
      if (w > 256.0) return INFINITY;
      return by_epilogue(5.36, 3.64, 5.4) + (0.45 + 0.081 * fill * fill) * steps;
    }
    default:
      // Two workgroups a unit: a third one waits for their place (700 x 3072 x 8960, 528 tiles: 92 us, 69 with 480; the deep tile 66).
      // In none of 837 products was this tile the fastest with more.
      if (w > 512.0) return INFINITY;
      return (w <= 256.0 ? 1.0 : 1.141 + 0.677 * (fill - 1.0)) * (by_epilogue(3.62, 2.26, 3.14) + 0.246 * steps);
  }
}

double tile_time(int tile, long m, int N, int K, int epi, int slices) {
  if (K > kMaxOffsetK && tile != kTile64) return INFINITY;
  return tiles_time(tile, tile_count(tile, m, N), K, epi, slices);
}

constexpr GemmParts kNoParts{nullptr, 0, nullptr, 0, nullptr};

struct GemmPlan {
  int tile;
  int slices;
  double time;
  bool chain = false;  // the slices add to the residual one behind the other
};

// Chained slices: steps that a slice is longer than the one in front of it (about what an update of the residual takes), and the time.
// Every slice needs a compute unit from the start. Fitted to 16 products: microseconds a step and what does not depend on K (the last
// update of the residual among it). Measured, best plan without / with a chain, us: 3271 x 1536 x 8960 114 to 118 / 84 to 92 (256 x 256,
// three slices), 4500 115 / 107 (two), 2352 72 / 71 (128 x 256, two), 2000 78 / 70, 1350 68 / 56 (three), 1100 50 / 46 (128 x 128, two), 480 31
// / 34; 1200 x 5120 x 13824 179 / 152 (256 x 256, two), 960 173 / 125 (three), 544 101 / 96 (128 x 256, two).
// 300 x 5120 x 5120 45 / 30 (128 x 128, two), 200 38 / 28 (three), 960 72 / 64 (256 x 256, three). With fewer steps a slice the updates are the
// larger part: 1200 x 1536 x 1536 14 to 16.5 / 17, 4500 28 / 39. (With slices by workgroup number; a ticket adds about 1.)
constexpr int kMaxChain = 4, kChainTiles = 256, kChainSteps = 16;
constexpr int chain_update(int tile) { return tile == kTile256 || tile == kTileWide ? 5 : 8; }
int chain_stagger(int tile, int K, int slices) {
  const int want = chain_update(tile), most = K / BK / slices;
  return want * (slices - 1) < most ? want : most / slices;  // the first slice keeps half of its steps
}
double chain_time(int tile, long m, int N, int K, int slices) {
  const long tiles = tile_count(tile, m, N);
  if (tile == kTile128 || K > kMaxOffsetK || N > 1 << 20 || tiles * slices > kChainTiles || K / BK / slices < kChainSteps) return INFINITY;
  const double fill = (double)(tiles * slices) / 256.0;
  // The whole update also where the slices are too short to be that far apart: it is waited for there (65 to 128 rows x 5120 x 5120,
  // four slices of 20 steps: a block with two of them 285 us at 78 rows, 273 with whole tiles).
  const double steps = (double)(K / BK) / slices + 0.5 * (slices - 1) * chain_update(tile);
  switch (tile) {
    case kTile256: return 16.3 + 5.0 * (slices - 2) + (1.17 + fmax(fill - 0.8, 0.0)) * steps;
    case kTileWide: return 15.0 + 2.0 * (slices - 2) + 0.72 * steps;
    case kTile128Deep: return 5.4 + 1.7 * (slices - 2) + (0.45 + 0.081 * fill * fill) * steps;
    default: return 6.0 + 2.5 * (slices - 2) + 0.246 * steps;
  }
}

// The fastest tile by the estimates. With scratch a gated-residual product may also be cut into slices of K: every slice
// but the last writes its fp32 result and a second launch adds them (about 6 TB/s from the caches, and the launch itself).
// Measured where N = 1536, K = 8960, slices against the best whole tile: 128 rows 17 / 41 us, 480 rows 31 / 37, 1200
// rows 46 / 66, 2000 and 2300 rows (two slices of 128 x 256 tiles) 75 / 72 and 77 / 79; beyond that a whole tile fills the chip.
GemmPlan plan_slices(long m, int N, int K, int epi, const GemmParts& parts) {
  GemmPlan best{kTile64, 1, INFINITY};
  for (int t = 0; t < kTiles; ++t) {
    const double v = tile_time(t, m, N, K, epi, 1);
    if (v < best.time) best = GemmPlan{t, 1, v};
  }
  if (epi != CHORUS_EPI_RESID || !parts.first || !aligned16(parts.first) || !aligned16(parts.rest)) return best;
  const double whole = best.time;
  const size_t one = (size_t)m * (size_t)N * sizeof(float);
  if (one > parts.first_bytes) return best;
  for (int sl = 2; sl <= kMaxSlices && sl <= K / BK; ++sl) {
    if (sl > 2 && (!parts.rest || (size_t)(sl - 2) * one > parts.rest_bytes)) break;
    const double add = 3.0 + (double)(2 * sl) * 4.0 * (double)m * N / 6.0e6;
    for (int t = 0; t < kTiles; ++t) {
      const double v = tile_time(t, m, N, K, epi, sl) + add;
      if (v < 0.95 * whole && v < best.time) best = GemmPlan{t, sl, v};
    }
  }
  return best;
}

// The same, or a chain where one may be taken and is estimated to be faster.
GemmPlan plan_gemm(long m, int N, int K, int epi, const GemmParts& parts) {
  GemmPlan best = plan_slices(m, N, K, epi, parts);
  if (!parts.counts || epi != CHORUS_EPI_RESID) return best;
  const double without = best.time;
  for (int sl = 2; sl <= kMaxChain && sl <= K / BK; ++sl)
    for (int t = 0; t < kTiles; ++t) {
      const double v = chain_time(t, m, N, K, sl);
      if (v < 0.97 * without && v < best.time) best = GemmPlan{t, sl, v, true};
    }
  return best;
}

// The groups of a chain: an XCD each, or two, four or all of them where their units would be fewer than their workgroups that way (three slices
// of 81 to 84 tiles: four groups; 880 x 1536 x 8960, 84 tiles: in one group a block 200.3 us, so 196.8).
int chain_groups(int tiles, int slices) {
  for (int groups = 8; groups > 1; groups /= 2)
    if ((tiles + groups - 1) / groups * groups * slices <= kChainTiles) return groups;
  return 1;
}

template <int WBM, int WBN, int C>
int32_t launch_chain(const uint16_t* A, const uint16_t* W, long M, int N, int K, const EpiArgs& ep, int slices, uint32_t* count,
                     int stagger, hipStream_t s) {
  constexpr int BM = 32 * WBM, BN = 32 * WBN;
  const long tm = (M + BM - 1) / BM;
  const int tn = (N + BN - 1) / BN;
  const size_t smem = (size_t)C * (BM + BN) / 2 * BK * sizeof(uint16_t);
  auto kern = gemm_w16_kernel<CHORUS_EPI_RESID, WBM, WBN, C, false, Chain>;
  static DynLdsOnce once;
  CHK_STATUS(once.ensure(reinterpret_cast<const void*>(kern), (int)smem));
  const int tiles = (int)(tm * tn), groups = chain_groups(tiles, slices);
  hipLaunchKernelGGL(kern, dim3((unsigned)align_up(tiles, groups), (unsigned)slices), dim3(256), smem, s, A, W, M, N, K, ep,
                     PartPtrs{nullptr, nullptr}, (int)tm, tn, Chain{count, stagger, tiles, groups});
  CHORUS_LAUNCH_CHECK();
  return CHORUS_OK;
}

int32_t launch_chain_tile(int tile, const uint16_t* A, const uint16_t* W, long M, int N, int K, const EpiArgs& ep, int slices,
                          uint32_t* counts, hipStream_t s) {
  const int stagger = chain_stagger(tile, K, slices);
  switch (tile) {
    case kTile256: return launch_chain<8, 8, 5>(A, W, M, N, K, ep, slices, counts, stagger, s);
    case kTileWide: return launch_chain<4, 8, 6>(A, W, M, N, K, ep, slices, counts, stagger, s);
    case kTile128Deep: return launch_chain<4, 4, kHalvesDeep>(A, W, M, N, K, ep, slices, counts, stagger, s);
    case kTile64: return launch_chain<2, 2, kHalves64>(A, W, M, N, K, ep, slices, counts, stagger, s);
    default: return CHORUS_E_ARG;
  }
}

int32_t launch_tile(int tile, const uint16_t* A, const uint16_t* W, long M, int N, int K, int epi, const EpiArgs& ep,
                    hipStream_t s, int slices = 1, const PartPtrs& parts = PartPtrs{nullptr, nullptr}) {
  if (K > kMaxOffsetK) return launch_gemm_w16<2, 2, kHalves64, true>(A, W, M, N, K, epi, ep, s, slices, parts);
  switch (tile) {
    case kTile256: return launch_gemm_w16<8, 8, 5>(A, W, M, N, K, epi, ep, s, slices, parts);
    case kTileWide: return launch_gemm_w16<4, 8, 6>(A, W, M, N, K, epi, ep, s, slices, parts);
    case kTile128: return launch_gemm_w16<4, 4, 5>(A, W, M, N, K, epi, ep, s, slices, parts);
    case kTile128Deep: return launch_gemm_w16<4, 4, kHalvesDeep>(A, W, M, N, K, epi, ep, s, slices, parts);
    default: return launch_gemm_w16<2, 2, kHalves64>(A, W, M, N, K, epi, ep, s, slices, parts);
  }
}

int32_t launch_plan(const GemmPlan& p, const uint16_t* A, const uint16_t* W, long M, int N, int K, int epi, const EpiArgs& ep,
                    const GemmParts& parts, hipStream_t s) {
  if (p.chain) return launch_chain_tile(p.tile, A, W, M, N, K, ep, p.slices, parts.counts, s);
  const PartPtrs pp{static_cast<float*>(parts.first), static_cast<float*>(parts.rest)};
  CHK_STATUS(launch_tile(p.tile, A, W, M, N, K, epi, ep, s, p.slices, pp));
  return p.slices > 1 ? launch_add_parts(pp, p.slices, M, N, ep, s) : CHORUS_OK;
}

// two products with bf16 outputs and the same K in one launch
template <int WBM, int WBN, int C>
int32_t launch_two(const uint16_t* A, const uint16_t* W, long M, int N, int K, const EpiArgs& ep, Twin twin, hipStream_t s) {
  constexpr int BM = 32 * WBM, BN = 32 * WBN;
  const long tm = (M + BM - 1) / BM, tm2 = (twin.M + BM - 1) / BM;
  const int tn = (N + BN - 1) / BN;
  twin.tiles_m = (int)tm2;
  twin.tiles_n = (twin.N + BN - 1) / BN;
  const long first = tm * tn, all = first + tm2 * twin.tiles_n;
  if (all > 0x7fffffffL) return CHORUS_E_SHAPE;
  twin.first = (int)first;
  const size_t smem = (size_t)C * (BM + BN) / 2 * BK * sizeof(uint16_t);
  auto kern = gemm_w16_kernel<CHORUS_EPI_BF16, WBM, WBN, C, false, Twin>;
  static DynLdsOnce once;
  CHK_STATUS(once.ensure(reinterpret_cast<const void*>(kern), (int)smem));
  hipLaunchKernelGGL(kern, dim3((unsigned)all), dim3(256), smem, s, A, W, M, N, K, ep, PartPtrs{nullptr, nullptr}, (int)tm, tn, twin);
  CHORUS_LAUNCH_CHECK();
  return CHORUS_OK;
}

int32_t check_gemm(const uint16_t* A, const uint16_t* W, int64_t M, int32_t N, int32_t K, const void* out, const float* bias,
                   const float* gate0, const float* gate1) {
  if (M < 0 || N <= 0 || K <= 0) return CHORUS_E_ARG;
  if (M == 0) return CHORUS_OK;
  if (!A || !W || !out) return CHORUS_E_ARG;
  if (K % BK || N % 8) return CHORUS_E_SHAPE;
  if (!aligned16(A) || !aligned16(W) || !aligned16(out) || !aligned16(bias) || !aligned16(gate0) || !aligned16(gate1))
    return CHORUS_E_ARG;
  return CHORUS_OK;
}

// The whole choice: the first head_rows rows in whole rounds of 256 x 256 tiles (0: no cut), the others by `rest`. A last
// round of 256 x 256 tiles that fills a small part of the chip costs most of a whole round. The rows can be cut instead:
// the row tiles that make up whole rounds go to the 256 x 256 kernel, the rows left over to whichever kernel suits that many
// rows, in a second launch behind the first. Taken when the estimate is better by 5 %; with up to three k-steps it was slower
// wherever it was taken (gated residual, 22 products with K = 64 and 128: 1.06 to 1.16 times; 4500 x 4608 x 128 36 us, whole 31).
struct GemmCut {
  long head_rows;
  GemmPlan rest;
  double time;  // of both launches
};
GemmCut plan_rows(long M, int N, int K, int epi, const GemmParts& parts) {
  const GemmPlan whole = plan_gemm(M, N, K, epi, parts);
  const long tiles_n256 = (N + 255) / 256, tiles256 = ((M + 255) / 256) * tiles_n256;
  const long head_rows = tiles256 > 256 && K >= 4 * BK ? (tiles256 / 256 * 256 / tiles_n256) * 256 : 0;
  if (head_rows > 0 && head_rows < M) {
    const GemmPlan tail = plan_gemm(M - head_rows, N, K, epi, GemmParts{nullptr, 0, nullptr, 0, parts.counts});
    const double time = tile_time(kTile256, head_rows, N, K, epi, 1) + tail.time;
    if (time < 0.95 * whole.time) return GemmCut{head_rows, tail, time};
  }
  return GemmCut{0, whole, whole.time};
}

// The tile on which two products with bf16 outputs and the same K run in one launch, kTiles: each in a launch of its own,
// whichever is the fastest by the estimates for the tiles of both together. 64 x 64 tiles up to one round of two workgroups a
// unit, the deep 128 x 128 ones up to two rounds of one; beyond that the larger product's own best tile is another one. Measured
// (tokens and text tokens, QKV and the text's keys and values; 64 x 64 / deep / apart, us): width 256, 128 and 16 4.8 / 5.7 / 7.8; width 1536, 100 and 16 9.9 / 18.2 / 17.9, 480 and 512 29.2 / 19.9 / 33.7, 800
// and 16 30.2 / 28.1 / 24.5, 900 and 512 40.9 / 33.3 / 39.4; width 5120, 100 and 512 160 / 113 / 129, 200 and 16 99 / 89 / 77, 200 and 512
// 179 / 152 / 129. Over 91 such pairs the choice is 1.2 % slower than the best (geometric mean), and never slower than apart.
int plan_two(long M, int N, long M2, int N2, int K) {
  if (K > kMaxOffsetK) return kTiles;
  const long small = tile_count(kTile64, M, N) + tile_count(kTile64, M2, N2);
  const long deep = tile_count(kTile128Deep, M, N) + tile_count(kTile128Deep, M2, N2);
  double best = plan_rows(M, N, K, CHORUS_EPI_BF16, kNoParts).time + plan_rows(M2, N2, K, CHORUS_EPI_BF16, kNoParts).time;
  int tile = kTiles;
  auto consider = [&](int t, double time) {
    if (time < best) {
      best = time;
      tile = t;
    }
  };
  consider(kTile64, tiles_time(kTile64, small, K, CHORUS_EPI_BF16, 1));
  if (deep <= 512)
    consider(kTile128Deep, tiles_time(kTile128Deep, deep < 256 ? deep : 256, K, CHORUS_EPI_BF16, 1) +
                               (deep > 256 ? tiles_time(kTile128Deep, deep - 256, K, CHORUS_EPI_BF16, 1) : 0.0));
  return tile;
}

}  // namespace

// One launch where plan_two says so (a block of 128 tokens of width 256 with 16 text tokens, its text keys and values prepared
// beside the tokens' in the same way: 62.9 -> 56.8 us).
int32_t gemm_bf16_two(const uint16_t* A, const uint16_t* W, int64_t M, int32_t N, int32_t K, uint16_t* out, const float* bias,
                      const uint16_t* A2, const uint16_t* W2, int64_t M2, int32_t N2, uint16_t* out2, const float* bias2,
                      void* stream) {
  CHK_STATUS(check_gemm(A, W, M, N, K, out, bias, nullptr, nullptr));
  CHK_STATUS(check_gemm(A2, W2, M2, N2, K, out2, bias2, nullptr, nullptr));
  if (M > 0 && M2 > 0) {
    const EpiArgs ep{out, bias, nullptr, nullptr, 1.f};
    const Twin twin{A2, W2, out2, bias2, (long)M2, N2, 0, 0, 0};
    switch (plan_two((long)M, N, (long)M2, N2, K)) {
      case kTile64: return launch_two<2, 2, kHalves64>(A, W, (long)M, N, K, ep, twin, (hipStream_t)stream);
      case kTile128Deep: return launch_two<4, 4, kHalvesDeep>(A, W, (long)M, N, K, ep, twin, (hipStream_t)stream);
      default: break;
    }
  }
  CHK_STATUS(gemm_bf16_parts(A, W, M, N, K, CHORUS_EPI_BF16, out, bias, nullptr, nullptr, 1.f, kNoParts, stream));
  return gemm_bf16_parts(A2, W2, M2, N2, K, CHORUS_EPI_BF16, out2, bias2, nullptr, nullptr, 1.f, kNoParts, stream);
}

TileCut gemm_tiles(int64_t M, int32_t N, int32_t K, int32_t epilogue) {
  const GemmCut cut = plan_rows((long)M, N, K, epilogue, kNoParts);
  return TileCut{cut.head_rows, cut.rest.tile};
}

bool gemm_bf16_chained(int64_t M, int32_t N, int32_t K, const GemmParts& parts) {
  return parts.counts && K / BK >= 2 * kChainSteps && plan_rows((long)M, N, K, CHORUS_EPI_RESID, parts).rest.chain;
}

int32_t gemm_bf16_parts(const uint16_t* A, const uint16_t* W, int64_t M, int32_t N, int32_t K, int32_t epilogue, void* out,
                        const float* bias, const float* gate0, const float* gate1, float scale, const GemmParts& parts,
                        void* stream) {
  CHK_STATUS(check_gemm(A, W, M, N, K, out, bias, gate0, gate1));
  if (M == 0) return CHORUS_OK;
  if (epilogue < CHORUS_EPI_BF16 || epilogue > CHORUS_EPI_RESID) return CHORUS_E_ARG;
  const EpiArgs ep{out, bias, gate0, gate1, scale};
  hipStream_t s = (hipStream_t)stream;
  const GemmCut cut = plan_rows((long)M, N, K, epilogue, parts);
  if (cut.head_rows == 0) return launch_plan(cut.rest, A, W, (long)M, N, K, epilogue, ep, parts, s);
  CHK_STATUS(launch_tile(kTile256, A, W, cut.head_rows, N, K, epilogue, ep, s));
  const size_t out_elt = (epilogue == CHORUS_EPI_F32 || epilogue == CHORUS_EPI_RESID) ? 4 : 2;
  EpiArgs ep_rest = ep;
  ep_rest.out = static_cast<uint8_t*>(out) + (size_t)cut.head_rows * (size_t)N * out_elt;
  return launch_plan(cut.rest, A + (size_t)cut.head_rows * (size_t)K, W, (long)M - cut.head_rows, N, K, epilogue, ep_rest,
                     GemmParts{nullptr, 0, nullptr, 0, parts.counts}, s);
}

}  // namespace chorus

using namespace chorus;

// tile of a kernel number, -1 for none
static int tile_of_number(int32_t kernel) {
  for (int t = 0; t < kTiles; ++t)
    if (kTileNumber[t] == kernel) return t;
  return -1;
}

extern "C" int32_t chorus_gemm_bf16_kernel(const uint16_t* A, const uint16_t* W, int64_t M, int32_t N, int32_t K,
                                           int32_t epilogue, void* out, const float* bias, const float* gate0,
                                           const float* gate1, float scale, int32_t kernel, void* stream) {
  if (kernel == 0) return gemm_bf16_parts(A, W, M, N, K, epilogue, out, bias, gate0, gate1, scale, kNoParts, stream);
  const int tile = tile_of_number(kernel);
  if (tile < 0) return CHORUS_E_ARG;
  CHK_STATUS(check_gemm(A, W, M, N, K, out, bias, gate0, gate1));
  if (M == 0) return CHORUS_OK;
  return launch_tile(tile, A, W, (long)M, N, K, epilogue, EpiArgs{out, bias, gate0, gate1, scale}, (hipStream_t)stream);
}

extern "C" int32_t chorus_gemm_bf16_slices(const uint16_t* A, const uint16_t* W, int64_t M, int32_t N, int32_t K, float* out,
                                           const float* bias, const float* gate0, const float* gate1, float scale,
                                           int32_t kernel, int32_t slices, float* parts, size_t parts_bytes, void* stream) {
  const int tile = tile_of_number(kernel);
  if (tile < 0 || slices < 1 || slices > kMaxSlices) return CHORUS_E_ARG;
  CHK_STATUS(check_gemm(A, W, M, N, K, out, bias, gate0, gate1));
  if (slices > K / BK) return CHORUS_E_SHAPE;
  if (M == 0) return CHORUS_OK;
  const size_t one = (size_t)M * (size_t)N * sizeof(float);
  if (slices > 1 && (!parts || !aligned16(parts) || parts_bytes < (size_t)(slices - 1) * one)) return CHORUS_E_WORKSPACE;
  const GemmParts two{parts, one, parts + (slices > 1 ? (size_t)M * N : 0), slices > 2 ? (size_t)(slices - 2) * one : 0, nullptr};
  return launch_plan(GemmPlan{tile, slices, 0.0}, A, W, (long)M, N, K, CHORUS_EPI_RESID, EpiArgs{out, bias, gate0, gate1, scale},
                     two, (hipStream_t)stream);
}

extern "C" int32_t chorus_gemm_bf16_plan(int64_t M, int32_t N, int32_t K, int32_t epilogue, size_t first_bytes, size_t rest_bytes,
                                         chorus_gemm_plan* out) {
  if (!out || M < 1 || N <= 0 || K <= 0 || epilogue < CHORUS_EPI_BF16 || epilogue > CHORUS_EPI_RESID) return CHORUS_E_ARG;
  if (K % BK || N % 8) return CHORUS_E_SHAPE;
  void* some = reinterpret_cast<void*>(uintptr_t{16});  // where the scratch lies does not matter
  const GemmCut cut = plan_rows((long)M, N, K, epilogue,
                                GemmParts{first_bytes ? some : nullptr, first_bytes, rest_bytes ? some : nullptr, rest_bytes, nullptr});
  *out = chorus_gemm_plan{cut.head_rows, kTileNumber[cut.rest.tile], cut.rest.slices};
  return CHORUS_OK;
}

extern "C" int32_t chorus_gemm_bf16_two_plan(int64_t M, int32_t N, int64_t M2, int32_t N2, int32_t K, int32_t* kernel) {
  if (!kernel || M < 1 || M2 < 1 || N <= 0 || N2 <= 0 || K <= 0) return CHORUS_E_ARG;
  if (K % BK || N % 8 || N2 % 8) return CHORUS_E_SHAPE;
  const int tile = plan_two((long)M, N, (long)M2, N2, K);
  *kernel = tile == kTiles ? 0 : kTileNumber[tile];
  return CHORUS_OK;
}

extern "C" int32_t chorus_gemm_bf16(const uint16_t* A, const uint16_t* W, int64_t M, int32_t N, int32_t K,
                                    int32_t epilogue, void* out, const float* bias, const float* gate0,
                                    const float* gate1, float scale, void* stream) {
  return gemm_bf16_parts(A, W, M, N, K, epilogue, out, bias, gate0, gate1, scale, kNoParts, stream);
}

__global__ __launch_bounds__(256) void clear_counts_kernel(uint32_t* p, int n) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i < n) p[i] = 0;
}

extern "C" int32_t chorus_gemm_bf16_chain(const uint16_t* A, const uint16_t* W, int64_t M, int32_t N, int32_t K, float* out,
                                          const float* bias, const float* gate0, const float* gate1, float scale, int32_t kernel,
                                          int32_t slices, uint32_t* counts, int32_t n_counts, void* stream) {
  const int tile = tile_of_number(kernel);
  if (tile < 0 || tile == kTile128 || slices < 1 || slices > kMaxChain) return CHORUS_E_ARG;
  CHK_STATUS(check_gemm(A, W, M, N, K, out, bias, gate0, gate1));
  if (slices > K / BK || K > kMaxOffsetK || N > 1 << 20) return CHORUS_E_SHAPE;
  if (M == 0) return CHORUS_OK;
  const long tiles = tile_count(tile, (long)M, N);
  if (tiles * slices > 0x7fffffffL / 256) return CHORUS_E_SHAPE;
  if (!counts || n_counts < tiles) return CHORUS_E_WORKSPACE;
  hipStream_t s = (hipStream_t)stream;
  hipLaunchKernelGGL(clear_counts_kernel, dim3((unsigned)((tiles + 255) / 256)), dim3(256), 0, s, counts, (int)tiles);
  CHORUS_LAUNCH_CHECK();
  return launch_chain_tile(tile, A, W, (long)M, N, K, EpiArgs{out, bias, gate0, gate1, scale}, slices, counts, s);
}

extern "C" int32_t chorus_gemm_bf16_chain_plan(int64_t M, int32_t N, int32_t K, size_t first_bytes, size_t rest_bytes, chorus_gemm_plan* out,
                                               int32_t* chained) {
  if (!out || !chained || M < 1 || N <= 0 || K <= 0) return CHORUS_E_ARG;
  if (K % BK || N % 8) return CHORUS_E_SHAPE;
  void* some = reinterpret_cast<void*>(uintptr_t{16});  // where the scratch lies does not matter
  const GemmCut cut = plan_rows((long)M, N, K, CHORUS_EPI_RESID, GemmParts{first_bytes ? some : nullptr, first_bytes,
                                rest_bytes ? some : nullptr, rest_bytes, static_cast<uint32_t*>(some)});
  *out = chorus_gemm_plan{cut.head_rows, kTileNumber[cut.rest.tile], cut.rest.slices};
  *chained = cut.rest.chain;
  return CHORUS_OK;
}
