// Products of a few rows with weight matrices, C = A W^T: what they take is the time to read the weights, once. A workgroup has a strip of 16 rows of
// W (of both matrices with NB = 2) and all rows of A; its waves share out K, in pieces of 256 bytes of each row, and request their next piece
// before they multiply this one. Weights go from memory straight into the registers that the matrix pipe reads, 16 rows of 64 bytes an
// instruction. Nothing is shared between workgroups but A, which stays in the L2s; the waves' sums meet in LDS and are added in the order
// of the waves. Loads that leave the caches alone (non-temporal) are slower where the last-level cache holds the weights from the call before
// (20480 x 4096 37 us, so 29) and no faster where it does not.
#pragma once
#include "gemm_tile.h"

namespace chorus {

constexpr int kSkinnyRows = 32;  // most rows of A: two blocks of 16
constexpr int kSkinnyWaves = 8;   // most waves of a workgroup

template <class MMA, int NB, int MB, class OUT>
__global__ __launch_bounds__(64 * kSkinnyWaves) void skinny_kernel(const uint16_t* __restrict__ A, const uint16_t* __restrict__ W,
                                                                   const uint16_t* __restrict__ W2, int M, int N, int K, OUT out) {
#if defined(__HIP_DEVICE_COMPILE__)
  typedef typename MMA::Acc Acc;
  constexpr int U = 2;  // groups of 64 units (128 bytes) of a row in a piece
  extern __shared__ __attribute__((aligned(16))) uint8_t smem_raw[];
  Acc* const part = reinterpret_cast<Acc*>(smem_raw);  // [waves][NB MB][64]
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), waves = blockDim.x >> 6;
  const int lj = lane & 15, lg = lane >> 4;
  const int n0 = 16 * xcd_remap(blockIdx.x, gridDim.x), row = n0 + lj < N ? n0 + lj : N - 1;
  const uint16_t* w[NB];
  w[0] = W + (size_t)row * K + 8 * lg;
  if (NB == 2) w[NB - 1] = W2 + (size_t)row * K + 8 * lg;
  const uint16_t* a[MB];
  bool live[MB];
#pragma unroll
  for (int mb = 0; mb < MB; ++mb) {
    live[mb] = 16 * mb + lj < M;
    a[mb] = A + (size_t)(live[mb] ? 16 * mb + lj : 0) * K + 8 * lg;
  }
  const int groups = K / BK;
  struct Piece {
    bf16x8 w[U][2][NB], a[U][2][MB];
  };
  auto load = [&](Piece& p, int g) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int at = (g + u < groups ? g + u : groups - 1) * BK + 32 * h;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
          p.w[u][h][nb] = *reinterpret_cast<const bf16x8*>(w[nb] + at);
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
          p.a[u][h][mb] = bf16x8{};
          if (live[mb]) p.a[u][h][mb] = *reinterpret_cast<const bf16x8*>(a[mb] + at);
        }
      }
  };
  Acc acc[NB][MB];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) acc[nb][mb] = Acc{};
  const int step = waves * U;
  Piece cur, next;
  int g = wave * U;
  if (g < groups) load(cur, g);
  for (; g < groups; g += step) {
    if (g + step < groups) load(next, g + step);
#pragma unroll
    for (int u = 0; u < U && g + u < groups; ++u)  // what is behind the last group is that one again
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int mb = 0; mb < MB; ++mb) acc[nb][mb] = MMA::mma(acc[nb][mb], cur.w[u][h][nb], cur.a[u][h][mb]);
    cur = next;
  }
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) part[(wave * NB * MB + nb * MB + mb) * 64 + lane] = acc[nb][mb];
  __syncthreads();
  for (int mb = wave; mb < MB; mb += waves) {
    Acc sum[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      sum[nb] = part[(nb * MB + mb) * 64 + lane];
      for (int k = 1; k < waves; ++k) sum[nb] += part[(k * NB * MB + nb * MB + mb) * 64 + lane];
    }
    const int m = 16 * mb + lj, n = n0 + 4 * lg;
    if (m < M && n < N) out(sum, (long)m, n);
  }
#endif
}

// Whether a product of M rows goes this way, N rows of all weight matrices. The 64 x 64 tiles of the other kernels read large matrices as fast, whatever the
// rows, and take four columns' worth of fewer workgroups where they are small. us, this kernel and 64 x 64 tiles: i8, 1 row, 1536 x 8960 7.9 / 16.4,
// 4096 x 4096 7.1 / 9.4, 30720 x 5120 27.1 / 23.9; 16 rows 10.6 / 16.3, 7.1 / 9.4, 39 / 24; 32 rows 14.3 / 16.3, 8.1 / 9.3, 56 / 25; pairs of
// bf16, 1 row, 20480 x 4096 29.1 / 30.9, 27648 x 5120 51 / 44; 16 rows, 5120 x 4096 14.3 / 15.3, 20480 x 4096 36 / 31; 32 rows, 5120 x 4096 18.0 / 15.1.
inline bool skinny_rows(int64_t M, int64_t N) { return N <= (M <= 4 ? 24576 : M <= 16 ? 8192 : M <= kSkinnyRows ? 4096 : 0); }

// N = rows of each weight matrix, K in units of 2 bytes.
template <class MMA, int NB, class OUT>
int32_t launch_skinny(const uint16_t* A, const uint16_t* W, const uint16_t* W2, int M, int N, int K, const OUT& out, hipStream_t s) {
  const int strips = (N + 15) / 16, groups = K / BK;
  // waves for all units at once where the strips are few, as long as each has a piece
  int waves = strips <= 1024 ? 8 : 4;
  while (waves > 1 && waves * 2 > groups) waves /= 2;
#define SKINNY(MB)                                                                                                                       \
  {                                                                                                                                      \
    auto kern = skinny_kernel<MMA, NB, MB, OUT>;                                                                                         \
    static DynLdsOnce once;                                                                                                              \
    CHK_STATUS(once.ensure(reinterpret_cast<const void*>(kern), kSkinnyWaves * NB * MB * 1024));                                           \
    hipLaunchKernelGGL(kern, dim3((unsigned)strips), dim3(64 * waves), (size_t)waves * NB * MB * 1024, s, A, W, W2, M, N, K, out);       \
  }
  if (M <= 16) SKINNY(1)
  else SKINNY(2)
#undef SKINNY
  CHORUS_LAUNCH_CHECK();
  return CHORUS_OK;
}

}  // namespace chorus
