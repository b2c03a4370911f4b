// Which blocks of keys a block of queries attends to: means over blocks of rows, and from the means of queries and keys the choice.
#include "chorus_ops.h"
#include "common.h"

namespace chorus {
namespace {

// Mean over blocks of `block` consecutive rows of a head, a wave a block: a lane sums one chunk of eight values of every 64 / (dh / 8)-th
// row, then the lanes of a chunk are added. HBM-bound: each row is read once, 16 bytes a lane.
template <int DH>
__global__ __launch_bounds__(256) void block_mean_kernel(const uint16_t* __restrict__ X, uint16_t* __restrict__ out, long L, long Lpad,
                                                         int block, long nb, long total) {
  constexpr int LANES = DH / 8, ROWS = 64 / LANES;
  const int lane = threadIdx.x & 63;
  const long id = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (id >= total) return;
  const long head = id / nb, b = id - head * nb;
  const long first = b * block;
  const int n = (int)(L - first < block ? L - first : block);
  const uint16_t* x = X + (head * Lpad + first) * DH + lane * 8;
  float s[8] = {};
  for (int r = lane / LANES, i = 0; r < n; r += ROWS, ++i) {
    const u32x4 u = *reinterpret_cast<const u32x4*>(x + (long)i * ROWS * DH);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      s[2 * k] += __uint_as_float(u[k] << 16);
      s[2 * k + 1] += __uint_as_float(u[k] & 0xffff0000u);
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if (LANES == 8) s[e] += row_rotate<8>(s[e]);
    s[e] += swap_rows16(s[e]);
    s[e] += swap_halves(s[e]);
  }
  if (lane < LANES) {
    u32x4 o;
#pragma unroll
    for (int k = 0; k < 4; ++k) o[k] = pack_bf16x2(s[2 * k] / (float)n, s[2 * k + 1] / (float)n);
    *reinterpret_cast<u32x4*>(out + (head * nb + b) * DH + lane * 8) = o;
  }
}

// Order-preserving bits of a score: NaN below every number, both zeros alike.
__device__ __forceinline__ uint64_t ordered(double s) {
  if (s != s) return 0;
  const uint64_t b = __builtin_bit_cast(uint64_t, s + 0.0);
  return b >> 63 ? ~b : b | (1ull << 63);
}

// A workgroup a row: the scores in fp64 (products of bf16 are exact there, and 128 of them add up without a rounding unless they are
// 2^30 apart), then one wave finds the keep-th of them bit by bit and writes the blocks above it and the first ones that equal it.
__global__ __launch_bounds__(256) void block_select_kernel(const uint16_t* __restrict__ Qm, const uint16_t* __restrict__ Km,
                                                           const uint8_t* __restrict__ rule, int* __restrict__ blocks, long nq, int nk,
                                                           int group, int dh, int keep) {
  extern __shared__ __attribute__((aligned(16))) uint8_t s_raw[];
  uint64_t* key = reinterpret_cast<uint64_t*>(s_raw);
  const long row = blockIdx.x, head = row / nq;
  const uint16_t* q = Qm + row * dh;
  const uint16_t* km = Km + head / group * nk * dh;
  for (int b = threadIdx.x; b < nk; b += 256) {
    double s = 0.0;
    for (int d = 0; d < dh; ++d) s = __builtin_fma((double)bf16_to_f32(q[d]), (double)bf16_to_f32(km[(long)b * dh + d]), s);
    key[b] = ordered(s);
  }
  __syncthreads();
  if (threadIdx.x >= 64) return;
  const int lane = threadIdx.x;
  int* to = blocks + row * keep;
  auto cls = [&](int b) { return rule ? (int)rule[b] : 0; };
  auto count = [&](auto of) {
    int n = 0;
    for (int b = lane; b < nk; b += 64) n += of(b);
    return wave_sum_i32(n);
  };
  const int always = count([&](int b) { return cls(b) == 1; }), plain = count([&](int b) { return cls(b) != 1 && cls(b) != 2; });
  // the class that the choice cuts, and how many of it are kept
  const int cut = always >= keep ? 1 : 0;
  int want = cut ? keep : keep - always;
  if (!cut && want > plain) want = plain;
  auto in_cut = [&](int b) { return cut ? cls(b) == 1 : cls(b) != 1 && cls(b) != 2; };
  uint64_t t = 0;  // the largest value that at least `want` of the class reach
  for (int bit = 63; bit >= 0; --bit) {
    const uint64_t up = t | (1ull << bit);
    if (count([&](int b) { return in_cut(b) && key[b] >= up; }) >= want) t = up;
  }
  int equal = want - count([&](int b) { return in_cut(b) && key[b] > t; });  // how many that equal it are kept
  int at = 0;
  for (int b0 = 0; b0 < nk; b0 += 64) {
    const int b = b0 + lane;
    const bool of = b < nk && in_cut(b), tie = of && key[b] == t;
    const uint64_t below = (1ull << lane) - 1, ties = __ballot(tie);
    const bool take = (b < nk && !cut && cls(b) == 1) || (of && key[b] > t) || (tie && __builtin_popcountll(ties & below) < equal);
    const uint64_t taken = __ballot(take);
    if (take) to[at + __builtin_popcountll(taken & below)] = b;
    at += __builtin_popcountll(taken);
    equal -= __builtin_popcountll(ties);
  }
  for (int i = at + lane; i < keep; i += 64) to[i] = -1;
}

}  // namespace
}  // namespace chorus

using namespace chorus;

extern "C" {

int32_t chorus_block_mean(const uint16_t* X, uint16_t* out, int64_t L, int64_t Lpad, int32_t H, int32_t dh, int32_t block, void* stream) {
  if (L < 0 || Lpad < L || H <= 0) return CHORUS_E_ARG;
  if ((dh != 64 && dh != 128) || (block != CHORUS_BLOCK_QUERIES && block != CHORUS_BLOCK_KEYS)) return CHORUS_E_SHAPE;
  if (L == 0) return CHORUS_OK;
  if (!X || !out || !aligned16(X) || !aligned16(out)) return CHORUS_E_ARG;
  const int64_t nb = (L + block - 1) / block;
  if (nb > 0x7fffffffL) return CHORUS_E_SHAPE;
  const int64_t total = nb * H, groups = (total + 3) / 4;
  if (groups > 0x7fffffffL) return CHORUS_E_SHAPE;
  const dim3 grid((unsigned)groups);
  if (dh == 128)
    hipLaunchKernelGGL(block_mean_kernel<128>, grid, dim3(256), 0, (hipStream_t)stream, X, out, (long)L, (long)Lpad, block, (long)nb, (long)total);
  else
    hipLaunchKernelGGL(block_mean_kernel<64>, grid, dim3(256), 0, (hipStream_t)stream, X, out, (long)L, (long)Lpad, block, (long)nb, (long)total);
  CHORUS_LAUNCH_CHECK();
  return CHORUS_OK;
}

int32_t chorus_block_select(const uint16_t* Qm, const uint16_t* Km, const uint8_t* rule, int32_t* blocks, int64_t nq, int64_t nk, int32_t H,
                            int32_t Hk, int32_t dh, int32_t keep, void* stream) {
  if (nq < 0 || nk < 0 || H <= 0 || Hk <= 0 || keep < 1) return CHORUS_E_ARG;
  if (H % Hk || (dh != 64 && dh != 128) || nk < 1 || nk > CHORUS_BLOCK_SELECT_MAX) return CHORUS_E_SHAPE;
  if (nq > 0x7fffffffL / H) return CHORUS_E_SHAPE;
  if (nq == 0) return CHORUS_OK;
  if (!Qm || !Km || !blocks || !aligned16(Qm) || !aligned16(Km) || !aligned16(blocks) || !aligned16(rule)) return CHORUS_E_ARG;
  static DynLdsOnce once;
  const size_t lds = (size_t)nk * sizeof(uint64_t);
  CHK_STATUS(once.ensure((const void*)block_select_kernel, CHORUS_BLOCK_SELECT_MAX * sizeof(uint64_t)));
  hipLaunchKernelGGL(block_select_kernel, dim3((unsigned)(nq * H)), dim3(256), lds, (hipStream_t)stream, Qm, Km, rule, blocks, (long)nq, (int)nk,
                     H / Hk, dh, keep);
  CHORUS_LAUNCH_CHECK();
  return CHORUS_OK;
}

}  // extern "C"
