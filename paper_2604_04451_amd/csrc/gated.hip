// The gated half of a feed-forward block, h = act(x Wg^T) * (x Wu^T), in one kernel, and its gradients.
#include <cmath>

#include "chorus_ops.h"
#include "common.h"
#include "gemm.h"
#include "gemm_tile.h"
#include "skinny.h"

namespace chorus {
namespace {

// act(x) = x s(x), s the logistic function of x (SiLU) or of 2 sqrt(2/pi) (x + 0.044715 x^3) (GELU, tanh form)
template <int ACT>
__device__ __forceinline__ float gate_exp(float x) {  // exp of minus the logistic function's argument
  if (ACT == CHORUS_ACT_SILU) return __builtin_amdgcn_exp2f(-1.4426950408889634f * x);
  return __builtin_amdgcn_exp2f(__builtin_fmaf(x * x, -0.10294324f, -2.3022082f) * x);
}
template <int ACT>
__device__ __forceinline__ float act(float x) {
  return x * __builtin_amdgcn_rcpf(1.0f + gate_exp<ACT>(x));
}
// act(x) and act'(x) = s + x s (1 - s) r'(x), r the logistic function's argument. Beyond 16 the GELU's s (1 - s) is 0 in fp32, and r'
// is kept finite there.
template <int ACT>
__device__ __forceinline__ void act_slope(float x, float& a, float& slope) {
  const float s = __builtin_amdgcn_rcpf(1.0f + gate_exp<ACT>(x));
  a = x * s;
  float rise = a * (1.0f - s);
  if (ACT == CHORUS_ACT_GELU) {
    const float c = fminf(fmaxf(x, -16.0f), 16.0f);
    rise *= __builtin_fmaf(c * c, 0.21406445f, 1.5957691f);  // 2 sqrt(2/pi) (1 + 3 0.044715 x^2)
  }
  slope = s + rise;
}

// A projection kept for the backward pass: 16 bits with a sign, 6 of exponent and 9 behind the point. Two bits more than bf16 has, of which the
// gradients' errors come half (relative norm of dW and dX against 64 bits 0.0030 with bf16, 0.0025 so, their own rounding 0.0017), for exponents that
// projections do not reach: 2^-40 to 2^24, 0 below, NaN beyond and for what is not finite.
__device__ __forceinline__ uint32_t keep16(float v) {
  const uint32_t bits = __float_as_uint(v);
  const int t = (int)(bits & 0x7fffffffu) - (87 << 23) + (1 << 13);  // halves away from zero
  const int c = t < 0 ? 0 : t > (0x7fff << 14) ? 0x7fff << 14 : t;
  return (bits >> 16 & 0x8000u) | (uint32_t)c >> 14;
}
__device__ __forceinline__ uint32_t keep16x2(float a, float b) { return keep16(a) | keep16(b) << 16; }
__device__ __forceinline__ float kept16(uint32_t w) {  // the low half
  const uint32_t c = w & 0x7fffu;
  const uint32_t v = c == 0 ? 0 : c == 0x7fffu ? 0x7fc00000u : (c << 14) + (87u << 23);
  return __uint_as_float(v | (w & 0x8000u) << 16);
}

// ---------------------------------------------------------------------------
// Forward: gemm16_loop with tiles whose columns are 16 of the gate and 16 of the other factor in turn, so that a lane's even blocks hold
// the gate at the very places where its odd ones hold the factor, and their product needs no exchange. x is read once for both. SAVE: the two
// projections go out as well, in 16 bits, for the backward pass.
// Bound as the product of as many columns is: 512 x 10240 x 4096 68 us with the weights in the last-level cache, 1260 TFLOP/s, 80 without; 4096 x 10240 x 4096
// with SAVE 560 us, 1230 TFLOP/s, of which the three outputs' 250 MB are 50.
// ---------------------------------------------------------------------------
template <int ACT, bool SAVE, int WBM, int WBN, int C>
__global__ __launch_bounds__(256, 1) void gated_kernel(const uint16_t* __restrict__ X, const uint16_t* __restrict__ W, uint16_t* __restrict__ H,
                                                       uint16_t* __restrict__ pre, long M, int F, int K, int tiles_m, int tiles_n) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int BM = 32 * WBM, BF = 16 * WBN;  // rows and columns of h in a tile
  extern __shared__ __attribute__((aligned(1024))) uint8_t smem_raw[];
  const TilePlace at = tile_place(xcd_remap(blockIdx.x, gridDim.x), tiles_m, tiles_n, K);
  const long m0 = (long)at.m * BM;
  const int f0 = at.n * BF;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  const int rows_a = M - m0 < BM ? (int)(M - m0) : BM, rows_b = F - f0 < BF ? F - f0 : BF;
  f32x4 acc[8][8];
  gemm16_loop<MmaBf16, SecondMatrix, WBM, WBN, C, false>(acc, reinterpret_cast<uint16_t*>(smem_raw), X + m0 * K, W + (long)f0 * K,
                                                         SecondMatrix{W + (long)(F + f0) * K}, rows_a, rows_b, K, 0, K / BK, wave, lane);
  const auto keep = [](f32x4 v) {
    if (WBM == 8) asm volatile("" : "+v"(v));  // one block at a time out of the accumulators
    return make_uint2(keep16x2(v[0], v[1]), keep16x2(v[2], v[3]));
  };
  uint16_t* const cw = reinterpret_cast<uint16_t*>(smem_raw) + wave * e16_bf_wave<WBN>();
  const long m = m0 + wm * 16 * WBM;
  const int f = f0 + wn * 8 * WBN;
  if constexpr (SAVE) {
    gemm16_rows_out<WBM, WBN / 2>([&](int nb, int mb) { return keep(acc[2 * nb][mb]); }, pre, cw, m, f, M, F, 2L * F, lane);
    gemm16_rows_out<WBM, WBN / 2>([&](int nb, int mb) { return keep(acc[2 * nb + 1][mb]); }, pre + F, cw, m, f, M, F, 2L * F, lane);
  }
  const auto product = [&](int nb, int mb) {
    f32x4 g = acc[2 * nb][mb], u = acc[2 * nb + 1][mb];
    if (WBM == 8) asm volatile("" : "+v"(g), "+v"(u));  // one block at a time out of the accumulators
#pragma unroll
    for (int e = 0; e < 4; ++e) g[e] = act<ACT>(g[e]) * u[e];
    return make_uint2(pack_bf16x2(g[0], g[1]), pack_bf16x2(g[2], g[3]));
  };
  gemm16_rows_out<WBM, WBN / 2>(product, H, cw, m, f, M, F, F, lane);
#endif
}

struct Call {
  const uint16_t* X;
  const uint16_t* W;
  uint16_t* H;
  uint16_t* pre;
  int act;
};

template <int WBM, int WBN, int C>
int32_t launch_gated(const Call& c, long M, int F, int K, hipStream_t s) {
  constexpr int BM = 32 * WBM, BF = 16 * WBN;
  const long tm = (M + BM - 1) / BM;
  const int tn = (F + BF - 1) / BF;
  if (tm * tn > 0x7fffffffL / 256) return CHORUS_E_SHAPE;
  const size_t smem = (size_t)C * (BM + 2 * BF) / 2 * BK * sizeof(uint16_t);
#define GATED(ACT, SAVE)                                                                                                              \
  {                                                                                                                                   \
    auto kern = gated_kernel<ACT, SAVE, WBM, WBN, C>;                                                                                 \
    static DynLdsOnce once;                                                                                                           \
    CHK_STATUS(once.ensure(reinterpret_cast<const void*>(kern), (int)smem));                                                          \
    hipLaunchKernelGGL(kern, dim3((unsigned)(tm * tn)), dim3(256), smem, s, c.X, c.W, c.H, c.pre, M, F, K, (int)tm, tn);              \
  }
  if (c.act == CHORUS_ACT_GELU) {
    if (c.pre) GATED(CHORUS_ACT_GELU, true)
    else GATED(CHORUS_ACT_GELU, false)
  } else {
    if (c.pre) GATED(CHORUS_ACT_SILU, true)
    else GATED(CHORUS_ACT_SILU, false)
  }
#undef GATED
  CHORUS_LAUNCH_CHECK();
  return CHORUS_OK;
}

constexpr int kTile192 = kTiles;  // 256 x 192, here alone

int32_t launch_gated_tile(int tile, const Call& c, long M, int F, int K, hipStream_t s) {
  switch (tile) {
    case kTile192: return launch_gated<8, 6, 5>(c, M, F, K, s);
    case kTile256: return launch_gated<8, 8, 5>(c, M, F, K, s);
    case kTileWide: return launch_gated<4, 8, 6>(c, M, F, K, s);
    case kTile128: return launch_gated<4, 4, 5>(c, M, F, K, s);
    case kTile128Deep: return launch_gated<4, 4, kHalvesDeep>(c, M, F, K, s);
    default: return launch_gated<2, 2, kHalves64>(c, M, F, K, s);
  }
}

// One round of 256 x 256 tiles that leaves units without one is a round of 256 x 192 tiles where all of those have a unit (F = 10240, K = 4096, 512
// rows, weights in the last-level cache: 160 tiles 75 us, 214 of these 68; not there: 85 and 80; 2048 x 2560 x 4096 75 and 67, x 1024 25 and 22). In all other products of 80 (M 100 to 3000, F 1024 to 13824) the
// choice by the estimates was the faster or as fast.
TileCut gated_tiles(int64_t M, int32_t F, int32_t K) {
  TileCut cut = gemm_tiles(M, 2 * F, K, CHORUS_EPI_GELU_BF16);
  if (cut.head_rows == 0 && cut.tile == kTile256 && (M + 255) / 256 * ((F + 95) / 96) <= 256) cut.tile = kTile192;
  return cut;
}

// few rows: the wave that joins a strip's sums
template <int ACT>
struct StripGated {
  uint16_t* H;
  uint16_t* pre;
  int F;
  __device__ __forceinline__ void operator()(const f32x4 (&sum)[2], long m, int f) const {
    const auto keep = [](uint16_t* at, const f32x4& v) { *reinterpret_cast<uint2*>(at) = make_uint2(keep16x2(v[0], v[1]), keep16x2(v[2], v[3])); };
    f32x4 h;
#pragma unroll
    for (int e = 0; e < 4; ++e) h[e] = act<ACT>(sum[0][e]) * sum[1][e];
    *reinterpret_cast<uint2*>(H + m * F + f) = make_uint2(pack_bf16x2(h[0], h[1]), pack_bf16x2(h[2], h[3]));
    if (pre) {
      keep(pre + m * 2 * F + f, sum[0]);
      keep(pre + (m * 2 + 1) * F + f, sum[1]);
    }
  }
};

// ---------------------------------------------------------------------------
// Backward. d = [dh u act'(g) | dh act(g)] as rows for dx = d W and as columns for dW = d^T x; W and x as columns too, so that both
// gradients are products of rows like every other one. All three are moves of memory: a wave has a tile of 64 x 64 values, a lane 8 x 8
// of them, which change places in its registers; a row of a tile is a line of 128 bytes on either side. 4096 x 10240 x 4096: 177 us, 5.6 TB/s; the two
// products behind it 470 and 500 us, 1460 and 1370 TFLOP/s.
// ---------------------------------------------------------------------------
// 8 rows of 8 values of bf16 in a lane's registers: rows to columns
__device__ __forceinline__ void transpose8(u32x4 (&x)[8]) {
  // 2 x 2 blocks of values, then of pairs, then of four
  uint32_t t[8][4];
#pragma unroll
  for (int r = 0; r < 8; r += 2)
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      t[r][c] = __builtin_amdgcn_perm(x[r + 1][c], x[r][c], 0x05040100);      // values 2c of both rows
      t[r + 1][c] = __builtin_amdgcn_perm(x[r + 1][c], x[r][c], 0x07060302);  // values 2c + 1
    }
  // t[2i + p][c]: rows 2i, 2i + 1 of column 2c + p
#pragma unroll
  for (int c = 0; c < 4; ++c)
#pragma unroll
    for (int p = 0; p < 2; ++p) x[2 * c + p] = u32x4{t[p][c], t[2 + p][c], t[4 + p][c], t[6 + p][c]};
}

// A transposition: rows [R, C] (R rows that count) -> columns [C, Rp], zeros behind R; C % 64 == 0, Rp % 64 == 0
struct Turn {
  const uint16_t* in;
  uint16_t* out;
  long R, Rp;
  int C;
  long tiles;  // Rp / 64 * C / 64, 0: none
};
__device__ __forceinline__ void turn_tile(const Turn& t, long tile, int lane) {
  const int a = lane >> 3, b = lane & 7, tiles_c = t.C / 64;
  const long r0 = tile / tiles_c * 64 + 8 * a;
  const int c0 = (int)(tile % tiles_c) * 64 + 8 * b;
  u32x4 x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = *reinterpret_cast<const u32x4*>(t.in + (r0 + i < t.R ? r0 + i : t.R - 1) * t.C + c0);
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (r0 + i >= t.R) x[i] = u32x4{0, 0, 0, 0};
  transpose8(x);
#pragma unroll
  for (int i = 0; i < 8; ++i) *reinterpret_cast<u32x4*>(t.out + (c0 + i) * t.Rp + r0) = x[i];
}

// All that the two products want laid out, in one launch: the gradients of the projections first, then W and x as columns.
struct Slopes {
  const uint16_t* pre;
  const uint16_t* dH;
  uint16_t* d;
  uint16_t* dt;
  long M, Mp, tiles;
  int F;
};
template <int ACT>
__global__ __launch_bounds__(256) void gated_layout_kernel(Slopes s, Turn w, Turn x) {
  long tile = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, a = lane >> 3, b = lane & 7;
  if (tile >= s.tiles) {
    tile -= s.tiles;
    if (tile < w.tiles) return turn_tile(w, tile, lane);
    tile -= w.tiles;
    if (tile < x.tiles) turn_tile(x, tile, lane);
    return;
  }
  const int F = s.F, tiles_f = F / 64;
  const long m0 = tile / tiles_f * 64 + 8 * a;
  const int f = (int)(tile % tiles_f) * 64 + 8 * b;
  u32x4 h[8], dg[8], du[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {  // rows behind the last are the last one, until they are zeros
    const long m = m0 + i < s.M ? m0 + i : s.M - 1;
    h[i] = *reinterpret_cast<const u32x4*>(s.dH + m * F + f);
    dg[i] = *reinterpret_cast<const u32x4*>(s.pre + m * 2 * F + f);
    du[i] = *reinterpret_cast<const u32x4*>(s.pre + (m * 2 + 1) * F + f);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const bool live = m0 + i < s.M;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float vg[2], vu[2];
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const float dh = __uint_as_float(p ? h[i][e] & 0xffff0000u : h[i][e] << 16);
        float value, slope;
        act_slope<ACT>(kept16(dg[i][e] >> 16 * p), value, slope);
        vg[p] = dh * kept16(du[i][e] >> 16 * p) * slope;
        vu[p] = dh * value;
      }
      dg[i][e] = live ? pack_bf16x2(vg[0], vg[1]) : 0;
      du[i][e] = live ? pack_bf16x2(vu[0], vu[1]) : 0;
    }
    if (live) {
      *reinterpret_cast<u32x4*>(s.d + (m0 + i) * 2 * F + f) = dg[i];
      *reinterpret_cast<u32x4*>(s.d + ((m0 + i) * 2 + 1) * F + f) = du[i];
    }
  }
  transpose8(dg);
  transpose8(du);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    *reinterpret_cast<u32x4*>(s.dt + (long)(f + i) * s.Mp + m0) = dg[i];
    *reinterpret_cast<u32x4*>(s.dt + (long)(F + f + i) * s.Mp + m0) = du[i];
  }
}

// Where a backward pass keeps what it lays out, in bytes from the workspace's start.
struct Layout {
  size_t d, dt, xt, wt, all;
  Layout(int64_t M, int32_t F, int32_t K) {
    const size_t mp = align_up((size_t)M, 64);
    d = 0;
    dt = d + align_up((size_t)M * 2 * (size_t)F * 2, 256);
    xt = dt + align_up(mp * 2 * (size_t)F * 2, 256);
    wt = xt + align_up(mp * (size_t)K * 2, 256);
    all = wt + align_up((size_t)2 * (size_t)F * (size_t)K * 2, 256);
  }
};

// Limits on sizes: a tile's bytes are within the 32-bit offsets of its loads, a launch of 64 x 64 tiles, a wave each, within 2^32 threads.
constexpr int kMostWidth = 1 << 20;
constexpr int64_t kMostTokens = 1 << 22, kMostTiles = 1 << 25;

int32_t check_gated(int64_t M, int32_t F, int32_t K, int32_t act) {
  if (M < 0 || F <= 0 || K <= 0 || (act != CHORUS_ACT_GELU && act != CHORUS_ACT_SILU)) return CHORUS_E_ARG;
  if (K % 64 || F % 64 || K > kMostWidth || F > kMostWidth || M > kMostTokens) return CHORUS_E_SHAPE;
  return CHORUS_OK;
}

}  // namespace
}  // namespace chorus

using namespace chorus;

extern "C" {

int32_t chorus_gated_ffn(const uint16_t* X, const uint16_t* W, int32_t act, uint16_t* H, uint16_t* pre, int64_t M, int32_t F, int32_t K, void* stream) {
  CHK_STATUS(check_gated(M, F, K, act));
  if (M == 0) return CHORUS_OK;
  if (!X || !W || !H || !aligned16(X) || !aligned16(W) || !aligned16(H) || !aligned16(pre)) return CHORUS_E_ARG;
  hipStream_t s = (hipStream_t)stream;
  if (skinny_rows(M, 2L * F)) {
    const uint16_t* W2 = W + (size_t)F * K;
    if (act == CHORUS_ACT_GELU) return launch_skinny<MmaBf16, 2>(X, W, W2, (int)M, F, K, StripGated<CHORUS_ACT_GELU>{H, pre, F}, s);
    return launch_skinny<MmaBf16, 2>(X, W, W2, (int)M, F, K, StripGated<CHORUS_ACT_SILU>{H, pre, F}, s);
  }
  const TileCut cut = gated_tiles(M, F, K);
  if (cut.head_rows) CHK_STATUS(launch_gated_tile(kTile256, Call{X, W, H, pre, act}, cut.head_rows, F, K, s));
  const size_t head = (size_t)cut.head_rows;
  return launch_gated_tile(cut.tile, Call{X + head * K, W, H + head * F, pre ? pre + head * 2 * F : nullptr, act}, (long)M - cut.head_rows, F, K, s);
}

int32_t chorus_gated_ffn_plan(int64_t M, int32_t F, int32_t K, chorus_gemm_plan* out) {
  CHK_STATUS(check_gated(M, F, K, CHORUS_ACT_GELU));
  if (!out || M == 0) return CHORUS_E_ARG;
  *out = chorus_gemm_plan{0, 0, 1};
  if (skinny_rows(M, 2L * F)) return CHORUS_OK;
  const TileCut cut = gated_tiles(M, F, K);
  out->head_rows = cut.head_rows;
  out->kernel = cut.tile == kTile192 ? 6 : kTileNumber[cut.tile];
  return CHORUS_OK;
}

size_t chorus_gated_ffn_backward_workspace_bytes(int64_t M, int32_t F, int32_t K) {
  return M < 1 || check_gated(M, F, K, CHORUS_ACT_GELU) != CHORUS_OK ? 0 : Layout(M, F, K).all;
}

int32_t chorus_gated_ffn_backward(const uint16_t* X, const uint16_t* W, const uint16_t* pre, const uint16_t* dH, int32_t act, uint16_t* dX, void* dW,
                                  int32_t dw_epilogue, int64_t M, int32_t F, int32_t K, void* ws, size_t ws_bytes, void* stream) {
  CHK_STATUS(check_gated(M, F, K, act));
  if (dw_epilogue != CHORUS_EPI_BF16 && dw_epilogue != CHORUS_EPI_F32 && dw_epilogue != CHORUS_EPI_RESID) return CHORUS_E_ARG;
  if (M == 0) return CHORUS_E_SHAPE;
  if (!X || !W || !pre || !dH || !aligned16(X) || !aligned16(W) || !aligned16(pre) || !aligned16(dH) || !aligned16(dX) || !aligned16(dW) || !aligned16(ws))
    return CHORUS_E_ARG;
  const Layout at(M, F, K);
  if (!ws || ws_bytes < at.all) return CHORUS_E_WORKSPACE;
  hipStream_t s = (hipStream_t)stream;
  uint8_t* const base = static_cast<uint8_t*>(ws);
  uint16_t* const d = reinterpret_cast<uint16_t*>(base + at.d);
  uint16_t* const dt = reinterpret_cast<uint16_t*>(base + at.dt);
  uint16_t* const xt = reinterpret_cast<uint16_t*>(base + at.xt);
  uint16_t* const wt = reinterpret_cast<uint16_t*>(base + at.wt);
  const long mp = (long)align_up((size_t)M, 64);
  const Slopes slopes{pre, dH, d, dt, (long)M, mp, mp / 64 * (F / 64), F};
  const Turn w{W, wt, 2L * F, 2L * F, K, dX ? 2L * F / 64 * (K / 64) : 0}, x{X, xt, (long)M, mp, K, dW ? mp / 64 * (K / 64) : 0};
  if (slopes.tiles + w.tiles + x.tiles > kMostTiles) return CHORUS_E_SHAPE;
  const dim3 grid((unsigned)((slopes.tiles + w.tiles + x.tiles + 3) / 4));
  if (act == CHORUS_ACT_GELU)
    hipLaunchKernelGGL(gated_layout_kernel<CHORUS_ACT_GELU>, grid, dim3(256), 0, s, slopes, w, x);
  else
    hipLaunchKernelGGL(gated_layout_kernel<CHORUS_ACT_SILU>, grid, dim3(256), 0, s, slopes, w, x);
  CHORUS_LAUNCH_CHECK();
  const GemmParts none{nullptr, 0, nullptr, 0, nullptr};
  if (dX) CHK_STATUS(gemm_bf16_parts(d, wt, M, K, 2 * F, CHORUS_EPI_BF16, dX, nullptr, nullptr, nullptr, 1.f, none, s));
  if (dW) CHK_STATUS(gemm_bf16_parts(dt, xt, 2L * F, K, (int)mp, dw_epilogue, dW, nullptr, nullptr, nullptr, 1.f, none, s));
  return CHORUS_OK;
}

}  // extern "C"
