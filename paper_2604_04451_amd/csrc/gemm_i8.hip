// Products of 8-bit integers with a scale for each row of either operand (each token and each output channel), and the quantisation
// of the rows: c = round(127 x / max|x|), y[m][n] = (sum_k c[m][k] w[n][k]) a[m] b[n]. The sums are whole numbers in 32 bits and so
// exact; the scales go in behind them, in fp32.
#include "chorus_ops.h"
#include "common.h"
#include "gemm.h"
#include "gemm_tile.h"
#include "skinny.h"

namespace chorus {
namespace {

constexpr int kStep = 128;              // values of a k-step: the 128 bytes that 64 of bf16 take
constexpr int kMostK = 131072 - kStep;  // 128 * 128 * K stays below 2^31
constexpr int kMostN = 1 << 24;         // sums of tiles and columns stay within 32 bits
constexpr float kTiny = 0x1p-100f, kHuge = 0x1p100f;

// ---------------------------------------------------------------------------
// Rows to codes: T threads a row, which stays in their registers between the search of its largest value and the rounding (V pieces
// of 8 values a thread; longer rows are read twice). One read, half as much written; memory bound: 32760 x 1536 34 us, 13103 x 8960 67, 4.4 and 5.3 TB/s with
// the codes, in a row of calls (in a trace of few of them 38 and 86); one row 4 us. The tokens are read past the caches, which have the codes for the product
// then: 67 and, for the product to fp32, 160 us each in a row of its own, 213 to 222 by card both in turn, 224 with tokens read as usual.
// The code is the whole number nearest to 127 x / max, halves to even, as if that quotient were exact. fp32 brings q = x (127 / max)
// to within 1.5 units in the last place, so that round(q) is off by one at most, near a half. What is left, 127 x - q max, is exact in an
// fma: 127 x and q max have 15 bits each, and for q != 0 their units are at most 2^9 apart. It is compared with max / 2.
// ---------------------------------------------------------------------------
struct RowScale {
  float max, by;  // 127 / max
};
__device__ __forceinline__ int code_of(float x, const RowScale& r) {
  const float q = __builtin_rintf(x * r.by);
  const float left = 2.0f * __builtin_fmaf(-q, r.max, 127.0f * x);
  const float away = __builtin_fabsf(left);
  const int n = (int)q, one = left < 0.f ? -1 : 1;
  return away > r.max || (away == r.max && (n & 1)) ? n + one : n;
}

template <int T, int V>
__global__ __launch_bounds__(256) void quant_rows_kernel(const uint16_t* __restrict__ X, long ld, int8_t* __restrict__ out, float* __restrict__ scale,
                                                         long M, int K, int Kp) {
  constexpr int ROWS = 256 / T;
  const int tid = threadIdx.x, at = tid % T;
  const long m = (long)blockIdx.x * ROWS + tid / T;
  if (T == 64 && m >= M) return;
  const u32x4* x = reinterpret_cast<const u32x4*>(X + m * ld);
  const int pieces = K / 8, padded = Kp / 8;
  u32x4 v[V];
  // the largest magnitude by its bits, which order as the values do; infinities and NaN are above all finite ones
  uint32_t most = 0;
  auto see = [&](const u32x4& p) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t lo = (p[e] << 16) & 0x7fffffffu, hi = p[e] & 0x7fff0000u;
      most = lo > most ? lo : most;
      most = hi > most ? hi : most;
    }
  };
#pragma unroll
  for (int i = 0; i < V; ++i) {
    v[i] = u32x4{0, 0, 0, 0};
    if (at + i * T < pieces) v[i] = __builtin_nontemporal_load(x + at + i * T);
    see(v[i]);
  }
  for (int p = at + V * T; p < pieces; p += T) see(x[p]);
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    const uint32_t o = (uint32_t)__shfl_xor((int)most, d);
    most = o > most ? o : most;
  }
  if (T > 64) {
    __shared__ uint32_t part[4];
    if ((tid & 63) == 0) part[tid >> 6] = most;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 4; ++w) most = part[w] > most ? part[w] : most;
  }
  const bool finite = most < 0x7f800000u;
  const float top = __uint_as_float(most);
  if (at == 0) scale[m] = finite ? top / 127.0f : __uint_as_float(0x7fc00000u);
  // far ends of the range by a power of two nearer to its middle, the values with them
  const float shift = top < kTiny ? kHuge : top > kHuge ? kTiny : 1.0f;
  RowScale r;
  r.max = top * shift;
  r.by = 127.0f / r.max;
  const bool plain = finite && most != 0;
  uint2* o = reinterpret_cast<uint2*>(out + m * Kp);
  auto put = [&](int p, const u32x4& a) {
    uint2 w = make_uint2(0, 0);
    if (plain && p < pieces) {
      uint32_t c[8];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        c[2 * e] = (uint32_t)code_of(__uint_as_float(a[e] << 16) * shift, r);
        c[2 * e + 1] = (uint32_t)code_of(__uint_as_float(a[e] & 0xffff0000u) * shift, r);
      }
      w.x = (c[0] & 255) | (c[1] & 255) << 8 | (c[2] & 255) << 16 | c[3] << 24;
      w.y = (c[4] & 255) | (c[5] & 255) << 8 | (c[6] & 255) << 16 | c[7] << 24;
    }
    o[p] = w;
  };
#pragma unroll
  for (int i = 0; i < V; ++i)
    if (at + i * T < padded) put(at + i * T, v[i]);
  for (int p = at + V * T; p < padded; p += T) put(p, p < pieces ? x[p] : u32x4{0, 0, 0, 0});
}

// ---------------------------------------------------------------------------
// The product: gemm16_loop with 8-bit operands, which takes 128 values in the bytes of 64. The scales go into the sums before the
// epilogue of the bf16 product, which adds the bias, takes the GELU or adds to the residual.
// Bound by the delivery of the operands, and by the epilogue where K is short, which nothing of the loop runs beside: 32760 x 8960 x 1536 with GELU 495 us,
// 1820 TOP/s (the loop alone 2870 TOP/s, GELU and its conversions 63 us, all of the epilogue 170), in bf16 774; 13103 x 1536 x 8960 to fp32 157 to 160 us, 2270
// TOP/s, with the gated residual 166, in bf16 302 and 304; 32760 x 1536 x 8960 with the gated residual 364, in bf16 670. Other tiles for either, and for 512 x 1536 x 4096 (11 us), were no faster.
// ---------------------------------------------------------------------------
template <int EPI, int WBM, int WBN, int C>
__global__ __launch_bounds__(256, 1) void gemm_i8_kernel(const uint16_t* __restrict__ A, const uint16_t* __restrict__ W, long M, int N, int K,
                                                         const float* __restrict__ a_scale, const float* __restrict__ w_scale, EpiArgs ep,
                                                         int tiles_m, int tiles_n) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int BM = 32 * WBM, BN = 32 * WBN, WTM = 16 * WBM, WTN = 16 * WBN;
  extern __shared__ __attribute__((aligned(1024))) uint8_t smem_raw[];
  const TilePlace at = tile_place(xcd_remap(blockIdx.x, gridDim.x), tiles_m, tiles_n, K);
  const long m0 = (long)at.m * BM;
  const int n0 = at.n * BN;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 1, wn = wave & 1, lj = lane & 15, lg = lane >> 4;
  const int rows_a = M - m0 < BM ? (int)(M - m0) : BM, rows_b = N - n0 < BN ? N - n0 : BN;
  i32x4 sums[8][8];
  gemm16_loop<MmaI8, OneMatrix, WBM, WBN, C, false>(sums, reinterpret_cast<uint16_t*>(smem_raw), A + m0 * K, W + (long)n0 * K, OneMatrix{}, rows_a,
                                                    rows_b, K, 0, K / BK, wave, lane);
  float as[8];
#pragma unroll
  for (int mb = 0; mb < WBM; ++mb) {
    const long m = m0 + wm * WTM + 16 * mb + lj;
    as[mb] = a_scale[m < M ? m : M - 1];
  }
  const auto scale_of = [&](int nb) {
    const int n = n0 + wn * WTN + 16 * nb + 4 * lg;
    return *reinterpret_cast<const f32x4*>(w_scale + (n < N ? n : 0));
  };
  const auto scaled = [&](int nb, int mb, const f32x4& ws) {
    i32x4 of = sums[nb][mb];
    if (WBM == 8) asm volatile("" : "+v"(of));  // turned into floats here: all at once, ahead of the stores, they spilled 16 to 40 bytes a lane
    f32x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = (float)of[e] * as[mb] * ws[e];
    return v;
  };
  if constexpr (EPI == CHORUS_EPI_F32) {
    // a lane stores its four consecutive columns of every block
#pragma unroll
    for (int nb = 0; nb < WBN; ++nb) {
      const int n = n0 + wn * WTN + 16 * nb + 4 * lg;
      if (n >= N) continue;
      const f32x4 ws = scale_of(nb);
      f32x4 bias = {0.f, 0.f, 0.f, 0.f};
      if (ep.bias) bias = *reinterpret_cast<const f32x4*>(ep.bias + n);
#pragma unroll
      for (int mb = 0; mb < WBM; ++mb) {
        const long m = m0 + wm * WTM + 16 * mb + lj;
        if (m < M) *reinterpret_cast<f32x4*>(static_cast<float*>(ep.out) + m * N + n) = scaled(nb, mb, ws) + bias;
      }
    }
  } else {
    f32x4 ws[8];
#pragma unroll
    for (int nb = 0; nb < WBN; ++nb) ws[nb] = scale_of(nb);
    gemm16_finish<EPI, WBM, WBN>([&](int nb, int mb) { return scaled(nb, mb, ws[nb]); }, ep, smem_raw, wave, wm, wn, m0, n0, M, N, lane);
  }
#endif
}

struct Operands {
  const uint16_t* A;
  const uint16_t* W;
  const float* a_scale;
  const float* w_scale;
};

template <int WBM, int WBN, int C>
int32_t launch_i8(const Operands& x, long M, int N, int K, int epi, const EpiArgs& ep, hipStream_t s) {
  constexpr int BM = 32 * WBM, BN = 32 * WBN;
  const long tm = (M + BM - 1) / BM;
  const int tn = (N + BN - 1) / BN;
  if (tm * tn > 0x7fffffffL / 256) return CHORUS_E_SHAPE;
  const size_t smem = (size_t)C * (BM + BN) / 2 * BK * sizeof(uint16_t);
#define GEMM_I8(E)                                                                                                                        \
  {                                                                                                                                       \
    auto kern = gemm_i8_kernel<E, WBM, WBN, C>;                                                                                           \
    static DynLdsOnce once;                                                                                                               \
    CHK_STATUS(once.ensure(reinterpret_cast<const void*>(kern), (int)smem));                                                              \
    hipLaunchKernelGGL(kern, dim3((unsigned)(tm * tn)), dim3(256), smem, s, x.A, x.W, M, N, K, x.a_scale, x.w_scale, ep, (int)tm, tn);    \
  }
  switch (epi) {
    case CHORUS_EPI_BF16: GEMM_I8(CHORUS_EPI_BF16); break;
    case CHORUS_EPI_GELU_BF16: GEMM_I8(CHORUS_EPI_GELU_BF16); break;
    case CHORUS_EPI_F32: GEMM_I8(CHORUS_EPI_F32); break;
    default: GEMM_I8(CHORUS_EPI_RESID); break;
  }
#undef GEMM_I8
  CHORUS_LAUNCH_CHECK();
  return CHORUS_OK;
}

int32_t launch_i8_tile(int tile, const Operands& x, long M, int N, int K, int epi, const EpiArgs& ep, hipStream_t s) {
  switch (tile) {
    case kTile256: return launch_i8<8, 8, 5>(x, M, N, K, epi, ep, s);
    case kTileWide: return launch_i8<4, 8, 6>(x, M, N, K, epi, ep, s);
    case kTile128: return launch_i8<4, 4, 5>(x, M, N, K, epi, ep, s);
    case kTile128Deep: return launch_i8<4, 4, kHalvesDeep>(x, M, N, K, epi, ep, s);
    default: return launch_i8<2, 2, kHalves64>(x, M, N, K, epi, ep, s);
  }
}

// Few rows: what is left to the wave that joins the sums of a strip of 16 columns.
template <int EPI>
struct StripI8 {
  const float* a_scale;
  const float* w_scale;
  EpiArgs ep;
  int N;
  __device__ __forceinline__ void operator()(const i32x4 (&sum)[1], long m, int n) const {
    const float as = a_scale[m];
    const f32x4 ws = *reinterpret_cast<const f32x4*>(w_scale + n);
    f32x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = (float)sum[0][e] * as * ws[e];
    if (ep.bias) v += *reinterpret_cast<const f32x4*>(ep.bias + n);
    if constexpr (EPI == CHORUS_EPI_BF16 || EPI == CHORUS_EPI_GELU_BF16) {
      if constexpr (EPI == CHORUS_EPI_GELU_BF16) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = gelu_tanh_fast(v[e]);
      }
      *reinterpret_cast<uint2*>(static_cast<uint16_t*>(ep.out) + m * N + n) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
    } else {
      f32x4* o = reinterpret_cast<f32x4*>(static_cast<float*>(ep.out) + m * N + n);
      if constexpr (EPI == CHORUS_EPI_RESID) {
        f32x4 gate = {1.f, 1.f, 1.f, 1.f};
        if (ep.gate0 || ep.gate1) {
          gate = f32x4{0.f, 0.f, 0.f, 0.f};
          if (ep.gate0) gate += *reinterpret_cast<const f32x4*>(ep.gate0 + n);
          if (ep.gate1) gate += *reinterpret_cast<const f32x4*>(ep.gate1 + n);
        }
        v = *o + gate * ep.scale * v;
      }
      *o = v;
    }
  }
};

int32_t check_i8(int64_t M, int32_t N, int32_t K, int32_t epilogue) {
  if (M < 0 || N <= 0 || K <= 0 || epilogue < CHORUS_EPI_BF16 || epilogue > CHORUS_EPI_RESID) return CHORUS_E_ARG;
  if (K % kStep || N % 8 || K > kMostK || N > kMostN) return CHORUS_E_SHAPE;
  return CHORUS_OK;
}

int32_t launch_i8_few(const Operands& x, long M, int N, int K, int epi, const EpiArgs& ep, hipStream_t s) {
#define FEW(E) return launch_skinny<MmaI8, 1>(x.A, x.W, nullptr, (int)M, N, K, StripI8<E>{x.a_scale, x.w_scale, ep, N}, s)
  switch (epi) {
    case CHORUS_EPI_BF16: FEW(CHORUS_EPI_BF16);
    case CHORUS_EPI_GELU_BF16: FEW(CHORUS_EPI_GELU_BF16);
    case CHORUS_EPI_F32: FEW(CHORUS_EPI_F32);
    default: FEW(CHORUS_EPI_RESID);
  }
#undef FEW
}

}  // namespace
}  // namespace chorus

using namespace chorus;

extern "C" {

int32_t chorus_quant_rows_i8(const uint16_t* X, int64_t ld, int8_t* out, float* scale, int64_t M, int32_t K, int32_t Kp, void* stream) {
  if (M < 0 || K <= 0 || Kp < K || ld < K) return CHORUS_E_ARG;
  if (K % 8 || Kp % 8 || ld % 8 || M > 0x7fffffffL / 256) return CHORUS_E_SHAPE;
  if (M == 0) return CHORUS_OK;
  if (!X || !out || !scale || !aligned16(X) || !aligned16(out) || !aligned16(scale)) return CHORUS_E_ARG;
  hipStream_t s = (hipStream_t)stream;
  // a wave a row where rows fill the GPU and fit its registers, a workgroup a row otherwise
  if (M >= 2048 && K <= 64 * 8 * 8)
    hipLaunchKernelGGL((quant_rows_kernel<64, 8>), dim3((unsigned)((M + 3) / 4)), dim3(256), 0, s, X, (long)ld, out, scale, (long)M, K, Kp);
  else
    hipLaunchKernelGGL((quant_rows_kernel<256, 6>), dim3((unsigned)M), dim3(256), 0, s, X, (long)ld, out, scale, (long)M, K, Kp);
  CHORUS_LAUNCH_CHECK();
  return CHORUS_OK;
}

int32_t chorus_gemm_i8(const int8_t* A, const float* a_scale, const int8_t* W, const float* w_scale, int64_t M, int32_t N, int32_t K,
                       int32_t epilogue, void* out, const float* bias, const float* gate0, const float* gate1, float scale, void* stream) {
  CHK_STATUS(check_i8(M, N, K, epilogue));
  if (M == 0) return CHORUS_OK;
  if (!A || !a_scale || !W || !w_scale || !out) return CHORUS_E_ARG;
  if (!aligned16(A) || !aligned16(a_scale) || !aligned16(W) || !aligned16(w_scale) || !aligned16(out) || !aligned16(bias) || !aligned16(gate0) ||
      !aligned16(gate1))
    return CHORUS_E_ARG;
  const Operands x{reinterpret_cast<const uint16_t*>(A), reinterpret_cast<const uint16_t*>(W), a_scale, w_scale};
  const EpiArgs ep{out, bias, gate0, gate1, scale};
  const int units = K / 2;  // a row in units of 2 bytes
  hipStream_t s = (hipStream_t)stream;
  if (skinny_rows(M, N)) return launch_i8_few(x, (long)M, N, units, epilogue, ep, s);
  const TileCut cut = gemm_tiles(M, N, units, epilogue);
  if (cut.head_rows) CHK_STATUS(launch_i8_tile(kTile256, x, cut.head_rows, N, units, epilogue, ep, s));
  const size_t elt = epilogue == CHORUS_EPI_F32 || epilogue == CHORUS_EPI_RESID ? 4 : 2;
  EpiArgs rest = ep;
  rest.out = static_cast<uint8_t*>(out) + (size_t)cut.head_rows * (size_t)N * elt;
  const Operands tail{x.A + (size_t)cut.head_rows * (size_t)units, x.W, a_scale + cut.head_rows, w_scale};
  return launch_i8_tile(cut.tile, tail, (long)M - cut.head_rows, N, units, epilogue, rest, s);
}

int32_t chorus_gemm_i8_plan(int64_t M, int32_t N, int32_t K, int32_t epilogue, chorus_gemm_plan* out) {
  CHK_STATUS(check_i8(M, N, K, epilogue));
  if (!out || M == 0) return CHORUS_E_ARG;
  *out = chorus_gemm_plan{0, 0, 1};
  if (skinny_rows(M, N)) return CHORUS_OK;
  const TileCut cut = gemm_tiles(M, N, K / 2, epilogue);
  out->head_rows = cut.head_rows;
  out->kernel = kTileNumber[cut.tile];
  return CHORUS_OK;
}

}  // extern "C"
