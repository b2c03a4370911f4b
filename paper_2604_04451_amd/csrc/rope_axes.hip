// Rotary positions with several axes: the rotation angles of a token come from its coordinates on up to any number of axes (time,
// height, width, ...), given as numbers, and from a frequency and an axis per pair of values. Optional RMSNorm over the row or over
// each head ahead of the rotation; token-major bf16 -> head-major bf16, as chorus_qk_norm_rope writes it.
//
//   y = x * rstd * gain;   angle_p = pos[axis_p] * freq_p;   (y1, y2) -> (y1 cos - y2 sin, y1 sin + y2 cos) * out_scale
//
// One rounding to bf16, at the end; all else in fp32. The angle is formed in fp64, in turns, and reduced to half a turn before it
// becomes fp32: a far position (10^5 and more on one axis) keeps the phase that fp32 products would lose.
#include "chorus_ops.h"
#include "common.h"

namespace chorus {
namespace {

constexpr float kEps = 1e-6f;

// Sum over the lanes that hold one head, `lanes` = 8 or 16 aligned neighbours.
__device__ __forceinline__ float head_sum(float v, int lanes) {
  auto dpp = [](float x, auto ctrl) {
    return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), decltype(ctrl)::value, 0xf, 0xf, false));
  };
  v += dpp(v, std::integral_constant<int, 0xb1>{});   // lane ^ 1
  v += dpp(v, std::integral_constant<int, 0x4e>{});   // lane ^ 2
  v += dpp(v, std::integral_constant<int, 0x141>{});  // mirrored in 8
  if (lanes == 16) v += dpp(v, std::integral_constant<int, 0x140>{});  // mirrored in 16
  return v;
}

__device__ __forceinline__ void unpack8(float (&x)[8], const u32x4& u) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    x[2 * k] = __uint_as_float(u[k] << 16);
    x[2 * k + 1] = __uint_as_float(u[k] & 0xffff0000u);
  }
}
__device__ __forceinline__ float sum_squares(const float (&x)[8]) {
  float s = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) s = __builtin_fmaf(x[e], x[e], s);
  return s;
}

// A wave a token; a lane takes chunks of eight values, so a head is 8 or 16 neighbouring lanes. HBM-bound: each row is read once
// and written once. NCH > 0: rows of more than 512 FULL and up to 512 NCH values, whose loads are all issued ahead of the angles
// and which stay in registers; NCH == 0: any number of heads, chunk by chunk, and twice (the second time from the cache) where the
// norm is over the row.
template <int NORM, bool HALVES, int NCH, int FULL>
__global__ __launch_bounds__(256) void rope_axes_kernel(const uint16_t* __restrict__ in, long ld, const float* __restrict__ gain,
                                                        uint16_t* __restrict__ out, long L, long Lpad, int H, int dh,
                                                        const float* __restrict__ pos, int n_axes, const double* __restrict__ freq,
                                                        const int* __restrict__ axis, int n_pairs, float out_scale) {
  __shared__ float s_cos[4][64], s_sin[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const long row = (long)blockIdx.x * 4 + wave;
  if (row >= Lpad) return;
  const int nchunk = H * dh >> 3, lanes = dh >> 3;
  if (row >= L) {
    for (int c = lane; c < nchunk; c += 64)
      *reinterpret_cast<u32x4*>(out + ((long)(c / lanes) * Lpad + row) * dh + c % lanes * 8) = u32x4{0, 0, 0, 0};
    return;
  }
  const uint16_t* r = in + row * ld;
  u32x4 rv[NCH > 0 ? NCH : 1];
  if (NCH > 0) {
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int c = lane + 64 * i;
      rv[i] = *reinterpret_cast<const u32x4*>(r + (i < FULL || c < nchunk ? c : nchunk - 1) * 8);
    }
  }
  uint64_t turning;  // the pairs that do; what stands beside a value in another pair, infinities and NaN too, is kept out of it
  {
    float cs = 1.f, sn = 0.f;
    const int a = lane < n_pairs ? axis[lane] : -1;
    turning = __ballot((unsigned)a < (unsigned)n_axes);
    if ((unsigned)a < (unsigned)n_axes) {
      const double turns = (double)pos[row * n_axes + a] * freq[lane] * 0.15915494309189535;  // / 2 pi
      sincospif(2.0f * (float)(turns - __builtin_rint(turns)), &sn, &cs);
    }
    s_cos[wave][lane] = cs;
    s_sin[wave][lane] = sn;
    __builtin_amdgcn_wave_barrier();
  }
  // With out_scale in it. Where there is no norm, out_scale is the gain and goes in ahead of the rotation, whose values fp32 may not
  // hold without it.
  float rstd = 1.0f;
  if (NORM == CHORUS_ROPE_NORM_WIDTH) {
    float ss = 0.f, x[8];
    if (NCH > 0) {
#pragma unroll
      for (int i = 0; i < NCH; ++i) {
        unpack8(x, rv[i]);
        const float s = sum_squares(x);
        ss += i < FULL || lane + 64 * i < nchunk ? s : 0.f;
      }
    } else {
      for (int c = lane; c < nchunk; c += 64) {
        unpack8(x, *reinterpret_cast<const u32x4*>(r + c * 8));
        ss += sum_squares(x);
      }
    }
    rstd = rsqrtf(wave_sum(ss) / (float)(H * dh) + kEps) * out_scale;
  }
  const int iters = NCH > 0 ? NCH : (nchunk + 63) / 64;
  constexpr int kTimes = NCH > 0 ? NCH : 1;
  const int d0 = lane % lanes * 8;  // in its head, whatever the chunk
  // Halves: a value's other half is in a lane of the same head, `off` values further. Gains go in ahead of the rotation and the
  // norm behind it, where a value takes it once (75600 x 5120, norm of the head 300 us, both halves normalised ahead 330; norm of
  // the row 302 and 337).
  const bool first = d0 < n_pairs;
  const int off = !HALVES || d0 >= 2 * n_pairs ? 0 : first ? n_pairs : -n_pairs;
  const uint32_t turns = HALVES ? (off != 0 ? (uint32_t)(turning >> (first ? d0 : d0 - n_pairs)) : 0u) : (uint32_t)(turning >> (d0 >> 1));
  float cs[8], sn[8];
  if (HALVES) {
    const int p = first ? d0 : d0 - n_pairs;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      cs[e] = off != 0 ? s_cos[wave][p + e] : 1.0f;
      sn[e] = off == 0 ? 0.f : first ? -s_sin[wave][p + e] : s_sin[wave][p + e];
    }
  }
#pragma unroll kTimes
  for (int it = 0; it < iters; ++it) {
    const int c0 = 64 * it;
    const bool live = it < FULL || c0 + lane < nchunk;
    const int c = live ? c0 + lane : nchunk - 1;  // lanes past the end keep the head's sum company and store nothing
    const int head = c / lanes;
    float x[8];
    u32x4 u;
    if (NCH > 0) u = rv[NCH > 0 ? it : 0];
    else u = *reinterpret_cast<const u32x4*>(r + c * 8);
    unpack8(x, u);
    if (NORM == CHORUS_ROPE_NORM_HEAD) rstd = rsqrtf(head_sum(sum_squares(x), lanes) / (float)dh + kEps) * out_scale;
    const float* g = NORM == CHORUS_ROPE_NORM_HEAD ? gain + d0 : gain + c * 8;
    auto gains = [&](float(&v)[8], int at) {
#pragma unroll
      for (int e = 0; e < 8; e += 4) {
        const f32x4 q = NORM == CHORUS_ROPE_NORM_NONE ? f32x4{out_scale, out_scale, out_scale, out_scale}
                                                      : *reinterpret_cast<const f32x4*>(g + at + e);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[e + i] = q[i];
      }
    };
    float own[8];
    gains(own, 0);
    if (HALVES) {
      float y[8];
      if (NORM == CHORUS_ROPE_NORM_WIDTH) {  // gains that change from chunk to chunk: exchanged with them, each is loaded once
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] *= own[e];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = __shfl(x[e], lane + off / 8, 64) * sn[e];
      } else {
        u32x4 other;
        float of[8];
#pragma unroll
        for (int k = 0; k < 4; ++k) other[k] = __shfl(u[k], lane + off / 8, 64);
        unpack8(y, other);
        gains(of, off);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          x[e] *= own[e];
          y[e] *= of[e] * sn[e];
        }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = turns >> e & 1 ? __builtin_fmaf(x[e], cs[e], y[e]) : x[e];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] *= rstd;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] *= rstd * own[e];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float c_ = s_cos[wave][(d0 >> 1) + k], s_ = s_sin[wave][(d0 >> 1) + k];
        const float a = x[2 * k], b = x[2 * k + 1];
        x[2 * k] = turns >> k & 1 ? a * c_ - b * s_ : a;
        x[2 * k + 1] = turns >> k & 1 ? a * s_ + b * c_ : b;
      }
    }
    u32x4 o;
#pragma unroll
    for (int k = 0; k < 4; ++k) o[k] = pack_bf16x2(x[2 * k], x[2 * k + 1]);
    if (live) *reinterpret_cast<u32x4*>(out + ((long)head * Lpad + row) * dh + d0) = o;
  }
}

}  // namespace
}  // namespace chorus

using namespace chorus;

extern "C" {

int32_t chorus_rope_axes_table(int32_t n_axes, const int32_t* dims, double theta, double* freq, int32_t* axis, int32_t* n_pairs) {
  if (n_axes < 1 || !dims || !freq || !axis || !n_pairs || !(theta > 0.0) || !(theta < INFINITY)) return CHORUS_E_ARG;
  int64_t sum = 0;
  for (int k = 0; k < n_axes; ++k) {
    if (dims[k] < 0 || dims[k] % 2) return CHORUS_E_ARG;
    sum += dims[k];
    if (sum > 128) return CHORUS_E_SHAPE;
  }
  int p = 0;
  for (int k = 0; k < n_axes; ++k)
    for (int i = 0; i < dims[k] / 2; ++i, ++p) {
      freq[p] = pow(theta, -2.0 * i / dims[k]);
      axis[p] = k;
    }
  *n_pairs = p;
  return CHORUS_OK;
}

int32_t chorus_rope_axes(const uint16_t* in, int64_t ld, const float* gain, int32_t norm, uint16_t* out, int64_t L, int64_t Lpad,
                         int32_t H, int32_t dh, const float* pos, int32_t n_axes, const double* freq, const int32_t* axis,
                         int32_t n_pairs, int32_t layout, float out_scale, void* stream) {
  if (L < 0 || Lpad < L || H <= 0 || dh <= 0 || n_axes < 1 || n_pairs < 0) return CHORUS_E_ARG;
  if (norm < CHORUS_ROPE_NORM_NONE || norm > CHORUS_ROPE_NORM_HEAD || (layout != CHORUS_ROPE_PAIRS && layout != CHORUS_ROPE_HALVES))
    return CHORUS_E_ARG;
  if (!(out_scale > 0.f) || !(out_scale < INFINITY)) return CHORUS_E_ARG;
  if ((dh != 64 && dh != 128) || H > (1 << 20) || 2 * (int64_t)n_pairs > dh) return CHORUS_E_SHAPE;
  if (layout == CHORUS_ROPE_HALVES && n_pairs % 8) return CHORUS_E_SHAPE;
  if (ld % 8 || ld < (int64_t)H * dh || Lpad > 0xffffffffL / 64 - 3) return CHORUS_E_SHAPE;  // 64 threads a row, of the 2^32 - 1 of a launch
  if (Lpad == 0) return CHORUS_OK;
  if (!out || !aligned16(out)) return CHORUS_E_ARG;
  if (L > 0 && (!in || !pos || (n_pairs && (!freq || !axis)) || (norm != CHORUS_ROPE_NORM_NONE && !gain))) return CHORUS_E_ARG;
  if (!aligned16(in) || !aligned16(pos) || !aligned16(freq) || !aligned16(axis) || !aligned16(gain)) return CHORUS_E_ARG;
  const int D = H * dh;
#define ROPE_ROWS(NORM, HALVES, NCH, FULL)                                                                                              \
  hipLaunchKernelGGL((rope_axes_kernel<NORM, HALVES, NCH, FULL>), dim3((unsigned)((Lpad + 3) / 4)), dim3(256), 0, (hipStream_t)stream, in, \
                     (long)ld, gain, out, (long)L, (long)Lpad, H, dh, pos, n_axes, freq, axis, n_pairs, out_scale)
  // by the width alone: up to 40 registers of a row, in steps that leave at most 3 of 10 chunks empty (20000 rows of 26 heads of
  // 128 and their norm: 53.5 us, chunk by chunk 63.3; 32760 rows of 12 heads 32.6)
#define ROPE(NORM, HALVES)                                  \
  do {                                                      \
    if (D <= 512) ROPE_ROWS(NORM, HALVES, 1, 0);            \
    else if (D <= 1024) ROPE_ROWS(NORM, HALVES, 2, 1);      \
    else if (D <= 1536) ROPE_ROWS(NORM, HALVES, 3, 2);      \
    else if (D <= 2048) ROPE_ROWS(NORM, HALVES, 4, 3);      \
    else if (D <= 2560) ROPE_ROWS(NORM, HALVES, 5, 4);      \
    else if (D <= 3584) ROPE_ROWS(NORM, HALVES, 7, 5);      \
    else if (D <= 5120) ROPE_ROWS(NORM, HALVES, 10, 7);     \
    else ROPE_ROWS(NORM, HALVES, 0, 0);                     \
  } while (0)
#define ROPE_LAYOUT(NORM)                                 \
  do {                                                    \
    if (layout == CHORUS_ROPE_HALVES) ROPE(NORM, true);   \
    else ROPE(NORM, false);                               \
  } while (0)
  if (norm == CHORUS_ROPE_NORM_WIDTH) ROPE_LAYOUT(CHORUS_ROPE_NORM_WIDTH);
  else if (norm == CHORUS_ROPE_NORM_HEAD) ROPE_LAYOUT(CHORUS_ROPE_NORM_HEAD);
  else ROPE_LAYOUT(CHORUS_ROPE_NORM_NONE);
#undef ROPE_LAYOUT
#undef ROPE
#undef ROPE_ROWS
  CHORUS_LAUNCH_CHECK();
  return CHORUS_OK;
}

}  // extern "C"
