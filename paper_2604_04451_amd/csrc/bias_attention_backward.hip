// Gradients of attention with a bias by distance. With P the weights, made again from the logits and the rows' logarithms of their sums,
//   delta_i = dO_i . O_i,  dS = P (dO V^T - delta),  dV = P^T dO,  dK = scale dS^T Q,  dQ = scale dS K,  dtable[c] = sum of dS where the bucket is c.
// Two passes over the logits, neither of which adds to memory that another workgroup adds to: queries stand still in the first (dQ, the
// sums of dS by distance, delta), keys in the second (dK and dV, over all heads that share them). A third kernel adds up the distances' sums.
#include "bias_attention.h"

namespace chorus {
namespace {

struct Delta {
  float* p;  // [B, H, Lq]
};

#if defined(__HIP_DEVICE_COMPILE__)
// A lane holds 4 values of a column of each of DB blocks of 16 rows: column l % 16, rows 4 (l / 16) on. Written as rows of bf16: four neighbouring
// lanes write 64 bytes of one, the column l % 16 / 4 * 4 + l / 16; `at` is where its values 8 (l % 4) .. + 8 of the first 32 go.
template <int DB>
__device__ __forceinline__ void put_columns(const f32x4 (&x)[DB], float factor, uint16_t* at, bool live, int lane) {
  const auto from_lane = [](int src, uint32_t v) { return (uint32_t)__builtin_amdgcn_ds_bpermute(4 * src, (int)v); };
  const int lq = lane & 15, g = lane >> 4, b4 = lq & 3;
  const int src = 16 * (b4 >> 1 | (b4 & 1) << 1) + (lq & 12) + g;
#pragma unroll
  for (int i = 0; i < DB / 2; ++i) {
    const f32x4 a = x[2 * i] * factor, b = x[2 * i + 1] * factor;
    const auto lo = __builtin_amdgcn_permlane16_swap(pack_bf16x2(a[0], a[1]), pack_bf16x2(b[0], b[1]), false, false);
    const auto hi = __builtin_amdgcn_permlane16_swap(pack_bf16x2(a[2], a[3]), pack_bf16x2(b[2], b[3]), false, false);
    const u32x4 v = {from_lane(src, lo[0]), from_lane(src, hi[0]), from_lane(src, lo[1]), from_lane(src, hi[1])};
    if (live) *reinterpret_cast<u32x4*>(at + 32 * i) = v;
  }
}
#endif

// The logarithm of a row's sum as the exponent that its weights lose; no weight is left to a row without keys or outside the matrix.
__device__ __forceinline__ float row_exponent(float lse, bool live) { return live && lse > -INFINITY ? lse * kLog2E : INFINITY; }

// ---------------------------------------------------------------------------
// Queries stand still: as the forward kernel, 32 queries a wave, keys 64 at a time. The products S^T = K Q^T and dP^T = V dO^T leave a lane with
// a query's logits and their gradients as the operand of dQ^T += K^T dS^T.
// Sums by distance: a wave's 64 x 32 gradients of a near tile are added up along their diagonals. Blocks of 16 x 16 on one diagonal are added
// in registers first, five diagonals of blocks; they go to LDS with row c of 16 shifted c places to the left, so that a column
// of the 95 places is a distance, and two places a lane are summed and added to the wave's own sums of distances. Tiles whose
// distances all share an end bucket cost one addition a value.
// ---------------------------------------------------------------------------
constexpr int kSkewPlaces = 95, kSkewRow = 97;

template <int DH>
__global__ __launch_bounds__(256, DH == 64 ? 2 : 1) void bias_dq_kernel(Rows Q, Rows K, Rows V, Rows O, const uint16_t* __restrict__ rest, Rows dO, RowsOut dQ,
                                                         const float* __restrict__ lse, Delta delta, float* __restrict__ part, BiasArgs bias, long Lq,
                                                         long Lk, int H, int group, int nq) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int KB = kTileKeys / 16, NC = kTileKeys / 32, KC = DH / 32, DB = DH / 16, RB = 2;
  constexpr int TILE = kTileKeys * DH;
  extern __shared__ __attribute__((aligned(16))) uint16_t smem[];  // [2][TILE] keys, [2][TILE] values, biases, sums of each wave, skewed rows of each
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lq = lane & 15, g = lane >> 4;
  const int width = bias.width(), far = bias.far;
  float* const s_bias = reinterpret_cast<float*>(smem + 4 * TILE);
  float* const s_sums = s_bias + width + wave * width;
  float* const s_skew = s_bias + 5 * width + wave * 16 * kSkewRow;

  const int unit = xcd_remap(blockIdx.x, gridDim.x);
  const int bh = unit / nq, qb = unit - bh * nq, b = bh / H, head = bh - b * H;
  const int n = __builtin_amdgcn_readfirstlane(bias.keys(b, Lk)), origin = __builtin_amdgcn_readfirstlane(bias.origin(b));
  const int q0 = qb * kTileQueries + wave * 32;
  const int last_q = (int)((long)(qb + 1) * kTileQueries < Lq ? (qb + 1) * kTileQueries : Lq) - 1;
  int most = n;
  if (bias.causal) {
    const int m = origin + last_q + 1;
    most = m < 0 ? 0 : m < n ? m : n;
  }
  const int steps = (most + kTileKeys - 1) / kTileKeys;

  TileStage<DH> k_in(tid, K.row), v_in(tid, V.row);
  const uint16_t* const k_base = K.p + (long)b * K.batch + (long)(head / group) * DH;
  const uint16_t* const v_base = V.p + (long)b * V.batch + (long)(head / group) * DH;
  auto fetch = [&](int t) {
    k_in.fetch(k_base + (long)t * kTileKeys * K.row, n - 1 - t * kTileKeys);
    v_in.fetch(v_base + (long)t * kTileKeys * V.row, n - 1 - t * kTileKeys);
  };
  auto store = [&](int buf) {
    k_in.store(smem + buf * TILE);
    v_in.store(smem + (2 + buf) * TILE);
  };
  if (steps > 0) fetch(0);
  for (int i = tid; i < width; i += 256) s_bias[i] = bias.bias(i, head, H);
  for (int i = lane; i < width; i += 64) s_sums[i] = 0.f;
  for (int i = lane; i < 16 * kSkewRow; i += 64) s_skew[i] = 0.f;

  const RowFragments<DH> rows(lane);
  const ColumnFragments<DH> columns(lane);
  bf16x8 qf[RB][KC], df[RB][KC];
  float ex[RB], dl[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const bool live = q0 + 16 * rb + lq < Lq;
    const long q = live ? q0 + 16 * rb + lq : Lq - 1;
    const uint16_t* qp = Q.p + (long)b * Q.batch + q * Q.row + (long)head * DH + 8 * g;
    const uint16_t* dp = dO.p + (long)b * dO.batch + q * dO.row + (long)head * DH + 8 * g;
    const long at = (long)b * O.batch + q * O.row + (long)head * DH + 8 * g;
    float sum = 0.f;
#pragma unroll
    for (int kc = 0; kc < KC; ++kc) {
      qf[rb][kc] = *reinterpret_cast<const bf16x8*>(qp + 32 * kc);
      df[rb][kc] = *reinterpret_cast<const bf16x8*>(dp + 32 * kc);
      const u32x4 o = *reinterpret_cast<const u32x4*>(O.p + at + 32 * kc), r = *reinterpret_cast<const u32x4*>(rest + at + 32 * kc);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        sum = __builtin_fmaf((float)df[rb][kc][e], both_halves((uint16_t)(o[e / 2] >> 16 * (e % 2)), (uint16_t)(r[e / 2] >> 16 * (e % 2))), sum);
    }
    sum += swap_rows16(sum);
    sum += swap_halves(sum);
    dl[rb] = sum;
    ex[rb] = row_exponent(lse[(long)bh * Lq + q], live);
    if (g == 0 && live) delta.p[(long)bh * Lq + q] = sum;
  }
  f32x4 dq[RB][DB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb)
#pragma unroll
    for (int db = 0; db < DB; ++db) dq[rb][db] = f32x4{0.f, 0.f, 0.f, 0.f};
  if (steps > 0) store(0);
  if (steps > 1) fetch(1);
  lds_barrier();
  const float below = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(s_bias[0])));
  const float above = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(s_bias[width - 1])));
  const float scale = bias.scale * kLog2E;
  float sum_below = 0.f, sum_above = 0.f;

  for (int t = 0, buf = 0; t < steps; ++t, buf ^= 1) {
    if (t + 1 < steps) store(buf ^ 1);
    if (t + 2 < steps) fetch(t + 2);
    const uint16_t* const k_tile = smem + buf * TILE;
    const uint16_t* const v_tile = smem + (2 + buf) * TILE;
    f32x4 s[KB][RB], dp[KB][RB];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        s[kb][rb] = f32x4{0.f, 0.f, 0.f, 0.f};
        dp[kb][rb] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
#pragma unroll
      for (int kc = 0; kc < KC; ++kc) {
        const bf16x8 kf = rows.read(k_tile, kb, kc), vf = rows.read(v_tile, kb, kc);
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          s[kb][rb] = mfma(kf, qf[rb][kc], s[kb][rb]);
          dp[kb][rb] = mfma(vf, df[rb][kc], dp[kb][rb]);
        }
      }
    }
    const int nearest = t * kTileKeys - (origin + q0);
    const bool near = nearest + 63 > -far && nearest - 31 < far;
    if (near) {
      const float* at = s_bias + (nearest + far + kPad + 4 * g - lq);
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[kb][rb][i] = __builtin_fmaf(s[kb][rb][i], scale, at[16 * (kb - rb) + i] - ex[rb]);
    } else {
      const float c = nearest > 0 ? above : below;
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[kb][rb][i] = __builtin_fmaf(s[kb][rb][i], scale, c - ex[rb]);
    }
    int end = n;
    if (bias.causal && origin + q0 + 1 < end) end = origin + q0 + 1;
    if ((t + 1) * kTileKeys > end) {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        int left = n;
        if (bias.causal && origin + q0 + 16 * rb + lq + 1 < n) left = origin + q0 + 16 * rb + lq + 1;
        left -= t * kTileKeys + 4 * g;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (16 * kb + i >= left) s[kb][rb][i] = -INFINITY;
      }
    }
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[kb][rb][i] = __builtin_amdgcn_exp2f(s[kb][rb][i]) * (dp[kb][rb][i] - dl[rb]);
    bf16x8 ds[NC][RB];
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int e = 0; e < 8; ++e) ds[c][rb][e] = (bf16_t)s[2 * c + (e >> 2)][rb][e & 3];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const bf16x8 kf = columns.read(k_tile, c, db);
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) dq[rb][db] = mfma(kf, ds[c][rb], dq[rb][db]);
      }
    if (near) {
      static_assert(KB == 4 && RB == 2, "five diagonals of blocks");
      float* const row = s_skew + lq * kSkewRow + 15 - lq + 4 * g;
#pragma unroll
      for (int d = 0; d < 5; ++d) {  // kb - rb = d - 1
        f32x4 v;
        if (d == 0) v = s[0][1];
        else if (d == 4) v = s[3][0];
        else v = s[d % 4][1] + s[(d + 3) % 4][0];
#pragma unroll
        for (int i = 0; i < 4; ++i) row[16 * d + i] = v[i];
      }
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
      float* const sums = s_sums + nearest - 31 + far + kPad;
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int p = lane + 64 * half;
        if (p < kSkewPlaces) {
          float a = 0.f;
#pragma unroll
          for (int c = 0; c < 16; ++c) a += s_skew[c * kSkewRow + p];
          sums[p] += a;
        }
      }
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    } else {
      float a = 0.f;
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int i = 0; i < 4; ++i) a += s[kb][rb][i];
      if (nearest > 0) sum_above += a;
      else sum_below += a;
    }
    lds_barrier();
  }
  sum_below = wave_sum(sum_below);
  sum_above = wave_sum(sum_above);
  if (lane == 0) {
    s_sums[0] += sum_below;
    s_sums[width - 1] += sum_above;
  }
  lds_barrier();
  for (int i = tid; i < width; i += 256) {
    float a = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) a += s_bias[(1 + w) * width + i];
    part[(long)unit * width + i] = a;
  }
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const long q = q0 + 16 * rb + (lq & 12) + g;
    put_columns<DB>(dq[rb], bias.scale, dQ.p + (long)b * dQ.batch + q * dQ.row + (long)head * DH + 8 * (lq & 3), q < Lq, lane);
  }
#endif
}

// ---------------------------------------------------------------------------
// Keys stand still: 32 keys and values a wave in registers, queries and their gradients 64 at a time through LDS, over all heads that share
// the keys. S = Q K^T and dP = dO V^T leave a lane with one key's logits as the operand of dV^T += dO^T P and dK^T += Q^T dS.
// ---------------------------------------------------------------------------
template <int DH>
__global__ __launch_bounds__(256, DH == 64 ? 2 : 1) void bias_dkv_kernel(Rows Q, Rows K, Rows V, Rows dO, RowsOut dK, RowsOut dV,
                                                                         const float* __restrict__ lse, Delta delta, BiasArgs bias, long Lq, long Lk,
                                                                         int H, int group, int nk) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int QB = kTileKeys / 16, NC = kTileKeys / 32, KC = DH / 32, DB = DH / 16, NB = 2;
  constexpr int TILE = kTileKeys * DH;
  extern __shared__ __attribute__((aligned(16))) uint16_t smem[];  // [2][TILE] queries, [2][TILE] their gradients, [2][2][64] exponents and deltas, biases
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lq = lane & 15, g = lane >> 4;
  float* const s_rows = reinterpret_cast<float*>(smem + 4 * TILE);
  float* const s_bias = s_rows + 4 * kTileKeys;
  const int width = bias.width(), far = bias.far, Hk = H / group;

  const int unit = xcd_remap(blockIdx.x, gridDim.x);
  const int bh = unit / nk, kt = unit - bh * nk, b = bh / Hk, kv_head = bh - b * Hk;
  const int n = __builtin_amdgcn_readfirstlane(bias.keys(b, Lk)), origin = __builtin_amdgcn_readfirstlane(bias.origin(b));
  const int k0 = kt * kTileQueries + wave * 32;  // the wave's first key
  const int tiles = (int)((Lq + kTileKeys - 1) / kTileKeys);
  int first_tile = 0;
  if (bias.causal) {
    const int q = kt * kTileQueries - origin;  // the first query that sees the workgroup's first key
    first_tile = q <= 0 ? 0 : q / kTileKeys < tiles ? q / kTileKeys : tiles;
  }
  const int each = kt * kTileQueries < n ? tiles - first_tile : 0, steps = each * group;

  TileStage<DH> q_in(tid, Q.row), d_in(tid, dO.row);
  float row_in = 0.f;
  auto fetch = [&](int i) {
    const int head = kv_head * group + i / each, t = first_tile + i % each;
    q_in.fetch(Q.p + (long)b * Q.batch + (long)t * kTileKeys * Q.row + (long)head * DH, (int)(Lq - 1) - t * kTileKeys);
    d_in.fetch(dO.p + (long)b * dO.batch + (long)t * kTileKeys * dO.row + (long)head * DH, (int)(Lq - 1) - t * kTileKeys);
    if (tid < 2 * kTileKeys) {
      const long q = (long)t * kTileKeys + (tid & 63);
      const bool live = q < Lq;
      const long at = ((long)b * H + head) * Lq + (live ? q : Lq - 1);
      row_in = tid < kTileKeys ? row_exponent(lse[at], live) : delta.p[at];
    }
  };
  auto store = [&](int buf) {
    q_in.store(smem + buf * TILE);
    d_in.store(smem + (2 + buf) * TILE);
    if (tid < 2 * kTileKeys) s_rows[buf * 2 * kTileKeys + tid] = row_in;
  };
  if (steps > 0) fetch(0);

  const RowFragments<DH> rows(lane);
  const ColumnFragments<DH> columns(lane);
  bf16x8 kf[NB][KC], vf[NB][KC];
  f32x4 dk[NB][DB], dv[NB][DB];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    long k = k0 + 16 * nb + lq;
    if (k > n - 1) k = n - 1;
    if (k < 0) k = 0;  // no keys at all: nothing is made of what is read
    const uint16_t* kp = K.p + (long)b * K.batch + k * K.row + (long)kv_head * DH + 8 * g;
    const uint16_t* vp = V.p + (long)b * V.batch + k * V.row + (long)kv_head * DH + 8 * g;
#pragma unroll
    for (int kc = 0; kc < KC; ++kc) {
      kf[nb][kc] = *reinterpret_cast<const bf16x8*>(kp + 32 * kc);
      vf[nb][kc] = *reinterpret_cast<const bf16x8*>(vp + 32 * kc);
    }
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      dk[nb][db] = f32x4{0.f, 0.f, 0.f, 0.f};
      dv[nb][db] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }
  const float scale = bias.scale * kLog2E;
  float below = 0.f, above = 0.f;
  if (steps > 0) store(0);
  if (steps > 1) fetch(1);

  for (int i = 0, buf = 0; i < steps; ++i, buf ^= 1) {
    const int t = first_tile + i % each;
    if (i % each == 0) {  // another head, other biases
      const int head = kv_head * group + i / each;
      if (i > 0) lds_barrier();
      for (int w = tid; w < width; w += 256) s_bias[w] = bias.bias(w, head, H);
      lds_barrier();
      below = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(s_bias[0])));
      above = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(s_bias[width - 1])));
    }
    if (i + 1 < steps) store(buf ^ 1);
    if (i + 2 < steps) fetch(i + 2);
    const uint16_t* const q_tile = smem + buf * TILE;
    const uint16_t* const d_tile = smem + (2 + buf) * TILE;
    const float* const ex = s_rows + buf * 2 * kTileKeys;
    f32x4 s[QB][NB], dp[QB][NB];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        s[qb][nb] = f32x4{0.f, 0.f, 0.f, 0.f};
        dp[qb][nb] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
#pragma unroll
      for (int kc = 0; kc < KC; ++kc) {
        const bf16x8 qf = rows.read(q_tile, qb, kc), df = rows.read(d_tile, qb, kc);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          s[qb][nb] = mfma(qf, kf[nb][kc], s[qb][nb]);
          dp[qb][nb] = mfma(df, vf[nb][kc], dp[qb][nb]);
        }
      }
    }
    const int nearest = k0 - (origin + t * kTileKeys);  // distance of the wave's first key from the tile's first query
    if (nearest + 31 > -far && nearest - 63 < far) {
      const float* at = s_bias + (nearest + far + kPad + lq - 4 * g);
#pragma unroll
      for (int qb = 0; qb < QB; ++qb)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[qb][nb][e] = __builtin_fmaf(s[qb][nb][e], scale, at[16 * (nb - qb) - e]);
    } else {
      const float c = nearest > 0 ? above : below;
#pragma unroll
      for (int qb = 0; qb < QB; ++qb)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[qb][nb][e] = __builtin_fmaf(s[qb][nb][e], scale, c);
    }
    if (bias.causal && nearest + 31 > 0) {
#pragma unroll
      for (int qb = 0; qb < QB; ++qb)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (nearest + 16 * (nb - qb) + lq - 4 * g - e > 0) s[qb][nb][e] = -INFINITY;
    }
    bf16x8 pf[NC][NB], ds[NC][NB];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(ex + 16 * qb + 4 * g), dl = *reinterpret_cast<const f32x4*>(ex + kTileKeys + 16 * qb + 4 * g);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p = __builtin_amdgcn_exp2f(s[qb][nb][e] - x[e]);
          pf[qb / 2][nb][4 * (qb % 2) + e] = (bf16_t)p;
          ds[qb / 2][nb][4 * (qb % 2) + e] = (bf16_t)(p * (dp[qb][nb][e] - dl[e]));
        }
    }
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const bf16x8 df = columns.read(d_tile, c, db), qf = columns.read(q_tile, c, db);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          dv[nb][db] = mfma(df, pf[c][nb], dv[nb][db]);
          dk[nb][db] = mfma(qf, ds[c][nb], dk[nb][db]);
        }
      }
    lds_barrier();
  }
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const long k = k0 + 16 * nb + (lq & 12) + g;
    const long at = (long)kv_head * DH + 8 * (lq & 3);
    // Keys behind the sequence: their columns hold those of its last key
    const bool counts = k0 + 16 * nb + lq < n;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        dk[nb][db][e] = counts ? dk[nb][db][e] : 0.f;
        dv[nb][db][e] = counts ? dv[nb][db][e] : 0.f;
      }
    put_columns<DB>(dk[nb], bias.scale, dK.p + (long)b * dK.batch + k * dK.row + at, k < Lk, lane);
    put_columns<DB>(dv[nb], 1.0f, dV.p + (long)b * dV.batch + k * dV.row + at, k < Lk, lane);
  }
#endif
}

// Adds up a head's sums by distance, a workgroup a head: over sequences and tiles of queries in order, then over the distances of a bucket.
__global__ __launch_bounds__(256) void bias_dtable_kernel(const float* __restrict__ part, float* __restrict__ dtable, BiasArgs bias, int B, int H, int nq) {
  __shared__ double s_sum[2 * (kMostFar + kPad) + 1];
  const int head = blockIdx.x, width = bias.width();
  for (int i = threadIdx.x; i < width; i += 256) {
    double a = 0.0;
    for (int b = 0; b < B; ++b) {
      const float* p = part + ((long)b * H + head) * nq * width + i;
      for (int q = 0; q < nq; ++q) a += (double)p[(long)q * width];
    }
    s_sum[i] = a;
  }
  __syncthreads();
  for (int c = threadIdx.x; c < bias.n_buckets; c += 256) {
    double a = 0.0;
    for (int i = 0; i < width; ++i) {
      int at = i - kPad;
      at = at < 0 ? 0 : at > 2 * bias.far ? 2 * bias.far : at;
      if (bias.bucket[at] == c) a += s_sum[i];
    }
    dtable[(long)c * H + head] = (float)a;
  }
}

struct BackwardLayout {
  size_t delta, part, all;
  int nq, nk;
  explicit BackwardLayout(const chorus_bias_attention& a) {
    nq = (int)((a.Lq + kTileQueries - 1) / kTileQueries);
    nk = (int)((a.Lk + kTileQueries - 1) / kTileQueries);
    delta = 0;
    part = align_up((size_t)a.B * a.H * (size_t)a.Lq * sizeof(float), 256);
    all = part + (size_t)a.B * a.H * nq * (size_t)(2 * (a.far + kPad) + 1) * sizeof(float);
  }
};

}  // namespace
}  // namespace chorus

using namespace chorus;

extern "C" {

size_t chorus_attention_bias_backward_workspace_bytes(const chorus_bias_attention* a) {
  return check_bias_sizes(a) != CHORUS_OK || a->B == 0 || a->Lq == 0 ? 0 : BackwardLayout(*a).all;
}

int32_t chorus_attention_bias_backward(const chorus_bias_attention* a, const chorus_bias_attention_steps* steps, const uint16_t* Q, const uint16_t* K,
                                       const uint16_t* V, const uint16_t* O, const uint16_t* rest, const float* lse, const uint16_t* dO,
                                       const float* table, const int32_t* bucket, const int32_t* lens, const int32_t* first, uint16_t* dQ, uint16_t* dK,
                                       uint16_t* dV, float* dtable, void* ws, size_t ws_bytes, void* stream) {
  BiasArgs bias;
  CHK_STATUS(check_bias_attention(a, table, bucket, lens, first, &bias));
  if (!steps) return CHORUS_E_ARG;
  if (!bias_step_ok(steps->do_row, steps->do_batch, a->H, a->dh) || !bias_step_ok(steps->dq_row, steps->dq_batch, a->H, a->dh) ||
      !bias_step_ok(steps->dk_row, steps->dk_batch, a->Hk, a->dh) || !bias_step_ok(steps->dv_row, steps->dv_batch, a->Hk, a->dh))
    return CHORUS_E_SHAPE;
  if (a->B == 0 || a->Lq == 0 || a->Lk == 0) return CHORUS_E_SHAPE;
  if (!Q || !K || !V || !O || !rest || !lse || !dO || !dQ || !dK || !dV || !dtable) return CHORUS_E_ARG;
  if (!aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(O) || !aligned16(rest) || !aligned16(lse) || !aligned16(dO) || !aligned16(dQ) ||
      !aligned16(dK) || !aligned16(dV) || !aligned16(dtable) || !aligned16(ws))
    return CHORUS_E_ARG;
  const BackwardLayout at(*a);
  if (!ws || ws_bytes < at.all) return CHORUS_E_WORKSPACE;
  const Rows q{Q, (long)a->q_row, (long)a->q_batch}, k{K, (long)a->k_row, (long)a->k_batch}, v{V, (long)a->v_row, (long)a->v_batch};
  const Rows o{O, (long)a->o_row, (long)a->o_batch}, d{dO, (long)steps->do_row, (long)steps->do_batch};
  const RowsOut gq{dQ, (long)steps->dq_row, (long)steps->dq_batch}, gk{dK, (long)steps->dk_row, (long)steps->dk_batch},
      gv{dV, (long)steps->dv_row, (long)steps->dv_batch};
  const Delta delta{reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + at.delta)};
  float* const part = reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + at.part);
  const int tiles = 4 * kTileKeys * a->dh * 2, most_width = 2 * (kMostFar + kPad) + 1;
  const int lds_q = tiles + (5 * bias.width() + 4 * 16 * kSkewRow) * 4, lds_k = tiles + (4 * kTileKeys + bias.width()) * 4;
  hipStream_t s = (hipStream_t)stream;
#define BACKWARD(DH)                                                                                                                          \
  do {                                                                                                                                        \
    static DynLdsOnce once_q, once_k;                                                                                                         \
    CHK_STATUS(once_q.ensure((const void*)bias_dq_kernel<DH>, tiles + (5 * most_width + 4 * 16 * kSkewRow) * 4));                             \
    CHK_STATUS(once_k.ensure((const void*)bias_dkv_kernel<DH>, tiles + (4 * kTileKeys + most_width) * 4));                                    \
    hipLaunchKernelGGL((bias_dq_kernel<DH>), dim3((unsigned)((long)a->B * a->H * at.nq)), dim3(256), lds_q, s, q, k, v, o, rest, d, gq, lse,  \
                       delta, part, bias, (long)a->Lq, (long)a->Lk, a->H, a->H / a->Hk, at.nq);                                               \
    CHORUS_LAUNCH_CHECK();                                                                                                                    \
    hipLaunchKernelGGL((bias_dkv_kernel<DH>), dim3((unsigned)((long)a->B * a->Hk * at.nk)), dim3(256), lds_k, s, q, k, v, d, gk, gv, lse,     \
                       delta, bias, (long)a->Lq, (long)a->Lk, a->H, a->H / a->Hk, at.nk);                                                     \
    CHORUS_LAUNCH_CHECK();                                                                                                                    \
  } while (0)
  if (a->dh == 128) BACKWARD(128);
  else BACKWARD(64);
#undef BACKWARD
  hipLaunchKernelGGL(bias_dtable_kernel, dim3((unsigned)a->H), dim3(256), 0, s, (const float*)part, dtable, bias, a->B, a->H, at.nq);
  CHORUS_LAUNCH_CHECK();
  return CHORUS_OK;
}

}  // extern "C"
