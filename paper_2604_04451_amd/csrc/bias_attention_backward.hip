// Gradients of attention with a bias by distance. With P the weights, made again from the logits and the rows' logarithms of their sums,
//   delta_i = sum_j P_ij (dO V^T)_ij = dO_i . O_i,  dS = P (dO V^T - delta),  dV = P^T dO,  dK = scale dS^T Q,  dQ = scale dS K,
//   dtable[c] = sum of dS where the bucket is c.
// Two passes over the logits, neither of which adds to memory that another workgroup adds to: queries stand still in the first (dQ), keys in
// the second (dK and dV, over all heads that share them, and the sums of dS by distance). Two small kernels add up the distances' sums.
// The sums over a bucket cancel to a small part of their terms, and an error of delta goes into all terms of a row alike. O has the roundings of
// the forward pass's weights in it; but a row's dS add up to 0, so that what those of the first pass add up to is what its delta was off by, and the
// second pass has it to fp32 (table's gradient, 8 x 512 tokens: relative error 5.8e-7, the plain form's in fp32 5.3e-7).
#include "bias_attention.h"

namespace chorus {
namespace {

// What the first pass leaves the second of every row: delta, and where it is out of the sums also its reference's first part, and the second with the logarithm
// of its sum; and which rows those are, a bit a row, 16 rows a word.
struct Delta {
  float* p;  // [3][B, H, Lq]
  long step;  // B * H * Lq
  uint32_t* apart;  // [B, H, 8 ceil(Lq / 128)]
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

// The logarithm of a row's sum as the exponent that its weights lose; no weight is left to a row without keys, outside the matrix or out of the sums.
__device__ __forceinline__ float row_exponent(float lse, bool live) {
  return live && lse > -INFINITY && !out_of_sums(lse * kLog2E) ? lse * kLog2E : INFINITY;
}

// ---------------------------------------------------------------------------
// Queries stand still: eight waves of 16 queries in registers, keys and values 64 at a time through LDS. The products S^T = K Q^T and dP^T = V dO^T leave a
// lane with a query's logits and their gradients as the operand of dQ^T += K^T dS^T. Fragments are read some slots before the MFMAs that use them, in
// the order written: left to itself the compiler reads them as they are needed, and a wave waits for the LDS at every one.
// Two waves on a SIMD take turns with the vector and the matrix pipe. With 32 queries a wave half the LDS reads would do, but one wave a SIMD is all that
// the registers hold then (heads of 128, 8191 tokens: first pass 788 us, second 1104; so 610 and 860). First pass in workgroups of four waves, two to a unit: 720;
// with four of the eight waves a phase behind the others, so that the pipes have different work: 800.
// ---------------------------------------------------------------------------
constexpr int kWaves = 8;

template <int DH>
__global__ __launch_bounds__(64 * kWaves, DH == 64 ? 4 : 2) void bias_dq_kernel(Rows Q, Rows K, Rows V, Rows O, const uint16_t* __restrict__ rest, Rows dO,
                                                                                RowsOut dQ, const float* __restrict__ lse, Delta delta, BiasArgs bias,
                                                                                long Lq, long Lk, int B, int H, int group, int nq) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int KB = kTileKeys / 16, NC = kTileKeys / 32, KC = DH / 32, DB = DH / 16, THREADS = 64 * kWaves;
  constexpr int TILE = kTileKeys * DH;
  extern __shared__ __attribute__((aligned(16))) uint16_t smem[];  // [2][TILE] keys, [2][TILE] values, biases
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lq = lane & 15, g = lane >> 4;
  const int width = bias.width(), far = bias.far;
  float* const s_bias = reinterpret_cast<float*>(smem + 4 * TILE);

  const Place place = place_of(blockIdx.x, gridDim.x, B, H, nq, 1);
  const int b = place.b, head = place.head, qb = place.tile;
  const long bh = (long)b * H + head;
  const int origin = __builtin_amdgcn_readfirstlane(bias.origin(b));
  const int q0 = qb * kTileQueries + wave * 16;
  const int last_q = (int)((long)(qb + 1) * kTileQueries < Lq ? (qb + 1) * kTileQueries : Lq) - 1;
  const int n = __builtin_amdgcn_readfirstlane(bias.seen(b, Lk, origin + last_q));  // keys that some query of the workgroup sees
  const int steps = (n + kTileKeys - 1) / kTileKeys;

  TileStage<DH, THREADS> k_in(tid, K.row), v_in(tid, V.row);
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
  BiasFill<THREADS> fill;
  fill.buckets(bias, tid);
  if (steps > 0) fetch(0);

  const RowFragments<DH> rows(lane);
  const ColumnFragments<DH> columns(lane);
  bf16x8 qf[KC], df[KC];
  const bool live = q0 + lq < (int)Lq;
  const int q = live ? q0 + lq : (int)Lq - 1;
  float dl = 0.f, over = 0.f;  // delta; what the row's gradients add up to, this lane's share
  {
    const uint16_t* qp = Q.p + (long)b * Q.batch + q * Q.row + (long)head * DH + 8 * g;
    const uint16_t* dp = dO.p + (long)b * dO.batch + q * dO.row + (long)head * DH + 8 * g;
    const long at = (long)b * O.batch + q * O.row + (long)head * DH + 8 * g;
    u32x4 o[KC], r[KC];
#pragma unroll
    for (int kc = 0; kc < KC; ++kc) {
      qf[kc] = *reinterpret_cast<const bf16x8*>(qp + 32 * kc);
      df[kc] = *reinterpret_cast<const bf16x8*>(dp + 32 * kc);
      o[kc] = *reinterpret_cast<const u32x4*>(O.p + at + 32 * kc);
      r[kc] = *reinterpret_cast<const u32x4*>(rest + at + 32 * kc);
    }
    fill.values(bias, head, H);
#pragma unroll
    for (int kc = 0; kc < KC; ++kc)
#pragma unroll
      for (int e = 0; e < 8; ++e)
        dl = __builtin_fmaf((float)df[kc][e], both_halves((uint16_t)(o[kc][e / 2] >> 16 * (e % 2)), (uint16_t)(r[kc][e / 2] >> 16 * (e % 2))), dl);
    dl += swap_rows16(dl);
    dl += swap_halves(dl);
  }
  // The exponent of the row's sum, in units of the products, and delta: what the sums of the matrix pipe start at.
  const float scale = bias.scale * kLog2E;
  const float row_lse = lse[bh * Lq + q], ex = -row_exponent(row_lse, live) / scale;
  const uint32_t apart = (uint32_t)__ballot(live && out_of_sums(row_lse * kLog2E)) & 0xffff;
  const f32x4 less_ex = {ex, ex, ex, ex}, less_dl = {-dl, -dl, -dl, -dl};
  f32x4 dq[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) dq[db] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int kc = 0; kc < KC; ++kc) asm volatile("" : "+v"(qf[kc]), "+v"(df[kc]));  // resident before the loop, which would wait for them at every tile otherwise
  fill.store(bias, s_bias, tid);
  if (steps > 0) store(0);
  if (steps > 1) fetch(1);
  lds_barrier();
  const float below = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(s_bias[0])));
  const float above = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(s_bias[width - 1])));

  for (int t = 0, buf = 0; t < steps; ++t, buf ^= 1) {
    if (t + 1 < steps) store(buf ^ 1);
    if (t + 2 < steps) fetch(t + 2);
    const uint16_t* const k_tile = smem + buf * TILE;
    const uint16_t* const v_tile = smem + (2 + buf) * TILE;
    f32x4 s[KB], dp[KB];
    {
      constexpr int SLOTS = KB * KC, kAhead = DH == 64 ? 2 : 4;
      bf16x8 kf[SLOTS], vf[SLOTS];
      auto read = [&](int f) {
        kf[f] = rows.read(k_tile, f / KC, f % KC);
        vf[f] = rows.read(v_tile, f / KC, f % KC);
      };
#pragma unroll
      for (int f = 0; f < kAhead; ++f) read(f);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int f = 0; f < SLOTS; ++f) {
        const int kb = f / KC, kc = f % KC;
        if (f + kAhead < SLOTS) read(f + kAhead);
        s[kb] = mfma(kf[f], qf[kc], kc == 0 ? less_ex : s[kb]);
        dp[kb] = mfma(vf[f], df[kc], kc == 0 ? less_dl : dp[kb]);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    constexpr int SLOTS2 = DB * NC, kAhead2 = DH == 64 ? 3 : 4;
    bf16x8 kt[SLOTS2];
    auto read2 = [&](int f) { kt[f] = columns.read(k_tile, f % NC, f / NC); };
#pragma unroll
    for (int f = 0; f < kAhead2; ++f) read2(f);
    __builtin_amdgcn_sched_barrier(0);
    const int nearest = t * kTileKeys - (origin + q0);  // distance of the tile's first key from the wave's first query
    if (nearest + 63 > -far && nearest - 15 < far) {
      const float* at = s_bias + (nearest + far + kPad + 4 * g - lq);
      f32x4 here[KB];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < 4; ++i) here[kb][i] = at[16 * kb + i];
      __builtin_amdgcn_sched_barrier(0);  // all of them requested before the first is used
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[kb][i] = __builtin_fmaf(s[kb][i], scale, here[kb][i]);
    } else {
      const float c = nearest > 0 ? above : below;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[kb][i] = __builtin_fmaf(s[kb][i], scale, c);
    }
    int end = n;  // first key that the wave's first query does not see
    if (bias.causal && origin + q0 + 1 < end) end = origin + q0 + 1;
    if ((t + 1) * kTileKeys > end) {
      int left = n;
      if (bias.causal && origin + q0 + lq + 1 < n) left = origin + q0 + lq + 1;
      left -= t * kTileKeys + 4 * g;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (16 * kb + i >= left) s[kb][i] = -INFINITY;
    }
    bf16x8 ds[NC];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float v = __builtin_amdgcn_exp2f(s[kb][i]) * dp[kb][i];
        over += v;
        ds[kb / 2][4 * (kb % 2) + i] = (bf16_t)v;
      }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int f = 0; f < SLOTS2; ++f) {
      if (f + kAhead2 < SLOTS2) read2(f + kAhead2);
      dq[f / NC] = mfma(kt[f], ds[f % NC], dq[f / NC]);
      __builtin_amdgcn_sched_barrier(0);
    }
    lds_barrier();
  }
  over += swap_rows16(over);
  over += swap_halves(over);
  // rows that are out of the sums, and those that are not finite though their result is, which may be so by an infinity or NaN times the weight 0 of a key
  // that they do not see
  float none = over * 0.f;
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int i = 0; i < 4; ++i) none = __builtin_fmaf(dq[db][i], 0.f, none);
  const uint32_t alone = apart | rows_of_lanes(__ballot(live && !(none == 0.f) && dl * 0.f == 0.f));
  if (g == 0 && live && !(alone >> lq & 1)) delta.p[bh * Lq + q] = dl + over;
  if (lane == 0) delta.apart[(bh * nq + qb) * kWaves + wave] = apart;
  const int row = q0 + (lq & 12) + g;
  if (__builtin_expect(alone != 0, 0)) {
    for (uint32_t left = alone; left; left &= left - 1) {
      const int r = q0 + __builtin_ctz(left), see = !bias.causal || origin + r + 1 > n ? n : origin + r + 1;
      const uint16_t* const dp = dO.p + (long)b * dO.batch + r * dO.row + (long)head * DH;
      ApartRow<DH> x{Q.p + (long)b * Q.batch + r * Q.row + (long)head * DH, k_base, K.row, s_bias, -(origin + r), far, scale, {0.f, 0.f}};
      x.refer(0, see, lane);
      float l = 0.f, d = 0.f, sum[DH / 64];
#pragma unroll 1
      for (int j = lane; j < see; j += 64) {
        const float w = __builtin_amdgcn_exp2f(x.logit(j));
        l += w;
        d = __builtin_fmaf(w, x.product(dp, v_base + (long)j * V.row), d);
      }
      l = wave_sum(l);
      const float by = l == 0.f ? 0.f : 1.0f / l;
      d = wave_sum(d) * by;
      ApartRow<DH>::weighted([&](int j) { return __builtin_amdgcn_exp2f(x.logit(j)) * by * (x.product(dp, v_base + (long)j * V.row) - d); }, k_base, K.row, 0, see,
                             lane, sum);
#pragma unroll
      for (int e = 0; e < DH / 64; ++e) dQ.p[(long)b * dQ.batch + r * dQ.row + (long)head * DH + lane + 64 * e] = f32_to_bf16(sum[e] * bias.scale);
      if (lane < 3) delta.p[lane * delta.step + bh * Lq + r] = lane == 0 ? d : lane == 1 ? x.ref.hi : x.ref.lo + __builtin_amdgcn_logf(l);
    }
  }
  put_columns<DB>(dq, bias.scale, dQ.p + (long)b * dQ.batch + row * dQ.row + (long)head * DH + 8 * (lq & 3),
                  row < (int)Lq && !(alone >> ((lq & 12) + g) & 1), lane);
#endif
}

// ---------------------------------------------------------------------------
// Keys stand still, 128 to a workgroup in registers, queries and their gradients 64 at a time through LDS, over all heads that share the keys.
// S = Q K^T and dP = dO V^T leave a lane with a key's logits as the operand of dV^T += dO^T P and dK^T += Q^T dS. Heads of 128 leave room for 16 keys a
// wave, eight waves; heads of 64 for 32, four waves.
// Sums by distance: a wave's gradients of a near tile are added up along their diagonals. Blocks of 16 x 16 on one diagonal are added in registers;
// then they go to LDS, a row for each of 16 keys, row c shifted c places, so that a column is a distance, which lanes sum and add to the wave's own sum of
// it. Written ahead of the products with dS and summed behind them, so that nobody waits for what was written. A tile whose distances all
// share an end bucket costs one addition a value.
// ---------------------------------------------------------------------------
constexpr int kNone = 32;
template <int DH>
struct KeyShape {
  static constexpr int kBlocks = DH == 64 ? 2 : 1, kWaves = 8 / kBlocks, kThreads = 64 * kWaves;  // blocks of 16 keys of a wave
  static constexpr int kDiagonals = 2 + kBlocks - 1, kPlaces = 16 * kDiagonals + 15, kRow = kPlaces + 2;  // of 32 queries
  static_assert(kPlaces <= 64, "a lane a place");
  static int lds(int width) { return 4 * kTileKeys * DH * 2 + (4 * kTileKeys + kNone + (1 + kWaves) * width + kWaves * 16 * kRow) * 4; }
};

template <int DH>
__global__ __launch_bounds__(KeyShape<DH>::kThreads, 2) void bias_dkv_kernel(Rows Q, Rows K, Rows V, Rows dO, RowsOut dK, RowsOut dV,
                                                                             const float* __restrict__ lse, Delta delta, float* __restrict__ part,
                                                                             BiasArgs bias, long Lq, long Lk, int B, int H, int group, int nk) {
#if defined(__HIP_DEVICE_COMPILE__)
  typedef KeyShape<DH> Shape;
  constexpr int QB = 2, KC = DH / 32, DB = DH / 16, NB = Shape::kBlocks, THREADS = Shape::kThreads;
  constexpr int TILE = kTileKeys * DH, ROW = Shape::kRow;
  extern __shared__ __attribute__((aligned(16))) uint16_t smem[];  // [2][TILE] queries, [2][TILE] their gradients, [2][2][64] exponents and deltas, biases,
                                                                   // sums of each wave, skewed rows of each
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lq = lane & 15, g = lane >> 4;
  const int width = bias.width(), far = bias.far;
  float* const s_rows = reinterpret_cast<float*>(smem + 4 * TILE);
  float* const s_none = s_rows + 4 * kTileKeys + kNone - 1;  // the last of as many biases of -inf
  float* const s_bias = s_none + 1;
  float* const s_sums = s_bias + width + wave * width;
  float* const s_skew = s_bias + (1 + Shape::kWaves) * width + wave * 16 * ROW;

  const Place place = place_of(blockIdx.x, gridDim.x, B, H / group, nk, 1);
  const int b = place.b, kv_head = place.head, kt = place.tile;
  const int origin = __builtin_amdgcn_readfirstlane(bias.origin(b));
  const int n = __builtin_amdgcn_readfirstlane(bias.seen(b, Lk, origin + (int)Lq - 1));  // keys that some query sees
  const int k0 = kt * kTileQueries + wave * 16 * NB;  // the wave's first key
  const int tiles = (int)((Lq + kTileKeys - 1) / kTileKeys);
  int first_tile = 0;
  if (bias.causal) {
    const int q = kt * kTileQueries - origin;  // the first query that sees the workgroup's first key
    first_tile = q <= 0 ? 0 : q / kTileKeys < tiles ? q / kTileKeys : tiles;
  }
  const int each = kt * kTileQueries < n ? tiles - first_tile : 0;
  // a column behind the last key has zeros for it, with a bias of -inf
  bool counts[NB];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) counts[nb] = k0 + 16 * nb + lq < n;

  TileStage<DH, THREADS> q_in(tid, Q.row), d_in(tid, dO.row);
  const float scale = bias.scale * kLog2E, per_scale = 1.0f / scale;
  float row_in = 0.f;
  bool row_live = false;
  auto fetch = [&](int head, int t) {
    q_in.fetch(Q.p + (long)b * Q.batch + (long)t * kTileKeys * Q.row + (long)head * DH, (int)(Lq - 1) - t * kTileKeys);
    d_in.fetch(dO.p + (long)b * dO.batch + (long)t * kTileKeys * dO.row + (long)head * DH, (int)(Lq - 1) - t * kTileKeys);
    if (wave < 2) {
      const float* const from = (wave == 0 ? lse : delta.p) + ((long)b * H + head) * Lq;
      const int q = t * kTileKeys + lane;
      row_live = q < (int)Lq;
      row_in = from[row_live ? q : (int)Lq - 1];  // looked at when it is stored: here the wave would wait for it
    }
  };
  auto store = [&](int buf) {
    q_in.store(smem + buf * TILE);
    d_in.store(smem + (2 + buf) * TILE);
    if (wave < 2) s_rows[buf * 2 * kTileKeys + tid] = wave == 0 ? -row_exponent(row_in, row_live) * per_scale : -row_in;
  };

  BiasFill<THREADS> fill;
  fill.buckets(bias, tid);
  const RowFragments<DH> rows(lane);
  const ColumnFragments<DH> columns(lane);
  bf16x8 kf[NB][KC], vf[NB][KC];
  f32x4 dk[NB][DB], dv[NB][DB];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    int k = k0 + 16 * nb + lq;
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
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
#pragma unroll
    for (int kc = 0; kc < KC; ++kc) {
      if (!counts[nb]) kf[nb][kc] = vf[nb][kc] = bf16x8{};
      asm volatile("" : "+v"(kf[nb][kc]), "+v"(vf[nb][kc]));  // resident before the loop, which would wait for them at every tile otherwise
    }
  for (int i = lane; i < 16 * ROW; i += 64) s_skew[i] = 0.f;
  if (tid < kNone) s_none[-tid] = -INFINITY;

  for (int in_group = 0; in_group < group; ++in_group) {
    const int head = kv_head * group + in_group;
    if (each > 0) fetch(head, first_tile);
    fill.values(bias, head, H);
    for (int i = lane; i < width; i += 64) s_sums[i] = 0.f;
    fill.store(bias, s_bias, tid);
    if (each > 0) store(0);
    if (each > 1) fetch(head, first_tile + 1);
    lds_barrier();
    const float below = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(s_bias[0])));
    const float above = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(s_bias[width - 1])));
    float sum_below = 0.f, sum_above = 0.f;
    for (int i = 0, buf = 0; i < each; ++i, buf ^= 1) {
      const int t = first_tile + i;
      if (i + 1 < each) store(buf ^ 1);
      if (i + 2 < each) fetch(head, t + 2);
      // half of the tile's queries at a time: logits and their gradients of all of them would not leave the registers that two waves a SIMD have
#pragma unroll 1
      for (int half = 0; half < 2; ++half) {
        const uint16_t* const q_tile = smem + buf * TILE + half * 32 * DH;
        const uint16_t* const d_tile = smem + (2 + buf) * TILE + half * 32 * DH;
        const float* const ex = s_rows + buf * 2 * kTileKeys + half * 32 + 4 * g;
        f32x4 s[QB][NB], dp[QB][NB];
        {
          constexpr int SLOTS = QB * KC, kAhead = NB == 2 ? 3 : 4;
          bf16x8 qf[SLOTS], df[SLOTS];
          auto read = [&](int f) {
            qf[f] = rows.read(q_tile, f / KC, f % KC);
            df[f] = rows.read(d_tile, f / KC, f % KC);
          };
          // what the sums of the matrix pipe start at: the rows' exponents, in units of the products, and deltas
          f32x4 less_ex[QB], less_dl[QB];
#pragma unroll
          for (int qb = 0; qb < QB; ++qb) {
            less_ex[qb] = *reinterpret_cast<const f32x4*>(ex + 16 * qb);
            less_dl[qb] = *reinterpret_cast<const f32x4*>(ex + kTileKeys + 16 * qb);
          }
#pragma unroll
          for (int f = 0; f < kAhead; ++f) read(f);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int f = 0; f < SLOTS; ++f) {
            const int qb = f / KC, kc = f % KC;
            if (f + kAhead < SLOTS) read(f + kAhead);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
              s[qb][nb] = mfma(qf[f], kf[nb][kc], kc == 0 ? less_ex[qb] : s[qb][nb]);
              dp[qb][nb] = mfma(df[f], vf[nb][kc], kc == 0 ? less_dl[qb] : dp[qb][nb]);
            }
            __builtin_amdgcn_sched_barrier(0);
          }
        }
        constexpr int kAhead2 = 3;
        bf16x8 qc[DB], dc[DB];
        auto read2 = [&](int f) {
          dc[f] = columns.read(d_tile, 0, f);
          qc[f] = columns.read(q_tile, 0, f);
        };
#pragma unroll
        for (int f = 0; f < kAhead2; ++f) read2(f);
        __builtin_amdgcn_sched_barrier(0);
        const int nearest = k0 - (origin + t * kTileKeys + 32 * half);  // distance of the wave's first key from the half's first query
        const bool near = nearest + 16 * NB - 1 > -far && nearest - 31 < far;
        if (near) {
          f32x4 here[NB][QB];
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            const float* at = counts[nb] ? s_bias + (nearest + 16 * nb + far + kPad + lq - 4 * g) : s_none;
#pragma unroll
            for (int qb = 0; qb < QB; ++qb)
#pragma unroll
              for (int e = 0; e < 4; ++e) here[nb][qb][e] = at[-16 * qb - e];
          }
          __builtin_amdgcn_sched_barrier(0);  // all of them requested before the first is used
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int qb = 0; qb < QB; ++qb)
#pragma unroll
              for (int e = 0; e < 4; ++e) s[qb][nb][e] = __builtin_fmaf(s[qb][nb][e], scale, here[nb][qb][e]);
        } else {
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            const float c = counts[nb] ? (nearest > 0 ? above : below) : -INFINITY;
#pragma unroll
            for (int qb = 0; qb < QB; ++qb)
#pragma unroll
              for (int e = 0; e < 4; ++e) s[qb][nb][e] = __builtin_fmaf(s[qb][nb][e], scale, c);
          }
        }
        if (bias.causal && nearest + 16 * NB - 1 > 0) {
#pragma unroll
          for (int qb = 0; qb < QB; ++qb)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (nearest + 16 * (nb - qb) + lq - 4 * g - e > 0) {
                  s[qb][nb][e] = -INFINITY;
                  dp[qb][nb][e] = 0.f;  // an infinity or NaN of the key is not the query's
                }
        }
        bf16x8 pf[NB], ds[NB];
#pragma unroll
        for (int qb = 0; qb < QB; ++qb)
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float p = __builtin_amdgcn_exp2f(s[qb][nb][e]);
              s[qb][nb][e] = p * dp[qb][nb][e];
              pf[nb][4 * qb + e] = (bf16_t)p;
              ds[nb][4 * qb + e] = (bf16_t)s[qb][nb][e];
            }
        if (near) {
          float* const row = s_skew + lq * (ROW + 1) + 15 - 4 * g;
#pragma unroll
          for (int d = 0; d < Shape::kDiagonals; ++d) {  // nb - qb = d - (QB - 1)
            f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
              const int qb = nb - d + QB - 1;
              if (qb >= 0 && qb < QB) v += s[qb][nb];
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) row[16 * d - e] = v[e];
          }
        } else {
          float a = 0.f;
#pragma unroll
          for (int qb = 0; qb < QB; ++qb)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) a += (s[qb][nb][0] + s[qb][nb][1]) + (s[qb][nb][2] + s[qb][nb][3]);
          if (nearest > 0) sum_above += a;
          else sum_below += a;
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int f = 0; f < DB; ++f) {
          if (f + kAhead2 < DB) read2(f + kAhead2);
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            dv[nb][f] = mfma(dc[f], pf[nb], dv[nb][f]);
            dk[nb][f] = mfma(qc[f], ds[nb], dk[nb][f]);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        if (near) {
          __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
          if (lane < Shape::kPlaces) {
            float a[16], *const sum = s_sums + (nearest - 31 + far + kPad + lane);
            const float before = *sum;
#pragma unroll
            for (int c = 0; c < 16; ++c) a[c] = s_skew[c * ROW + lane];
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int n2 = 8; n2 > 0; n2 /= 2)
#pragma unroll
              for (int c = 0; c < n2; ++c) a[c] += a[c + n2];
            *sum = before + a[0];
          }
          __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
        }
      }
      lds_barrier();
    }
    // rows that are out of the sums: 16 of a word, a key a lane, whose four lanes share its values
    const int words = (int)((Lq + kTileQueries - 1) / kTileQueries) * kWaves;
    const uint32_t* const apart = delta.apart + ((long)b * H + head) * words;
    uint32_t some = 0;
    for (int i = lane; i < words; i += 64) some |= apart[i];
    if (__builtin_expect(each > 0 && __any(some), 0)) {
#pragma unroll 1
      for (int w = 0; w < words; ++w) {
#pragma unroll 1
        for (uint32_t left = (uint32_t)__builtin_amdgcn_readfirstlane((int)apart[w]); left; left &= left - 1) {
          const int r = 16 * w + __builtin_ctz(left);
          const float* const of = delta.p + ((long)b * H + head) * Lq + r;
          const float dl = of[0], ref = of[delta.step], log_sum = of[2 * delta.step];
          const uint16_t* const qp = Q.p + (long)b * Q.batch + r * Q.row + (long)head * DH;
          const uint16_t* const dp = dO.p + (long)b * dO.batch + r * dO.row + (long)head * DH;
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            float x = 0.f, y = 0.f;
#pragma unroll
            for (int kc = 0; kc < KC; ++kc) {
              const bf16x8 qv = *reinterpret_cast<const bf16x8*>(qp + 32 * kc + 8 * g), dv8 = *reinterpret_cast<const bf16x8*>(dp + 32 * kc + 8 * g);
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                x = __builtin_fmaf((float)qv[e], (float)kf[nb][kc][e], x);
                y = __builtin_fmaf((float)dv8[e], (float)vf[nb][kc][e], y);
              }
            }
            x += swap_rows16(x);
            x += swap_halves(x);
            y += swap_rows16(y);
            y += swap_halves(y);
            const int dist = k0 + 16 * nb + lq - (origin + r), at = dist + far + kPad;
            const bool sees = counts[nb] && !(bias.causal && dist > 0);
            const float bias_here = s_bias[at < 0 ? 0 : at < width ? at : width - 1];
            const float pw = sees ? __builtin_amdgcn_exp2f(__builtin_fmaf(x, products_by(scale, ref), (bias_here - ref) - log_sum)) : 0.f;
            const float dsw = sees ? pw * (y - dl) : 0.f;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                dv[nb][db][e] = __builtin_fmaf(pw, bf16_to_f32(dp[16 * db + 4 * g + e]), dv[nb][db][e]);
                dk[nb][db][e] = __builtin_fmaf(dsw, bf16_to_f32(qp[16 * db + 4 * g + e]), dk[nb][db][e]);
              }
            if (g == 0) {  // 16 distances, each of one lane
              if (at < 0) sum_below += dsw;
              else if (at >= width) sum_above += dsw;
              else s_sums[at] += dsw;
            }
          }
        }
      }
    }
    sum_below = wave_sum(sum_below);
    sum_above = wave_sum(sum_above);
    if (lane == 0) {
      s_sums[0] += sum_below;
      s_sums[width - 1] += sum_above;
    }
    lds_barrier();
    for (int i = tid; i < width; i += THREADS) {
      float a = 0.f;
#pragma unroll
      for (int w = 0; w < Shape::kWaves; ++w) a += s_bias[(1 + w) * width + i];
      part[(((long)b * H + head) * nk + kt) * width + i] = a;
    }
    lds_barrier();
  }
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    if (!counts[nb]) {  // zeros, and no infinity or NaN of a gradient times 0
#pragma unroll
      for (int db = 0; db < DB; ++db) dk[nb][db] = dv[nb][db] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const int k = k0 + 16 * nb + (lq & 12) + g;
    const long at = (long)kv_head * DH + 8 * (lq & 3);
    put_columns<DB>(dk[nb], bias.scale, dK.p + (long)b * dK.batch + k * dK.row + at, k < (int)Lk, lane);
    put_columns<DB>(dv[nb], 1.0f, dV.p + (long)b * dV.batch + k * dV.row + at, k < (int)Lk, lane);
  }
#endif
}

// Adds up the sums by distance. First, 64 distances of a head a workgroup, whose four waves share out sequences and tiles of keys; then a wave a
// bucket and head over the distances of the bucket. Every order depends on the sizes alone.
__global__ __launch_bounds__(256) void bias_distances_kernel(const float* __restrict__ part, double* __restrict__ sums, int width, int B, int H, int nk) {
  __shared__ double s_sum[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, head = blockIdx.y, i = blockIdx.x * 64 + lane;
  const long n = (long)B * nk;
  double a = 0.0;
  if (i < width)
#pragma unroll 8
    for (long k = wave; k < n; k += 4) {
      const long b = k / nk;
      a += (double)part[((b * H + head) * nk + (k - b * nk)) * width + i];
    }
  s_sum[wave][lane] = a;
  __syncthreads();
  if (wave == 0 && i < width) sums[(long)head * width + i] = (s_sum[0][lane] + s_sum[1][lane]) + (s_sum[2][lane] + s_sum[3][lane]);
}
__global__ __launch_bounds__(256) void bias_dtable_kernel(const double* __restrict__ sums, float* __restrict__ dtable, BiasArgs bias, int H) {
  const int lane = threadIdx.x & 63, c = blockIdx.x * 4 + (threadIdx.x >> 6), head = blockIdx.y, width = bias.width();
  if (c >= bias.n_buckets) return;
  double a = 0.0;
  for (int i = lane; i < width; i += 64) {
    int at = i - kPad;
    at = at < 0 ? 0 : at > 2 * bias.far ? 2 * bias.far : at;
    if (bias.bucket[at] == c) a += sums[(long)head * width + i];
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) a += __shfl_xor(a, d);
  if (lane == 0) dtable[(long)c * H + head] = (float)a;
}

// Both in one launch, a workgroup a head, where sequences times tiles of keys are few: a pass with both directions, which the host's side bounds then, takes 44.9
// us with one tile of keys and 48.0 with two launches, 46.4 and 48.5 with 8, 148.3 and 149.6 with 16 of 64 heads; 90.6 and 89.9 with 32, 1176 and 1125 with 1024.
constexpr long kFewParts = 16;
constexpr int kTableThreads = 1024;
__global__ __launch_bounds__(kTableThreads) void bias_table_kernel(const float* __restrict__ part, float* __restrict__ dtable, BiasArgs bias, int B, int H,
                                                                   int nk) {
  constexpr int HALF = kTableThreads / 2, MOST = 2 * (kMostFar + kPad) + 1;
  __shared__ double s_sum[2][MOST];
  __shared__ int s_bucket[MOST];
  const int tid = threadIdx.x, head = blockIdx.x, width = bias.width(), n = B * nk, share = tid / HALF;
  for (int i = tid; i < width; i += kTableThreads) s_bucket[i] = bias.bucket_of(i);
  for (int i = tid % HALF; i < width; i += HALF) {
    double a = 0.0;
#pragma unroll 8
    for (int k = share; k < n; k += 2) {
      const int b = k / nk;
      a += (double)part[(((long)b * H + head) * nk + (k - b * nk)) * width + i];
    }
    s_sum[share][i] = a;
  }
  __syncthreads();
  const int lane = tid & 63;
  for (int c = tid >> 6; c < bias.n_buckets; c += kTableThreads / 64) {
    double a = 0.0;
    for (int i = lane; i < width; i += 64)
      if (s_bucket[i] == c) a += s_sum[0][i] + s_sum[1][i];
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) a += __shfl_xor(a, d);
    if (lane == 0) dtable[(long)c * H + head] = (float)a;
  }
}

struct BackwardLayout {
  size_t delta, apart, part, sums, all;
  int nq, nk;
  explicit BackwardLayout(const chorus_bias_attention& a) {
    nq = (int)((a.Lq + kTileQueries - 1) / kTileQueries);
    nk = (int)((a.Lk + kTileQueries - 1) / kTileQueries);
    delta = 0;
    apart = align_up((size_t)a.B * a.H * (size_t)a.Lq * 3 * sizeof(float), 256);
    part = apart + align_up((size_t)a.B * a.H * nq * kWaves * sizeof(uint32_t), 256);
    const size_t width = (size_t)(2 * (a.far + kPad) + 1);
    sums = part + align_up((size_t)a.B * a.H * nk * width * sizeof(float), 256);
    all = sums + (size_t)a.H * width * sizeof(double);
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
  if (a->B > 1 && (steps->dq_batch == 0 || steps->dk_batch == 0 || steps->dv_batch == 0)) return CHORUS_E_SHAPE;
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
  const Delta delta{reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + at.delta), (long)a->B * a->H * (long)a->Lq,
                    reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(ws) + at.apart)};
  float* const part = reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + at.part);
  const int tiles = 4 * kTileKeys * a->dh * 2, most_width = 2 * (kMostFar + kPad) + 1;
  const int lds_q = tiles + bias.width() * 4;
  hipStream_t s = (hipStream_t)stream;
#define BACKWARD(DH)                                                                                                                          \
  do {                                                                                                                                        \
    static DynLdsOnce once_q, once_k;                                                                                                         \
    CHK_STATUS(once_q.ensure((const void*)bias_dq_kernel<DH>, tiles + most_width * 4));                             \
    CHK_STATUS(once_k.ensure((const void*)bias_dkv_kernel<DH>, KeyShape<DH>::lds(most_width)));                                    \
    hipLaunchKernelGGL((bias_dq_kernel<DH>), dim3((unsigned)((long)a->B * a->H * at.nq)), dim3(64 * kWaves), lds_q, s, q, k, v, o, rest, d, gq, lse,  \
                       delta, bias, (long)a->Lq, (long)a->Lk, a->B, a->H, a->H / a->Hk, at.nq);                                               \
    CHORUS_LAUNCH_CHECK();                                                                                                                    \
    hipLaunchKernelGGL((bias_dkv_kernel<DH>), dim3((unsigned)((long)a->B * a->Hk * at.nk)), dim3(KeyShape<DH>::kThreads),                             \
                       KeyShape<DH>::lds(bias.width()), s, q, k, v, d, gk, gv, lse, delta, part, bias, (long)a->Lq, (long)a->Lk, a->B, a->H,          \
                       a->H / a->Hk, at.nk);                                                                                                          \
    CHORUS_LAUNCH_CHECK();                                                                                                                    \
  } while (0)
  if (a->dh == 128) BACKWARD(128);
  else BACKWARD(64);
#undef BACKWARD
  if ((long)a->B * at.nk <= kFewParts) {
    hipLaunchKernelGGL(bias_table_kernel, dim3((unsigned)a->H), dim3(kTableThreads), 0, s, (const float*)part, dtable, bias, a->B, a->H, at.nk);
    CHORUS_LAUNCH_CHECK();
    return CHORUS_OK;
  }
  double* const sums = reinterpret_cast<double*>(static_cast<uint8_t*>(ws) + at.sums);
  hipLaunchKernelGGL(bias_distances_kernel, dim3((unsigned)((bias.width() + 63) / 64), (unsigned)a->H), dim3(256), 0, s, (const float*)part, sums,
                     bias.width(), a->B, a->H, at.nk);
  CHORUS_LAUNCH_CHECK();
  hipLaunchKernelGGL(bias_dtable_kernel, dim3((unsigned)((a->n_buckets + 3) / 4), (unsigned)a->H), dim3(256), 0, s, (const double*)sums, dtable, bias, a->H);
  CHORUS_LAUNCH_CHECK();
  return CHORUS_OK;
}

}  // extern "C"
