// Attention whose logits get a learned bias by the bucket of the distance between query and key, forward: O = softmax(scale Q K^T + bias) V, over
// the keys of each sequence of a padded batch, causal or not, one query or many.
//
// The tiled kernel: a workgroup of four waves takes 128 queries of a head, 32 a wave in registers, and walks over the keys 64 at a time, in
// tiles in LDS that come from the rows as a projection leaves them. S^T = K Q^T leaves a lane with the logits of one query row in the order in
// which its weights are the operand of O^T += V^T P^T; V^T comes out of the rows of V by transposing LDS reads. A step has two phases:
// the weights on the vector pipe; then this tile's share of the result and the next one's logits on the matrix pipe, the next tiles on
// their way in registers meanwhile. One barrier a step; two or three waves a SIMD take turns with the pipes.
// The bias of a distance is in LDS, in powers of two, `far` and a tile's width to either side. A wave's 64 x 32 logits read it only where some
// distance is below `far`; tiles beyond have one value. The sums of the matrix pipe start at minus the row's reference, so that a logit
// becomes the exponent of its weight in one fma.
// Measured: two prompts of 512 and 256 tokens, 64 heads of 64, 17 to 18 us; of that 7.5 before the first and behind the last step, for which the lengths, the biases
// and the first tiles are fetched one behind the other; a step 1.1 us, bound by the vector pipe's 160 instructions and 32 exponentials for 32
// MFMAs. Halving the rows of a workgroup changed nothing. 8191 tokens, 12 heads of 128, weights in two parts: 612 us, 1010 TFLOP/s with the second parts' products.
#include "bias_attention.h"

namespace chorus {
namespace {

constexpr int kMostSlices = 64;  // the join holds a slice a lane

// Tiles of 128 queries whose workgroups leave compute units idle are cut into slices of the keys: about two workgroups for every unit, none of less
// than four steps.
int slices_of(long tiles, long Lk) {
  const long steps = (Lk + kTileKeys - 1) / kTileKeys;
  long s = tiles >= 256 ? 1 : (512 + tiles - 1) / tiles;
  if (s > steps / 4) s = steps / 4;
  return s < 1 ? 1 : s > kMostSlices ? kMostSlices : (int)s;
}
size_t slice_bytes(long tiles, int slices, int dh, int rows) {
  return slices > 1 ? (size_t)tiles * slices * rows * (dh * sizeof(float) + sizeof(Share)) : 0;
}

struct Outputs {
  RowsOut o;
  uint16_t* rest;  // as o, the other half of the bits
  float* lse;      // [B, H, Lq]
};

// SPLIT: for the backward pass a weight goes to the matrix pipe in two parts of 8 bits, 16 together, and the other half of the result's bits goes out as well:
// delta = dO . O then has 16 bits in the products for dQ (relative error of dQ against 64 bits 0.0024, 0.0025 with weights of 8 bits; 8191 tokens, 12 heads of
// 128 486 to 612 us). The second pass and the table's sums have their delta from the first one's sums, whatever that of dO . O was.
template <int DH, bool SPLIT>
__global__ __launch_bounds__(256, DH == 64 ? 3 : 2) void bias_attention_kernel(Rows Q, Rows K, Rows V, Outputs out, BiasArgs bias, float* __restrict__ part, long Lq,
                                                                long Lk, int B, int H, int group, int nq, int slices) {
#if defined(__HIP_DEVICE_COMPILE__)  // the buffer descriptors below are types of the device compiler's alone
  constexpr int KB = kTileKeys / 16, NC = kTileKeys / 32, KC = DH / 32, DB = DH / 16, RB = 2, PARTS = SPLIT ? 2 : 1;
  constexpr int TILE = kTileKeys * DH;
  extern __shared__ __attribute__((aligned(16))) uint16_t smem[];  // [2][TILE] keys, [2][TILE] values, biases
  float* const s_bias = reinterpret_cast<float*>(smem + 4 * TILE);

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lq = lane & 15, g = lane >> 4;
  const Place place = place_of(blockIdx.x, gridDim.x, B, H, nq, slices);
  const int b = place.b, head = place.head, qb = place.tile, slice = place.slice, unit = ((head * B + b) * nq + qb) * slices + slice;
  const int origin = __builtin_amdgcn_readfirstlane(bias.origin(b));
  const int q0 = qb * kTileQueries + wave * 32;  // the wave's first query
  const int last_q = (int)((long)(qb + 1) * kTileQueries < Lq ? (qb + 1) * kTileQueries : Lq) - 1;
  const int n = __builtin_amdgcn_readfirstlane(bias.seen(b, Lk, origin + last_q));  // keys that some query of the workgroup sees
  const int steps = (n + kTileKeys - 1) / kTileKeys;
  const int t0 = slices > 1 ? steps * slice / slices : 0, t1 = slices > 1 ? steps * (slice + 1) / slices : steps;  // at most 2^22 steps and 64 slices

  BiasFill<256> fill;
  fill.buckets(bias, tid);
  TileStage<DH, 256> k_in(tid, K.row), v_in(tid, V.row);
  const uint16_t* const k_base = K.p + (long)b * K.batch + (long)(head / group) * DH;
  const uint16_t* const v_base = V.p + (long)b * V.batch + (long)(head / group) * DH;
  auto fetch_k = [&](int t) { k_in.fetch(k_base + (long)t * kTileKeys * K.row, n - 1 - t * kTileKeys); };
  auto fetch_v = [&](int t) { v_in.fetch(v_base + (long)t * kTileKeys * V.row, n - 1 - t * kTileKeys); };
  if (t0 < t1) {
    fetch_k(t0);
    fetch_v(t0);
  }
  const int width = bias.width(), far = bias.far;
  const RowFragments<DH> k_at(lane);
  const ColumnFragments<DH> v_at(lane);
  bf16x8 qf[RB][KC];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    int q = q0 + 16 * rb + lq;
    if (q > (int)Lq - 1) q = (int)Lq - 1;
    const uint16_t* qp = Q.p + (long)b * Q.batch + q * Q.row + (long)head * DH + 8 * g;
#pragma unroll
    for (int kc = 0; kc < KC; ++kc) qf[rb][kc] = *reinterpret_cast<const bf16x8*>(qp + 32 * kc);
  }
  fill.values(bias, head, H);
#pragma unroll
  for (int rb = 0; rb < RB; ++rb)
#pragma unroll
    for (int kc = 0; kc < KC; ++kc) asm volatile("" : "+v"(qf[rb][kc]));  // resident before the loop, which would wait for them at every tile otherwise
  if (t0 < t1) {
    k_in.store(smem);
    v_in.store(smem + 2 * TILE);
    if (t0 + 1 < t1) fetch_k(t0 + 1);
  }
  f32x4 o[DB][RB], s[KB][RB];
  // A row's reference, in powers of two, and the sum of its weights: in every lane, made by the matrix pipe of the rounded ones, which are what weights
  // the values; SPLIT: of the exact ones, a lane's share
  float m_run[RB], l_run[RB];
  f32x4 l_sum[RB];
  bf16x8 ones;
#pragma unroll
  for (int e = 0; e < 8; ++e) ones[e] = (bf16_t)1.0f;
  f32x4 less_m[RB];  // minus the reference, in units of the products: what the sums of the matrix pipe start at
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    m_run[rb] = 0.f;
    l_run[rb] = 0.f;
    l_sum[rb] = f32x4{0.f, 0.f, 0.f, 0.f};
    less_m[rb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int db = 0; db < DB; ++db) o[db][rb] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  bool fresh = true;       // some row of the wave has seen no finite logit
  bool seen[RB] = {false, false};
  const float scale = bias.scale * kLog2E;

  fill.store(bias, s_bias, tid);
  lds_barrier();
  const float below = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(s_bias[0])));
  const float above = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(s_bias[width - 1])));
  if (t0 < t1) {
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        s[kb][rb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kc = 0; kc < KC; ++kc) s[kb][rb] = mfma(k_at.read(smem, kb, kc), qf[rb][kc], s[kb][rb]);
      }
  }
  if (t0 + 1 < t1) {
    k_in.store(smem + TILE);
    fetch_v(t0 + 1);
    if (t0 + 2 < t1) fetch_k(t0 + 2);
  }
  lds_barrier();

  // logits of tile t: scaled, with their bias, less the reference
  auto logits = [&](int t) {
    const int nearest = t * kTileKeys - (origin + q0);  // distance of the tile's first key from the wave's first query
    if (nearest + 63 > -far && nearest - 31 < far) {
      const float* at = s_bias + (nearest + far + kPad + 4 * g - lq);
      f32x4 here[KB + RB - 1];
#pragma unroll
      for (int d = 0; d < KB + RB - 1; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) here[d][i] = at[16 * (d - RB + 1) + i];
      __builtin_amdgcn_sched_barrier(0);  // all of them requested before the first is used
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[kb][rb][i] = __builtin_fmaf(s[kb][rb][i], scale, here[kb - rb + RB - 1][i]);
    } else {
      const float c = nearest > 0 ? above : below;
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[kb][rb][i] = __builtin_fmaf(s[kb][rb][i], scale, c);
    }
    int end = n;  // first key that the wave's first query does not see
    if (bias.causal && origin + q0 + 1 < end) end = origin + q0 + 1;
    if ((t + 1) * kTileKeys > end) {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        int rest = n;
        if (bias.causal && origin + q0 + 16 * rb + lq + 1 < n) rest = origin + q0 + 16 * rb + lq + 1;
        rest -= t * kTileKeys + 4 * g;
        asm volatile("" : "+v"(rest));  // compared here: hoisted, the results would fill the scalar registers
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (16 * kb + i >= rest) s[kb][rb][i] = -INFINITY;
      }
    }
  };
  // The reference moves when a row exceeds it by more than 2^8, and to the first finite logit of a row, or to kLeastReference if that is less.
  auto move = [&]() {
    float mx[RB];
    bool far_up = fresh;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      mx[rb] = s[0][rb][0];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < 4; ++i) mx[rb] = fmaxf(mx[rb], s[kb][rb][i]);
      far_up = far_up || mx[rb] > 8.0f;
    }
    if (!__any(far_up)) return;
    bool none = false;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      float m = fmaxf(mx[rb], swap_rows16(mx[rb]));
      m = fmaxf(m, swap_halves(m));
      const bool finite = m > -INFINITY;
      const float delta = !seen[rb] ? (finite ? fmaxf(m, kLeastReference) : 0.f) : fmaxf(m, 0.f);
      const float alpha = !seen[rb] ? 1.0f : __builtin_amdgcn_exp2f(-delta);
      seen[rb] = seen[rb] || finite;
      none = none || !seen[rb];
      m_run[rb] += delta;
      const float from = -m_run[rb] / scale;
      less_m[rb] = f32x4{from, from, from, from};
      if (SPLIT) l_run[rb] *= alpha;
      else l_sum[rb] *= alpha;
#pragma unroll
      for (int db = 0; db < DB; ++db) o[db][rb] *= alpha;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) s[kb][rb] -= delta;
    }
    fresh = __any(none);
  };

  int buf = 0;
  for (int t = t0; t < t1; ++t, buf ^= 1) {
    // ================= vector phase: the weights of this tile =================
    __builtin_amdgcn_sched_barrier(0);
    logits(t);
    move();
    bf16x8 pf[PARTS][NC][RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int c = 0; c < NC; ++c) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float p = __builtin_amdgcn_exp2f(s[2 * c + (e >> 2)][rb][e & 3]);
          if (SPLIT) l_run[rb] += p;
          pf[0][c][rb][e] = (bf16_t)p;
          if (SPLIT) pf[PARTS - 1][c][rb][e] = (bf16_t)(p - (float)pf[0][c][rb][e]);
        }
      }
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int a = 0; a < PARTS; ++a) asm volatile("" : "+v"(pf[a][c][rb]));  // here and not where they are used
    // what was requested a step ago: the keys behind the next tile's over this tile's, whose logits are made, the next tile's values
    // beside this one's
    if (t + 2 < t1) k_in.store(smem + buf * TILE);
    if (t + 1 < t1) v_in.store(smem + (2 + (buf ^ 1)) * TILE);
    if (t + 3 < t1) fetch_k(t + 3);
    if (t + 2 < t1) fetch_v(t + 2);
    __builtin_amdgcn_sched_barrier(0);
    // ================= matrix phase: this tile's share of the result, and the logits of the next one =================
    // A slot is two MFMAs and the read of the fragment that is used kAhead slots on.
    __builtin_amdgcn_s_setprio(1);
    constexpr int VS = DB * NC, SLOTS = VS + KB * KC, kAhead = DH == 64 ? 3 : 4;
    bf16x8 fr[SLOTS];
    auto read = [&](int f) {
      fr[f] = f < VS ? v_at.read(smem + (2 + buf) * TILE, f % NC, f / NC) : k_at.read(smem + (buf ^ 1) * TILE, (f - VS) / KC, (f - VS) % KC);
    };
#pragma unroll
    for (int f = 0; f < kAhead; ++f) read(f);
    __builtin_amdgcn_sched_barrier(0);
    if (!SPLIT) {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int c = 0; c < NC; ++c) l_sum[rb] = mfma(ones, pf[0][c][rb], l_sum[rb]);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        if (i < VS) {
          const int db = i / NC, rb = i % NC, c = u;
#pragma unroll
          for (int a = 0; a < PARTS; ++a) o[db][rb] = mfma(fr[db * NC + c], pf[a][c][rb], o[db][rb]);
        } else {
          const int kb = (i - VS) / KC, at = (i - VS) % KC * 2 + u, rb = at / KC, kc = at % KC;
          s[kb][rb] = mfma(fr[VS + kb * KC + kc], qf[rb][kc], kc == 0 ? less_m[rb] : s[kb][rb]);
        }
      }
      if (i + kAhead < SLOTS) read(i + kAhead);
      __builtin_amdgcn_sched_barrier(0);
    }
    static_assert(NC == 2 && RB == 2 && SLOTS > kAhead, "a slot's two MFMAs");
    __builtin_amdgcn_s_setprio(0);
    lds_barrier();
    __builtin_amdgcn_sched_barrier(0);
  }

  // On the way out four neighbouring lanes write 64 bytes of a row: they get them from the lanes of that row.
  const auto from_lane = [](int src, uint32_t v) { return (uint32_t)__builtin_amdgcn_ds_bpermute(4 * src, (int)v); };
  int out_lane = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
  asm volatile("" : "+v"(out_lane));  // the lane again: what is made of it would take registers that the loop needs
  const int out_q = out_lane & 15, out_g = out_lane >> 4, row0 = q0 + (out_q & 12) + out_g, b4 = out_q & 3;
  uint32_t all_apart = 0;
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    if (SPLIT) {
      l_run[rb] += swap_rows16(l_run[rb]);
      l_run[rb] += swap_halves(l_run[rb]);
    }
    const float l = SPLIT ? l_run[rb] : l_sum[rb][0], inv = l == 0.f ? 0.f : 1.0f / l;  // no key at all: a row of zeros
    const int row = row0 + 16 * rb, mine = q0 + 16 * rb + out_q, count = (int)Lq;
    // rows that are out of the sums: all their logits are far below the reference, or it is too large. And rows that are not finite though their weights are,
    // which may be so by an infinity or NaN times the weight 0 of a key that they do not see, or the other part of a weight.
    float none = 0.f;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int i = 0; i < 4; ++i) none = __builtin_fmaf(o[db][rb][i], 0.f, none);
    const uint32_t apart = rows_of_lanes(__ballot(mine < count && ((!(none == 0.f) && l * 0.f == 0.f) || (seen[rb] && (l < kLeastSum || out_of_sums(m_run[rb]))))));
    all_apart |= apart << 16 * rb;
    const bool live = row < count && !(apart >> ((out_q & 12) + out_g) & 1), mine_live = mine < count && !(apart >> out_q & 1);
    if (slices > 1) {
      const long at = (long)unit * kTileQueries;
      float* op = part + (at + (row - qb * kTileQueries)) * DH + 4 * b4;
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        f32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = __uint_as_float(from_lane(16 * b4 + (out_q & 12) + out_g, __float_as_uint(o[db][rb][e])));
        if (live) *reinterpret_cast<f32x4*>(op + 16 * db) = v;
      }
      if (out_g == 0 && mine_live)
        reinterpret_cast<Share*>(part + (long)gridDim.x * kTileQueries * DH)[at + (mine - qb * kTileQueries)] = Share{{m_run[rb], 0.f}, l};
      continue;
    }
    const long to = (long)b * out.o.batch + row * out.o.row + (long)head * DH + 8 * b4;
    const int src = 16 * (b4 >> 1 | (b4 & 1) << 1) + (out_q & 12) + out_g;
    auto put = [&](uint16_t* p, bool rest) {
#pragma unroll
      for (int i = 0; i < DB / 2; ++i) {
        // 4 values of block 2i and 4 of 2i + 1 here, and as many with the lane 16 further: after the swap eight of the one here, of
        // the other there
        const f32x4 x = o[2 * i][rb] * inv, y = o[2 * i + 1][rb] * inv;
        const auto two = [&](float a, float b) {
          return SPLIT && rest ? (uint32_t)left_off(a) | (uint32_t)left_off(b) << 16 : pack_bf16x2(a, b);
        };
        const auto lo = __builtin_amdgcn_permlane16_swap(two(x[0], x[1]), two(y[0], y[1]), false, false);
        const auto hi = __builtin_amdgcn_permlane16_swap(two(x[2], x[3]), two(y[2], y[3]), false, false);
        const u32x4 v = {from_lane(src, lo[0]), from_lane(src, hi[0]), from_lane(src, lo[1]), from_lane(src, hi[1])};
        if (live) *reinterpret_cast<u32x4*>(p + to + 32 * i) = v;
      }
    };
    put(out.o.p, false);
    if (SPLIT) put(out.rest, true);
    if (out.lse && out_g == 0 && mine_live) out.lse[((long)b * H + head) * Lq + mine] = l == 0.f ? -INFINITY : kLn2 * (m_run[rb] + __builtin_amdgcn_logf(l));
  }
  if (__builtin_expect(all_apart != 0, 0)) {
    // places worked out again: kept from the start they would take registers that the loop needs
    int b2 = __builtin_amdgcn_readfirstlane(b), head2 = __builtin_amdgcn_readfirstlane(head), qb2 = __builtin_amdgcn_readfirstlane(qb), at2 = out_lane;
    asm volatile("" : "+s"(b2), "+s"(head2), "+s"(qb2), "+v"(at2));
    const uint16_t* const keys = K.p + (long)b2 * K.batch + (long)(head2 / group) * DH;
    const uint16_t* const values = V.p + (long)b2 * V.batch + (long)(head2 / group) * DH;
    for (uint32_t left = all_apart; left; left &= left - 1) {
      const int r = wave * 32 + __builtin_ctz(left), q = qb2 * kTileQueries + r, see = !bias.causal || origin + q + 1 > n ? n : origin + q + 1;
      const int j0 = t0 * kTileKeys, j1 = t1 * kTileKeys < see ? t1 * kTileKeys : see;
      ApartRow<DH> x{Q.p + (long)b2 * Q.batch + q * Q.row + (long)head2 * DH, keys, K.row, s_bias, -(origin + q), far, scale, {0.f, 0.f}};
      x.refer(j0, j1, at2);
      float sum[DH / 64], total = 0.f;
      ApartRow<DH>::weighted([&](int j) {
        const float w = __builtin_amdgcn_exp2f(x.logit(j));
        total += w;
        return w;
      }, values, V.row, j0, j1, at2, sum);
      total = wave_sum(total);
      const bool some = total != 0.f;
      const long row = (long)(((head2 * B + b2) * nq + qb2) * slices + slice) * kTileQueries + r;
#pragma unroll
      for (int e = 0; e < DH / 64; ++e) {
        if (slices > 1) {
          part[row * DH + at2 + 64 * e] = some ? sum[e] : 0.f;
        } else {
          const float v = some ? sum[e] / total : 0.f;
          const long to = (long)b2 * out.o.batch + q * out.o.row + (long)head2 * DH + at2 + 64 * e;
          out.o.p[to] = f32_to_bf16(v);
          if (SPLIT) out.rest[to] = left_off(v);
        }
      }
      if (at2 == 0) {
        if (slices > 1) reinterpret_cast<Share*>(part + (long)gridDim.x * kTileQueries * DH)[row] = Share{x.ref, total};
        else if (out.lse) out.lse[((long)b2 * H + head2) * Lq + q] = some ? kLn2 * (x.ref.hi + (x.ref.lo + __builtin_amdgcn_logf(total))) : -INFINITY;
      }
    }
  }
#endif
}

// ---------------------------------------------------------------------------
// Few queries: what they take is the time to read the keys and values. Up to 16 rows, the queries of as many of the heads that share keys as fit, make
// one block of columns for the matrix pipe; the eight waves of a workgroup take every eighth tile of 64 keys each, by themselves: keys straight into
// the registers that the matrix pipe reads, values through a region of LDS of the wave's own for their columns, both requested a tile ahead. No barrier
// but for the join of the waves at the end. Four sequences of 64 heads of 64, one query each over 1025 to 4097 keys: 35 us, 4.8 TB/s; 48 where no cache holds a part
// of them, for the longest sequence's workgroups. Two slices of each were 4 % faster there and 1 % slower here, four 25 % slower here.
// ---------------------------------------------------------------------------
constexpr int kFewRows = 16, kFewWaves = 8;

// Where the rows of a workgroup stand: `heads` neighbouring heads of those that share keys, Lq queries each.
struct FewPlace {
  int heads, parts;  // of a workgroup; workgroups for the heads that share keys
};

template <int DH>
__global__ __launch_bounds__(64 * kFewWaves, 2) void bias_few_kernel(Rows Q, Rows K, Rows V, Outputs out, BiasArgs bias, float* __restrict__ part, int Lq,
                                                                     long Lk, int H, int group, FewPlace place, int slices) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int KB = kTileKeys / 16, NC = kTileKeys / 32, KC = DH / 32, DB = DH / 16, TILE = kTileKeys * DH;
  extern __shared__ __attribute__((aligned(16))) uint16_t smem[];  // [waves][TILE] values, then the waves' results; biases of each head
  float* const s_bias = reinterpret_cast<float*>(smem + kFewWaves * TILE);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lq = lane & 15, g = lane >> 4, Hk = H / group, width = bias.width(), far = bias.far;
  const int unit = blockIdx.x, tile = slices > 1 ? unit / slices : unit, slice = unit - tile * slices;
  const int in_group = tile % place.parts, bk = tile / place.parts, b = bk / Hk, kv_head = bk - b * Hk;
  const int head0 = kv_head * group + in_group * place.heads;
  const int heads = group - in_group * place.heads < place.heads ? group - in_group * place.heads : place.heads;
  const int origin = __builtin_amdgcn_readfirstlane(bias.origin(b)), n = __builtin_amdgcn_readfirstlane(bias.seen(b, Lk, origin + Lq - 1));
  const int live_rows = heads * Lq, row = lq < live_rows ? lq : live_rows - 1, of_head = row / Lq, q = row - of_head * Lq;
  const int steps = (n + kTileKeys - 1) / kTileKeys;
  const int t0 = (slices > 1 ? steps * slice / slices : 0) + wave, t1 = slices > 1 ? steps * (slice + 1) / slices : steps;
  int t = t0;

  BiasFill<64 * kFewWaves> fill;
  fill.buckets(bias, tid);
  TileStage<DH, 64> v_in(lane, V.row);
  const uint16_t* const k_base = K.p + (long)b * K.batch + (long)kv_head * DH;
  const uint16_t* const v_base = V.p + (long)b * V.batch + (long)kv_head * DH;
  const int k_bytes = (int)(K.row * 2);
  u32x4 kf[KB][KC];
  auto fetch_k = [&](int at) {
    const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(uniform(k_base + (long)at * kTileKeys * K.row), 0, -1, 0x00027000);
    const int rest = n - 1 - at * kTileKeys;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      const int r = 16 * kb + lq;
      const int from = (r < rest ? r : rest) * k_bytes + 16 * g;
#pragma unroll
      for (int kc = 0; kc < KC; ++kc) kf[kb][kc] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, from, 64 * kc, 0));
    }
  };
  auto fetch_v = [&](int at) { v_in.fetch(v_base + (long)at * kTileKeys * V.row, n - 1 - at * kTileKeys); };
  if (t < t1) {
    fetch_k(t);
    fetch_v(t);
  }
  bf16x8 qf[KC];
  {
    const uint16_t* qp = Q.p + (long)b * Q.batch + (long)q * Q.row + (long)(head0 + of_head) * DH + 8 * g;
#pragma unroll
    for (int kc = 0; kc < KC; ++kc) qf[kc] = *reinterpret_cast<const bf16x8*>(qp + 32 * kc);
  }
  for (int h = 0; h < heads; ++h) {
    fill.values(bias, head0 + h, H);
    fill.store(bias, s_bias + h * width, tid);
  }
  lds_barrier();
  const float* const my_bias = s_bias + of_head * width;
  const float below = my_bias[0], above = my_bias[width - 1];
  const float scale = bias.scale * kLog2E;
  const ColumnFragments<DH> v_at(lane);
  uint16_t* const v_tile = smem + wave * TILE;
  int end = n;  // first key that this lane's query does not see
  if (bias.causal && origin + q + 1 < end) end = origin + q + 1;

  f32x4 o[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) o[db] = f32x4{0.f, 0.f, 0.f, 0.f};
  Reference ref{0.f, 0.f};  // in powers of two
  float l_run = 0.f;        // this lane's share of the sum of the weights
  bool holds = false;       // something is left of that sum
  for (; t < t1; t += kFewWaves) {
    f32x4 s[KB];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      s[kb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kc = 0; kc < KC; ++kc) s[kb] = mfma(__builtin_bit_cast(bf16x8, kf[kb][kc]), qf[kc], s[kb]);
    }
    v_in.store(v_tile);
    if (t + kFewWaves < t1) {
      fetch_k(t + kFewWaves);
      fetch_v(t + kFewWaves);
    }
    const int nearest = t * kTileKeys - origin;  // distance of the tile's first key from query 0
    f32x4 here[KB];
    if (nearest + 63 > -far && nearest - (kFewRows - 1) < far) {
      const float* at = my_bias + (nearest - q + far + kPad + 4 * g);
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < 4; ++i) here[kb][i] = at[16 * kb + i];
      __builtin_amdgcn_sched_barrier(0);
    } else {
      const float c = nearest > 0 ? above : below;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) here[kb] = f32x4{c, c, c, c};
    }
    const int left = end - t * kTileKeys - 4 * g;
    if (__any(left < kTileKeys)) {
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (16 * kb + i >= left) {
            here[kb][i] = -INFINITY;
            s[kb][i] = 0.f;
          }
    }
    // Bias less reference first: both can be of a size that leaves nothing of the products. For the same reason a row's first reference, and one that has gone
    // far up, from a mask's size to that of the keys behind it, is looked at once more: the largest logit was off by a rounding of the mask then. As there is
    // nothing in the sums, it may go down.
    const auto exponent = [&](int kb, int i, float by) { return __builtin_fmaf(s[kb][i], by, (here[kb][i] - ref.hi) - ref.lo); };
    bool finite = false;
#pragma unroll 1
    for (int again = 0; again < 2; ++again) {
      const float by = products_by(scale, ref.hi);
      float mx = -INFINITY;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < 4; ++i) mx = fmaxf(mx, exponent(kb, i, by));
      if (!__any(!holds || mx > 8.0f)) break;  // as in the tiled kernel
      float m = fmaxf(mx, swap_rows16(mx));
      m = fmaxf(m, swap_halves(m));
      finite = m > -INFINITY;
      const float up = holds ? fmaxf(m, 0.f) : finite ? m : 0.f;
      const float alpha = holds ? __builtin_amdgcn_exp2f(-up) : 1.0f;
      holds = holds && alpha > 0.f;
      ref.move(up);
      l_run *= alpha;
#pragma unroll
      for (int db = 0; db < DB; ++db) o[db] *= alpha;
    }
    holds = holds || finite;
    const float by = products_by(scale, ref.hi);
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int i = 0; i < 4; ++i) s[kb][i] = exponent(kb, i, by);
    bf16x8 pf[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float p = __builtin_amdgcn_exp2f(s[2 * c + (e >> 2)][e & 3]);
        l_run += p;
        pf[c][e] = (bf16_t)p;
      }
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int c = 0; c < NC; ++c) o[db] = mfma(v_at.read(v_tile, c, db), pf[c], o[db]);
  }
  l_run += swap_rows16(l_run);
  l_run += swap_halves(l_run);

  // the waves' results, [wave][row][DH] and their shares: put together in the order of the waves
  lds_barrier();
  float* const s_o = reinterpret_cast<float*>(smem);
  Share* const s_share = reinterpret_cast<Share*>(s_o + kFewWaves * kFewRows * (DH + 4));
#pragma unroll
  for (int db = 0; db < DB; ++db) *reinterpret_cast<f32x4*>(s_o + (wave * kFewRows + lq) * (DH + 4) + 16 * db + 4 * g) = o[db];
  if (g == 0) s_share[wave * kFewRows + lq] = Share{ref, l_run};
  // Rows that are not finite though their weights are: made again of the keys that they see, as in the tiled kernel: this wave's part of them, with its weights.
  float none = 0.f;
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int i = 0; i < 4; ++i) none = __builtin_fmaf(o[db][i], 0.f, none);
  for (uint32_t left = rows_of_lanes(__ballot(lq < live_rows && !(none == 0.f) && l_run * 0.f == 0.f)); __builtin_expect(left != 0, 0); left &= left - 1) {
    const int r = __builtin_ctz(left), of = r / Lq, qi = r - of * Lq, see = !bias.causal || origin + qi + 1 > n ? n : origin + qi + 1;
    const Reference at{__uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ref.hi), r)), __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ref.lo), r))};
    const ApartRow<DH> x{Q.p + (long)b * Q.batch + (long)qi * Q.row + (long)(head0 + of) * DH, k_base, K.row, s_bias + of * width, -(origin + qi), far, scale, at};
    float sum[DH / 64] = {};
    for (int i = t0; i < t1; i += kFewWaves) {
      const int j0 = i * kTileKeys, j1 = j0 + kTileKeys < see ? j0 + kTileKeys : see;
      float here[DH / 64];
      ApartRow<DH>::weighted([&](int j) { return __builtin_amdgcn_exp2f(x.logit(j)); }, v_base, V.row, j0, j1, lane, here);
#pragma unroll
      for (int e = 0; e < DH / 64; ++e) sum[e] += here[e];
    }
#pragma unroll
    for (int e = 0; e < DH / 64; ++e) s_o[(wave * kFewRows + r) * (DH + 4) + lane + 64 * e] = sum[e];
  }
  lds_barrier();
  constexpr int PER = 64 * kFewWaves / kFewRows, E = DH / PER;  // threads of a row; values of a thread
  const int r = tid / PER, d0 = tid % PER * E;
  if (r >= live_rows) return;
  Reference top{-INFINITY, -INFINITY};
  float total = 0.f, sum[E] = {};
#pragma unroll
  for (int w = 0; w < kFewWaves; ++w) {
    const Share x = s_share[w * kFewRows + r];
    if (x.sum != 0.f) top.hi = fmaxf(top.hi, x.ref.hi);
  }
#pragma unroll
  for (int w = 0; w < kFewWaves; ++w) {
    const Share x = s_share[w * kFewRows + r];
    if (x.sum != 0.f) top.lo = fmaxf(top.lo, (x.ref.hi - top.hi) + x.ref.lo);
  }
#pragma unroll
  for (int w = 0; w < kFewWaves; ++w) {
    const Share x = s_share[w * kFewRows + r];
    const float f = x.sum != 0.f ? __builtin_amdgcn_exp2f((x.ref.hi - top.hi) + x.ref.lo - top.lo) : 0.f;
    total = __builtin_fmaf(f, x.sum, total);
#pragma unroll
    for (int e = 0; e < E; ++e) sum[e] = __builtin_fmaf(f, s_o[(w * kFewRows + r) * (DH + 4) + d0 + e], sum[e]);
  }
  if (slices > 1) {
    float* op = part + ((long)unit * kFewRows + r) * DH + d0;
#pragma unroll
    for (int e = 0; e < E; ++e) op[e] = sum[e];
    if (d0 == 0) reinterpret_cast<Share*>(part + (long)gridDim.x * kFewRows * DH)[(long)unit * kFewRows + r] = Share{top, total};
    return;
  }
  const int head = head0 + r / Lq, qi = r % Lq;
  const float inv = total == 0.f ? 0.f : 1.0f / total;
  uint16_t* op = out.o.p + (long)b * out.o.batch + (long)qi * out.o.row + (long)head * DH + d0;
#pragma unroll
  for (int e = 0; e < E; ++e) op[e] = f32_to_bf16(sum[e] * inv);
  if (out.lse && d0 == 0) out.lse[((long)b * H + head) * Lq + qi] = total == 0.f ? -INFINITY : kLn2 * (top.hi + (top.lo + __builtin_amdgcn_logf(total)));
#endif
}

// Puts the slices of a row together, a wave a row: the largest reference, then the slices' results and sums by their distance from it, in
// an order that depends on nothing but their number. FEW: rows of several heads, as bias_few_kernel has them; otherwise queries of one.
template <int DH, bool FEW>
__global__ __launch_bounds__(256) void bias_join_kernel(const float* __restrict__ part, Outputs out, long Lq, int B, int H, int group, int nq,
                                                        FewPlace place, int slices, long units) {
  constexpr int E = DH / 64, ROWS = FEW ? kFewRows : kTileQueries;  // values of a lane; rows of a unit
  const int lane = threadIdx.x & 63;
  const long at = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
  const long tile = at / ROWS;
  const int row = (int)(at - tile * ROWS);
  if (tile >= units / slices) return;
  long b, q;
  int head;
  if (FEW) {
    const int Hk = H / group, in_group = (int)(tile % place.parts);
    const long bk = tile / place.parts;
    b = bk / Hk;
    const int of_group = in_group * place.heads + row / (int)Lq;
    if (row >= place.heads * (int)Lq || of_group >= group) return;
    head = (int)(bk - b * Hk) * group + of_group;
    q = row % (int)Lq;
  } else {
    const long hb = tile / nq;
    head = (int)(hb / B);
    b = hb - (long)head * B;
    q = (tile - hb * nq) * ROWS + row;
    if (q >= Lq) return;
  }
  const long first = tile * slices * ROWS + row;
  Share x{{0.f, 0.f}, 0.f};
  if (lane < slices) x = reinterpret_cast<const Share*>(part + units * ROWS * DH)[first + (long)lane * ROWS];
  const bool some = x.sum != 0.f;  // a slice without a key has no reference
  const float hi = wave_max(some ? x.ref.hi : -INFINITY), behind = (x.ref.hi - hi) + x.ref.lo, lo = wave_max(some ? behind : -INFINITY);
  const float w = some ? __builtin_amdgcn_exp2f(behind - lo) : 0.f;
  const float total = wave_sum(w * x.sum), inv = total == 0.f ? 0.f : 1.0f / total;
  float sum[E] = {};
  for (int s = 0; s < slices; ++s) {
    const float ws = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), s));
    const float* p = part + (first + (long)s * ROWS) * DH + E * lane;
#pragma unroll
    for (int e = 0; e < E; ++e) sum[e] = __builtin_fmaf(ws, p[e], sum[e]);
  }
  const long to = b * out.o.batch + q * out.o.row + (long)head * DH + E * lane;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const float v = sum[e] * inv;
    out.o.p[to + e] = f32_to_bf16(v);
    if (out.rest) out.rest[to + e] = left_off(v);
  }
  if (out.lse && lane == 0) out.lse[((long)b * H + head) * Lq + q] = total == 0.f ? -INFINITY : kLn2 * (hi + (lo + __builtin_amdgcn_logf(total)));
}

struct ForwardPlan {
  bool few;  // a workgroup for the few queries of some heads; otherwise one for 128 queries of a head
  FewPlace place;
  long tiles;
  int nq, slices;
  size_t bytes;
};
// The few queries' kernel takes whole workgroups' worth of keys; slices of the keys where the workgroups would leave compute units idle (two are counted to a
// unit), of at least two tiles for each wave.
ForwardPlan forward_plan(const chorus_bias_attention& a, bool training) {
  ForwardPlan p{};
  p.few = !training && a.Lq <= kFewRows;
  p.nq = (int)((a.Lq + kTileQueries - 1) / kTileQueries);
  if (!p.few) {
    p.tiles = (long)a.B * a.H * p.nq;
    p.slices = slices_of(p.tiles, (long)a.Lk);
    p.bytes = slice_bytes(p.tiles, p.slices, a.dh, kTileQueries);
    return p;
  }
  const int group = a.H / a.Hk;
  p.place.heads = kFewRows / (int)a.Lq < group ? kFewRows / (int)a.Lq : group;
  // the heads' biases have to fit beside the values
  const int room = (160 * 1024 - kFewWaves * kTileKeys * a.dh * 2) / (int)((2 * (a.far + kPad) + 1) * sizeof(float));
  if (p.place.heads > room) p.place.heads = room;
  p.place.parts = (group + p.place.heads - 1) / p.place.heads;
  p.tiles = (long)a.B * a.Hk * p.place.parts;
  const long steps = (a.Lk + kTileKeys - 1) / kTileKeys;
  long s = p.tiles >= 256 ? 1 : (512 + p.tiles - 1) / p.tiles;
  if (s > steps / (2 * kFewWaves)) s = steps / (2 * kFewWaves);
  p.slices = s < 1 ? 1 : s > kMostSlices ? kMostSlices : (int)s;
  p.bytes = slice_bytes(p.tiles, p.slices, a.dh, kFewRows);
  return p;
}
constexpr int64_t kMostTiles = 1 << 22;

}  // namespace

bool bias_step_ok(int64_t row, int64_t batch, int64_t heads, int32_t dh) {
  return row >= heads * dh && row <= (1 << 23) && row % 8 == 0 && batch >= 0 && batch % 8 == 0;
}

int32_t check_bias_sizes(const chorus_bias_attention* a) {
  if (!a) return CHORUS_E_ARG;
  if (a->B < 0 || a->Lq < 0 || a->Lk < 0 || a->H <= 0 || a->Hk <= 0 || a->n_buckets <= 0 || a->far < 0) return CHORUS_E_ARG;
  if (!(a->scale >= 0x1p-30f && a->scale <= 0x1p30f)) return CHORUS_E_ARG;
  if ((a->dh != 64 && a->dh != 128) || a->H % a->Hk || a->far > kMostFar || a->Lq > kMostTokens || a->Lk > kMostTokens) return CHORUS_E_SHAPE;
  if (a->H >= (1 << 16) || a->B > (1 << 20) || a->n_buckets > (1 << 16)) return CHORUS_E_SHAPE;
  if (!bias_step_ok(a->q_row, a->q_batch, a->H, a->dh) || !bias_step_ok(a->k_row, a->k_batch, a->Hk, a->dh) || !bias_step_ok(a->v_row, a->v_batch, a->Hk, a->dh) ||
      !bias_step_ok(a->o_row, a->o_batch, a->H, a->dh) || (a->B > 1 && a->o_batch == 0))
    return CHORUS_E_SHAPE;
  const int64_t nq = (a->Lq + kTileQueries - 1) / kTileQueries, nk = (a->Lk + kTileQueries - 1) / kTileQueries;
  if (nq * a->H > kMostTiles || nk * a->H > kMostTiles || nq * a->H * a->B > kMostTiles || nk * a->H * a->B > kMostTiles) return CHORUS_E_SHAPE;
  return CHORUS_OK;
}

int32_t check_bias_attention(const chorus_bias_attention* a, const float* table, const int32_t* bucket, const int32_t* lens, const int32_t* first,
                             BiasArgs* out) {
  CHK_STATUS(check_bias_sizes(a));
  if (a->B == 0 || a->Lq == 0) return CHORUS_OK;
  if (!table || !bucket || !aligned16(table) || !aligned16(bucket) || !aligned16(lens) || !aligned16(first)) return CHORUS_E_ARG;
  *out = BiasArgs{table, bucket, lens, first, a->n_buckets, a->far, a->causal != 0, a->scale};
  return CHORUS_OK;
}

}  // namespace chorus

using namespace chorus;

extern "C" {

// Steps of the logarithm by the condition (n / near)^steps >= (far / near)^k, whose two sides are the same number only where both are powers of
// one root; long double keeps them to 10^-17 of their size, and two that differ are further apart for every far that the call takes.
int32_t chorus_bias_buckets(int32_t n_buckets, int32_t far, int32_t both_sides, int32_t* bucket) {
  const int side = both_sides ? n_buckets / 2 : n_buckets, near = side / 2, steps = side - near;
  if (n_buckets < 2 || !bucket || (both_sides && n_buckets % 2) || near < 1) return CHORUS_E_ARG;
  if (far > kMostFar || far <= near) return CHORUS_E_SHAPE;
  for (int d = -far; d <= far; ++d) {
    const int n = both_sides ? (d < 0 ? -d : d) : (d < 0 ? -d : 0);
    int of = n;
    if (n >= near) {
      const long double at = (long double)steps * __builtin_logl((long double)n / near) / __builtin_logl((long double)far / near);
      int k = (int)(at + 1e-12L);
      of = near + (k < steps - 1 ? k : steps - 1);
    }
    bucket[d + far] = of + (both_sides && d > 0 ? side : 0);
  }
  return CHORUS_OK;
}

size_t chorus_attention_bias_workspace_bytes(const chorus_bias_attention* a) {
  if (check_bias_sizes(a) != CHORUS_OK || a->B == 0 || a->Lq == 0) return 0;
  const size_t serving = forward_plan(*a, false).bytes, training = forward_plan(*a, true).bytes;
  return serving > training ? serving : training;
}

int32_t chorus_attention_bias(const chorus_bias_attention* a, const uint16_t* Q, const uint16_t* K, const uint16_t* V, uint16_t* O, uint16_t* rest,
                              float* lse, const float* table, const int32_t* bucket, const int32_t* lens, const int32_t* first, void* ws,
                              size_t ws_bytes, void* stream) {
  BiasArgs bias;
  CHK_STATUS(check_bias_attention(a, table, bucket, lens, first, &bias));
  if (a->B == 0 || a->Lq == 0) return CHORUS_OK;
  if (!Q || !O || (a->Lk > 0 && (!K || !V))) return CHORUS_E_ARG;
  if (!aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(O) || !aligned16(rest) || !aligned16(lse) || !aligned16(ws)) return CHORUS_E_ARG;
  const ForwardPlan p = forward_plan(*a, rest != nullptr);
  if (p.bytes && (!ws || ws_bytes < p.bytes)) return CHORUS_E_WORKSPACE;
  const Rows q{Q, (long)a->q_row, (long)a->q_batch}, k{K, (long)a->k_row, (long)a->k_batch}, v{V, (long)a->v_row, (long)a->v_batch};
  const Outputs out{RowsOut{O, (long)a->o_row, (long)a->o_batch}, rest, lse};
  const long units = p.tiles * p.slices;
  const int few_tiles = kFewWaves * kTileKeys * a->dh * 2;
  const int lds = 4 * kTileKeys * a->dh * 2 + bias.width() * 4, most = 4 * kTileKeys * a->dh * 2 + (2 * (kMostFar + kPad) + 1) * 4;
  hipStream_t s = (hipStream_t)stream;
#define ATTEND(DH, SPLIT)                                                                                                               \
  do {                                                                                                                                  \
    static DynLdsOnce once;                                                                                                             \
    CHK_STATUS(once.ensure((const void*)bias_attention_kernel<DH, SPLIT>, most));                                                              \
    hipLaunchKernelGGL((bias_attention_kernel<DH, SPLIT>), dim3((unsigned)units), dim3(256), lds, s, q, k, v, out, bias, (float*)ws,           \
                       (long)a->Lq, (long)a->Lk, a->B, a->H, a->H / a->Hk, p.nq, p.slices);                                                   \
    CHORUS_LAUNCH_CHECK();                                                                                                              \
  } while (0)
#define JOIN(DH, FEW, ROWS)                                                                                                            \
  hipLaunchKernelGGL((bias_join_kernel<DH, FEW>), dim3((unsigned)((p.tiles * ROWS + 3) / 4)), dim3(256), 0, s, (const float*)ws, out, \
                     (long)a->Lq, a->B, a->H, a->H / a->Hk, p.nq, p.place, p.slices, units)
#define FEW(DH)                                                                                                                        \
  do {                                                                                                                                 \
    static DynLdsOnce once;                                                                                                            \
    CHK_STATUS(once.ensure((const void*)bias_few_kernel<DH>, 160 * 1024));                                                             \
    hipLaunchKernelGGL((bias_few_kernel<DH>), dim3((unsigned)units), dim3(64 * kFewWaves), few_tiles + p.place.heads * bias.width() * 4, s, q, k, \
                       v, out, bias, (float*)ws, (int)a->Lq, (long)a->Lk, a->H, a->H / a->Hk, p.place, p.slices);                      \
    CHORUS_LAUNCH_CHECK();                                                                                                             \
    if (p.slices > 1) JOIN(DH, true, kFewRows);                                                                                        \
  } while (0)
  if (p.few) {
    if (a->dh == 128) FEW(128);
    else FEW(64);
    CHORUS_LAUNCH_CHECK();
    return CHORUS_OK;
  }
  if (a->dh == 128) {
    if (rest) ATTEND(128, true);
    else ATTEND(128, false);
  } else {
    if (rest) ATTEND(64, true);
    else ATTEND(64, false);
  }
  if (p.slices > 1) {
    if (a->dh == 128) JOIN(128, false, kTileQueries);
    else JOIN(64, false, kTileQueries);
    CHORUS_LAUNCH_CHECK();
  }
#undef ATTEND
#undef FEW
#undef JOIN
  return CHORUS_OK;
}

}  // extern "C"
