// Attention over listed blocks of keys: O = softmax(Q K^T / sqrt(dh)) V, a query seeing the keys of the blocks in the list of its
// block of 128 queries and head, and no others. bf16 operands on the matrix pipe, fp32 online softmax, logits never leave
// registers.
//
// A workgroup of four waves takes a list: a wave holds 32 of the 128 queries (two blocks of 16, in registers) and all walk over the
// list a block of 64 keys at a time, in tiles in LDS. A compute unit holds two workgroups of heads of 128, a wave of each on every
// SIMD (and four of heads of 64, which take 120 to 128 registers and 32 KB). They get half a step apart by themselves, the matrix
// phase going ahead of the other's vector phase: while the waves of one make the weights of a tile on the vector pipe, those of the
// other keep the matrix pipe busy (O += V P, then the next tile's S = K Q^T). Held apart by barriers across both, as one workgroup
// with two lists, they are no faster where lists are alike (32760 queries 1026 us, 1014 as they are) and wait for each other where
// they are not (13104 queries with 30 to 60 blocks, 12 heads: 236 us, 215). Neighbouring lists meet many of the same blocks, which
// then come from the L2.
//
// What a step has to fit into: 68 MFMAs a wave (1088 cycles of the pipe), 32 exponentials (512) and about 90 other vector
// instructions. Measured (cycles a step, 32760 queries, 103 blocks each, 12 heads): vector phase 1240, matrix phase 1435, so the
// matrix pipe is busy three quarters of the time at the clock that the power management leaves; 1014 us, 1310 TFLOP/s, where the
// dense kernel has 1380 over 13184 keys and 1170 over as many as these lists hold (all three a few percent apart from card to
// card). Queries that are not scaled before cost 32 multiplications a step more, 1085 us where scaled ones took 1046 on the same
// card. Heads of 64 have half the MFMAs but all the exponentials: 590 us and 633 unscaled, 1124 TFLOP/s, the vector pipe issuing 70
// % of the time (52 with heads of 128) and the matrix pipe busy 63 % (72). The probabilities are rounded to bf16 for the matrix
// pipe, once, and their sum is taken over the rounded ones. On the way there: the next logits made beside the exponentials of this
// tile 1165 (the two pipes hardly overlap inside a wave); loops that were unrolled by two for constant buffer addresses 1060 (the
// register allocator gives every MFMA result a new home then, and reads wait for the old ones).
//
// The operand layouts are those of the dense kernel on v_mfma_f32_16x16x32_bf16: S^T = K Q^T leaves a lane with the logits of one query
// row, and in the order in which V^T is stored (chorus_v_transpose) its probabilities are the B operand of O^T += V^T P^T as they stand:
//   lane l: query row l % 16 of each block, g = l / 16; S^T block kb of a tile (16 keys x 16 queries): the K fragment's row r is key
//   32 (kb / 2) + 16 (r / 8) + 8 (kb % 2) + r % 8, so the lane holds keys 32 (kb / 2) + 16 (g / 2) + 8 (kb % 2) + 4 (g % 2) + i.
#include "chorus_ops.h"
#include "common.h"

namespace chorus {
namespace {

constexpr int BQ = CHORUS_BLOCK_QUERIES, BK = CHORUS_BLOCK_KEYS;
constexpr int64_t kMostKeys = 1 << 22;  // a head's keys and values in bytes stay within the 32-bit offsets of the loads
constexpr int kMostSlices = 64;         // the join holds a slice a lane
constexpr int64_t kMostLists = (1 << 24) - 512 * kMostSlices - 2;  // with the last round's slices, 256 threads each, within the 2^32 of a launch

// How a launch goes: the first `whole` lists by one workgroup each, the others cut into `slices` (entry e of a list goes to slice
// e % slices, so that a short list with its end full of -1 is cut evenly), whose results are joined by a second launch.
struct BlockPlan {
  long whole;
  int cut, slices;
};
// Lists that leave the last round of workgroups (two on a compute unit) partly empty, or the only one, are cut into as many slices
// as make that round the shortest. A block takes a workgroup of heads of 128 about 1.2 us alone on its unit and 1.5 beside another,
// heads of 64 seven tenths of that, with two counted to a unit though four fit: the more there are the longer a step of each takes,
// and counted as four the cut comes out worse (us, lists of blocks: 600 of 100 126 as it is, 146 with four; 516 of 200 210, 237;
// 768 of 60 102, 96). A slice costs its fp32 result on the way out and in (3 TB/s), the join 8 us. us, lists of blocks, dh: 40 of
// 118, 128: 6 slices 36, 1 124, 12 40; 32 of 30, 64: 6 slices 15, 1 26, 16 20; 256 of 100, 128: 2 slices 97, 1 122, 4 107; 312 of
// 20, 128: whole 36, 2 slices 49.
BlockPlan block_plan(long lists, int dh, int keep) {
  constexpr long units = 256, places = 2 * units;
  const long cut = lists % places;
  BlockPlan best{lists, 0, 1};
  auto cost = [&](long s) {
    const long n = cut * s, rounds = n / places, rest = n % places;
    const double last = rest == 0 ? 0.0 : rest <= units && n == rest && lists < places ? 1.2 : 1.5;
    return (1.5 * (double)rounds + last) * (dh == 128 ? 1.0 : 0.7) * (double)((keep + s - 1) / s) +
           (s > 1 ? 8.0 + (double)n * BQ * dh * 8.0 / 3e6 : 0.0);
  };
  double least = cost(1);
  for (int s = 2; cut > 0 && s <= kMostSlices && s <= keep; ++s)
    if (cost(s) < 0.9 * least) {
      least = cost(s);
      best = BlockPlan{lists - cut, (int)cut, s};
    }
  return best;
}
size_t plan_bytes(const BlockPlan& p, int dh) {
  return p.slices > 1 ? (size_t)p.cut * p.slices * BQ * (dh * sizeof(float) + sizeof(float2)) : 0;
}

// The blocks of a list in turn, every stride-th entry, 64 of them in the wave's lanes at a time; entries outside [0, nk) are passed over.
struct List {
  const int* at;
  int left, stride, nk, lane, v;
  uint64_t mask;
  __device__ List(const int* list, int entries, int stride_, int nk_, int lane_)
      : at(list), left(entries), stride(stride_), nk(nk_), lane(lane_), v(-1), mask(0) {}
  __device__ int next() {  // -1 behind the last
    while (mask == 0) {
      if (left <= 0) return -1;
      v = lane < left ? at[(long)lane * stride] : -1;
      mask = __ballot((unsigned)v < (unsigned)nk);
      at += 64L * stride;
      left -= 64;
    }
    const int i = __builtin_ctzll(mask);
    mask &= mask - 1;
    return __builtin_amdgcn_readlane(v, i);
  }
};

// PRE: the queries hold log2(e) / sqrt(dh) already, and a logit leaves the matrix pipe as the exponent of its weight.
template <int DH, bool PRE>
__global__ __launch_bounds__(256, 2) void attention_blocks_kernel(const uint16_t* __restrict__ Q, const uint16_t* __restrict__ K,
                                                                  const uint16_t* __restrict__ Vt, uint16_t* __restrict__ O,
                                                                  const int* __restrict__ blocks, float* __restrict__ part, long Lq,
                                                                  long Lk, long LqPad, long LkPad, int H, int group, int nq, int nk, int keep,
                                                                  int whole, int slices, float scale_log2) {
#if defined(__HIP_DEVICE_COMPILE__)  // the buffer descriptors below are types of the device compiler's alone
  constexpr int KB = BK / 16, NC = BK / 32, KC = DH / 32, DB = DH / 16, RB = 2;
  constexpr int K_LD = DH / 32, V_LD = DH / 32;  // 1 KB loads of a wave for a tile
  constexpr int TILE = BK * DH;                  // elements of a tile of keys or values
  extern __shared__ __attribute__((aligned(16))) uint16_t smem[];  // [2][TILE] keys, [2][TILE] values
  typedef __attribute__((address_space(3))) void* Lds;

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lq = lane & 15, g = lane >> 4;
  // cut lists come last, in ranges of their own on every XCD: with the others' they would all be on the last one
  const int units = gridDim.x, front = whole < units ? whole : 0;
  const int unit = (int)blockIdx.x < front ? xcd_remap(blockIdx.x, front) : front + xcd_remap(blockIdx.x - front, units - front);
  const bool sliced = unit >= whole;
  const int tile = sliced ? whole + (unit - whole) / slices : unit, slice = sliced ? (unit - whole) % slices : 0;
  const int head = tile / nq, qb = tile - head * nq;

  // ---- a tile's way into LDS: each wave instruction fills 1 KB in order, and a lane fetches the 16 bytes that belong at its place. Rows of
  // keys (DH values) and of values (64) hold their 16-byte pieces at position piece ^ swizzle(row), such that the 16 rows of a
  // fragment read meet all banks. The rows of a wave's i-th load are those of the first and i times those of four waves further on, which
  // only the swizzle of the keys may see, in every other load.
  const auto k_swizzle = [](int row) { return DH == 128 ? (row & 7) | (row >> 4 & 1) << 3 : (row >> 1 & 3) | (row >> 4 & 1) << 2; };
  const auto v_swizzle = [](int row) { return row >> 1 & 7; };
  constexpr int PIECES = DH / 8, K_ROWS = 4 * 64 / PIECES, K_WAYS = K_ROWS == 16 ? 2 : 1;
  uint32_t k_from[K_WAYS], v_from;
#pragma unroll
  for (int i = 0; i < K_WAYS; ++i) {
    const int row = i * K_ROWS + wave * (64 / PIECES) + lane / PIECES;
    k_from[i] = (uint32_t)(row * DH * 2 + (lane % PIECES ^ k_swizzle(row)) * 16);
  }
  {
    const int row = wave * 8 + lane / 8;
    v_from = (uint32_t)(row * (int)LkPad * 2 + (lane % 8 ^ v_swizzle(row)) * 16);
  }
  const int v_step = 32 * (int)LkPad * 2;
  const auto k_rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)(K + (long)(head / group) * LkPad * DH), 0, (int)(LkPad * DH * 2), 0x00027000);
  const auto v_rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)(Vt + (long)(head / group) * LkPad * DH), 0, (int)(LkPad * DH * 2), 0x00027000);
  auto load_k = [&](int b, int buf) {
#pragma unroll
    for (int i = 0; i < K_LD; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(k_rsrc, (Lds)(smem + buf * TILE + (4 * i + wave) * 512), 16, k_from[i % K_WAYS],
                                               b * (TILE * 2) + i / K_WAYS * K_WAYS * K_ROWS * DH * 2, 0, 0);
  };
  auto load_v = [&](int b, int buf, int i) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(v_rsrc, (Lds)(smem + (2 + buf) * TILE + (4 * i + wave) * 512), 16, v_from,
                                             b * (BK * 2) + i * v_step, 0, 0);
  };
  // ---- and out of it
  int k_at[KC], v_at[NC];
#pragma unroll
  for (int kc = 0; kc < KC; ++kc) {
    const int row = 16 * (lq >> 3) + (lq & 7);
    k_at[kc] = row * DH + ((4 * kc + g) ^ k_swizzle(row)) * 8;
    asm volatile("" : "+v"(k_at[kc]));  // kept in registers, not made again from the lane in every matrix phase
  }
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    v_at[c] = lq * BK + ((4 * c + g) ^ v_swizzle(lq)) * 8;
    asm volatile("" : "+v"(v_at[c]));
  }
  auto k_frag = [&](int buf, int kb, int kc) {
    return *reinterpret_cast<const bf16x8*>(&smem[buf * TILE + (32 * (kb >> 1) + 8 * (kb & 1)) * DH + k_at[kc]]);
  };
  auto v_frag = [&](int buf, int db, int c) { return *reinterpret_cast<const bf16x8*>(&smem[(2 + buf) * TILE + 16 * db * BK + v_at[c]]); };

  bf16x8 qf[RB][KC];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    // four neighbouring lanes read 64 bytes of a row, which is a request; what they hold is another lane's, where lq % 4 and g
    // change places
    long q = (long)qb * BQ + wave * 32 + 16 * rb + (lq & 12) + g;
    if (q > Lq - 1) q = Lq - 1;
    const uint16_t* qp = Q + ((long)head * LqPad + q) * DH + 8 * (lq & 3);
#pragma unroll
    for (int kc = 0; kc < KC; ++kc) qf[rb][kc] = *reinterpret_cast<const bf16x8*>(qp + 32 * kc);
  }
  f32x4 o[DB][RB], s[KB][RB];
  // A row's reference, in units of its logits, and the sum of its weights (in every element; the matrix pipe adds up the rounded
  // weights, which are what weights the values: 64 cycles there against 128 of the busier vector phase). S^T accumulators start at minus
  // the reference.
  float m_run[RB];
  f32x4 l_run[RB];
  bf16x8 ones;
#pragma unroll
  for (int e = 0; e < 8; ++e) ones[e] = (bf16_t)1.0f;
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    m_run[rb] = 0.f;
    l_run[rb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int db = 0; db < DB; ++db) o[db][rb] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  bool fresh = true;  // some row of the wave has seen no finite logit
  auto mask = [&](int b) {  // keys behind the last
    int rest = (int)(Lk - (long)b * BK) - (16 * (g >> 1) + 4 * (g & 1));
    asm volatile("" : "+v"(rest));  // compared here: hoisted, the results would fill the scalar registers
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (32 * (kb >> 1) + 8 * (kb & 1) + i >= rest) {
#pragma unroll
          for (int rb = 0; rb < RB; ++rb) s[kb][rb][i] = -INFINITY;
        }
  };
  // The reference moves when a row exceeds it by more than 2^8, and to the first finite logit of a row whatever that is. Each lane looks
  // at its own logits; those of a row's four lanes meet only when it moves.
  const float most = PRE ? 8.0f : 8.0f / scale_log2;
  auto move = [&]() {
    float mx[RB];
    bool far = fresh;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      mx[rb] = s[0][rb][0];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < 4; ++i) mx[rb] = fmaxf(mx[rb], s[kb][rb][i]);
      far = far || mx[rb] > most;
    }
    if (!__any(far)) return;
    bool none = false;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      float m = fmaxf(mx[rb], swap_rows16(mx[rb]));
      m = fmaxf(m, swap_halves(m));
      const bool first = l_run[rb][0] == 0.f, finite = m > -INFINITY;
      const float delta = first ? (finite ? m : 0.f) : fmaxf(m, 0.f);
      const float alpha = first ? 1.0f : __builtin_amdgcn_exp2f(-delta * (PRE ? 1.0f : scale_log2));
      none = none || (first && !finite);
      m_run[rb] += delta;
      l_run[rb] *= alpha;
#pragma unroll
      for (int db = 0; db < DB; ++db) o[db][rb] *= alpha;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) s[kb][rb] -= delta;
    }
    fresh = __any(none);
  };

  List list(blocks + (long)tile * keep + slice, sliced ? (keep - slice + slices - 1) / slices : keep, sliced ? slices : 1, nk, lane);
  const int tail = Lk % BK ? nk - 1 : -2;  // the block that is not full
  int b0 = list.next(), b1 = -1, b2 = -1;  // this tile and the two behind it; behind the last, this one is loaded again and not used
  if (b0 >= 0) {
    b1 = list.next();
    if (b1 >= 0) b2 = list.next();
    load_k(b0, 0);
#pragma unroll
    for (int i = 0; i < V_LD; ++i) load_v(b0, 0, i);
    load_k(b1 < 0 ? b0 : b1, 1);
  }
#pragma unroll
  for (int rb = 0; rb < RB; ++rb)
#pragma unroll
    for (int kc = 0; kc < KC; ++kc) {
      u32x4 u = __builtin_bit_cast(u32x4, qf[rb][kc]);
#pragma unroll
      for (int e = 0; e < 4; ++e) u[e] = __builtin_amdgcn_ds_bpermute(4 * (16 * (lq & 3) + (lq & 12) + g), u[e]);
      qf[rb][kc] = __builtin_bit_cast(bf16x8, u);
      asm volatile("" : "+v"(qf[rb][kc]));  // resident before the loop, which would wait for them otherwise
    }
  asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
  if (b0 >= 0) {
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        s[kb][rb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kc = 0; kc < KC; ++kc) s[kb][rb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k_frag(0, kb, kc), qf[rb][kc], s[kb][rb], 0, 0, 0);
      }
  }
  asm volatile("s_barrier" ::: "memory");

  for (int buf = 0; b0 >= 0; buf ^= 1) {
    // ================= vector phase: the weights of this tile =================
    __builtin_amdgcn_sched_barrier(0);
    load_k(b2 < 0 ? b0 : b2, buf);  // over this tile's keys, whose logits are made
    if (b0 == tail) mask(b0);
    move();
    bf16x8 pf[NC][RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int c = 0; c < NC; ++c) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float x = s[2 * c + (e >> 2)][rb][e & 3];
          pf[c][rb][e] = (bf16_t)__builtin_amdgcn_exp2f(PRE ? x : x * scale_log2);
        }
      }
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) asm volatile("" : "+v"(pf[c][rb]));  // here and not where they are used
    const int v_next = b1 < 0 ? b0 : b1;
    b0 = b1;
    b1 = b2;
    if (b1 >= 0) b2 = list.next();
    __builtin_amdgcn_sched_barrier(0);
    // this tile's values and the next one's keys, requested a step ago, are in LDS for all four waves; the keys requested above are
    // not waited for
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(K_LD) : "memory");
    __builtin_amdgcn_sched_barrier(0);
    // ================= matrix phase: this tile's share of the result, and the logits of the next one =================
    // Written out in the order in which it is to run: the compiler moves no LDS read across a load into LDS. A slot is two MFMAs and the
    // read of the fragment that is used kAhead slots on; every fourth also requests a piece of the next tile's values.
    __builtin_amdgcn_s_setprio(1);
    constexpr int VS = DB * NC, SLOTS = VS + KB * KC, kAhead = 4, kFirst = 2, kEvery = 4;
    bf16x8 fr[SLOTS];
    auto read = [&](int f) { fr[f] = f < VS ? v_frag(buf, f / NC, f % NC) : k_frag(buf ^ 1, (f - VS) / KC, (f - VS) % KC); };
#pragma unroll
    for (int f = 0; f < kAhead; ++f) read(f);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int c = 0; c < NC; ++c) l_run[rb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pf[c][rb], l_run[rb], 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        if (i < VS) {
          const int db = i / NC, rb = i % NC, c = u;
          o[db][rb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fr[db * NC + c], pf[c][rb], o[db][rb], 0, 0, 0);
        } else {
          const int kb = (i - VS) / KC, at = (i - VS) % KC * 2 + u, rb = at / KC, kc = at % KC;
          if (kc == 0) s[kb][rb] = f32x4{-m_run[rb], -m_run[rb], -m_run[rb], -m_run[rb]};
          s[kb][rb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fr[VS + kb * KC + kc], qf[rb][kc], s[kb][rb], 0, 0, 0);
        }
      }
      if (i + kAhead < SLOTS) read(i + kAhead);
      if (i % kEvery == kFirst && i / kEvery < V_LD) load_v(v_next, buf ^ 1, i / kEvery);
      __builtin_amdgcn_sched_barrier(0);
    }
    static_assert(NC == 2 && RB == 2 && (V_LD - 1) * kEvery + kFirst < SLOTS && SLOTS > kAhead, "a slot's two MFMAs, and all the loads, have their places");
    __builtin_amdgcn_s_setprio(0);
    asm volatile("s_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // no load may land in the LDS of a workgroup that has ended

  // On the way out, as with the queries, four neighbouring lanes write 64 bytes of a row: they get them from the lanes of that row.
  const auto from_lane = [](int src, uint32_t v) { return (uint32_t)__builtin_amdgcn_ds_bpermute(4 * src, (int)v); };
  const int row0 = wave * 32 + (lq & 12) + g, b4 = lq & 3;
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int row = row0 + 16 * rb;
    const bool live = (long)qb * BQ + row < Lq;
    const float l = l_run[rb][0];
    if (sliced) {
      const long at = (long)(unit - whole) * BQ;
      float* op = part + (at + row) * DH + 4 * b4;
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        f32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = __uint_as_float(from_lane(16 * b4 + (lq & 12) + g, __float_as_uint(o[db][rb][e])));
        if (live) *reinterpret_cast<f32x4*>(op + 16 * db) = v;
      }
      if (g == 0 && (long)qb * BQ + wave * 32 + 16 * rb + lq < Lq)
        reinterpret_cast<float2*>(part + (long)(units - whole) * BQ * DH)[at + wave * 32 + 16 * rb + lq] = make_float2(m_run[rb], l);
    } else {
      const float inv = l == 0.f ? 0.f : 1.0f / l;  // no key at all: a row of zeros
      uint16_t* op = O + ((long)qb * BQ + row) * ((long)H * DH) + (long)head * DH + 8 * b4;
      const int src = 16 * (b4 >> 1 | (b4 & 1) << 1) + (lq & 12) + g;
#pragma unroll
      for (int i = 0; i < DB / 2; ++i) {
        // 4 values of block 2i and 4 of 2i + 1 here, and as many with the lane 16 further: after the swap eight of the one here, of
        // the other there
        const f32x4 x = o[2 * i][rb] * inv, y = o[2 * i + 1][rb] * inv;
        const auto lo = __builtin_amdgcn_permlane16_swap(pack_bf16x2(x[0], x[1]), pack_bf16x2(y[0], y[1]), false, false);
        const auto hi = __builtin_amdgcn_permlane16_swap(pack_bf16x2(x[2], x[3]), pack_bf16x2(y[2], y[3]), false, false);
        const u32x4 v = {from_lane(src, lo[0]), from_lane(src, hi[0]), from_lane(src, lo[1]), from_lane(src, hi[1])};
        if (live) *reinterpret_cast<u32x4*>(op + 32 * i) = v;
      }
    }
  }
#endif
}

// Puts the slices of a row together, W waves a row: the largest reference, then the slices' results and sums by their distance from
// it, in an order that depends on nothing but their number. Bound by the way to them: with one wave a row, its 42 slices were 10
// reads one behind the other (60 rows, 12 heads 10.4 us).
template <int DH, int W>
__global__ __launch_bounds__(256) void attention_blocks_join_kernel(const float* __restrict__ part, uint16_t* __restrict__ O, long Lq, int H, int nq,
                                                                    int whole, int slices, int cut, float scale_log2) {
  constexpr int ROWS = 4 / W, E = DH / 64;  // of a workgroup; values of a lane
  __shared__ float s_sum[4][DH];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int at = blockIdx.x / (BQ / ROWS), row = blockIdx.x % (BQ / ROWS) * ROWS + wave / W, share = wave % W;
  const int tile = whole + at, head = tile / nq;
  const long q = (long)(tile - head * nq) * BQ + row;
  const bool live = q < Lq;
  if (W == 1 && !live) return;
  const long first = (long)at * slices * BQ + row;
  const float2 ml = live && lane < slices ? reinterpret_cast<const float2*>(part + (long)cut * slices * BQ * DH)[first + (long)lane * BQ] : make_float2(0.f, 0.f);
  const float m = ml.y != 0.f ? ml.x : -INFINITY;  // a slice without a key has no reference
  const float top = wave_max(m);
  const float w = ml.y != 0.f ? __builtin_amdgcn_exp2f((m - top) * scale_log2) : 0.f;
  const float total = wave_sum(w * ml.y);
  const float inv = total == 0.f ? 0.f : 1.0f / total;
  float sum[E] = {};
  for (int s = share; live && s < slices; s += W) {
    const float* p = part + (first + (long)s * BQ) * DH + E * lane;
    const float ws = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), s));
    float v[E];
    if (E == 2) {
      const float2 two = *reinterpret_cast<const float2*>(p);
      v[0] = two.x;
      v[E - 1] = two.y;
    } else {
      v[0] = *p;
    }
#pragma unroll
    for (int e = 0; e < E; ++e) sum[e] = __builtin_fmaf(ws, v[e], sum[e]);
  }
  if (W > 1) {
#pragma unroll
    for (int e = 0; e < E; ++e) s_sum[wave][E * lane + e] = sum[e];
    __syncthreads();
    if (share != 0 || !live) return;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      sum[e] = 0.f;
#pragma unroll
      for (int i = 0; i < W; ++i) sum[e] += s_sum[wave + i][E * lane + e];
    }
  }
  uint16_t* op = O + q * (long)H * DH + (long)head * DH;
  if (E == 2) reinterpret_cast<uint32_t*>(op)[lane] = pack_bf16x2(sum[0] * inv, sum[E - 1] * inv);
  else op[lane] = f32_to_bf16(sum[0] * inv);
}

}  // namespace
}  // namespace chorus

using namespace chorus;

extern "C" {

size_t chorus_attention_blocks_workspace_bytes(int64_t Lq, int32_t H, int32_t dh, int32_t keep) {
  if (Lq <= 0 || H <= 0 || (dh != 64 && dh != 128) || keep < 1 || Lq > 0x7fffffffL) return 0;
  const int64_t nq = (Lq + BQ - 1) / BQ;
  return nq > kMostLists / H ? 0 : plan_bytes(block_plan((long)(nq * H), dh, keep), dh);
}

int32_t chorus_attention_blocks(const uint16_t* Q, const uint16_t* K, const uint16_t* Vt, uint16_t* O, const int32_t* blocks, int32_t keep,
                                int64_t Lq, int64_t Lk, int64_t LqPad, int64_t LkPad, int32_t H, int32_t Hk, int32_t dh, int32_t prescaled,
                                void* ws, size_t ws_bytes, void* stream) {
  if (Lq < 0 || Lk < 0 || LqPad < Lq || LkPad < Lk || H <= 0 || Hk <= 0 || keep < 1) return CHORUS_E_ARG;
  if ((dh != 64 && dh != 128) || H % Hk || Lk < 1 || LkPad % BK || LkPad > kMostKeys) return CHORUS_E_SHAPE;
  if (Lq > 0x7fffffffL) return CHORUS_E_SHAPE;
  const int64_t nq = (Lq + BQ - 1) / BQ, nk = (Lk + BK - 1) / BK;
  if (nq > kMostLists / H || keep > 0x7fffffff - kMostSlices) return CHORUS_E_SHAPE;
  if (Lq == 0) return CHORUS_OK;
  if (!Q || !K || !Vt || !O || !blocks) return CHORUS_E_ARG;
  if (!aligned16(Q) || !aligned16(K) || !aligned16(Vt) || !aligned16(O) || !aligned16(blocks) || !aligned16(ws)) return CHORUS_E_ARG;
  const BlockPlan p = block_plan((long)(nq * H), dh, keep);
  const size_t need = plan_bytes(p, dh);
  if (need && (!ws || ws_bytes < need)) return CHORUS_E_WORKSPACE;
  const float scale_log2 = prescaled ? 1.0f : CHORUS_ATTENTION_Q_PRESCALE(dh);
  const dim3 grid((unsigned)(p.whole + (long)p.cut * p.slices));
#define ATTEND(DH, PRE)                                                                                                                 \
  do {                                                                                                                                  \
    static DynLdsOnce once;                                                                                                             \
    constexpr int lds = 4 * BK * DH * 2;                                                                                                \
    CHK_STATUS(once.ensure((const void*)attention_blocks_kernel<DH, PRE>, lds));                                                        \
    hipLaunchKernelGGL((attention_blocks_kernel<DH, PRE>), grid, dim3(256), lds, (hipStream_t)stream, Q, K, Vt, O, blocks, (float*)ws,   \
                       (long)Lq, (long)Lk, (long)LqPad, (long)LkPad, H, H / Hk, (int)nq, (int)nk, keep, (int)p.whole, p.slices, \
                       scale_log2);                                                                                                     \
  } while (0)
  if (dh == 128) {
    if (prescaled) ATTEND(128, true);
    else ATTEND(128, false);
  } else {
    if (prescaled) ATTEND(64, true);
    else ATTEND(64, false);
  }
#undef ATTEND
  CHORUS_LAUNCH_CHECK();
  if (need) {
    // Four waves a row as long as all of them are on the GPU at once (32 a unit): 12 lists in 12 slices 15.0 us the call, 17.6 with
    // one; 40 lists 23.0, 21.5.
    const int waves = p.cut * BQ * 4 <= 256 * 32 && p.slices >= 4 ? 4 : 1;
    const dim3 join((unsigned)(p.cut * (BQ / 4 * waves)));
#define JOIN(DH, W)                                                                                                                      \
  hipLaunchKernelGGL((attention_blocks_join_kernel<DH, W>), join, dim3(256), 0, (hipStream_t)stream, (const float*)ws, O, (long)Lq, H, (int)nq, \
                     (int)p.whole, p.slices, p.cut, scale_log2)
    if (dh == 128) {
      if (waves == 4) JOIN(128, 4);
      else JOIN(128, 1);
    } else {
      if (waves == 4) JOIN(64, 4);
      else JOIN(64, 1);
    }
#undef JOIN
    CHORUS_LAUNCH_CHECK();
  }
  return CHORUS_OK;
}

}  // extern "C"
