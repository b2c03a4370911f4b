// Attention over listed blocks of keys: O = softmax(Q K^T / sqrt(dh)) V, a query seeing the keys of the blocks in the list of its block of
// 128 queries and head, and no others. bf16 operands on the matrix pipe, fp32 online softmax, logits never leave registers.
//
// A workgroup of four waves owns the 128 queries of one list (32 a wave, as two blocks of 16, held in registers) and walks over
// the list a block of 64 keys at a time. The operand layouts are those of the dense kernel on v_mfma_f32_16x16x32_bf16: S^T = K Q^T
// leaves a lane with the logits of one query row, and in the order in which V^T is stored (chorus_v_transpose) its probabilities are the B
// operand of O^T += V^T P^T as they stand:
//   lane l: query row l % 16 of each block, g = l / 16; S^T block kb of a tile (16 keys x 16 queries): the K fragment's row r is key
//   32 (kb / 2) + 16 (r / 8) + 8 (kb % 2) + r % 8, so the lane holds keys 32 (kb / 2) + 16 (g / 2) + 8 (kb % 2) + 4 (g % 2) + i.
#include <type_traits>

#include "chorus_ops.h"
#include "common.h"

namespace chorus {
namespace {

constexpr int BQ = CHORUS_BLOCK_QUERIES, BK = CHORUS_BLOCK_KEYS;
constexpr int64_t kMostKeys = 1 << 22;  // a head's keys and values in bytes stay within the 32-bit offsets of the loads

// The blocks of a list in turn, 64 entries in the wave's lanes at a time; entries outside [0, nk) are passed over.
struct List {
  const int* at;
  int left, nk, lane, v;
  uint64_t mask;
  __device__ List(const int* list, int keep, int nk_, int lane_) : at(list), left(keep), nk(nk_), lane(lane_), v(-1), mask(0) {}
  __device__ int next() {  // -1 behind the last
    while (mask == 0) {
      if (left <= 0) return -1;
      v = lane < left ? at[lane] : -1;
      mask = __ballot((unsigned)v < (unsigned)nk);
      at += 64;
      left -= 64;
    }
    const int i = __builtin_ctzll(mask);
    mask &= mask - 1;
    return __builtin_amdgcn_readlane(v, i);
  }
};

template <int DH, bool PRE>
__global__ __launch_bounds__(256, 2) void attention_blocks_kernel(const uint16_t* __restrict__ Q, const uint16_t* __restrict__ K,
                                                                  const uint16_t* __restrict__ Vt, uint16_t* __restrict__ O,
                                                                  const int* __restrict__ blocks, long Lq, long Lk, long LqPad,
                                                                  long LkPad, int H, int group, int nq, int nk, int keep,
                                                                  float scale_log2) {
#if defined(__HIP_DEVICE_COMPILE__)  // the buffer descriptors below are types of the device compiler's alone
  constexpr int KB = BK / 16, NC = BK / 32, KC = DH / 32, DB = DH / 16, RB = 2;
  constexpr int K_LD = DH / 32, V_LD = DH / 32;  // 1 KB loads of a wave for a tile
  constexpr int TILE = BK * DH;                  // elements of a tile of keys or values
  extern __shared__ __attribute__((aligned(16))) uint16_t smem[];  // [2][TILE] keys, [2][TILE] values
  typedef __attribute__((address_space(3))) void* Lds;

  const int tile = xcd_remap(blockIdx.x, H * nq);
  const int head = tile / nq, qb = tile - head * nq;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lq = lane & 15, g = lane >> 4;

  // ---- a tile's way into LDS: each wave instruction fills 1 KB in order, and a lane fetches the 16 bytes that belong at its place. Rows of
  // keys (DH values) and of values (64) hold their 16-byte pieces at position piece ^ swizzle(row), such that the 16 rows of a
  // fragment read meet all banks.
  const auto k_swizzle = [](int row) { return DH == 128 ? (row & 7) | (row >> 4 & 1) << 3 : (row >> 1 & 3) | (row >> 4 & 1) << 2; };
  const auto v_swizzle = [](int row) { return row >> 1 & 7; };
  uint32_t k_from[K_LD], v_from[V_LD];
#pragma unroll
  for (int i = 0; i < K_LD; ++i) {
    constexpr int PIECES = DH / 8;
    const int row = (4 * i + wave) * (64 / PIECES) + lane / PIECES;
    k_from[i] = (uint32_t)(row * DH * 2 + (lane % PIECES ^ k_swizzle(row)) * 16);
  }
#pragma unroll
  for (int i = 0; i < V_LD; ++i) {
    const int row = (4 * i + wave) * 8 + lane / 8;
    v_from[i] = (uint32_t)(row * (int)LkPad * 2 + (lane % 8 ^ v_swizzle(row)) * 16);
  }
  const auto k_rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)(K + (long)(head / group) * LkPad * DH), 0, (int)(LkPad * DH * 2), 0x00027000);
  const auto v_rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)(Vt + (long)(head / group) * LkPad * DH), 0, (int)(LkPad * DH * 2), 0x00027000);
  auto load_k = [&](int b, int buf) {
#pragma unroll
    for (int i = 0; i < K_LD; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(k_rsrc, (Lds)(smem + buf * TILE + (4 * i + wave) * 512), 16, k_from[i], b * (TILE * 2), 0, 0);
  };
  auto load_v = [&](int b, int buf) {
#pragma unroll
    for (int i = 0; i < V_LD; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(v_rsrc, (Lds)(smem + (2 + buf) * TILE + (4 * i + wave) * 512), 16, v_from[i], b * (BK * 2), 0, 0);
  };
  // ---- and out of it
  int k_at[KC], v_at[NC];
#pragma unroll
  for (int kc = 0; kc < KC; ++kc) {
    const int row = 16 * (lq >> 3) + (lq & 7);
    k_at[kc] = row * DH + ((4 * kc + g) ^ k_swizzle(row)) * 8;
  }
#pragma unroll
  for (int c = 0; c < NC; ++c) v_at[c] = lq * BK + ((4 * c + g) ^ v_swizzle(lq)) * 8;

  bf16x8 qf[RB][KC];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    long q = (long)qb * BQ + wave * 32 + 16 * rb + lq;
    if (q > Lq - 1) q = Lq - 1;
    const uint16_t* qp = Q + ((long)head * LqPad + q) * DH + 8 * g;
#pragma unroll
    for (int kc = 0; kc < KC; ++kc) qf[rb][kc] = *reinterpret_cast<const bf16x8*>(qp + 32 * kc);
  }
  f32x4 o[DB][RB];
  // A row's reference, in units of its logits, and this lane's part of the sum of its weights. S^T accumulators start at minus the
  // reference, so a logit leaves the matrix pipe as the exponent of its weight (but for scale_log2 where the queries do not hold it).
  float m_run[RB], l_run[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    m_run[rb] = 0.f;
    l_run[rb] = 0.f;
#pragma unroll
    for (int db = 0; db < DB; ++db) o[db][rb] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  bool fresh = true;  // some row of the wave has seen no finite logit
  f32x4 s[2][KB][RB];
  auto compute_s = [&](f32x4(&s)[KB][RB], int buf) {
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      bf16x8 kf[KC];
#pragma unroll
      for (int kc = 0; kc < KC; ++kc)
        kf[kc] = *reinterpret_cast<const bf16x8*>(&smem[buf * TILE + (32 * (kb >> 1) + 8 * (kb & 1)) * DH + k_at[kc]]);
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        f32x4 acc = {-m_run[rb], -m_run[rb], -m_run[rb], -m_run[rb]};
#pragma unroll
        for (int kc = 0; kc < KC; ++kc) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[kc], qf[rb][kc], acc, 0, 0, 0);
        s[kb][rb] = acc;
      }
    }
  };
  auto mask = [&](f32x4(&s)[KB][RB], int b) {  // keys behind the last
    int rest = (int)(Lk - (long)b * BK) - (16 * (g >> 1) + 4 * (g & 1));
    asm volatile("" : "+v"(rest));  // compared here: hoisted, the 32 results would fill the scalar registers
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (32 * (kb >> 1) + 8 * (kb & 1) + i >= rest) {
#pragma unroll
          for (int rb = 0; rb < RB; ++rb) s[kb][rb][i] = -INFINITY;
        }
  };
  auto maximum = [&](float(&mx)[RB], const f32x4(&s)[KB][RB]) {
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      float m = s[0][rb][0];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < 4; ++i) m = fmaxf(m, s[kb][rb][i]);
      m = fmaxf(m, swap_rows16(m));
      mx[rb] = fmaxf(m, swap_halves(m));
    }
  };
  // The reference moves when a row exceeds it by more than 2^8, and to the first finite logit of a row whatever that is.
  const float most = PRE ? 8.0f : 8.0f / scale_log2;
  auto move = [&](f32x4(&s)[KB][RB], const float(&mx)[RB]) {
    bool far = fresh;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) far = far || mx[rb] > most;
    if (!__any(far)) return;
    bool none = false;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      float l = l_run[rb] + swap_rows16(l_run[rb]);
      l += swap_halves(l);
      const bool first = l == 0.f;
      const float delta = first ? (mx[rb] > -INFINITY ? mx[rb] : 0.f) : fmaxf(mx[rb], 0.f);
      const float alpha = first ? 1.0f : __builtin_amdgcn_exp2f(-delta * (PRE ? 1.0f : scale_log2));
      none = none || (first && !(mx[rb] > -INFINITY));
      m_run[rb] += delta;
      l_run[rb] *= alpha;
#pragma unroll
      for (int db = 0; db < DB; ++db) o[db][rb] *= alpha;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) s[kb][rb] -= delta;
    }
    fresh = __any(none);
  };

  List list(blocks + (long)tile * keep, keep, nk, lane);
  const int tail = Lk % BK ? nk - 1 : -2;  // the block that is not full
  int b1 = list.next(), b2 = -1;           // the next tile and the one behind it
  // One tile: its weights while the matrix pipe makes the next one's logits, then its share of the result. b1, b2: the tiles behind it.
  auto step = [&](auto parity) {
    constexpr int buf = decltype(parity)::value;
    b1 = b2;
    if (b1 >= 0) {
      b2 = list.next();
      if (b2 >= 0) load_k(b2, buf);
      load_v(b1, buf ^ 1);
    }
    __builtin_amdgcn_sched_barrier(0);
    bf16x8 pf[NC][RB];
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float x = s[buf][2 * c + (e >> 2)][rb][e & 3];
          const float p = __builtin_amdgcn_exp2f(PRE ? x : x * scale_log2);
          l_run[rb] += p;
          pf[c][rb][e] = (bf16_t)p;
        }
    compute_s(s[buf ^ 1], buf ^ 1);
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) asm volatile("" : "+v"(pf[c][rb]));  // here and not where they are used
    __builtin_amdgcn_sched_group_barrier(0x100, 6, 0);
#pragma unroll
    for (int i = 0; i < KB * KC * RB; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x002, PRE ? 3 : 4, 0);
      if (i % 2 && i / 2 < KB * KC - 6) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (b1 >= 0 && b1 == tail) mask(s[buf ^ 1], b1);
    float mx[RB];
    maximum(mx, s[buf ^ 1]);
#pragma unroll
    for (int db = 0; db < DB; ++db) {
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const bf16x8 vf = *reinterpret_cast<const bf16x8*>(&smem[(2 + buf) * TILE + 16 * db * BK + v_at[c]]);
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) o[db][rb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[c][rb], o[db][rb], 0, 0, 0);
      }
    }
    __builtin_amdgcn_sched_group_barrier(0x100, 6, 1);
#pragma unroll
    for (int i = 0; i < DB * NC * RB; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 1);
      __builtin_amdgcn_sched_group_barrier(0x002, 2, 1);
      if (i % 2 && i / 2 < DB * NC - 6) __builtin_amdgcn_sched_group_barrier(0x100, 1, 1);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (b1 >= 0) move(s[buf ^ 1], mx);
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
  };
  if (b1 >= 0) {
    b2 = list.next();
    load_k(b1, 0);
    load_v(b1, 0);
    if (b2 >= 0) load_k(b2, 1);
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int kc = 0; kc < KC; ++kc) asm volatile("" : "+v"(qf[rb][kc]));  // resident before the loop, which would wait for them otherwise
    asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
    compute_s(s[0], 0);
    if (b1 == tail) mask(s[0], b1);
    float mx[RB];
    maximum(mx, s[0]);
    move(s[0], mx);
    asm volatile("s_barrier" ::: "memory");
      while (true) {
      step(std::integral_constant<int, 0>{});
      if (b1 < 0) break;
      step(std::integral_constant<int, 1>{});
      if (b1 < 0) break;
    }
  }

  const int D = H * DH;
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    float l = l_run[rb] + swap_rows16(l_run[rb]);
    l += swap_halves(l);
    const float inv = l == 0.f ? 0.f : 1.0f / l;  // no key at all: a row of zeros
    const long q = (long)qb * BQ + wave * 32 + 16 * rb + lq;
    if (q < Lq) {
      uint16_t* op = O + q * (long)D + (long)head * DH + 4 * g;
#pragma unroll
      for (int db = 0; db < DB; ++db)
        *reinterpret_cast<uint2*>(op + 16 * db) = make_uint2(pack_bf16x2(o[db][rb][0] * inv, o[db][rb][1] * inv),
                                                             pack_bf16x2(o[db][rb][2] * inv, o[db][rb][3] * inv));
    }
  }
#endif
}

}  // namespace
}  // namespace chorus

using namespace chorus;

extern "C" {

size_t chorus_attention_blocks_workspace_bytes(int64_t Lq, int32_t H, int32_t dh, int32_t keep) {
  (void)Lq, (void)H, (void)dh, (void)keep;
  return 0;
}

int32_t chorus_attention_blocks(const uint16_t* Q, const uint16_t* K, const uint16_t* Vt, uint16_t* O, const int32_t* blocks, int32_t keep,
                                int64_t Lq, int64_t Lk, int64_t LqPad, int64_t LkPad, int32_t H, int32_t Hk, int32_t dh, int32_t prescaled,
                                void* ws, size_t ws_bytes, void* stream) {
  if (Lq < 0 || Lk < 0 || LqPad < Lq || LkPad < Lk || H <= 0 || Hk <= 0 || keep < 1) return CHORUS_E_ARG;
  if ((dh != 64 && dh != 128) || H % Hk || Lk < 1 || LkPad % BK || LkPad > kMostKeys) return CHORUS_E_SHAPE;
  if (Lq > 0x7fffffffL) return CHORUS_E_SHAPE;
  const int64_t nq = (Lq + BQ - 1) / BQ, nk = (Lk + BK - 1) / BK;
  if (nq > 0x7fffffffL / H) return CHORUS_E_SHAPE;
  if (Lq == 0) return CHORUS_OK;
  if (!Q || !K || !Vt || !O || !blocks) return CHORUS_E_ARG;
  if (!aligned16(Q) || !aligned16(K) || !aligned16(Vt) || !aligned16(O) || !aligned16(blocks) || !aligned16(ws)) return CHORUS_E_ARG;
  (void)ws_bytes;
  const float scale_log2 = prescaled ? 1.0f : CHORUS_ATTENTION_Q_PRESCALE(dh);
  const dim3 grid((unsigned)(nq * H));
#define ATTEND(DH, PRE)                                                                                                                  \
  do {                                                                                                                                  \
    static DynLdsOnce once;                                                                                                             \
    constexpr int lds = 4 * BK * DH * 2;                                                                                                \
    CHK_STATUS(once.ensure((const void*)attention_blocks_kernel<DH, PRE>, lds));                                                        \
    hipLaunchKernelGGL((attention_blocks_kernel<DH, PRE>), grid, dim3(256), lds, (hipStream_t)stream, Q, K, Vt, O, blocks, (long)Lq,     \
                       (long)Lk, (long)LqPad, (long)LkPad, H, H / Hk, (int)nq, (int)nk, keep, scale_log2);                              \
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
  return CHORUS_OK;
}

}  // extern "C"
