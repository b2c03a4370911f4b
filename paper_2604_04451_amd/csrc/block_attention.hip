// Attention over listed blocks of keys: O = softmax(Q K^T / sqrt(dh)) V, a query seeing the keys of the blocks in the list of its block of
// 128 queries and head, and no others. bf16 operands on the matrix pipe, fp32 online softmax, logits never leave registers.
//
// A workgroup of four waves owns the 128 queries of one list (32 a wave, as two blocks of 16, held in registers) and walks over
// the list a block of 64 keys at a time. The operand layouts are those of the dense kernel on v_mfma_f32_16x16x32_bf16: S^T = K Q^T
// leaves a lane with the logits of one query row, and in the order in which V^T is stored (chorus_v_transpose) its probabilities are the B
// operand of O^T += V^T P^T as they stand:
//   lane l: query row l % 16 of each block, g = l / 16; S^T block kb of a tile (16 keys x 16 queries): the K fragment's row r is key
//   32 (kb / 2) + 16 (r / 8) + 8 (kb % 2) + r % 8, so the lane holds keys 32 (kb / 2) + 16 (g / 2) + 8 (kb % 2) + 4 (g % 2) + i.
#include "chorus_ops.h"
#include "common.h"

namespace chorus {
namespace {

constexpr int BQ = CHORUS_BLOCK_QUERIES, BK = CHORUS_BLOCK_KEYS;
// Where a running maximum starts: finite, so that a block of keys whose logits are all -inf leaves a row as it was (-inf less -inf would
// be a NaN), and below every finite logit.
constexpr float kLowest = -3.402823466e38f;

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

template <int DH>
__global__ __launch_bounds__(256, 2) void attention_blocks_kernel(const uint16_t* __restrict__ Q, const uint16_t* __restrict__ K,
                                                                  const uint16_t* __restrict__ Vt, uint16_t* __restrict__ O,
                                                                  const int* __restrict__ blocks, long Lq, long Lk, long LqPad,
                                                                  long LkPad, int H, int group, int nq, int nk, int keep,
                                                                  float scale_log2) {
  constexpr int NT = 256;
  constexpr int KS = DH + 16, VS = BK + 16;  // padded LDS row strides (elements)
  constexpr int KB = BK / 16, NC = BK / 32, KC = DH / 32, DB = DH / 16, RB = 2;
  constexpr int K_LD = BK * (DH / 8) / NT, V_LD = DH * (BK / 8) / NT;
  __shared__ __attribute__((aligned(16))) uint16_t smk[BK * KS];
  __shared__ __attribute__((aligned(16))) uint16_t smv[DH * VS];

  const int tile = xcd_remap(blockIdx.x, H * nq);
  const int head = tile / nq, qb = tile - head * nq;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int lq = lane & 15, g = lane >> 4;
  const uint16_t* Kh = K + (long)(head / group) * LkPad * DH;
  const uint16_t* Vh = Vt + (long)(head / group) * DH * LkPad;

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
  float m_run[RB], l_run[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    m_run[rb] = kLowest;
    l_run[rb] = 0.f;
#pragma unroll
    for (int db = 0; db < DB; ++db) o[db][rb] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  u32x4 rk[K_LD], rv[V_LD];
  auto load = [&](int b) {
#pragma unroll
    for (int i = 0; i < K_LD; ++i) rk[i] = *reinterpret_cast<const u32x4*>(Kh + (long)b * BK * DH + (tid + NT * i) * 8);
#pragma unroll
    for (int i = 0; i < V_LD; ++i) {
      const int id = tid + NT * i;
      rv[i] = *reinterpret_cast<const u32x4*>(Vh + (long)(id / (BK / 8)) * LkPad + (long)b * BK + id % (BK / 8) * 8);
    }
  };
  const int krow0 = 16 * (lq >> 3) + (lq & 7);
  List list(blocks + (long)tile * keep, keep, nk, lane);
  int b = list.next();
  if (b >= 0) load(b);
  while (b >= 0) {
#pragma unroll
    for (int i = 0; i < K_LD; ++i) {
      const int id = tid + NT * i;
      *reinterpret_cast<u32x4*>(&smk[id / (DH / 8) * KS + id % (DH / 8) * 8]) = rk[i];
    }
#pragma unroll
    for (int i = 0; i < V_LD; ++i) {
      const int id = tid + NT * i;
      *reinterpret_cast<u32x4*>(&smv[id / (BK / 8) * VS + id % (BK / 8) * 8]) = rv[i];
    }
    const int next = list.next();
    if (next >= 0) load(next);
    __syncthreads();
    f32x4 s[KB][RB];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      bf16x8 kf[KC];
#pragma unroll
      for (int kc = 0; kc < KC; ++kc)
        kf[kc] = *reinterpret_cast<const bf16x8*>(&smk[(32 * (kb >> 1) + 8 * (kb & 1) + krow0) * KS + 32 * kc + 8 * g]);
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kc = 0; kc < KC; ++kc) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[kc], qf[rb][kc], acc, 0, 0, 0);
        s[kb][rb] = acc;
      }
    }
    const int rest = (int)(Lk - (long)b * BK < BK ? Lk - (long)b * BK : BK);  // keys of this block
    bf16x8 pf[NC][RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      float mx = -INFINITY;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (32 * (kb >> 1) + 16 * (g >> 1) + 8 * (kb & 1) + 4 * (g & 1) + i >= rest) s[kb][rb][i] = -INFINITY;
          mx = fmaxf(mx, s[kb][rb][i]);
        }
      mx = fmaxf(mx, swap_rows16(mx));
      mx = fmaxf(mx, swap_halves(mx)) * scale_log2;
      const float m_new = fmaxf(m_run[rb], mx);
      const float alpha = __builtin_amdgcn_exp2f(m_run[rb] - m_new);
      m_run[rb] = m_new;
      l_run[rb] *= alpha;
#pragma unroll
      for (int db = 0; db < DB; ++db) o[db][rb] *= alpha;
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[2 * c + (e >> 2)][rb][e & 3], scale_log2, -m_new));
          l_run[rb] += p;
          pf[c][rb][e] = (bf16_t)p;
        }
    }
#pragma unroll
    for (int db = 0; db < DB; ++db) {
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const bf16x8 vf = *reinterpret_cast<const bf16x8*>(&smv[(16 * db + lq) * VS + 32 * c + 8 * g]);
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) o[db][rb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[c][rb], o[db][rb], 0, 0, 0);
      }
    }
    __syncthreads();
    b = next;
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
  if ((dh != 64 && dh != 128) || H % Hk || Lk < 1 || LkPad % BK || LkPad > 0x7fffffffL) return CHORUS_E_SHAPE;
  if (Lq > 0x7fffffffL) return CHORUS_E_SHAPE;
  const int64_t nq = (Lq + BQ - 1) / BQ, nk = (Lk + BK - 1) / BK;
  if (nq > 0x7fffffffL / H) return CHORUS_E_SHAPE;
  if (Lq == 0) return CHORUS_OK;
  if (!Q || !K || !Vt || !O || !blocks) return CHORUS_E_ARG;
  if (!aligned16(Q) || !aligned16(K) || !aligned16(Vt) || !aligned16(O) || !aligned16(blocks) || !aligned16(ws)) return CHORUS_E_ARG;
  (void)ws_bytes;
  const float scale_log2 = prescaled ? 1.0f : CHORUS_ATTENTION_Q_PRESCALE(dh);
  const dim3 grid((unsigned)(nq * H));
#define ATTEND(DH)                                                                                                                      \
  hipLaunchKernelGGL(attention_blocks_kernel<DH>, grid, dim3(256), 0, (hipStream_t)stream, Q, K, Vt, O, blocks, (long)Lq, (long)Lk,    \
                     (long)LqPad, (long)LkPad, H, H / Hk, (int)nq, (int)nk, keep, scale_log2)
  if (dh == 128) ATTEND(128);
  else ATTEND(64);
#undef ATTEND
  CHORUS_LAUNCH_CHECK();
  return CHORUS_OK;
}

}  // extern "C"
