// The main loop of the tiled products C = A W^T, A [M, K] and W [N, K] both K-contiguous: tiles straight from global memory into LDS,
// accumulators of 16 x 16 blocks in registers. Shared by the products of bf16 (gemm.hip, gated.hip) and of 8-bit integers (gemm_i8.hip).
#pragma once
#include "chorus_ops.h"
#include "common.h"

namespace chorus {

// s_waitcnt operand that waits for at most n vector memory operations in flight and for nothing else
constexpr int vmcnt_imm(int n) { return (n & 15) | ((n >> 4) << 14) | 0x0F70; }

constexpr int BK = 64;  // values of bf16 in a k-step; of other types as many as 128 bytes hold

// The same address in scalar registers: the compiler does not see that a value worked out from the workgroup's id by a
// division is one for the whole wave, and would walk over the lanes with every descriptor made from it.
__device__ __forceinline__ void* uniform_address(const uint16_t* p) {
  const uint64_t u = reinterpret_cast<uint64_t>(p);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(u >> 32)), lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)u);
  return reinterpret_cast<void*>(((uint64_t)hi << 32) | lo);
}

// Row and column tile of a logical tile number: groups of 8 row tiles. Within a group the tiles that run together on one XCD share
// operands in its L2. Normally they are taken row tile fastest (8 row tiles x 4 column tiles at a time). When the activation rows are
// long and the weight matrix is only a few tiles wide, column tile fastest is better: all column tiles of a row tile run together, so
// every activation panel, the operand too big for any cache, leaves HBM once. K in units of 2 bytes.
struct TilePlace {
  int m, n;
};
__device__ __forceinline__ TilePlace tile_place(int tile, int tiles_m, int tiles_n, int K) {
  constexpr int GM = 8;
  const int per_group = GM * tiles_n;
  const int group = tile / per_group;
  const int first_m = group * GM;
  const int gsz = (tiles_m - first_m) < GM ? (tiles_m - first_m) : GM;
  const int in_group = tile - group * per_group;
  const bool n_fastest = tiles_n <= 8 && K >= 4096;
  return TilePlace{n_fastest ? first_m + in_group / tiles_n : first_m + in_group % gsz, n_fastest ? in_group % tiles_n : in_group / gsz};
}

// A 16 x 16 block of results plus the product of 16 rows of W and 16 of A over the 64 bytes of a half-step's row. Volatile and in place.
struct MmaBf16 {
  typedef f32x4 Acc;
  static __device__ __forceinline__ void add(f32x4& c, const bf16x8& w, const bf16x8& a) {
    asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(w), "v"(a));
  }
  static __device__ __forceinline__ f32x4 mma(const f32x4& c, const bf16x8& w, const bf16x8& a) {  // where the compiler may place it
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, a, c, 0, 0, 0);
  }
};
// 64 products of 8-bit integers instead of 32 of bf16, in the same registers and lanes; sums in 32 bits
typedef __attribute__((__vector_size__(4 * sizeof(int32_t)))) int32_t i32x4;
struct MmaI8 {
  typedef i32x4 Acc;
  static __device__ __forceinline__ void add(i32x4& c, const bf16x8& w, const bf16x8& a) {
    asm volatile("v_mfma_i32_16x16x64_i8 %0, %1, %2, %0" : "+a"(c) : "v"(w), "v"(a));
  }
  static __device__ __forceinline__ i32x4 mma(const i32x4& c, const bf16x8& w, const bf16x8& a) {
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, w), __builtin_bit_cast(i32x4, a), c, 0, 0, 0);
  }
};

// Where the tile's rows of W come from: N consecutive ones, or 16 of one matrix and 16 of a second one in turn, so that a wave's even
// blocks of columns are products with the first and the odd ones with the second, for the same places of both.
struct OneMatrix {
  static constexpr bool kPair = false;
};
struct SecondMatrix {
  const uint16_t* first;  // its first row of the tile
  static constexpr bool kPair = true;
};

// ---------------------------------------------------------------------------
// Large-problem kernel: 256 x 256 x 64 tiles, four waves (one per SIMD), each wave a 128 x 128 quadrant as 8 x 8
// accumulators of v_mfma_f32_16x16x32_bf16 (256 accumulator registers). Per unit of work a 16x16x32 MFMA reads and
// writes half the accumulator registers of a 32x32x16 one (k = 32 per instruction instead of 16), which is what the
// power-managed part rewards; a 16-byte LDS fragment (16 rows x 8 k per quarter wave) feeds eight MFMAs.
//
// Both operands stream global -> LDS directly (buffer_load_dwordx4 ... lds: no register staging, no LDS store
// instructions, one lane offset per load for all steps) into a ring of five half steps of 32 KB, the whole 160 KB: rows 0-127
// of A and of W are one half of a k-step, rows 128-255 the other. A direct load writes the 64 lanes' 16-byte pieces to
// consecutive LDS addresses, i.e. 8 unpadded rows of 128 bytes. Bank conflicts are avoided by an XOR swizzle instead of padding: the
// 16-byte chunk c of row r lives at chunk position c ^ ((r >> 1) & 7); the loading lane for position p of row r
// fetches global chunk p ^ ((r >> 1) & 7). (A 16-byte-per-lane LDS read is served 16 lanes a cycle: the four-lane
// groups of one half wave whose group index has the same bit parity, groups 0, 3, 5, 6 together and 1, 2, 4, 7. With
// lane = 16 * chunk + row those are rows 0-3 and 12-15 of one chunk with rows 4-11 of its neighbour, which this
// swizzle spreads over all 64 banks: measured, no conflict cycles.)
//
// Operand layout of v_mfma_f32_16x16x32_bf16: lane l supplies row (or column) l % 16 and the 8 k-values
// 8 (l / 16) .. + 8; it receives column l % 16 and rows 4 (l / 16) .. + 4 of the 16 x 16 result. The weight fragment is
// the row operand and the activation fragment the column operand, so a lane holds one output row m and four
// consecutive output columns n.
//
// One loop iteration per k-step, hand-laid for a single wave per SIMD (nothing else hides a gap between two MFMAs):
// half-step 0 (64 MFMAs) with the LDS reads of half-step 1's fragments; wait + barrier; half-step 1 (64 MFMAs) with the LDS
// reads of the next step's first fragments. Either half issues the 8 loads of a half step, one every eight MFMAs: those of
// half-step 0 land 1 to 1.5 steps later, those of half-step 1 half a step to a step. Every read and load stands alone
// between two MFMAs. What bounds the loop is the delivery of the operands: with all 16 loads of a step in its second half and
// two whole stages in LDS it ran at 1310 TFLOP/s (8192 x 8192 x 8192), so at 1510; with the loads aimed at two steps
// that stay in the L2 at 1530, without any loads at 1780. Measured and not taken: 16 loads in the first half of half-step
// 1 (1.04 of the time), one load per wave and step that fetches lines into the L2 four steps ahead (1.04), workgroups that
// stay and take the next tile's first steps behind the last ones of this tile's (0.99 to 1.02), later starts for some of the XCDs
// so that not all epilogues write at once (they cost what they save).
// The MFMAs are volatile assembly, in place on their accumulators: left to the register allocator every result gets
// a new home, at the price of several hundred accumulator moves per k-step.
// ---------------------------------------------------------------------------
// WBM, WBN = 16 x 16 blocks along the rows (M) and columns (N) of a wave's quadrant: 8, 8 (256 x 256 tiles), 4, 4 (128 x
// 128), 2, 2 (64 x 64) or 4, 8 (128 x 256).
// C = half steps in LDS: the loads of a half step are issued C - 4 to C - 2 half-steps before the barrier that they must have
// landed at. Five leave room for two 128 x 128 workgroups on a compute unit, which then hide each other's waits; a launch with
// fewer tiles than units has no second workgroup there, and seven (112 KB) take its place: 1200 x 1536 x 8960 100 -> 67 us. More
// measured the same: from there on the unit's L1, not the distance, sets the rate.
// Sizes and places are in units of 2 bytes, whatever the type: A, W at the first value of the tile's first row that this workgroup
// multiplies, rows of K units of which k_first stand in front of A; rows_a, rows_b: rows of the tile inside the matrices (with a second
// matrix: of each); KTN k-steps. Leaves the wave's sums in acc and LDS free for the epilogue.
template <class MMA, class WROWS, int WBM, int WBN, int C, bool FAR>
__device__ __forceinline__ void gemm16_loop(typename MMA::Acc (&acc)[8][8], uint16_t* smem, const uint16_t* A, const uint16_t* W,
                                            WROWS second, int rows_a, int rows_b, int K, int k_first, int KTN, int wave, int lane) {
#if defined(__HIP_DEVICE_COMPILE__)  // the buffer descriptors below are types of the device compiler's alone
  static_assert(!(FAR && WROWS::kPair), "rows out of reach of the offsets come from one matrix");
  constexpr int WTM = 16 * WBM, WTN = 16 * WBN;  // rows and columns of a wave's quadrant
  constexpr int HA = WTM * BK, HB = WTN * BK;    // elements of half a step's rows of A and of W
  const int wm = wave >> 1, wn = wave & 1;
  const int lj = lane & 15, lg = lane >> 4;

  // ---- loader: load i of half h covers 8 of the tile's rows from WTM h + 4 WBM wave + 8 i on (of W: WTN h + 4 WBN wave + 8
  // i); lane -> (row, position). One lane offset per load serves every step: the step's place in the rows is a scalar, and
  // rows past the matrix's end are past the descriptor's too (such loads fetch nothing; their results are never stored).
  const int lr = lane >> 3, lp = lane & 7;
  constexpr int LA = WBM / 2, LB = WBN / 2;  // loads of a half step
  // (the arrays that the lambdas below capture have the large tile's size for either tile: a bound that depends on
  // the template parameter loses the kernel's host-side stub)
  int oa[8], ob[8];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
#pragma unroll
    for (int i = 0; i < LA; ++i) {
      const int r = WTM * h + 4 * WBM * wave + 8 * i + lr;
      const int at = (lp ^ ((r >> 1) & 7)) * 16;  // the global chunk that belongs at position lp
      oa[LA * h + i] = FAR ? (r < rows_a ? r : rows_a - 1) : r * (2 * K) + at;
    }
#pragma unroll
    for (int i = 0; i < LB; ++i) {
      const int r = WTN * h + 4 * WBN * wave + 8 * i + lr;
      const int at = (lp ^ ((r >> 1) & 7)) * 16, from = WROWS::kPair ? (r >> 5) * 16 + (r & 15) : r;
      ob[LB * h + i] = FAR ? (r < rows_b ? r : rows_b - 1) : from * (2 * K) + at;
    }
  }
  void* const base_a = uniform_address(A);
  void* const base_b = uniform_address(W);
  void* base_c = base_b;
  if constexpr (WROWS::kPair) base_c = uniform_address(second.first);
  const int bytes_a = __builtin_amdgcn_readfirstlane(FAR ? 0 : (rows_a * K - k_first * BK) * 2);
  const int bytes_b = __builtin_amdgcn_readfirstlane(FAR ? 0 : (rows_b * K - k_first * BK) * 2);
  // load t (A's first, then W's) of half step hs (half hs % 2 of the rows of step hs / 2), into the ring at slot
  auto issue = [&](int hs, int h, int slot, int t) {
    const bool of_w = t >= LA;
    const int i = of_w ? t - LA : t, kt = hs >> 1;
    void* const base_w = WROWS::kPair && ((4 * WBN * wave + 8 * i) & 16) ? base_c : base_b;
    __attribute__((address_space(3))) void* const dst =
        (__attribute__((address_space(3))) void*)(smem + (of_w ? C * HA + slot * HB + (4 * WBN * wave + 8 * i) * BK
                                                                : slot * HA + (4 * WBM * wave + 8 * i) * BK));
    if constexpr (FAR) {
      const int r = of_w ? ob[LB * h + i] : oa[LA * h + i];
      const int row = (of_w ? WTN * h + 4 * WBN * wave : WTM * h + 4 * WBM * wave) + 8 * i + lr;
      const uint16_t* src = reinterpret_cast<const uint16_t*>(of_w ? base_w : base_a) + (long)r * K +
                            (long)(kt < KTN ? kt : KTN - 1) * BK + (lp ^ ((row >> 1) & 7)) * 8;
      __builtin_amdgcn_global_load_lds(src, dst, 16, 0, 0);
    } else {
      // past the last step an empty descriptor: the loads keep their place in the count and fetch nothing
      const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(of_w ? base_w : base_a, 0, kt < KTN ? (of_w ? bytes_b : bytes_a) : 0, 0x00027000);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, dst, 16, of_w ? ob[LB * h + i] : oa[LA * h + i], kt * (2 * BK), 0, 0);
    }
  };

  // ---- fragment read offsets (elements): row l % 16 of a 16-row block, 16-byte chunk 4 h + l / 16, swizzled by the row
  const int sw = (lj >> 1) & 7;
  int koff[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) koff[h] = ((4 * h + lg) ^ sw) * 8 + lj * BK;

#pragma unroll
  for (int nb = 0; nb < WBN; ++nb)
#pragma unroll
    for (int mb = 0; mb < WBM; ++mb) acc[nb][mb] = typename MMA::Acc{};

  bf16x8 af[2][8], bfr[2][8];
  // fragment f of a half-step: 0 .. WBM-1 the activation blocks (m), then the WBN weight blocks (n); sa, sb: where the wave's
  // rows of the step start
  auto read_frag = [&](int sa, int sb, int h, int set, int f) {
    if (f < WBM)
      af[set][f] = *reinterpret_cast<const bf16x8*>(smem + sa + koff[h] + f * 16 * BK);
    else
      bfr[set][f - WBM] = *reinterpret_cast<const bf16x8*>(smem + sb + koff[h] + (f - WBM) * 16 * BK);
  };
  // MFMAs g0 .. g1-1 of the WBM * WBN of a half-step, weight block major: g = WBM nb + mb. In place on the accumulator
  // registers (left to itself the register allocator gives every result a new home and pays with hundreds of
  // accumulator moves per k-step); being volatile they also keep their place between the loads written around them.
  auto mfmas = [&](int set, int g0, int g1) {
#pragma unroll
    for (int g = g0; g < g1; ++g)
      MMA::add(acc[g / WBM][g % WBM], bfr[set][g / WBM], af[set][g % WBM]);
  };
  // order in which the fragments of a half-step are fetched: what its first MFMAs need comes first (the first weight
  // block, the activation blocks, the other weight blocks)
  auto frag_order = [](int i) { return i == 0 ? WBM : (i <= WBM ? i - 1 : i); };

  // Schedule of one k-step (square tiles, WB = WBM = WBN: 2 WB^2 MFMAs a wave in 4 WB slots of WB / 2, 128 MFMAs in 32
  // slots of four for the large tile). Either half-step issues the loads of one half step further on, one every other slot.
  // The barrier sits between the two half-steps. In the first half a wave fetches its fragments of the second half (same
  // step); at the barrier every wave holds all its fragments of the current step in registers, so that the step's two
  // places in the ring are free behind it, and the whole next step is in LDS: what was requested behind that step, C - 4
  // half steps, stays in flight. The second half fetches the next step's first fragments. Fragment reads are
  // packed into the first kReadSlots slots of a half so that the last of them has returned when the half ends. With one
  // wave per SIMD nothing else feeds the matrix pipe while this wave issues something that is not an MFMA, so reads and
  // loads stand one at a time between single MFMAs, where they issue in the shadow of the MFMA in front of them, and
  // the wave index is kept in a scalar register so that the LDS address of a load costs no vector instruction.
  // A rectangular tile has no whole number of MFMAs per slot: its reads stand behind MFMAs spread evenly over the first
  // three quarters of a half, its loads over all of it.
  constexpr int NS = WBM + WBN;            // slots of a half-step = fragments of a half-step
  constexpr int NH = NS / 2;               // loads of a half step
  constexpr int G = WBM * WBN;             // MFMAs of a half-step
  constexpr int MPS = WBM / 2;             // MFMAs of a slot
  constexpr int kReadSlots = 3 * WBM / 2;  // 12 of 16 (6 of 8, 3 of 4)
  // reads of slot f: one fragment, two in the first NS - kReadSlots slots (which = 0: the first, 1: the second)
  auto read_of_slot = [&](int sa, int sb, int h, int set, int f, int which) {
    constexpr int kDouble = NS - kReadSlots;
    if (f < kDouble)
      read_frag(sa, sb, h, set, frag_order(2 * f + which));
    else if (f < kReadSlots && which == 0)
      read_frag(sa, sb, h, set, frag_order(f + kDouble));
  };
  // half-step h: its MFMAs, the fragments of the half-step behind it from sa, sb, the loads of half step hs into slot
  auto half_step = [&](int h, int sa, int sb, int hs, int slot) {
    if constexpr (WBM == WBN) {
#pragma unroll
      for (int f = 0; f < NS; ++f) {
        mfmas(h, MPS * f, MPS * f + 1);
        __builtin_amdgcn_sched_barrier(0);
        read_of_slot(sa, sb, 1 - h, 1 - h, f, 0);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (MPS > 1) mfmas(h, MPS * f + 1, MPS * f + 2);
        __builtin_amdgcn_sched_barrier(0);
        read_of_slot(sa, sb, 1 - h, 1 - h, f, 1);
        __builtin_amdgcn_sched_barrier(0);
        mfmas(h, MPS * f + 2, MPS * f + MPS - 1);  // (none for the small tiles)
        __builtin_amdgcn_sched_barrier(0);
        if (f & 1) issue(hs, (C - 1 + h) & 1, slot, f >> 1);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (MPS > 2) mfmas(h, MPS * f + MPS - 1, MPS * f + MPS);
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
#pragma unroll
      for (int g = 0; g < G; ++g) {
        mfmas(h, g, g + 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < NS; ++i)
          if (i * 3 * G / (4 * NS) == g) read_frag(sa, sb, 1 - h, 1 - h, frag_order(i));
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < NH; ++i)
          if ((2 * i + 1) * G / (2 * NH) == g) issue(hs, (C - 1 + h) & 1, slot, i);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };
  auto wrap = [](int slot) { return slot >= C ? slot - C : slot; };

#pragma unroll
  for (int hs = 0; hs < C - 1; ++hs)
#pragma unroll
    for (int t = 0; t < NH; ++t) issue(hs, hs & 1, hs, t);
  // the first step's pieces are in LDS, the later ones may be in flight (the barrier alone: a fence would wait for them)
  asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(NH * (C - 3)) : "memory");
  __builtin_amdgcn_sched_barrier(0);
  int first = 0;  // slot of the first half of step kt
  int sa = wm * HA, sb = C * HA + wn * HB;
#pragma unroll
  for (int f = 0; f < NS; ++f) read_frag(sa, sb, 0, 0, frag_order(f));
  __builtin_amdgcn_sched_barrier(0);

  for (int kt = 0; kt < KTN; ++kt) {
    const int next = wrap(first + 2);
    const int san = wrap(next + wm) * HA, sbn = C * HA + wrap(next + wn) * HB;
    half_step(0, sa, sb, 2 * kt + C - 1, wrap(first + C - 1));
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(NH * (C - 4)) : "memory");
    __builtin_amdgcn_sched_barrier(0);
    half_step(1, san, sbn, 2 * kt + C, first);
    first = next;
    sa = san;
    sb = sbn;
  }

  __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));  // no direct load may land in the staging regions of the epilogue
  // The compiler does not know the assembly above for MFMAs and so keeps no distance between the last of them and the
  // first instruction that reads an accumulator: cover the longest such distance explicitly. The wait is tied to the
  // accumulators of the last four MFMAs (operands of the statement), so that no copy or spill of one of them can be
  // placed in front of it; every other accumulator was written at least four MFMAs earlier.
  asm volatile("s_nop 15\n\ts_nop 15\n\ts_nop 15"
               : "+a"(acc[WBN - 1][WBM - 1]), "+a"(acc[WBN - 1][WBM - 2]), "+a"(acc[WBM > 2 ? WBN - 1 : 0][WBM > 2 ? WBM - 3 : 1]),
                 "+a"(acc[WBM > 2 ? WBN - 1 : 0][WBM > 2 ? WBM - 4 : 0]));
  lds_barrier();  // the staging regions of the epilogue overlay the operands
#endif
}

__device__ __forceinline__ float gelu_tanh_fast(float x) {
  // 0.5 x (1 + tanh(u)) = x / (1 + exp(-2u)),  u = sqrt(2/pi) (x + 0.044715 x^3); the exponent is taken in base 2:
  // -2u log2(e) = -x (2.3022082 + 0.10294324 x^2)
  const float t = x * x;
  const float p = __builtin_fmaf(t, -0.10294324f, -2.3022082f);
  const float e = __builtin_amdgcn_exp2f(p * x);
  return x * __builtin_amdgcn_rcpf(1.0f + e);
}

struct EpiArgs {
  void* out;
  const float* bias;
  const float* gate0;
  const float* gate1;
  float scale;
};

// Results of 16 bits on their way out: 32 output rows at a time go through a private LDS region as [32][16 WBN] (row stride 16 WBN + 8), then
// leave as full row segments of the quadrant (256, 128 or 64 bytes). words(nb, mb): a lane's four values of a block. ld: values from row to
// row of the output.
template <int WBN> constexpr int e16_bf_stride() { return 16 * WBN + 8; }
template <int WBN> constexpr int e16_bf_wave() { return 32 * e16_bf_stride<WBN>(); }  // elements per wave
template <int WBM, int WBN, class WORDS>
__device__ __forceinline__ void gemm16_rows_out(const WORDS& words, uint16_t* out, uint16_t* cw, long m_wave0, int n_wave0, long M, int N, long ld,
                                                int lane) {
  constexpr int E16_BF_STRIDE = e16_bf_stride<WBN>();
  constexpr int LPR = 2 * WBN;  // read-back: LPR lanes x 16 bytes per row
  const int lj = lane & 15, lg = lane >> 4;
#pragma unroll
  for (int mp = 0; mp < WBM / 2; ++mp) {  // pairs of 16-row blocks
#pragma unroll
    for (int mh = 0; mh < 2; ++mh)
#pragma unroll
      for (int nb = 0; nb < WBN; ++nb)
        *reinterpret_cast<uint2*>(cw + (16 * mh + lj) * E16_BF_STRIDE + 16 * nb + 4 * lg) = words(nb, 2 * mp + mh);
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
#pragma unroll
    for (int it = 0; it < LPR / 2; ++it) {
      const int row = (64 * it + lane) / LPR, rcol = (64 * it + lane) % LPR * 8;
      const long m = m_wave0 + 32 * mp + row;
      const int n = n_wave0 + rcol;
      const u32x4 v = *reinterpret_cast<const u32x4*>(cw + row * E16_BF_STRIDE + rcol);
      // streaming store: an output tile is not read again by this kernel, and left to the default policy the written
      // lines push the operand panels that the next tiles share out of the L2 (measured: 14-19 % on the widest output)
      if (m < M && n < N) __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(out + m * ld + n));
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    __builtin_amdgcn_sched_barrier(0);
  }
}

// bf16 (optionally GELU) epilogue of the 16x16 layout, block(nb, mb) being a lane's part of a block of results
template <int EPI, int WBM, int WBN, class BLOCK>
__device__ __forceinline__ void gemm16_epilogue_bf16(const BLOCK& block, const EpiArgs& ep, uint16_t* cw, long m_wave0, int n_wave0, long M, int N,
                                                     int lane) {
  const int lg = lane >> 4;
  float4 bias[WBN];
#pragma unroll
  for (int nb = 0; nb < WBN; ++nb) {
    const int n = n_wave0 + 16 * nb + 4 * lg;
    bias[nb] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (ep.bias && n < N) bias[nb] = *reinterpret_cast<const float4*>(ep.bias + n);
  }
  const auto words = [&](int nb, int mb) {
    f32x4 a = block(nb, mb);
    // one block at a time out of the accumulators: of the large tile's, fetched together, 8 to 12 bytes a lane spilled
    if (WBM == 8 && (mb & 1)) asm volatile("" : "+v"(a));
    float v0 = a[0] + bias[nb].x, v1 = a[1] + bias[nb].y, v2 = a[2] + bias[nb].z, v3 = a[3] + bias[nb].w;
    if (EPI == CHORUS_EPI_GELU_BF16) {
      v0 = gelu_tanh_fast(v0); v1 = gelu_tanh_fast(v1); v2 = gelu_tanh_fast(v2); v3 = gelu_tanh_fast(v3);
    }
    return make_uint2(pack_bf16x2(v0, v1), pack_bf16x2(v2, v3));
  };
  gemm16_rows_out<WBM, WBN>(words, reinterpret_cast<uint16_t*>(ep.out), cw, m_wave0, n_wave0, M, N, N, lane);
}

// fp32 gated-residual epilogue of the 16x16 layout: 16 output rows at a time through a private LDS region as
// [16][16 WBN] fp32 (row stride 16 WBN + 4), read back with 4 WBN lanes per row; the residual rows are requested before the
// LDS round trip. out[m][n] += gate[n] * scale * (acc + bias[n]).
template <int WBN> constexpr int e16_f32_stride() { return 16 * WBN + 4; }
template <int WBN> constexpr int e16_f32_wave() { return 16 * e16_f32_stride<WBN>(); }  // floats per wave
// CHAIN: what another workgroup of the tile wrote is read and what the next one reads is written past the L2s (agent scope).
template <int WBM, int WBN, bool CHAIN = false, class BLOCK>
__device__ __forceinline__ void gemm16_epilogue_resid(const BLOCK& block, const EpiArgs& ep, float* cw, long m_wave0,
                                                      int n_wave0, long M, int N, int lane) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int E16_F32_STRIDE = e16_f32_stride<WBN>();
  constexpr int LPR = 4 * WBN, RPI = 64 / LPR;  // read-back: LPR lanes x 16 bytes per row, RPI rows per instruction
  const int lj = lane & 15, lg = lane >> 4;
  const int rrow = lane / LPR, rcol = (lane % LPR) * 4;
  const int n = n_wave0 + rcol;
  const bool n_ok = n < N;
  f32x4 bias = {0.f, 0.f, 0.f, 0.f}, gate = {1.f, 1.f, 1.f, 1.f};
  if (n_ok) {
    if (ep.bias) bias = *reinterpret_cast<const f32x4*>(ep.bias + n);
    if (ep.gate0 || ep.gate1) {
      gate = f32x4{0.f, 0.f, 0.f, 0.f};
      if (ep.gate0) gate += *reinterpret_cast<const f32x4*>(ep.gate0 + n);
      if (ep.gate1) gate += *reinterpret_cast<const f32x4*>(ep.gate1 + n);
    }
    gate *= ep.scale;
  }
  float* out = reinterpret_cast<float*>(ep.out);
  constexpr int kAgent = 16;  // cache policy bit sc1
  const long m_base = m_wave0 < M ? m_wave0 : M - 1;  // never in front of the descriptor's first row
  const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(uniform_address(reinterpret_cast<const uint16_t*>(out + m_base * N)), 0, -1, 0x00027000);
  auto offset = [&](long m) { return ((int)(m - m_base) * N + n) * 4; };
  // The residual rows of block mb + 1 are requested before the results of block mb are stored: memory operations
  // retire in order, so a load issued behind a block's stores could only be consumed once those stores had drained.
  f32x4 cur[2][WBN];
  auto fetch = [&](int mb, f32x4 (&dst)[WBN]) {
#pragma unroll
    for (int it = 0; it < WBN; ++it) {
      long m = m_wave0 + 16 * mb + RPI * it + rrow;
      if (m > M - 1) m = M - 1;  // rows past the end read the last row (never stored)
      if constexpr (CHAIN)
        dst[it] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, offset(m) - (n_ok ? 0 : 4 * n), 0, kAgent));
      else
        dst[it] = *reinterpret_cast<const f32x4*>(out + m * N + (n_ok ? n : 0));
    }
  };
  fetch(0, cur[0]);
#pragma unroll
  for (int mb = 0; mb < WBM; ++mb) {
#pragma unroll
    for (int nb = 0; nb < WBN; ++nb) *reinterpret_cast<f32x4*>(cw + lj * E16_F32_STRIDE + 16 * nb + 4 * lg) = block(nb, mb);
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    if (mb + 1 < WBM) fetch(mb + 1, cur[(mb + 1) & 1]);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int it = 0; it < WBN; ++it) {
      const f32x4 v = *reinterpret_cast<const f32x4*>(cw + (RPI * it + rrow) * E16_F32_STRIDE + rcol);
      const long m = m_wave0 + 16 * mb + RPI * it + rrow;
      const f32x4 r = cur[mb & 1][it] + gate * (v + bias);
      if constexpr (CHAIN) {
        if (n_ok && m < M) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, r), rsrc, offset(m), 0, kAgent);
      } else {
        if (n_ok && m < M) *reinterpret_cast<f32x4*>(out + m * N + n) = r;
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    __builtin_amdgcn_sched_barrier(0);
  }
#endif
}

// Epilogue of the 4-wave 16x16 kernels, block(nb, mb) being a lane's part of a block of results: wave (wm, wn) holds rows m0 + 16 WBM wm .. + 16 WBM, columns
// n0 + 16 WBN wn .. + 16 WBN.
template <int EPI, int WBM, int WBN, class BLOCK>
__device__ __forceinline__ void gemm16_finish(const BLOCK& block, const EpiArgs& ep, uint8_t* smem_raw, int wave, int wm, int wn,
                                              long m0, int n0, long M, int N, int lane) {
  constexpr int WTM = 16 * WBM, WTN = 16 * WBN;  // rows and columns of a wave's quadrant
  uint16_t* smem = reinterpret_cast<uint16_t*>(smem_raw);
  const int lj = lane & 15, lg = lane >> 4;
  if constexpr (EPI == CHORUS_EPI_BF16 || EPI == CHORUS_EPI_GELU_BF16) {
    gemm16_epilogue_bf16<EPI, WBM, WBN>(block, ep, smem + wave * e16_bf_wave<WBN>(), m0 + wm * WTM, n0 + wn * WTN, M, N, lane);
  } else if constexpr (EPI == CHORUS_EPI_RESID) {
    gemm16_epilogue_resid<WBM, WBN>(block, ep, reinterpret_cast<float*>(smem_raw) + wave * e16_f32_wave<WBN>(), m0 + wm * WTM,
                                    n0 + wn * WTN, M, N, lane);
  } else {
    // plain fp32: a lane stores its four consecutive columns of every block
#pragma unroll
    for (int nb = 0; nb < WBN; ++nb) {
      const int n = n0 + wn * WTN + 16 * nb + 4 * lg;
      if (n >= N) continue;
      f32x4 bias = {0.f, 0.f, 0.f, 0.f};
      if (ep.bias) bias = *reinterpret_cast<const f32x4*>(ep.bias + n);
#pragma unroll
      for (int mb = 0; mb < WBM; ++mb) {
        const long m = m0 + wm * WTM + 16 * mb + lj;
        if (m < M) *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(ep.out) + m * N + n) = block(nb, mb) + bias;
      }
    }
  }
}

}  // namespace chorus
