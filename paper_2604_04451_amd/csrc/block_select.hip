// Which blocks of keys a block of queries attends to: means over blocks of rows, and from the means of queries and keys the choice.
#include "chorus_ops.h"
#include "common.h"

namespace chorus {
namespace {

// Mean over blocks of BLOCK consecutive rows of a head, a wave a block: a lane sums one chunk of eight values of every 64 / (dh /
// 8)-th row, each divided by BLOCK ahead of the sum, which is exact and keeps sums of the largest values finite, then the lanes of
// a chunk are added. HBM-bound: each row is read once, 16 bytes a lane, eight rows of a lane in flight (75600 x 5120 135 us, 5.8
// TB/s; 3271 x 1536 3.9 us, with one behind the other, where few blocks wait a memory latency a row, 6.8).
template <int DH, int BLOCK>
__global__ __launch_bounds__(256) void block_mean_kernel(const uint16_t* __restrict__ X, uint16_t* __restrict__ out, long L, long Lpad,
                                                         long nb, long total) {
  constexpr int LANES = DH / 8, ROWS = 64 / LANES, TIMES = BLOCK / ROWS;
  const int lane = threadIdx.x & 63;
  const long id = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (id >= total) return;
  const long head = id / nb, b = id - head * nb;
  const long first = b * BLOCK;
  const int n = (int)(L - first < BLOCK ? L - first : BLOCK), mine = lane / LANES;
  const uint16_t* x = X + (head * Lpad + first) * DH + lane * 8;
  float s[8] = {};
  auto add = [&](const u32x4& u) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      s[2 * k] = __builtin_fmaf(__uint_as_float(u[k] << 16), 1.0f / BLOCK, s[2 * k]);
      s[2 * k + 1] = __builtin_fmaf(__uint_as_float(u[k] & 0xffff0000u), 1.0f / BLOCK, s[2 * k + 1]);
    }
  };
  if (n == BLOCK) {
#pragma unroll
    for (int i0 = 0; i0 < TIMES; i0 += 8) {
      u32x4 u[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) u[i] = *reinterpret_cast<const u32x4*>(x + (i0 + i) * ROWS * DH);
#pragma unroll
      for (int i = 0; i < 8; ++i) add(u[i]);
    }
  } else {
    for (int i0 = 0; i0 * ROWS < n; i0 += 8) {  // a short last block: its last row stands for those behind its end, which are not added
      u32x4 u[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int row = (i0 + i) * ROWS + mine;
        u[i] = *reinterpret_cast<const u32x4*>(x + ((row < n ? row : n - 1) - mine) * DH);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if ((i0 + i) * ROWS + mine < n) add(u[i]);
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if (LANES == 8) s[e] += row_rotate<8>(s[e]);
    s[e] += swap_rows16(s[e]);
    s[e] += swap_halves(s[e]);
  }
  if (lane < LANES) {
    u32x4 o;
#pragma unroll
    for (int k = 0; k < 4; ++k) o[k] = pack_bf16x2(s[2 * k] / (float)n * BLOCK, s[2 * k + 1] / (float)n * BLOCK);
    *reinterpret_cast<u32x4*>(out + (head * nb + b) * DH + lane * 8) = o;
  }
}

// ---------------------------------------------------------------------------
// The choice. Scores decide between neighbours, so they are compared as their exact values; the matrix pipe gives them to fp32 only. A
// workgroup makes the fp32 scores of R rows of queries with every block of keys (16 x 16 tiles, the keys' fragments straight from
// memory: a head's means stay in its XCD's L2) into LDS, and then a wave takes a row: it finds the W-th largest score, and where the next
// one is further away than both can be off, which is nearly always, the choice stands. Elsewhere the scores within that distance are made
// again in fp64 and decide among themselves.
//
// How far a score can be off: products of bf16 are exact in fp32, and whatever the order of a sum of DH <= 128 of them, each of its
// additions is off by at most 2^-23 of the sum of magnitudes, itself at most |q| |k|: kBound |q| max |k|, and a trace for values
// that are flushed. Norms come from the same pipe (the largest entry of K K^T, which is on its diagonal) and are within 2^-16 of
// their values, which kBound has room for. Where |q| |k| is a number below 1e38 every score is one; where it is not (infinities,
// NaN, sums that fp32 does not hold) all scores are made in fp64.
//
// Two fifths of a workgroup's time go into the sweep over the keys (20K of 48K cycles at 591 x 1182 blocks, 40 heads: 77 us), the rest into its
// rows; there the vector and the scalar pipe share the work, 20 comparisons and 40 counts for each look at a row. The search therefore stays
// in floats, with no more than a mean between two looks (compared and bisected as integers, for a sure end, it took a quarter longer): a block
// that is in whatever its score (`always`) scores +inf, one that is out -inf.
// ---------------------------------------------------------------------------
constexpr uint32_t kIn = 0xffffffffu, kOut = 0u;  // the same two as codes: no finite float has them
constexpr float kBound = 1.05f / 65536.0f;
constexpr float kTrace = 2e-36f;  // more than 128 squares that fp32 does not hold

// A score as 64 bits whose unsigned order is that of the scores: both zeros alike, NaN below every number.
__device__ __forceinline__ uint64_t ordered(double s) {
  if (s != s) return 0;
  const uint64_t b = __builtin_bit_cast(uint64_t, s + 0.0);
  return b >> 63 ? ~b : b | (1ull << 63);
}

__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
  auto of = [](uint32_t a, uint32_t b) { return a > b ? a : b; };
  const auto h = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  v = of(h[0], h[1]);
  const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = of(r[0], r[1]);
  v = of(v, __builtin_amdgcn_update_dpp(0, v, 0x128, 0xf, 0xf, false));
  v = of(v, __builtin_amdgcn_update_dpp(0, v, 0x124, 0xf, 0xf, false));
  v = of(v, __builtin_amdgcn_update_dpp(0, v, 0x122, 0xf, 0xf, false));
  return __builtin_amdgcn_readfirstlane(of(v, __builtin_amdgcn_update_dpp(0, v, 0x121, 0xf, 0xf, false)));
}
__device__ __forceinline__ int lanes_below(uint64_t mask, int more) {  // of the mask's lanes, and `more`
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, more));
}

// Eight products, each exact in fp64, added one after the other.
__device__ __forceinline__ double dot8(const u32x4& x, const u32x4& y) {
  double s = 0.0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    s = __builtin_fma((double)__uint_as_float(x[e] << 16), (double)__uint_as_float(y[e] << 16), s);
    s = __builtin_fma((double)__uint_as_float(x[e] & 0xffff0000u), (double)__uint_as_float(y[e] & 0xffff0000u), s);
  }
  return s;
}

// The score of a row of queries and a block of keys in fp64: exact, unless terms are 2^30 apart. Beyond that the order of
// the additions decides, and it is close_border's, so that a row's choice is the same by either: eight values one after the
// other, then sums that are half of them apart, a quarter, ... and neighbours.
template <int DH>
__device__ __forceinline__ uint64_t exact_score(const uint16_t* __restrict__ q, const uint16_t* __restrict__ k) {
  constexpr int LANES = DH / 8;
  auto piece = [&](int l) { return dot8(*reinterpret_cast<const u32x4*>(q + 8 * l), *reinterpret_cast<const u32x4*>(k + 8 * l)); };
  double pair = 0.0, sum = 0.0;
#pragma unroll 1  // the sums 0, 2, 1, 3 of four, with few of the pieces in registers
  for (int i = 0; i < 4; ++i) {
    const int l = i >> 1 | (i & 1) << 1;
    double s = piece(l) + piece(l + LANES / 2);
    if (LANES == 16) s += piece(l + 4) + piece(l + 12);
    pair = i & 1 ? pair + s : s;
    if (i & 1) sum += pair;
  }
  return ordered(sum);
}

// Loops over a lane's scores that count across the wave: unrolled where the scores are in registers; in LDS, of a length not known
// before, they cannot be.
template <int NV>
constexpr int kTimesOf = NV > 0 ? NV : 1;

// A row's scores, one in 64 a lane: in registers (NV of them), or in LDS where there are more.
template <int NV>
struct Scores {
  float reg[NV > 0 ? NV : 1];
  uint32_t* at;  // the row in LDS, this lane's first
  int n;         // scores a lane
  __device__ __forceinline__ int count() const { return NV > 0 ? NV : n; }
  __device__ __forceinline__ float get(int i) const { return NV > 0 ? reg[NV > 0 ? i : 0] : __uint_as_float(at[64 * i]); }
  __device__ __forceinline__ void set(int i, float v) {
    if (NV > 0) reg[NV > 0 ? i : 0] = v;
    else at[64 * i] = __float_as_uint(v);
  }
  __device__ __forceinline__ int reach(float t) const {  // how many of the wave's scores reach t
    int c = 0, i = 0;
    if (NV == 0) {  // eight reads in flight
      for (; i + 8 <= n; i += 8) {
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = get(i + j);
#pragma unroll
        for (int j = 0; j < 8; ++j) c += __builtin_popcountll(__ballot(x[j] >= t));
      }
    }
#pragma unroll kTimesOf<NV>
    for (; i < count(); ++i) c += __builtin_popcountll(__ballot(get(i) >= t));
    return c;
  }
  // Where the border of the W largest is, `in` of the scores being +inf and `all` not -inf: `reached` of them reach `low`, W or
  // more, and fewer than W lie above `high`. Bisection between -bound and bound, beyond which there are finite scores on neither
  // side: first at twice the usual size of a score and at 0, then in the middle (a row's scores are spread like a bell, and halves
  // of their range come near in a few steps), until W are left above, or no more is to be had from scores that are `off` from
  // exact. As soon as the border lies among 64 scores or fewer they move to a lane each, and a step costs one comparison. With W
  // reached low = high is the W-th score, and `next` the one behind.
  struct Border {
    float low, high, next;
    int reached;
  };
  __device__ __forceinline__ Border border(int W, int in, int all, float bound, float usual, float off, float* __restrict__ list, int lane) const {
    float lo = -bound, hi = 1.01f * bound;
    int reach_lo = all, reach_hi = in;
    float mid = 2.0f * usual;
    while (reach_lo != W && hi - lo > off && reach_lo - reach_hi > 64) {
      const int c = reach(mid);
      const bool low = c >= W;
      reach_lo = low ? c : reach_lo;
      reach_hi = low ? reach_hi : c;
      lo = low ? mid : lo;
      hi = low ? hi : mid;
      mid = lo < 0.f && hi == 2.0f * usual ? 0.f : 0.5f * lo + 0.5f * hi;
    }
    float least = INFINITY, next = -INFINITY;
    if (reach_lo == W) {
#pragma unroll
      for (int i = 0; i < count(); ++i) {
        const float x = get(i);
        least = fminf(least, x >= lo ? x : INFINITY);
        next = fmaxf(next, x >= lo ? -INFINITY : x);
      }
    } else if (reach_lo - reach_hi <= 64) {
      int at = 0;
#pragma unroll kTimesOf<NV>
      for (int i = 0; i < count(); ++i) {
        const float x = get(i);
        const bool of = x >= lo && x < hi;
        const uint64_t taken = __ballot(of);
        if (of) list[lanes_below(taken, at)] = x;
        at += __builtin_popcountll(taken);
      }
      __builtin_amdgcn_wave_barrier();
      const float x = lane < at ? list[lane] : -INFINITY;
      __builtin_amdgcn_wave_barrier();
      const int above = reach_hi;
      while (reach_lo != W && hi - lo > off) {
        mid = 0.5f * lo + 0.5f * hi;
        const int c = above + __builtin_popcountll(__ballot(x >= mid));
        const bool low = c >= W;
        reach_lo = low ? c : reach_lo;
        lo = low ? mid : lo;
        hi = low ? hi : mid;
      }
      least = x >= lo ? x : INFINITY;
      next = x < lo ? x : -INFINITY;
    }
    if (reach_lo != W) return Border{lo, hi, lo, reach_lo};
    least = -wave_max(-least);
    return Border{least, least, wave_max(next), W};
  }
};

// Writes a row's choice, the blocks whose `take` holds: ascending, then -1.
template <int NV, class TAKE>
__device__ __forceinline__ void put_row(int n, TAKE take, int* __restrict__ to, int keep, int lane) {
  int put = 0;
#pragma unroll kTimesOf<NV>
  for (int i = 0; i < n; ++i) {
    const bool t = take(i);
    const uint64_t taken = __ballot(t);
    if (t) to[lanes_below(taken, put)] = lane + 64 * i;
    put += __builtin_popcountll(taken);
  }
  for (int i = put + lane; i < keep; i += 64) to[i] = -1;
}

// The scores from `down` to `up`, which the others leave open, kMostOpen of them at most, become +inf or -inf by their exact
// values: 8 values of a row a lane, so 8 or 16 lanes a block make its score, which is two reads and a sum away; then each open
// block's lane counts those in front. Returns false, with nothing done, where more are open.
constexpr int kMostOpen = 32;
template <int DH, int NV>
__device__ __forceinline__ bool close_border(Scores<NV>& v, int W, float down, float up, uint64_t* __restrict__ keys, const uint16_t* __restrict__ q,
                                             const uint16_t* __restrict__ km, int lane) {
  uint32_t* list = reinterpret_cast<uint32_t*>(keys);
  int open = 0, before = 0;
#pragma unroll kTimesOf<NV>
  for (int i = 0; i < v.count(); ++i) {
    const float x = v.get(i);
    before += __builtin_popcountll(__ballot(x > up));
    const uint64_t mask = __ballot(x >= down && x <= up);
    if (mask == 0) continue;
    const int place = lanes_below(mask, open);
    if (mask >> lane & 1 && place < kMostOpen) list[place] = lane + 64 * i;
    open += __builtin_popcountll(mask);
  }
  if (open > kMostOpen) return false;
  __builtin_amdgcn_wave_barrier();
  const int mine = lane < open ? (int)list[lane] : 0;
  __builtin_amdgcn_wave_barrier();
  constexpr int LANES = DH / 8;  // of a block
  for (int base = 0; base < open; base += 64 / LANES) {
    const int of = base + lane / LANES, b = __shfl(mine, of, 64);
    const u32x4 x = *reinterpret_cast<const u32x4*>(q + lane % LANES * 8), y = *reinterpret_cast<const u32x4*>(km + (long)b * DH + lane % LANES * 8);
    double s = dot8(x, y);
#pragma unroll
    for (int d = LANES / 2; d > 0; d /= 2) s += __shfl_xor(s, d, 64);
    if (lane % LANES == 0 && of < open) keys[of] = ordered(s);
  }
  __builtin_amdgcn_wave_barrier();
  const uint64_t key = lane < open ? keys[lane] : 0;
  for (int j = 0; j < open; ++j) {  // listed in ascending order of index: equal scores go to the lower lane
    const uint32_t hi = __builtin_amdgcn_readlane((uint32_t)(key >> 32), j), lo = __builtin_amdgcn_readlane((uint32_t)key, j);
    const uint64_t other = (uint64_t)hi << 32 | lo;
    before += other > key || (other == key && j < lane);
  }
  const uint64_t kept = __ballot(lane < open && before < W);
  __builtin_amdgcn_wave_barrier();
  open = 0;
#pragma unroll kTimesOf<NV>
  for (int i = 0; i < v.count(); ++i) {
    const float x = v.get(i);
    const uint64_t mask = __ballot(x >= down && x <= up);
    if (mask == 0) continue;
    if (mask >> lane & 1) v.set(i, kept >> lanes_below(mask, open) & 1 ? INFINITY : -INFINITY);
    open += __builtin_popcountll(mask);
  }
  return true;
}

// The choice of W where fp32 scores say nothing (`odd`), or are as good as equal by the dozen, from `down` to `up`. It is rare,
// works in LDS and stays out of the row loop's registers. The row there holds scores (+inf: in, -inf: out).
template <int DH>
__device__ __noinline__ void put_row_exactly(uint32_t* __restrict__ at, int n, int W, bool odd, float down, float up, const uint16_t* __restrict__ q,
                                             const uint16_t* __restrict__ km, int* __restrict__ to, int keep, int lane) {
  // codes: kIn, kOut, or 1 for what the exact scores decide
#pragma unroll 4
  for (int i = 0; i < n; ++i) {
    const uint32_t bits = at[64 * i];
    const float f = __uint_as_float(bits);
    const bool is_in = bits == 0x7f800000u || (!odd && f > up), is_out = bits == 0xff800000u || (!odd && f < down);
    at[64 * i] = is_in ? kIn : is_out ? kOut : 1u;
  }
  // the 64 bits of the scores in three parts, each among those that are alike in the part before; what is alike in all goes by index
  uint32_t from = 1, tied = kOut;
  int equal = 0;
  auto reach = [&](uint32_t t) {
    int c = 0;
    for (int i = 0; i < n; ++i) c += __builtin_popcountll(__ballot(at[64 * i] >= t));
    return c;
  };
  for (int part = 0; part < 3; ++part) {
    for (int i = 0; i < n; ++i) {
      const uint32_t x = at[64 * i];
      if (x != kOut && x != kIn) {
        const uint64_t e = exact_score<DH>(q, km + (long)(lane + 64 * i) * DH);
        at[64 * i] = 1u + (part == 0 ? (uint32_t)(e >> 33) : part == 1 ? (uint32_t)(e >> 2) & 0x7fffffffu : (uint32_t)e & 3u);
      }
    }
    uint32_t lo = 1, hi = kIn;  // all that are open reach the one, fewer than W the other
    int reached = reach(lo);
    while (reached != W && hi - lo > 1) {
      const uint32_t mid = lo + (hi - lo) / 2;
      const int c = reach(mid);
      if (c >= W) {
        lo = mid;
        reached = c;
      } else {
        hi = mid;
      }
    }
    from = lo;
    tied = kOut;
    if (reached == W) break;
    tied = lo;
    from = kIn;
    equal = W - reach(lo + 1);
    for (int i = 0; i < n; ++i) {
      const uint32_t x = at[64 * i];
      if (x != kOut && x != kIn && x != tied) at[64 * i] = x > tied ? kIn : kOut;
    }
  }
  put_row<0>(n, [&](int i) {
    const uint32_t x = at[64 * i];
    const uint64_t ties = __ballot(tied != kOut && x == tied);
    const bool take = x >= from || (tied != kOut && x == tied && lanes_below(ties, 0) < equal);
    equal -= __builtin_popcountll(ties);
    return take;
  }, to, keep, lane);
}

// T: 16-row tiles of queries, R = 16 T rows or fewer where T is 1. THREADS: 1024, four waves a SIMD of 128 registers a lane, but
// where a lane holds 40 scores. With 20 it takes a little more than there are: 1 to 9 values of a lane wait in scratch memory (16
// to 48 bytes), written once ahead of the sweep over the keys and read once behind it, and 71 scalar values in lanes of vector
// registers (188 with 40 scores, 22 with 8).
template <int DH, int NV, int T, int THREADS>
__global__ __launch_bounds__(THREADS, THREADS == 1024 ? 4 : 2) void block_select_kernel(const uint16_t* __restrict__ Qm, const uint16_t* __restrict__ Km,
                                                                                        const uint8_t* __restrict__ rule, int* __restrict__ blocks, int nq,
                                                                                        int nk, int group, int keep, int R, int stride, int tiles) {
  constexpr int KC = DH / 32, WAVES = THREADS / 64;
  extern __shared__ __attribute__((aligned(16))) uint32_t score[];  // [R][stride]
  __shared__ uint32_t s_k2[WAVES];        // the largest squared norm of a block of keys that a wave met
  __shared__ float s_q2[16 * T];          // the rows' squared norms
  __shared__ uint64_t s_list[WAVES][kMostOpen];  // 64 scores at a border, then the exact ones of the blocks that are open
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int at = xcd_remap(blockIdx.x, gridDim.x), head = at / tiles, first = (at - head * tiles) * R;
  const uint16_t* q0 = Qm + (long)head * nq * DH;
  const uint16_t* km = Km + (long)(head / group) * nk * DH;
  const int strips = (nk + 15) / 16, last = strips - 1;
  // the rules of this lane's blocks, on their way while the scores are made
  uint32_t of_block[NV > 0 ? NV : 1];
  auto rule_of = [&](int i) { return lane + 64 * i >= nk ? 2u : rule ? (uint32_t)rule[lane + 64 * i] : 0u; };
#pragma unroll
  for (int i = 0; i < (NV > 0 ? NV : 1); ++i) of_block[i] = rule_of(i);
  {
    const int l16 = lane & 15, g = lane >> 4;
    // A lane's KC fragments are neighbouring pieces of 16 bytes of its row. Read as they stand, each lane would be a request of its
    // own, which is what the sweep then waits for (591 x 1182 blocks, 40 heads, 91 us instead of 77; 256 x 512, 12 heads, 14.8
    // instead of 11.8); so KC neighbouring lanes read the pieces of one row, KC rows in turn, and exchange them.
    const int r0 = l16 / KC * KC, piece = KC * g + l16 % KC;
    bf16x8 qf[T][KC];
#pragma unroll
    for (int t = 0; t < T; ++t) {
#pragma unroll
      for (int j = 0; j < KC; ++j) {
        const int of = 16 * t + r0 + j < R ? 16 * t + r0 + j : R - 1, row = first + of < nq ? first + of : nq - 1;
        qf[t][j] = *reinterpret_cast<const bf16x8*>(q0 + (long)row * DH + piece * 8);
      }
      transpose_lanes(qf[t], lane);
    }
    // strips of 16 keys, two in flight behind the one in use; behind the last strip one key for all lanes, which costs next to nothing
    const uint32_t whole = (r0 * DH + piece * 8) * 2;
    bf16x8 kf[3][KC];
    auto fetch = [&](bf16x8(&to)[KC], int strip) {
      const char* from = reinterpret_cast<const char*>(km + (long)(strip > last ? 0 : strip) * 16 * DH);
      if (KC == 4 && strip < last) {  // one address for four loads; two are not worth the branch
#pragma unroll
        for (int j = 0; j < KC; ++j) to[j] = *reinterpret_cast<const bf16x8*>(from + whole + j * DH * 2);
      } else {
        const int most = strip > last ? 0 : strip == last ? nk - 1 - 16 * last : 15;
#pragma unroll
        for (int j = 0; j < KC; ++j) to[j] = *reinterpret_cast<const bf16x8*>(from + (uint32_t)((r0 + j < most ? r0 + j : most) * DH + piece * 8) * 2);
      }
    };
    uint32_t k2 = 0;  // as bits: a NaN is above all numbers, and the sign of one is dropped
    uint32_t* to = score + (long)l16 * stride + 4 * g;
    auto use = [&](bf16x8(&kf)[KC], int strip) {
      transpose_lanes(kf, lane);
      f32x4 s[T], n2 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int t = 0; t < T; ++t) s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kc = 0; kc < KC; ++kc) {
#pragma unroll
        for (int t = 0; t < T; ++t) s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[kc], qf[t][kc], s[t], 0, 0, 0);
        n2 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[kc], kf[kc], n2, 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t bits = __float_as_uint(n2[i]) & 0x7fffffffu;
        k2 = bits > k2 ? bits : k2;
      }
#pragma unroll
      for (int t = 0; t < T; ++t)
        if (T > 1 || l16 < R) *reinterpret_cast<u32x4*>(to + (long)t * 16 * stride + strip * 16) = __builtin_bit_cast(u32x4, s[t]);
    };
    fetch(kf[0], wave);
    fetch(kf[1], wave + WAVES);
    // behind the last strip, what a wave reads of a row is zeros
    const int pad = (64 - strips * 16 % 64) % 64;
    for (int row = wave; row < R; row += WAVES)
      if (lane < pad) score[(long)row * stride + strips * 16 + lane] = 0;
    for (int strip = wave; strip <= last; strip += 3 * WAVES) {
      fetch(kf[2], strip + 2 * WAVES);
      use(kf[0], strip);
      if (strip + WAVES > last) break;
      fetch(kf[0], strip + 3 * WAVES);
      use(kf[1], strip + WAVES);
      if (strip + 2 * WAVES > last) break;
      fetch(kf[1], strip + 4 * WAVES);
      use(kf[2], strip + 2 * WAVES);
    }
    k2 = wave_max_u32(k2);
    if (lane == 0) s_k2[wave] = k2;
    if (wave == 0) {
#pragma unroll
      for (int t = 0; t < T; ++t) {
        float q2 = 0.f;
#pragma unroll
        for (int kc = 0; kc < KC; ++kc)
#pragma unroll
          for (int e = 0; e < 8; ++e) q2 = __builtin_fmaf((float)qf[t][kc][e], (float)qf[t][kc][e], q2);
        q2 += swap_rows16(q2);
        q2 += swap_halves(q2);
        if (g == 0) s_q2[16 * t + l16] = q2;
      }
    }
  }
  // 0, or +inf or -inf whatever the score
  const int n = NV > 0 ? NV : (nk + 63) / 64;
  int always = 0, ordinary = nk;
  if (rule) {
    ordinary = 0;
#pragma unroll kTimesOf<NV>
    for (int i = 0; i < n; ++i) {
      const uint32_t c = NV > 0 ? of_block[NV > 0 ? i : 0] : rule_of(i);
      always += __builtin_popcountll(__ballot(c == 1));
      ordinary += __builtin_popcountll(__ballot(c != 1 && c != 2));
    }
  }
  const bool among_always = always >= keep;  // the choice is among those alone
  const int in = among_always ? 0 : always, all = among_always ? always : always + ordinary, W = keep < all ? keep : all;
  auto place = [&](uint32_t c) { return c == 1 ? (among_always ? 0.f : INFINITY) : c == 2 || among_always ? -INFINITY : 0.f; };
  float by_rule[NV > 0 ? NV : 1];
#pragma unroll
  for (int i = 0; i < (NV > 0 ? NV : 1); ++i) by_rule[i] = place(of_block[i]);
  __syncthreads();
  const float k_norm = sqrtf(__uint_as_float(wave_max_u32(s_k2[lane % WAVES])) + kTrace);

  for (int r = wave; r < R && first + r < nq; r += WAVES) {
    Scores<NV> v;
    v.at = score + (long)r * stride + lane;
    v.n = n;
    const float q_norm = sqrtf(__uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(s_q2[r]))) + kTrace);
    const float off = kBound * q_norm * k_norm + 7.7e-34f * (1.0f + q_norm) * (1.0f + k_norm);
    const float bound = 1.01f * q_norm * k_norm + off;
    const bool odd = !(bound < 1e38f);  // room for a search between -bound and a little more than bound
    const bool every = W == all;  // all that may be chosen are
#pragma unroll
    for (int i = 0; i < v.count(); ++i) {
      const float p = NV > 0 ? by_rule[NV > 0 ? i : 0] : place(rule_of(i));
      float f = 0.f;
      if (!every && !odd && 64 * i < nk) f = __uint_as_float(v.at[64 * i]);
      v.set(i, f + p);
    }
    int* to = blocks + ((long)head * nq + first + r) * keep;
    const uint16_t* q = q0 + (long)(first + r) * DH;
    float from = -3.402823466e38f, down = 0.f;
    bool clear = every;
    if (!every && !odd) {
      const auto border = v.border(W, in, all, bound, bound * (DH == 128 ? 0.088f : 0.125f), off, reinterpret_cast<float*>(s_list[wave]), lane);
      from = border.low;
      clear = border.reached == W && border.low - border.next > 2.0f * off;
      if (!clear) {
        down = border.low - 2.0f * off;
        from = border.high + 2.0f * off;  // nothing is left between `down` and this
        clear = close_border<DH>(v, W, down, from, s_list[wave], q, km, lane);
      }
    }
    if (clear) {
      put_row<NV>(v.count(), [&](int i) { return v.get(i) >= from; }, to, keep, lane);
    } else {
#pragma unroll
      for (int i = 0; i < v.count(); ++i)
        if (64 * i < nk) v.at[64 * i] = __float_as_uint(v.get(i));
      put_row_exactly<DH>(v.at, (nk + 63) / 64, W, odd, down, from, q, km, to, keep, lane);
    }
  }
}

// The rows of a workgroup. All of them share one sweep over a head's keys, which is what the call waits for (1182 blocks of 128
// values are 300 KB, from the L2, and a compute unit holds one workgroup): as few as let the launch run in one round of workgroups,
// and where it takes more than one, 32 (two matrix tiles) or as many as their scores leave room for in the LDS, down to two rows of
// CHORUS_BLOCK_SELECT_MAX scores (128 KB). 103 x 205 blocks, 12 heads: 8 rows 9.2 us, 4 rows (312 workgroups) half as long again.
int select_rows(long nq, int H, int stride) {
  int R = 4;
  while (R < 32 && (nq + R - 1) / R * H > 256) R *= 2;
  while (R > 1 && (size_t)R * stride * 4 > 155 * 1024) R /= 2;
  return R;
}

}  // namespace
}  // namespace chorus

using namespace chorus;

extern "C" {

int32_t chorus_block_mean(const uint16_t* X, uint16_t* out, int64_t L, int64_t Lpad, int32_t H, int32_t dh, int32_t block, void* stream) {
  if (L < 0 || Lpad < L || H <= 0) return CHORUS_E_ARG;
  if ((dh != 64 && dh != 128) || (block != CHORUS_BLOCK_QUERIES && block != CHORUS_BLOCK_KEYS)) return CHORUS_E_SHAPE;
  if (L == 0) return CHORUS_OK;
  if (!X || !out || !aligned16(X) || !aligned16(out)) return CHORUS_E_ARG;
  const int64_t nb = L / block + (L % block != 0);
  if (nb > 0x7fffffffL) return CHORUS_E_SHAPE;
  const int64_t total = nb * H, groups = (total + 3) / 4;
  if (groups > 0xffffffffL / 256) return CHORUS_E_SHAPE;  // the threads of a launch
  const dim3 grid((unsigned)groups);
#define MEAN(DH, BLOCK) \
  hipLaunchKernelGGL((block_mean_kernel<DH, BLOCK>), grid, dim3(256), 0, (hipStream_t)stream, X, out, (long)L, (long)Lpad, (long)nb, (long)total)
  if (dh == 128) {
    if (block == CHORUS_BLOCK_QUERIES) MEAN(128, CHORUS_BLOCK_QUERIES);
    else MEAN(128, CHORUS_BLOCK_KEYS);
  } else {
    if (block == CHORUS_BLOCK_QUERIES) MEAN(64, CHORUS_BLOCK_QUERIES);
    else MEAN(64, CHORUS_BLOCK_KEYS);
  }
#undef MEAN
  CHORUS_LAUNCH_CHECK();
  return CHORUS_OK;
}

int32_t chorus_block_select(const uint16_t* Qm, const uint16_t* Km, const uint8_t* rule, int32_t* blocks, int64_t nq, int64_t nk, int32_t H,
                            int32_t Hk, int32_t dh, int32_t keep, void* stream) {
  if (nq < 0 || nk < 0 || H <= 0 || Hk <= 0 || keep < 1) return CHORUS_E_ARG;
  if (H % Hk || (dh != 64 && dh != 128) || nk < 1 || nk > CHORUS_BLOCK_SELECT_MAX) return CHORUS_E_SHAPE;
  // a workgroup of up to 1024 threads for each row at the most, of the 2^32 - 1 of a launch
  if (nq > 0xffffffffL / 1024 / H || keep > 0x7fffffff - 64) return CHORUS_E_SHAPE;
  if (nq == 0) return CHORUS_OK;
  if (!Qm || !Km || !blocks || !aligned16(Qm) || !aligned16(Km) || !aligned16(blocks) || !aligned16(rule)) return CHORUS_E_ARG;
  const int stride = (int)((nk + 63) / 64 * 64) + 4;  // rows 4 banks apart
  const int R = select_rows((long)nq, H, stride);
  const int64_t tiles = (nq + R - 1) / R;
  const size_t lds = (size_t)R * stride * sizeof(float);
#define SELECT(DH, NV, T, THREADS)                                                                                                        \
  do {                                                                                                                                   \
    static DynLdsOnce once;                                                                                                              \
    CHK_STATUS(once.ensure((const void*)block_select_kernel<DH, NV, T, THREADS>, 155 * 1024));                                           \
    hipLaunchKernelGGL((block_select_kernel<DH, NV, T, THREADS>), dim3((unsigned)(tiles * H)), dim3(THREADS), lds, (hipStream_t)stream, Qm, \
                       Km, rule, blocks, (int)nq, (int)nk, H / Hk, keep, R, stride, (int)tiles);                                         \
  } while (0)
#define SELECT_ROWS(DH, NV, THREADS)           \
  do {                                         \
    if (R == 32) SELECT(DH, NV, 2, THREADS);   \
    else SELECT(DH, NV, 1, THREADS);           \
  } while (0)
  // A lane holds the scores of its row in 8, 20 or 40 registers, the fewest of these that do, and behind that reads them from LDS
  // at each look (2 rows of 9000 blocks: 88 us). At the borders, 12 heads: 256 rows of 512 blocks 11.1 us with 8 registers, 16.6
  // with 20; 600 of 1280 37.4 with 20, 64.0 with 40; 600 of 2560 104 with 40, 141 from LDS. More steps would pay between them: 300
  // rows of 600 blocks 17.5 us, 13.3 with 12 registers; 450 of 1000 27.5, 24.4 with 16.
#define SELECT_LENGTH(DH)                           \
  do {                                              \
    if (nk <= 64 * 8) SELECT_ROWS(DH, 8, 1024);     \
    else if (nk <= 64 * 20) SELECT_ROWS(DH, 20, 1024); \
    else if (nk <= 64 * 40) SELECT(DH, 40, 1, 512); \
    else SELECT(DH, 0, 1, 1024);                    \
  } while (0)
  if (dh == 128) SELECT_LENGTH(128);
  else SELECT_LENGTH(64);
#undef SELECT_LENGTH
#undef SELECT_ROWS
#undef SELECT
  CHORUS_LAUNCH_CHECK();
  return CHORUS_OK;
}

}  // extern "C"
