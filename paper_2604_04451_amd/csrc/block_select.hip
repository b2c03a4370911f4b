// Which blocks of keys a block of queries attends to: means over blocks of rows, and from the means of queries and keys the choice.
#include "chorus_ops.h"
#include "common.h"

namespace chorus {
namespace {

// Mean over blocks of `block` consecutive rows of a head, a wave a block: a lane sums one chunk of eight values of every 64 / (dh / 8)-th
// row, then the lanes of a chunk are added. HBM-bound: each row is read once, 16 bytes a lane.
template <int DH>
__global__ __launch_bounds__(256) void block_mean_kernel(const uint16_t* __restrict__ X, uint16_t* __restrict__ out, long L, long Lpad,
                                                         int block, long nb, long total) {
  constexpr int LANES = DH / 8, ROWS = 64 / LANES;
  const int lane = threadIdx.x & 63;
  const long id = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (id >= total) return;
  const long head = id / nb, b = id - head * nb;
  const long first = b * block;
  const int n = (int)(L - first < block ? L - first : block);
  const uint16_t* x = X + (head * Lpad + first) * DH + lane * 8;
  float s[8] = {};
  for (int r = lane / LANES, i = 0; r < n; r += ROWS, ++i) {
    const u32x4 u = *reinterpret_cast<const u32x4*>(x + (long)i * ROWS * DH);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      s[2 * k] += __uint_as_float(u[k] << 16);
      s[2 * k + 1] += __uint_as_float(u[k] & 0xffff0000u);
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
    for (int k = 0; k < 4; ++k) o[k] = pack_bf16x2(s[2 * k] / (float)n, s[2 * k + 1] / (float)n);
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
// that are flushed. Norms come from the same pipe (the diagonal of K K^T) and are within 2^-16 of their values, which kBound has room for.
//
// A score is held as 32 bits whose unsigned order is the order of the floats; 0 stands for "out" and kIn for "in", which no finite
// float has. Under `always` a block is in from the start, under `never` out.
// ---------------------------------------------------------------------------
constexpr uint32_t kIn = 0xffffffffu, kOut = 0u;
constexpr float kBound = 1.05f / 65536.0f;
constexpr int kSelectThreads = 512;

__device__ __forceinline__ uint32_t ordered(float f) {
  const uint32_t b = __float_as_uint(f + 0.0f);
  return b >> 31 ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t v) { return __uint_as_float(v >> 31 ? v & 0x7fffffffu : ~v); }
// NaN below every number, both zeros alike
__device__ __forceinline__ uint64_t ordered(double s) {
  if (s != s) return 0;
  const uint64_t b = __builtin_bit_cast(uint64_t, s + 0.0);
  return b >> 63 ? ~b : b | (1ull << 63);
}

template <bool MAX>
__device__ __forceinline__ uint32_t wave_extreme(uint32_t v) {
  auto of = [](uint32_t a, uint32_t b) { return (a > b) == MAX ? a : b; };
  const auto h = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  v = of(h[0], h[1]);
  const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = of(r[0], r[1]);
  v = of(v, __builtin_amdgcn_update_dpp(0, v, 0x128, 0xf, 0xf, false));
  v = of(v, __builtin_amdgcn_update_dpp(0, v, 0x124, 0xf, 0xf, false));
  v = of(v, __builtin_amdgcn_update_dpp(0, v, 0x122, 0xf, 0xf, false));
  return __builtin_amdgcn_readfirstlane(of(v, __builtin_amdgcn_update_dpp(0, v, 0x121, 0xf, 0xf, false)));
}

// The score of a row of queries and a block of keys in fp64: exact, unless terms are 2^30 apart.
template <int DH>
__device__ __forceinline__ uint64_t exact_score(const uint16_t* __restrict__ q, const uint16_t* __restrict__ k) {
  double s = 0.0;
#pragma unroll 4
  for (int d = 0; d < DH; d += 8) {
    const u32x4 a = *reinterpret_cast<const u32x4*>(q + d), b = *reinterpret_cast<const u32x4*>(k + d);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      s = __builtin_fma((double)__uint_as_float(a[e] << 16), (double)__uint_as_float(b[e] << 16), s);
      s = __builtin_fma((double)__uint_as_float(a[e] & 0xffff0000u), (double)__uint_as_float(b[e] & 0xffff0000u), s);
    }
  }
  return ordered(s);
}

// The row's scores, one in 64 a lane: in registers (NV of them), or in LDS where there are more.
template <int NV>
struct Scores {
  uint32_t reg[NV > 0 ? NV : 1];
  uint32_t* at;  // the row in LDS, this lane's first
  int n;         // scores a lane
  __device__ __forceinline__ int count() const { return NV > 0 ? NV : n; }
  __device__ __forceinline__ uint32_t get(int i) const { return NV > 0 ? reg[NV > 0 ? i : 0] : at[64 * i]; }
  __device__ __forceinline__ void set(int i, uint32_t v) {
    if (NV > 0) reg[NV > 0 ? i : 0] = v;
    else at[64 * i] = v;
  }
  template <class OF>
  __device__ __forceinline__ int how_many(OF of) const {  // of the wave's scores
    int c = 0;
#pragma unroll
    for (int i = 0; i < count(); ++i) c += __builtin_popcountll(__ballot(of(get(i))));
    return c;
  }
  // The largest t that at least W scores reach, or one that exactly W reach. Bisection between the least and the largest score, of values
  // where they are floats (a row's scores are spread like a bell, so halves of its range leave their order of magnitude in a few
  // steps, as halves of the order of the bits do not), of the order otherwise; the latter always ends.
  __device__ __forceinline__ uint32_t find(int W, bool floats, int& reached) const {
    uint32_t least = kIn, most = kOut;
#pragma unroll
    for (int i = 0; i < count(); ++i) {
      const uint32_t v = get(i);
      if (v != kOut && v < least) least = v;
      if (v != kIn && v > most) most = v;
    }
    uint32_t lo = wave_extreme<false>(least), hi = wave_extreme<true>(most) + 1;
    reached = how_many([&](uint32_t v) { return v >= lo; });
    for (int step = 0; reached != W && hi - lo > 1; ++step) {
      uint32_t mid = lo + (hi - lo) / 2;
      if (floats && step < 16) {
        const uint32_t m = ordered(0.5f * unordered(lo) + 0.5f * unordered(hi));
        if (m > lo && m < hi) mid = m;
      }
      const int c = how_many([&](uint32_t v) { return v >= mid; });
      if (c >= W) {
        lo = mid;
        reached = c;
      } else {
        hi = mid;
      }
    }
    return lo;
  }
};

// Writes the row's choice: what reaches `from`, and the first `equal` of those that are `tied`, which is below it; ascending, then -1.
template <int NV>
__device__ __forceinline__ void put_row(const Scores<NV>& v, uint32_t from, uint32_t tied, int equal, int* __restrict__ to, int keep,
                                        int lane) {
  int put = 0;
  const uint64_t below = (1ull << lane) - 1;
#pragma unroll
  for (int i = 0; i < v.count(); ++i) {
    const uint32_t x = v.get(i);
    const uint64_t ties = __ballot(x == tied && x < from);
    const bool take = x >= from || (x == tied && __builtin_popcountll(ties & below) < equal);
    const uint64_t taken = __ballot(take);
    if (take) to[put + __builtin_popcountll(taken & below)] = lane + 64 * i;
    put += __builtin_popcountll(taken);
    equal -= __builtin_popcountll(ties);
  }
  for (int i = put + lane; i < keep; i += 64) to[i] = -1;
}

// The choice of W by exact scores among those that are neither in nor out. Their 64 bits are compared in three parts, each among those that
// are alike in the part before; what is alike in all goes by index. In LDS, as this is rare and its loops are long.
template <int DH>
__device__ __noinline__ void put_row_exactly(Scores<0> v, int W, const uint16_t* __restrict__ q, const uint16_t* __restrict__ km,
                                             int* __restrict__ to, int keep, int lane) {
  uint32_t from = 1, tied = kIn;
  int equal = 0;
  for (int part = 0; part < 3; ++part) {
    for (int i = 0; i < v.n; ++i) {
      const uint32_t x = v.get(i);
      if (x != kOut && x != kIn) {
        const uint64_t e = exact_score<DH>(q, km + (long)(lane + 64 * i) * DH);
        v.set(i, 1u + (part == 0 ? (uint32_t)(e >> 33) : part == 1 ? (uint32_t)(e >> 2) & 0x7fffffffu : (uint32_t)e & 3u));
      }
    }
    int reached;
    from = v.find(W, false, reached);
    if (reached == W) break;
    tied = from;
    from = kIn;
    equal = W - v.how_many([&](uint32_t x) { return x > tied; });
    for (int i = 0; i < v.n; ++i) {
      const uint32_t x = v.get(i);
      if (x != kOut && x != kIn && x != tied) v.set(i, x > tied ? kIn : kOut);
    }
  }
  put_row(v, from, tied, from == kIn ? equal : 0, to, keep, lane);
}

template <int DH, int NV>
__global__ __launch_bounds__(kSelectThreads) void block_select_kernel(const uint16_t* __restrict__ Qm, const uint16_t* __restrict__ Km,
                                                                      const uint8_t* __restrict__ rule, int* __restrict__ blocks, int nq,
                                                                      int nk, int group, int keep, int R, int stride, int tiles) {
  constexpr int KC = DH / 32, WAVES = kSelectThreads / 64;
  extern __shared__ __attribute__((aligned(16))) uint8_t s_raw[];
  float* score = reinterpret_cast<float*>(s_raw);  // [R][stride]
  __shared__ uint32_t s_k2;                        // the largest squared norm of a block of keys
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int at = xcd_remap(blockIdx.x, gridDim.x), head = at / tiles, first = (at - head * tiles) * R;
  const uint16_t* q0 = Qm + (long)head * nq * DH;
  const uint16_t* km = Km + (long)(head / group) * nk * DH;
  if (threadIdx.x == 0) s_k2 = 0;
  __syncthreads();
  {
    const int l16 = lane & 15, g = lane >> 4;
    bf16x8 qf[KC];
    const int row = first + l16 < nq ? first + l16 : nq - 1;
#pragma unroll
    for (int kc = 0; kc < KC; ++kc) qf[kc] = *reinterpret_cast<const bf16x8*>(q0 + (long)row * DH + 32 * kc + 8 * g);
    float k2 = 0.f;
    for (int strip = wave; strip * 16 < nk; strip += WAVES) {
      const int key = strip * 16 + l16 < nk ? strip * 16 + l16 : nk - 1;
      bf16x8 kf[KC];
#pragma unroll
      for (int kc = 0; kc < KC; ++kc) kf[kc] = *reinterpret_cast<const bf16x8*>(km + (long)key * DH + 32 * kc + 8 * g);
      f32x4 s = {0.f, 0.f, 0.f, 0.f}, n2 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kc = 0; kc < KC; ++kc) {
        s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[kc], qf[kc], s, 0, 0, 0);
        n2 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[kc], kf[kc], n2, 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (4 * g + i == l16) k2 = n2[i] >= k2 || n2[i] != n2[i] ? n2[i] : k2;  // a NaN stays
      if (l16 < R) *reinterpret_cast<f32x4*>(score + (long)l16 * stride + strip * 16 + 4 * g) = s;
    }
    if (k2 != k2) k2 = INFINITY;
    atomicMax(&s_k2, __float_as_uint(k2));
  }
  __syncthreads();
  const float k_norm = sqrtf(__uint_as_float(s_k2));

  for (int r = wave; r < R && first + r < nq; r += WAVES) {
    const uint16_t* q = q0 + (long)(first + r) * DH;
    Scores<NV> v;
    v.at = reinterpret_cast<uint32_t*>(score + (long)r * stride) + lane;
    v.n = (nk + 63) / 64;
    float q2 = 0.f;
    if (lane < DH / 2) {
      const uint32_t two = *reinterpret_cast<const uint32_t*>(q + 2 * lane);
      const float a = __uint_as_float(two << 16), b = __uint_as_float(two & 0xffff0000u);
      q2 = a * a + b * b;
    }
    const float q_norm = sqrtf(wave_sum(q2));
    const float off = kBound * q_norm * k_norm + 7.7e-34f * (1.0f + q_norm) * (1.0f + k_norm);
    int always = 0, free_ = 0;
    if (rule) {
      for (int b = lane; b < v.n * 64; b += 64) {
        const int c = b < nk ? rule[b] : 2;
        always += __builtin_popcountll(__ballot(c == 1));
        free_ += __builtin_popcountll(__ballot(c != 1 && c != 2));
      }
    } else {
      free_ = nk;
    }
    const bool among_always = always >= keep;  // the choice is among those alone
    const int W = among_always ? keep : always + free_ < keep ? always + free_ : keep;
    bool odd = !(off < INFINITY);  // scores that fp32 does not hold
#pragma unroll
    for (int i = 0; i < v.count(); ++i) {
      const int b = lane + 64 * i;
      uint32_t x = kOut;
      if (b < nk) {
        const float f = score[(long)r * stride + b];
        const int c = rule ? rule[b] : 0;
        if (c == 1) x = among_always ? ordered(f) : kIn;
        else if (c != 2 && !among_always) x = ordered(f);
        if (!(fabsf(f) < INFINITY)) {
          odd = true;
          if (x != kOut && x != kIn) x = 1;
        }
      }
      v.set(i, x);
    }
    odd = __any(odd);
    int* to = blocks + ((long)head * nq + first + r) * keep;
    const int some = v.how_many([](uint32_t x) { return x != kOut; });
    if (W >= some) {
      put_row(v, 1u, kIn, 0, to, keep, lane);
      continue;
    }
    if (!odd) {
      int reached;
      const uint32_t t = v.find(W, true, reached);
      uint32_t least = kIn, next = kOut;  // the W-th, and what comes behind it
#pragma unroll
      for (int i = 0; i < v.count(); ++i) {
        const uint32_t x = v.get(i);
        if (x >= t && x < least) least = x;
        if (x < t && x > next) next = x;
      }
      const float last = unordered(wave_extreme<false>(least)), behind = unordered(wave_extreme<true>(next));
      if (reached == W && last - behind > 2.0f * off) {
        put_row(v, t, kIn, 0, to, keep, lane);
        continue;
      }
      const uint32_t up = ordered(last + 2.0f * off), down = ordered(last - 2.0f * off);
#pragma unroll
      for (int i = 0; i < v.count(); ++i) {
        const uint32_t x = v.get(i);
        if (x != kOut && x != kIn) v.set(i, x > up ? kIn : x < down ? kOut : 1u);
      }
      if (v.how_many([](uint32_t x) { return x != kOut; }) == W) {
        put_row(v, 1u, kIn, 0, to, keep, lane);
        continue;
      }
    }
    Scores<0> all;
    all.at = v.at;
    all.n = v.n;
#pragma unroll
    for (int i = 0; i < v.count(); ++i)
      if (i < v.n) all.set(i, v.get(i));
    put_row_exactly<DH>(all, W, q, km, to, keep, lane);
  }
}

// The rows of a workgroup: 16, one matrix tile, as long as their scores leave room for two workgroups on a compute unit and the launch has
// two for each; fewer otherwise, down to one row of CHORUS_BLOCK_SELECT_MAX scores (64 KB).
int select_rows(long nq, int H, int stride) {
  int R = 16;
  while (R > 1 && (size_t)R * stride * 4 > 80 * 1024) R /= 2;
  while (R > 4 && (nq + R - 1) / R * H < 512) R /= 2;
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
  const int64_t nb = (L + block - 1) / block;
  if (nb > 0x7fffffffL) return CHORUS_E_SHAPE;
  const int64_t total = nb * H, groups = (total + 3) / 4;
  if (groups > 0x7fffffffL) return CHORUS_E_SHAPE;
  const dim3 grid((unsigned)groups);
  if (dh == 128)
    hipLaunchKernelGGL(block_mean_kernel<128>, grid, dim3(256), 0, (hipStream_t)stream, X, out, (long)L, (long)Lpad, block, (long)nb, (long)total);
  else
    hipLaunchKernelGGL(block_mean_kernel<64>, grid, dim3(256), 0, (hipStream_t)stream, X, out, (long)L, (long)Lpad, block, (long)nb, (long)total);
  CHORUS_LAUNCH_CHECK();
  return CHORUS_OK;
}

int32_t chorus_block_select(const uint16_t* Qm, const uint16_t* Km, const uint8_t* rule, int32_t* blocks, int64_t nq, int64_t nk, int32_t H,
                            int32_t Hk, int32_t dh, int32_t keep, void* stream) {
  if (nq < 0 || nk < 0 || H <= 0 || Hk <= 0 || keep < 1) return CHORUS_E_ARG;
  if (H % Hk || (dh != 64 && dh != 128) || nk < 1 || nk > CHORUS_BLOCK_SELECT_MAX) return CHORUS_E_SHAPE;
  if (nq > 0x7fffffffL / H) return CHORUS_E_SHAPE;
  if (nq == 0) return CHORUS_OK;
  if (!Qm || !Km || !blocks || !aligned16(Qm) || !aligned16(Km) || !aligned16(blocks) || !aligned16(rule)) return CHORUS_E_ARG;
  const int stride = (int)((nk + 63) / 64 * 64) + 4;  // rows 4 banks apart
  const int R = select_rows((long)nq, H, stride);
  const int64_t tiles = (nq + R - 1) / R;
  const size_t lds = (size_t)R * stride * sizeof(float);
#define SELECT(DH, NV)                                                                                                                   \
  do {                                                                                                                                   \
    static DynLdsOnce once;                                                                                                              \
    CHK_STATUS(once.ensure((const void*)block_select_kernel<DH, NV>, 80 * 1024));                                                        \
    hipLaunchKernelGGL((block_select_kernel<DH, NV>), dim3((unsigned)(tiles * H)), dim3(kSelectThreads), lds, (hipStream_t)stream, Qm, Km, \
                       rule, blocks, (int)nq, (int)nk, H / Hk, keep, R, stride, (int)tiles);                                             \
  } while (0)
#define SELECT_LENGTH(DH)                  \
  do {                                     \
    if (nk <= 64 * 4) SELECT(DH, 4);       \
    else if (nk <= 64 * 8) SELECT(DH, 8);  \
    else if (nk <= 64 * 20) SELECT(DH, 20); \
    else if (nk <= 64 * 40) SELECT(DH, 40); \
    else SELECT(DH, 0);                    \
  } while (0)
  if (dh == 128) SELECT_LENGTH(128);
  else SELECT_LENGTH(64);
#undef SELECT_LENGTH
#undef SELECT
  CHORUS_LAUNCH_CHECK();
  return CHORUS_OK;
}

}  // extern "C"
