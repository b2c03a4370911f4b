// Attention with a learned bias by the distance between query and key: what its forward and backward kernels share.
#pragma once
#include "chorus_ops.h"
#include "common.h"

namespace chorus {

constexpr int kTileKeys = 64;      // keys (or, where keys stand still, queries) of a step, in LDS
constexpr int kTileQueries = 128;  // queries (or keys) of a workgroup
constexpr int kPad = 96;           // a near tile's distances reach 63 + 31 behind the farthest
constexpr int kMostFar = 512;  // biases and a wave's sums of every distance fit the LDS beside the tiles
constexpr int64_t kMostTokens = 1 << 28;
constexpr float kLog2E = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// A row's reference, or the exponent of its sum, goes into the sums of the matrix pipe, whose roundings are of its size then: 2^-14 each at this limit, in
// powers of two. Rows beyond it, which a large finite bias is all that is left to (or a large positive one), have no weights in the loops; a wave makes them
// by itself behind those, in fp32, taking the reference off the bias before the product is added, by a reference in two parts (Reference). No reference in the
// loops is below kLeastReference: a row that has seen only keys with a bias of -10000, or of the lowest value of the type, has lost nothing when it sees others.
constexpr float kMostInSums = 1024.f, kLeastReference = -32.f, kLeastSum = 0x1p-90f;
// What multiplies the products of a row: nothing is left of them beside a reference of a size that leaves nothing of them in 64 bits either. A row that has
// nothing but biases of the lowest value of the type has all its keys alike.
__device__ __forceinline__ float products_by(float scale, float reference) { return __builtin_fabsf(reference) < 0x1p60f ? scale : 0.f; }
__device__ __forceinline__ bool out_of_sums(float exponent) {
  return __builtin_fabsf(exponent) > kMostInSums && __builtin_fabsf(exponent) < INFINITY;
}

// What is taken off the logits of a row, in two parts: beside a bias of -1e10 one number in fp32 has no room for a product of 100. hi is near the largest
// bias, so that bias - hi is exact where it matters, and lo what is left of the largest logit.
struct Reference {
  float hi, lo;
  // up by so much; what the sum's rounding leaves off goes to lo
  __device__ __forceinline__ void move(float up) {
    const float t = lo + up, to = hi + t, moved = to - hi;
    lo = (hi - (to - moved)) + (t - moved);
    hi = to;
  }
};
// A share of a row: its reference and the sum of its weights, 0 where it has no key.
struct Share {
  Reference ref;
  float sum;
};

// A tensor of heads as the kernels see it: value (b, row, head, i) at p + b * batch + row * row_step + head * dh + i.
struct Rows {
  const uint16_t* p;
  long row, batch;
};
struct RowsOut {
  uint16_t* p;
  long row, batch;
};

struct BiasArgs {
  const float* table;     // [n_buckets, H]
  const int* bucket;      // [2 far + 1]
  const int* lens;        // [B] or null
  const int* first;       // [B] or null
  int n_buckets, far, causal;
  float scale;
  __device__ __forceinline__ int keys(int b, long Lk) const {
    if (!lens) return (int)Lk;
    const int n = lens[b];
    return n < 0 ? 0 : n > (int)Lk ? (int)Lk : n;
  }
  __device__ __forceinline__ int origin(int b) const {  // position of query 0 among the keys
    const int most = 1 << 29;
    const int f = first ? first[b] : 0;
    return f < -most ? -most : f > most ? most : f;
  }
  // keys that a query at position `last` or ahead of it sees: those behind are as if they were not there
  __device__ __forceinline__ int seen(int b, long Lk, int last) const {
    const int n = keys(b, Lk);
    return !causal || last + 1 > n ? n : last < 0 ? 0 : last + 1;
  }
  __host__ __device__ int width() const { return 2 * (far + kPad) + 1; }  // distances that a bias or a sum is kept for, the ends repeated
  // bucket of distance i - (far + kPad)
  __device__ __forceinline__ int bucket_of(int i) const {
    const int at = i - kPad;
    return bucket[at < 0 ? 0 : at > 2 * far ? 2 * far : at];
  }
};

// A head's biases on their way to LDS: buckets, then their values, each requested well ahead of its use. One for each distance from -(far + kPad) to far +
// kPad, in powers of two; a bucket outside the table has none. Finite ones end at +-2^90, so that the lowest value of the type, and differences of
// biases in units of the products, stay finite.
template <int THREADS>
struct BiasFill {
  static constexpr int kEach = (2 * (kMostFar + kPad) + THREADS) / THREADS;
  int c[kEach];
  float v[kEach];
  __device__ __forceinline__ void buckets(const BiasArgs& a, int tid) {
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      c[j] = -1;
      if (tid + j * THREADS < a.width()) c[j] = a.bucket_of(tid + j * THREADS);
    }
  }
  __device__ __forceinline__ void values(const BiasArgs& a, int head, int H) {
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      v[j] = 0.f;
      if ((unsigned)c[j] < (unsigned)a.n_buckets) v[j] = a.table[(long)c[j] * H + head];
    }
  }
  __device__ __forceinline__ void store(const BiasArgs& a, float* to, int tid) const {
#pragma unroll
    for (int j = 0; j < kEach; ++j)
      if (tid + j * THREADS < a.width())
        to[tid + j * THREADS] = __builtin_fabsf(v[j]) < INFINITY ? fminf(fmaxf(v[j] * kLog2E, -0x1p90f), 0x1p90f) : v[j];
  }
};

// Which of `n` tiles of a head and sequence a workgroup has, and which slice of it. Workgroups are dealt out to the XCDs in turn; where heads divide
// among them, an XCD has its share of the heads for all sequences, sequence by sequence, so that it has some of every length and a compute unit
// that takes two or three workgroups gets them of different sequences. The tiles of one head and sequence stay together.
struct Place {
  int b, head, tile, slice;
};
__device__ __forceinline__ Place place_of(int block, int blocks, int B, int H, int n, int slices) {
  Place p{0, 0, 0, 0};
  int at = H % 8 ? xcd_remap(block, blocks) : block / 8;
  if (slices > 1) {
    p.slice = at % slices;
    at /= slices;
  }
  const int of = at / n;
  p.tile = at - of * n;
  if (H % 8) {
    p.head = of / B;
    p.b = of - p.head * B;
  } else {
    p.b = of / (H / 8);
    p.head = block % 8 * (H / 8) + of - p.b * (H / 8);
  }
  // in scalar registers, where divisions do not leave them
  p.b = __builtin_amdgcn_readfirstlane(p.b);
  p.head = __builtin_amdgcn_readfirstlane(p.head);
  p.tile = __builtin_amdgcn_readfirstlane(p.tile);
  p.slice = __builtin_amdgcn_readfirstlane(p.slice);
  return p;
}

// A tile of rows in LDS: DH values a row, its 16-byte pieces at position piece ^ swizzle(row), such that 16 rows of a piece and its
// neighbour, which a fragment of rows takes, meet all banks, and so do 8 rows of 32 bytes, which a fragment of columns takes.
template <int DH>
__device__ __forceinline__ int tile_swizzle(int row) {
  return DH == 128 ? (row & 7) << 1 : (row >> 1 & 3) << 1;
}
typedef __attribute__((__vector_size__(4 * sizeof(short)))) short i16x4;

__device__ __forceinline__ void* uniform(const void* p) {
  const uint64_t u = reinterpret_cast<uint64_t>(p);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(u >> 32)), lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)u);
  return reinterpret_cast<void*>(((uint64_t)hi << 32) | lo);
}

#if defined(__HIP_DEVICE_COMPILE__)  // buffer descriptors are types of the device compiler's alone
// 64 rows of DH values on their way from global memory to LDS, through registers: a copy straight into LDS would make the compiler wait for
// all of them ahead of every transposing read. Each thread fetches the 16 bytes that belong at its place of the tile. Rows behind the last are
// the last one again: nothing behind it is read.
template <int DH, int THREADS>
struct TileStage {
  static constexpr int kPieces = DH / 8, kRows = THREADS / kPieces, kLoads = kTileKeys / kRows;  // of a row; of the workgroup's loads; of a thread for a tile
  int row, piece, row_bytes, to;
  u32x4 v[kLoads];
  __device__ __forceinline__ TileStage(int tid, long row_step) {
    row = tid / kPieces;
    piece = (tid % kPieces ^ tile_swizzle<DH>(row)) * 16;
    row_bytes = (int)(row_step * 2);
    to = tid * 8;
  }
  // the tile whose first row is at p, of which `rest` more rows exist
  __device__ __forceinline__ void fetch(const uint16_t* p, int rest) {
    const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(uniform(p), 0, -1, 0x00027000);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int r = row + i * kRows;  // row is below kRows, a power of two: their bits do not meet
      const int from = (r < rest ? r : rest) * row_bytes + (piece ^ tile_swizzle<DH>(i * kRows) * 16);
      v[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, from, 0, 0));
    }
  }
  __device__ __forceinline__ void store(uint16_t* tile) const {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) *reinterpret_cast<u32x4*>(tile + to + i * (THREADS * 8)) = v[i];
  }
};
#endif

// 16 rows of a tile as an operand of v_mfma_f32_16x16x32_bf16: lane l has row l % 16, values 32 kc + 8 (l / 16) .. + 8
template <int DH>
struct RowFragments {
  int at[DH / 32];
  __device__ __forceinline__ explicit RowFragments(int lane) {
    const int r = lane & 15, g = lane >> 4;
#pragma unroll
    for (int kc = 0; kc < DH / 32; ++kc) at[kc] = r * DH + ((4 * kc + g) ^ tile_swizzle<DH>(r)) * 8;
  }
  __device__ __forceinline__ bf16x8 read(const uint16_t* tile, int block, int kc) const {
    return *reinterpret_cast<const bf16x8*>(tile + block * 16 * DH + at[kc]);
  }
};
// 16 columns of 32 rows: lane l has column 16 db + l % 16, of rows 32 c + 4 (l / 16) + {0..3} and 16 further. One instruction takes 4 rows of 32 bytes
// for 16 lanes, lane i of them 8 bytes from row i / 4, and hands lane i column i.
template <int DH>
struct ColumnFragments {
  int at[DH / 16];
  __device__ __forceinline__ explicit ColumnFragments(int lane) {
    const int j = lane & 15, r = 4 * (lane >> 4) + (j >> 2);
#pragma unroll
    for (int db = 0; db < DH / 16; ++db) at[db] = r * DH + ((2 * db + (j >> 1 & 1)) ^ tile_swizzle<DH>(r)) * 8 + (j & 1) * 4;
  }
  __device__ __forceinline__ bf16x8 read(const uint16_t* tile, int c, int db) const {
    typedef __attribute__((address_space(3))) i16x4* Lds4;
    const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds4)(tile + 32 * c * DH + at[db]));
    const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds4)(tile + (32 * c + 16) * DH + at[db]));
    bf16x8 v;
    const bf16x4 a = __builtin_bit_cast(bf16x4, lo), b = __builtin_bit_cast(bf16x4, hi);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[e] = a[e];
      v[4 + e] = b[e];
    }
    return v;
  }
};

// A row by itself, made by a wave of the keys that it sees: a key a lane for the logits, a value of the result (of each 64) a lane for what is weighted by them.
template <int DH>
struct ApartRow {
  const uint16_t* q;      // the row
  const uint16_t* k;      // key 0, from row to row k_row
  long k_row;
  const float* s_bias;    // biases in powers of two, as BiasFill leaves them
  int nearest, far;       // distance of key 0 from the row
  float scale;            // with log2 e

  static __device__ __forceinline__ float product(const uint16_t* a, const uint16_t* b) {
    float sum = 0.f;
#pragma unroll 1
    for (int i = 0; i < DH; i += 8) {
      const bf16x8 x = *reinterpret_cast<const bf16x8*>(a + i), y = *reinterpret_cast<const bf16x8*>(b + i);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum = __builtin_fmaf((float)x[e], (float)y[e], sum);
    }
    return sum;
  }
  Reference ref;          // of its keys, once refer() has found it

  __device__ __forceinline__ int place(int j) const {  // of key j's bias
    const int at = nearest + j + far + kPad, last = 2 * (far + kPad);
    return at < 0 ? 0 : at < last ? at : last;
  }
  // logit of key j less the reference
  __device__ __forceinline__ float logit(int j) const {
    return __builtin_fmaf(product(q, k + (long)j * k_row), products_by(scale, ref.hi), (s_bias[place(j)] - ref.hi) - ref.lo);
  }
  __device__ __forceinline__ void refer(int j0, int j1, int lane) {
    float m = -INFINITY;
    for (int i = place(j0) + lane, last = place(j1 - 1); i <= last; i += 64) m = fmaxf(m, s_bias[i]);
    m = wave_max(m);
    ref = Reference{m > -INFINITY ? m : 0.f, 0.f};
    m = -INFINITY;
#pragma unroll 1
    for (int j = j0 + lane; j < j1; j += 64) m = fmaxf(m, logit(j));
    m = wave_max(m);
    ref.lo = m > -INFINITY ? m : 0.f;
  }
  // sum[e] = the sum over keys j0 .. j1 of weight(j) rows[j][lane + 64 e]; weight(j) is asked of lane j - j0 - 64 i
  template <class WEIGHT>
  static __device__ __forceinline__ void weighted(const WEIGHT& weight, const uint16_t* rows, long row_step, int j0, int j1, int lane, float (&sum)[DH / 64]) {
#pragma unroll
    for (int e = 0; e < DH / 64; ++e) sum[e] = 0.f;
#pragma unroll 1
    for (int at = j0; at < j1; at += 64) {
      float w = 0.f;
      if (at + lane < j1) w = weight(at + lane);
      const int count = j1 - at < 64 ? j1 - at : 64;
#pragma unroll 1
      for (int j = 0; j < count; ++j) {
        const float wj = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), j));
#pragma unroll
        for (int e = 0; e < DH / 64; ++e) sum[e] = __builtin_fmaf(wj, bf16_to_f32(rows[(long)(at + j) * row_step + lane + 64 * e]), sum[e]);
      }
    }
  }
};

// Rows l % 16 of which some lane l has the bit
__device__ __forceinline__ uint32_t rows_of_lanes(uint64_t lanes) {
  lanes |= lanes >> 32;
  return (uint32_t)(lanes | lanes >> 16) & 0xffff;
}

__device__ __forceinline__ f32x4 mfma(const bf16x8& a, const bf16x8& b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ float lane_value(int src, float v) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_ds_bpermute(4 * src, (int)__float_as_uint(v)));
}

// The 16 bits of an fp32 value that its rounding to bf16 leaves off, as the whole number that the rounded one's bits, 16 places further up, are short of
// the value's: both together are the value, but for a half that was rounded down, which is short of one in the last place.
__device__ __forceinline__ uint16_t left_off(float v) {
  const int d = (int)(__float_as_uint(v) - ((uint32_t)f32_to_bf16(v) << 16));
  return (uint16_t)(d < 0x7fff ? d : 0x7fff);
}
__device__ __forceinline__ float both_halves(uint16_t rounded, uint16_t rest) {
  return __uint_as_float(((uint32_t)rounded << 16) + (uint32_t)(int)(int16_t)rest);
}

bool bias_step_ok(int64_t row, int64_t batch, int64_t heads, int32_t dh);
int32_t check_bias_sizes(const chorus_bias_attention* a);
// The checks that both directions share; sets the kernels' view.
int32_t check_bias_attention(const chorus_bias_attention* a, const float* table, const int32_t* bucket, const int32_t* lens, const int32_t* first,
                             BiasArgs* out);

}  // namespace chorus
