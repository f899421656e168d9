// ntc_linear_tile.h -- the tiled matrix products of linear layers over bins, on MFMA.
//
// One kernel, three products of two row-major operands P and Q:
//   kForward  out[s][n]    = sum_k P[s][k] Q_e[n][k]     P = x rows by slot, Q = weight
//   kInput    out[s][c]    = sum_n P[s][n] Q_e[n][c]     P = dz rows by slot, Q = weight
//   kWeight   out_e[m][c]  = sum_s P[s][m] Q[s][c]       P = dz rows, Q = x rows, s over e's bin
// An operand whose contraction runs along its rows ("along": P of the first two, Q of
// the first) is staged as rows of 64 contraction values; one whose contraction runs
// across its rows ("across") as 64 rows of the tile's columns.
#pragma once

#include <type_traits>

#include "ntc_experts.h"

namespace ntc {

enum Product { kForward, kInput, kWeight };

// How rows are found.  kDense: slots in order, a row each.  kGather: through perm or
// slots_per_row, offsets from the operand's start within 4 GiB.  kFar: the same with
// 64-bit addresses.
enum Access { kDense, kGather, kFar };

// Which of a product's 256 x 256 tiles a launch takes: all; those that fill whole rounds of
// the 256 CUs; or the others, each cut into smaller ones, where they come to at most half a
// round (else the whole rounds' launch has them too).
enum Part { kAll, kWhole, kRest };

// Division of slots (below 2^31) by a constant: d = 1 .. 2^31 - 1, L = ceil(log2 d),
// m = ceil(2^(31 + L) / d), which fits 32 bits; floor(s m / 2^(31 + L)) is exact because
// m d - 2^(31 + L) < 2^L.
struct Divisor {
  uint32_t m, shift;
};
__device__ __forceinline__ uint32_t divided(uint32_t s, Divisor d) {
  return __umulhi(s << 1, d.m) >> d.shift;
}

struct TileArgs {
  const void *p, *q;          // 16-byte aligned, strides multiples of 8 elements
  int64_t p_stride, q_stride; // elements between rows
  int64_t q_expert;           // elements between experts' Q (kForward, kInput)
  Divisor p_div, q_div;       // row of a slot
  const uint32_t *bin_offset, *perm;
  uint32_t perm_capacity;
  int32_t n_experts;
  uint32_t n;                 // slots
  int32_t rows, cols, contr;  // out rows (kWeight), out columns, contraction (padded to 8)
  int64_t p_rows, q_rows;     // rows of P, of Q (kForward, kInput: of an expert's)
  int32_t p_width, q_width;   // elements of a row that may be read
  void *out;
  int64_t out_stride, out_expert;
  int32_t out_f32;
  int32_t vec;                // the epilogue's rows take 8 elements at a time
  // kForward's epilogue
  const void *bias;
  int32_t activation;
  float slope;
  const void *residual;
  int64_t residual_stride;
  void *pre;
  int64_t pre_stride;
  uint32_t *written;          // kInput: set to 0 at every slot written (may be NULL)
  Part part;                  // of the tiles
};

// What out-of-range lanes read instead.
static __device__ const uint4v kZeros = {0u, 0u, 0u, 0u};

typedef float float16v __attribute__((ext_vector_type(16)));

template <class T> struct Frag;
template <> struct Frag<_Float16> {
  typedef half8 type;
  static __device__ __forceinline__ float16v mfma(half8 a, half8 b, float16v c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
  }
};
template <> struct Frag<__bf16> {
  typedef bf16x8 type;
  static __device__ __forceinline__ float16v mfma(bf16x8 a, bf16x8 b, float16v c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
};

// ------------------------------------------------------------- activations

// 1 - Phi(size) of the normal distribution, size >= 0, erf by formula 7.1.26 (its
// coefficients halved) of Abramowitz and Stegun, "Handbook of Mathematical Functions"
// (absolute error of erf below 1.5e-7; the result is rounded to 16 bits or scaled by z).
__device__ __forceinline__ float normal_tail(float size, float *density_exp) {
  const float t = __builtin_amdgcn_rcpf(1.f + 0.3275911f * 0.70710678f * size);
  const float e = __builtin_amdgcn_exp2f(size * size * -0.72134752f);  // exp(-size^2 / 2)
  *density_exp = e;
  return e * (t * (0.127414796f +
                   t * (-0.142248368f + t * (0.7107068705f +
                                             t * (-0.7265760135f + t * 0.5307027145f)))));
}

// z kept within +-10^4, where every activation has reached its limit (16-bit types hold
// larger numbers only of no further effect on the factor): infinities get the limit's
// value instead of infinity times 0; NaN stays.
__device__ __forceinline__ float bounded(float z) {
  const float size = fabsf(z) > 1e4f ? 1e4f : fabsf(z);
  return __builtin_copysignf(size, z);
}

__device__ __forceinline__ float logistic(float z) {
  return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * -1.44269504f));
}

template <int V>
__device__ __forceinline__ void activate_all(float (&z)[V], int act, float slope) {
  float e;
  if (act == NTC_ACT_RELU) {
#pragma unroll
    for (int j = 0; j < V; ++j) z[j] = z[j] < 0.f ? 0.f : z[j];  // NaN stays
  } else if (act == NTC_ACT_LEAKY_RELU) {
#pragma unroll
    for (int j = 0; j < V; ++j) z[j] = z[j] > 0.f ? z[j] : slope * z[j];
  } else if (act == NTC_ACT_GELU) {
#pragma unroll
    for (int j = 0; j < V; ++j) {  // z Phi(z) on either side of 0
      const float size = fabsf(bounded(z[j]));
      z[j] = fmaxf(z[j], 0.f) - size * normal_tail(size, &e);
    }
  } else if (act == NTC_ACT_SILU) {
#pragma unroll
    for (int j = 0; j < V; ++j) z[j] = (z[j] < -1e4f ? -1e4f : z[j]) * logistic(z[j]);
  }
}

__device__ __forceinline__ float activation_slope(float z, int act, float slope) {
  z = bounded(z);
  switch (act) {
    case NTC_ACT_RELU: return z > 0.f ? 1.f : 0.f;
    case NTC_ACT_LEAKY_RELU: return z > 0.f ? 1.f : slope;
    case NTC_ACT_GELU: {
      float e;
      const float tail = normal_tail(fabsf(z), &e);
      return (z < 0.f ? tail : 1.f - tail) + z * e * 0.39894228f;
    }
    case NTC_ACT_SILU: {
      const float t = logistic(z);
      return t * (1.f + z * (1.f - t));
    }
    default: return 1.f;
  }
}

// V consecutive outputs of a row from their sums: bias, pre, activation, residual, store.
// ALIGNED: the rows start on whole runs; else on elements, which memory accesses of more
// than one element take as well, only slower.
template <class T, int V, bool ALIGNED>
struct __attribute__((packed, aligned(ALIGNED ? sizeof(T) * V : sizeof(T)))) Run {
  T v[V];
};

template <class T, Product PRODUCT, int V, bool ALIGNED>
__device__ __forceinline__ void finish(const TileArgs &a, int expert, int64_t row, int col,
                                       float (&v)[V]) {
  if constexpr (PRODUCT == kForward) {
    if (a.bias) {
      const Run<T, V, ALIGNED> b = *(const Run<T, V, ALIGNED> *)((const T *)a.bias + (int64_t)expert * a.cols + col);
#pragma unroll
      for (int j = 0; j < V; ++j) v[j] += (float)b.v[j];
    }
    if (a.pre) {
      Run<T, V, ALIGNED> z;
#pragma unroll
      for (int j = 0; j < V; ++j) z.v[j] = (T)v[j];
      *(Run<T, V, ALIGNED> *)((T *)a.pre + row * a.pre_stride + col) = z;
    }
    activate_all<V>(v, a.activation, a.slope);
    if (a.residual) {
      const int64_t at = row * a.residual_stride + col;
      if (a.out_f32) {
        const Run<float, V, ALIGNED> r = *(const Run<float, V, ALIGNED> *)((const float *)a.residual + at);
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] += r.v[j];
      } else {
        const Run<T, V, ALIGNED> r = *(const Run<T, V, ALIGNED> *)((const T *)a.residual + at);
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] += (float)r.v[j];
      }
    }
  }
  const int64_t at = row * a.out_stride + col +
                     (PRODUCT == kWeight ? (int64_t)expert * a.out_expert : 0);
  if (a.out_f32) {
    Run<float, V, ALIGNED> o;
#pragma unroll
    for (int j = 0; j < V; ++j) o.v[j] = v[j];
    *(Run<float, V, ALIGNED> *)((float *)a.out + at) = o;
  } else {
    Run<T, V, ALIGNED> o;
#pragma unroll
    for (int j = 0; j < V; ++j) o.v[j] = (T)v[j];
    *(Run<T, V, ALIGNED> *)((T *)a.out + at) = o;
  }
}

// The same for the columns that exist.
template <class T, Product PRODUCT, int V>
__device__ __forceinline__ void finish_some(const TileArgs &a, int expert, int64_t row, int col,
                                            float (&v)[V]) {
  if (a.vec) {  // whole runs only
    if (col < a.cols) finish<T, PRODUCT, V, true>(a, expert, row, col, v);
  } else if (col + V <= a.cols) {
    finish<T, PRODUCT, V, false>(a, expert, row, col, v);
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j) {
      float one[1] = {v[j]};
      if (col + j < a.cols) finish<T, PRODUCT, 1, true>(a, expert, row, col + j, one);
    }
  }
}

// ------------------------------------------------------------------- staging

// 16 bytes a lane from memory to LDS, past the registers: lane i's land at `to` + 16 i.
__device__ __forceinline__ void to_lds(const void *from, void *to) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from,
                                   (__attribute__((address_space(3))) void *)to, 16, 0, 0);
}

// Until all but the YOUNGER youngest loads of every wave, and its LDS reads, are done.
template <int YOUNGER>
__device__ __forceinline__ void staged_barrier() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(YOUNGER) : "memory");
}

// LDS order of 16-byte pieces.  Along: rows of 8 pieces, piece c of row r at
// c ^ ((r >> 1) & 7), so that 16 rows' pieces read at once lie in different banks.
// Across: rows of COLS / 8 pieces, piece c of row r at c ^ 4 (r & 3), for the four rows
// and four pieces that half a wave's transposing read takes (64 columns: two rows lie in
// different banks as they are, c ^ 4 ((r >> 1) & 1)).
__device__ __forceinline__ int along_swizzle(int r) { return (r >> 1) & 7; }
template <int COLS>
__device__ __forceinline__ int across_swizzle(int r) {
  return COLS == 64 ? 4 * ((r >> 1) & 1) : 4 * (r & 3);
}

typedef short short4v __attribute__((ext_vector_type(4)));
typedef short short8v __attribute__((ext_vector_type(8)));

// Eight contraction values of column i (of 16): rows 0-3 and 4-7 below `at`, one
// transposing read each.
template <class T, int ROW_BYTES>
__device__ __forceinline__ typename Frag<T>::type across_frag(const char *at) {
  typedef __attribute__((address_space(3))) short4v *Lds;
  const short4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)at);
  const short4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(at + 4 * ROW_BYTES));
  return __builtin_bit_cast(typename Frag<T>::type, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4,
                                                                            5, 6, 7));
}

// ------------------------------------------------------------ expert of a tile

// Finds the expert and first slot position of row tile `tile` among all experts' tiles
// of 2^log slots, in LDS; returns the number of tiles.  Every thread of the workgroup calls.
struct TileSpot {
  int expert;
  uint32_t begin, end;  // positions in perm
};

template <int THREADS>
__device__ __forceinline__ uint32_t count_tiles(const TileArgs &a, int log, uint32_t *scratch,
                                                uint32_t &before, uint32_t &mine) {
  const uint32_t side = 1u << log;
  const int t = threadIdx.x, per = (a.n_experts + THREADS - 1) / THREADS;
  mine = 0;
  for (int e = t * per; e < (t + 1) * per && e < a.n_experts; ++e) {
    const uint32_t lo = min(a.bin_offset[e], a.perm_capacity);
    const uint32_t hi = min(a.bin_offset[e + 1], a.perm_capacity);
    mine += hi > lo ? (hi - lo + side - 1) >> log : 0;
  }
  // exclusive sum over the workgroup
  uint32_t sum = mine;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const uint32_t up = __shfl_up(sum, d);
    if ((t & 63) >= d) sum += up;
  }
  if ((t & 63) == 63) scratch[t >> 6] = sum;
  __syncthreads();
  uint32_t base = 0, total = 0;
  for (int w = 0; w < THREADS / 64; ++w) {
    if (w < (t >> 6)) base += scratch[w];
    total += scratch[w];
  }
  before = base + sum - mine;
  return total;
}

template <int THREADS>
__device__ __forceinline__ void find_tile(const TileArgs &a, int log, uint32_t tile, uint32_t before,
                                          uint32_t mine, TileSpot *spot) {
  const uint32_t side = 1u << log;
  if (tile >= before && tile < before + mine) {
    const int per = (a.n_experts + THREADS - 1) / THREADS;
    uint32_t left = tile - before;
    for (int e = threadIdx.x * per; e < ((int)threadIdx.x + 1) * per && e < a.n_experts; ++e) {
      const uint32_t lo = min(a.bin_offset[e], a.perm_capacity);
      const uint32_t hi = min(a.bin_offset[e + 1], a.perm_capacity);
      const uint32_t tiles = hi > lo ? (hi - lo + side - 1) >> log : 0;
      if (left < tiles) {
        spot->expert = e;
        spot->begin = lo + left * side;
        spot->end = hi;
        break;
      }
      left -= tiles;
    }
  }
  __syncthreads();
}

// ---------------------------------------------------------------- the kernel

// TM x TN outputs per workgroup of 2 x 2 waves, contraction in steps of 64 through two
// LDS buffers, each step multiplied in two halves of 32 from registers.  A half's
// fragments are read from LDS while the half before is multiplied, so that no MFMA waits
// for LDS.  After a step's second half has been read its buffer takes the pieces of the
// step after next, spread over more than a half's MFMAs; they have until the next step's
// first half ends.  One barrier a step covers both.  Steps of 64 and not 32: pieces of
// whole 128-byte lines (with 64-byte pieces the L2 was asked twice for every line).  At
// 8192 x 4096 x 4096 bf16 a forward product takes 211 us (1.30 PFLOP/s, MFMA 85 % busy
// in long contractions; with 64-byte pieces 228), the input gradient 208, the weight
// gradient 197.  A 64 x 64 tile multiplies a step too fast for the next one's pieces to
// come from memory meanwhile: it has four buffers (128 x 4096 x 4096: 32 us with two, 15
// with four).  MFMA takes Q's rows as its first operand, so a lane ends up with four
// consecutive output columns of one row.
template <class T, Product PRODUCT, Access ACCESS, int TM, int TN>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(TM > 128 ? 1 : 2)))
void tile_product(TileArgs a) {
#ifdef __HIP_DEVICE_COMPILE__  // the host's pass knows no buffer resources in lambdas
  constexpr int kWaves = 4, kThreads = 256, WN = 2;
  constexpr bool kPAcross = PRODUCT == kWeight, kQAcross = PRODUCT != kForward;
  constexpr int FM = TM / 64, FN = TN / 64;  // fragments of 32 per wave
  constexpr int kPBytes = TM * 128, kQBytes = TN * 128, kBuffer = kPBytes + kQBytes;
  constexpr int kRing = TM > 64 ? 2 : 4;  // buffers
  typedef typename Frag<T>::type F;
  // objects of their own, so that the compiler sees that reads of one don't wait for
  // pieces on their way to another
  __shared__ __align__(16) char lds0[kBuffer], lds1[kBuffer];
  __shared__ __align__(16) char lds2[kRing > 2 ? kBuffer : 16], lds3[kRing > 2 ? kBuffer : 16];
  __shared__ uint32_t scratch[kWaves];
  __shared__ TileSpot spot;

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  // which tile
  int expert = 0;
  uint32_t begin, end;   // slot positions: the tile's rows, or kWeight's contraction
  int32_t row0 = 0, col0;
  if constexpr (PRODUCT == kWeight) {
    const uint32_t row_tiles = (uint32_t)(a.rows + TM - 1) / TM;
    const uint32_t col_tiles = (uint32_t)(a.cols + TN - 1) / TN;
    const uint32_t each = row_tiles * col_tiles;
    // an eighth of every expert's tiles on each XCD: experts differ in length
    const uint32_t share = (each + 7) / 8;
    expert = (int)(blockIdx.x / 8 / share);
    const uint32_t in = blockIdx.x % 8 * share + blockIdx.x / 8 % share;
    if (in >= each) return;
    const uint32_t group = in / (8 * col_tiles), inside = in % (8 * col_tiles);
    const uint32_t high = min(8u, row_tiles - group * 8);
    row0 = (int32_t)(group * 8 + inside % high) * TM;
    col0 = (int32_t)(inside / high) * TN;
    begin = 0;
    end = a.n;
    if (ACCESS != kDense && a.perm) {
      begin = min(a.bin_offset[expert], a.perm_capacity);
      end = max(begin, min(a.bin_offset[expert + 1], a.perm_capacity));
    }
  } else {
    constexpr int kLog = TM == 64 ? 6 : TM == 128 ? 7 : 8;
    static_assert(TM == TN, "");
    constexpr uint32_t kCut = 256 / TM;
    const bool rest = kCut > 1 && ACCESS != kFar && a.part == kRest;
    const int log = rest ? 8 : kLog;
    const uint32_t side = 1u << log;
    const uint32_t col_tiles = ((uint32_t)a.cols + side - 1) >> log;
    uint32_t before = 0, mine = 0;
    uint32_t tiles;
    if (ACCESS != kDense && a.perm) tiles = count_tiles<kThreads>(a, log, scratch, before, mine);
    else tiles = (uint32_t)(((uint64_t)a.n + side - 1) >> log);
    const uint64_t total = (uint64_t)tiles * col_tiles;
    const uint64_t over = a.part != kAll && total % 256 <= 128 ? total % 256 : 0;
    const uint64_t count = rest ? over * (kCut * kCut) : total - over;  // of this launch
    if (blockIdx.x >= count) return;
    uint32_t b = xcd_local_block(blockIdx.x, (uint32_t)count), cut = 0;
    if (rest) {
      cut = b % (kCut * kCut);
      b = (uint32_t)(total - over) + b / (kCut * kCut);
    }
    // groups of 8 row tiles, column tiles within: 8 row tiles share a Q tile at a time
    const uint32_t group = b / (8 * col_tiles), in = b % (8 * col_tiles);
    const uint32_t high = min(8u, tiles - group * 8);
    const uint32_t tile = group * 8 + in % high;
    col0 = (int32_t)((in / high * side) + cut % kCut * TN);
    if (ACCESS != kDense && a.perm) {
      find_tile<kThreads>(a, log, tile, before, mine, &spot);
      expert = __builtin_amdgcn_readfirstlane(spot.expert);
      begin = __builtin_amdgcn_readfirstlane(spot.begin) + cut / kCut * TM;
      end = __builtin_amdgcn_readfirstlane(spot.end);
      if (begin >= end || a.perm[begin] == NTC_PAD) return;  // padding past the bin's last slot
    } else {
      begin = tile * side + cut / kCut * TM;
      end = a.n;
    }
    if (begin >= end || col0 >= a.cols) return;  // a tile's cut
  }

  const char *P = (const char *)a.p;
  const char *Q = (const char *)a.q;
  if constexpr (PRODUCT != kWeight) Q += (int64_t)expert * a.q_expert * 2;
  const char *zeros = (const char *)&kZeros;
  // the slot at a position; NTC_PAD past the end and for slots that don't exist
  auto slot_at = [&](uint32_t pos) -> uint32_t {
    uint32_t s = pos < end ? pos : begin;
    if (ACCESS != kDense && a.perm) {
      s = a.perm[s];
      asm("" : "+v"(s));  // loaded for every lane: a select, not a branch
    }
    return pos < end && s < a.n ? s : NTC_PAD;
  };
  const uint32_t contr = PRODUCT == kWeight ? end - begin : (uint32_t)a.contr;
  const uint32_t steps = contr / 64 + (contr % 64 != 0);

  // Staging: piece i of this wave covers 1 KB of a buffer, 16 bytes a lane.  Addresses are
  // a base that moves on with the step, in scalar registers, and an offset a lane; what
  // lies past the operand's end reads as 0, and so does the offset kNothing.  Rows and
  // columns of outputs that don't exist may read anything, contraction values that
  // don't exist have to read 0 from both operands.
  constexpr int kPLoads = TM / 8 / kWaves, kQLoads = TN / 8 / kWaves;
  constexpr int kLoads = kPLoads + kQLoads;
  constexpr int kPRow = 512 / TM, kQRow = 512 / TN;  // across: rows a piece covers
  constexpr uint32_t kNothing = 0xFFFFFFFFu, kLimit = 0xFFFFFFF0u;
  // kFar, and the operands whose rows come by slot in kWeight
  constexpr bool kPFar = ACCESS == kFar, kQFar = ACCESS == kFar && PRODUCT == kWeight;
  constexpr bool kBySlot = PRODUCT == kWeight && ACCESS != kDense;
  const int64_t p_bytes = a.p_stride * 2, q_bytes = a.q_stride * 2;
  const int64_t p_step = kPAcross ? (kBySlot ? 0 : 64 * p_bytes) : 128;
  const int64_t q_step = kQAcross ? (kBySlot ? 0 : 64 * q_bytes) : 128;
  // first rows: along P starts at its first slot's, along Q at col0, across at the columns
  uint32_t p_first = 0;
  if constexpr (!kPAcross && ACCESS != kGather) p_first = ACCESS == kDense ? begin : 0;
  if constexpr (kPAcross && !kBySlot) p_first = begin;
  const uint32_t q_first = PRODUCT == kForward ? (uint32_t)col0
                           : PRODUCT == kWeight && !kBySlot ? begin : 0;
  const char *p_base = P + (int64_t)p_first * p_bytes + (kPAcross ? row0 * 2 : 0);
  const char *q_base = Q + (int64_t)q_first * q_bytes + (kQAcross ? col0 * 2 : 0);
  const int64_t p_size = (a.p_rows - 1 - (int64_t)p_first) * p_bytes + a.p_width * 2 -
                         (kPAcross ? row0 * 2 : 0);
  const int64_t q_size = (a.q_rows - 1 - (int64_t)q_first) * q_bytes + a.q_width * 2 -
                         (kQAcross ? col0 * 2 : 0);

  uint32_t offset[kLoads];
  const char *far[kPFar ? kPLoads : 1];  // along P of kFar: the row itself
  bool far_on[kPFar ? kPLoads : 1];
  // along: the column of every piece of this lane
  const int along_c = ((lane & 7) ^ along_swizzle(wave * 8 + (lane >> 3))) * 8;
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const bool is_p = i < kPLoads;
    const int piece = (is_p ? i : i - kPLoads) * kWaves + wave;
    const uint32_t bytes = (uint32_t)(is_p ? p_bytes : q_bytes);
    if (is_p ? kPAcross : kQAcross) {
      const int per = (is_p ? TM : TN) / 8;  // pieces a row
      const int r = piece * (is_p ? kPRow : kQRow) + lane / per;
      offset[i] = ((lane % per) ^ (is_p ? across_swizzle<TM>(r) : across_swizzle<TN>(r))) * 16 + (kBySlot ? 0 : r * bytes);
    } else {
      const int r = piece * 8 + (lane >> 3);
      offset[i] = r * bytes + along_c * 2;
      if constexpr (ACCESS != kDense) {
        if (is_p) {
          const uint32_t s = slot_at(begin + r);
          const uint32_t row = divided(s, a.p_div);
          if constexpr (kPFar) {
            far_on[i] = s != NTC_PAD;
            far[i] = P + (far_on[i] ? (int64_t)row * p_bytes + along_c * 2 : 0);
          } else {
            offset[i] = s != NTC_PAD ? row * bytes + along_c * 2 : kNothing;
          }
        }
      }
    }
  }
  // kWeight by slot: the slots of a step's pieces, read kRing / 2 steps before they are
  // staged.  With TM == TN a piece of P and the piece of Q with its number cover the same.
  static_assert(PRODUCT != kWeight || TM == TN, "");
  constexpr int kSlots = kBySlot ? kPLoads : 1;
  auto read_slots = [&](uint32_t (&slot)[kSlots], uint32_t index) {
    if constexpr (kBySlot) {
#pragma unroll
      for (int i = 0; i < kSlots; ++i) {
        const uint32_t pos = begin + index * 64 + (i * kWaves + wave) * kPRow + lane / (TM / 8);
        slot[i] = pos < end ? pos : begin;
        if (a.perm) slot[i] = a.perm[slot[i]];  // looked at when it is used
      }
    }
  };
  // The operand as a buffer resource.  Steps move on by the instruction's scalar offset,
  // which the range check counts; a weight past 4 GiB (kFar's kInput) by its base.
  constexpr bool kQMoves = kPFar && PRODUCT == kInput;
  auto window = [&](const char *base, int64_t size) {
    const int64_t rest = size > 0 ? size : 0;
    return __builtin_amdgcn_make_buffer_rsrc(
        const_cast<char *>(base), 0,
        (int)(uint32_t)(rest < (int64_t)kLimit ? rest : (int64_t)kLimit), 0x00020000);
  };
  const auto p_all = window(p_base, p_size), q_all = window(q_base, q_size);
  // before a step's pieces: along pieces past the contraction's end read 0 from now on
  auto open_step = [&](uint32_t index) {
    if constexpr (!kPAcross || !kQAcross) {
      if ((index + 1) * 64 > contr) {
        const bool off = index * 64 + along_c >= contr;
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
          if (!(i < kPLoads ? kPAcross : kQAcross)) {
            if (off) offset[i] = kNothing;
            if constexpr (kPFar && !kPAcross)
              if (i < kPLoads && off) far_on[i] = false;
          }
      }
    }
  };
  auto stage = [&](int i, char *buffer, uint32_t index,
                   uint32_t (&slot)[kSlots]) __attribute__((always_inline)) {
    const bool is_p = i < kPLoads;
    const int piece = (is_p ? i : i - kPLoads) * kWaves + wave;
    char *to = buffer + (is_p ? 0 : kPBytes) + piece * 1024;
    uint32_t at = offset[i], row = 0;
    bool on = true;
    if constexpr (kBySlot) {
      const int j = is_p ? i : i - kPLoads;
      row = slot[j];
      on = row < a.n &&
           index * 64 + (j * kWaves + wave) * kPRow + lane / (TM / 8) < contr;
      if (!is_p) row = divided(row, a.q_div);  // dz has a row for every slot
    }
    if (is_p ? kPFar : kQFar) {
      const char *from;
      if constexpr (kBySlot) {
        from = (is_p ? p_base + (int64_t)row * p_bytes : q_base + (int64_t)row * q_bytes) + at;
        on = on && (is_p ? row0 * 2 + at < (uint32_t)a.p_width * 2
                         : col0 * 2 + at < (uint32_t)a.q_width * 2);
      } else {
        from = far[kPFar ? i : 0] + (uint64_t)index * 128;
        on = far_on[kPFar ? i : 0];
      }
      asm("" : "+v"(from));  // computed for every lane: a select, not a branch
      to_lds(on ? from : zeros, to);
    } else {
      if constexpr (kBySlot) {
        at += row * (uint32_t)(is_p ? p_bytes : q_bytes);
        asm("" : "+v"(at));
        at = on ? at : kNothing;
      }
      const uint32_t moved = index * (uint32_t)(is_p ? p_step : q_step);
      if (!is_p && kQMoves) {
        const int64_t gone = (int64_t)index * q_step;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(
            window(q_base + gone, q_size - gone),
            (__attribute__((address_space(3))) void *)to, 16, (int)at, 0, 0, 0);
      } else {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(
            is_p ? p_all : q_all, (__attribute__((address_space(3))) void *)to, 16, (int)at,
            (int)moved, 0, 0);
      }
    }
  };

  // fragments of 32 rows or columns by 16 contraction values: this lane's LDS offsets
  const int wm = wave / WN * (TM / 2), wn = wave % WN * (TN / 2);
  const int fr = lane & 31, fk = lane >> 5;  // row or column, contraction half
  auto along_at = [&](int first, int k16) {  // first: multiple of 32
    return (first + fr) * 128 + (((k16 * 2 + fk) ^ along_swizzle(fr)) << 4);
  };
  auto across_at = [&](auto columns, int first, int k16) {
    constexpr int kColumns = columns.value, row_bytes = kColumns * 2;
    const int r = fk * 8 + ((lane & 15) >> 2);
    const int c = first / 8 + ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
    return (k16 * 16 + r) * row_bytes + ((c ^ across_swizzle<kColumns>(r)) << 4) + (lane & 1) * 8;
  };
  // fragment j of a half: the P and Q fragments of its first 16 values, then the second's
  constexpr int kFrags = 2 * (FM + FN);
  auto read = [&](int j, const char *buffer, int half,
                  F (&to)[kFrags]) __attribute__((always_inline)) {
    const char *lp = buffer, *lq = buffer + kPBytes;
    const int k16 = half * 2 + j / (FM + FN), f = j % (FM + FN);
    if (f < FM) {
      if constexpr (kPAcross) to[j] = across_frag<T, TM * 2>(lp + across_at(std::integral_constant<int, TM>(), wm + f * 32, k16));
      else to[j] = *(const F *)(lp + along_at(wm + f * 32, k16));
    } else {
      const int first = wn + (f - FM) * 32;
      if constexpr (kQAcross) to[j] = across_frag<T, TN * 2>(lq + across_at(std::integral_constant<int, TN>(), first, k16));
      else to[j] = *(const F *)(lq + along_at(first, k16));
    }
  };

  float16v acc[FM][FN] = {};
  // A half's MFMAs with, between them, the reads of the next half's fragments (early: the
  // last must be there when this half ends) and pieces of a coming step: its first ones in
  // a second half, the others in the first half that follows.
  constexpr int kMfmas = 2 * FM * FN;
  constexpr int kReadSlots = kMfmas > 2 ? kMfmas * 3 / 4 : 1;
  constexpr int kStageSlots = kRing == 2 ? kMfmas * 3 / 2 : kMfmas;
  auto run_half = [&](auto half, F (&now)[kFrags], F (&next)[kFrags], const char *from, char *to,
                      uint32_t index, uint32_t (&slot)[kSlots]) __attribute__((always_inline)) {
    constexpr int kPast = half.value ? 0 : kMfmas;
#pragma unroll
    for (int m = 0; m < kMfmas; ++m) {
      const int k = m / (FM * FN), fm = m / FN % FM, fn = m % FN;
      acc[fm][fn] = Frag<T>::mfma(now[k * (FM + FN) + FM + fn], now[k * (FM + FN) + fm],
                                  acc[fm][fn]);
#pragma unroll
      for (int j = m * kFrags / kReadSlots; j < (m + 1) * kFrags / kReadSlots; ++j)
        if (j < kFrags) read(j, from, 1 - half.value, next);
#pragma unroll
      for (int i = (m + kPast) * kLoads / kStageSlots; i < (m + kPast + 1) * kLoads / kStageSlots;
           ++i)
        if (i < kLoads) stage(i, to, index, slot);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  constexpr int kEarly = kMfmas * kLoads / kStageSlots;  // pieces staged in a second half

  if (steps > 0) {
    F first[kFrags], second[kFrags];  // fragments of a step's halves
    char *const ring[4] = {lds0, lds1, kRing > 2 ? lds2 : lds0, kRing > 2 ? lds3 : lds1};
    uint32_t slot[kRing][kSlots];  // by step % kRing
    // the ring's pieces, but for those that the first step's halves stage
#pragma unroll
    for (int b = 0; b < kRing; ++b) {
      read_slots(slot[b], b);
      open_step(b);
#pragma unroll
      for (int i = 0; i < (kRing == 2 && b == 1 ? kEarly : kLoads); ++i)
        stage(i, ring[b], b, slot[b]);
    }
    read_slots(slot[0], kRing);
    if (kRing == 4) read_slots(slot[1], 5);
    constexpr int kYounger = kRing == 2 ? 0 : 2 * kLoads;  // pieces of later steps
    staged_barrier<kRing == 2 ? kEarly : 3 * kLoads>();
#pragma unroll
    for (int j = 0; j < kFrags; ++j) read(j, lds0, 0, first);
    // index % kRing == at
    auto run_step = [&](auto where, uint32_t index) __attribute__((always_inline)) {
      constexpr int at = where.value;
      char *own = ring[at], *other = ring[(at + 1) % 4];
      run_half(std::integral_constant<int, 0>(), first, second, own, other, index + 1,
               slot[(at + 1) % kRing]);
      staged_barrier<kYounger>();
      read_slots(slot[(at + kRing + kRing / 2) % kRing], index + kRing + kRing / 2);
      open_step(index + kRing);
      run_half(std::integral_constant<int, 1>(), second, first, other, own, index + kRing,
               slot[at]);
    };
    // Several steps at a time, past the last one with zeros: with a second way out the
    // compiler keeps the accumulators in scratch.
    for (uint32_t index = 0; index < steps; index += kRing) {
      run_step(std::integral_constant<int, 0>(), index);
      run_step(std::integral_constant<int, 1>(), index + 1);
      if constexpr (kRing == 4) {
        run_step(std::integral_constant<int, 2>(), index + 2);
        run_step(std::integral_constant<int, 3>(), index + 3);
      }
    }
    staged_barrier<0>();
  }

  // Out: a lane holds out row wm + fm * 32 + fr, columns wn + fn * 32 + j * 8 + fk * 4
  // + 0..3.  Two row fragments at a time go through LDS (the wave's part of one buffer
  // each) and leave as whole rows; piece c of four columns of row r lies at c ^ (r & 15)
  // (of 8 pieces a row: & 7), against bank conflicts.
  constexpr int kCols = TN / 2, kTurn = kCols / 4 < 16 ? kCols / 4 - 1 : 15;
  constexpr int kPair = FM < 2 ? FM : 2;
  static_assert(4 * 32 * kCols * 4 <= kBuffer, "");
#pragma unroll
  for (int pair = 0; pair < FM; pair += kPair) {
    const int first = wm + pair * 32;
    uint32_t own_slot = 0;  // of row `lane` of the fragments
    if constexpr (PRODUCT != kWeight) own_slot = slot_at(begin + first + lane % (kPair * 32));
#pragma unroll
    for (int f = 0; f < kPair; ++f)
#pragma unroll
      for (int fn = 0; fn < FN; ++fn)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float16v v = acc[pair + f][fn];
          const float4v part = {v[j * 4], v[j * 4 + 1], v[j * 4 + 2], v[j * 4 + 3]};
          float *patch = (float *)(f == 0 ? lds0 : lds1) + wave * 32 * kCols;
          *(float4v *)(patch + fr * kCols + ((fn * 8 + j * 2 + fk) ^ (fr & kTurn)) * 4) = part;
        }
    wave_shares();
    auto leave = [&](auto run) __attribute__((always_inline)) {
      constexpr int V = run.value;         // columns a lane takes: 16 bytes of them
      constexpr int kLanes = kCols / V, kRowsAtOnce = 64 / kLanes;
      constexpr int kTurns = kPair * 32 / kRowsAtOnce, kBatch = 2;
      const int piece = lane % kLanes * (V / 4);
      // A short loop: its code comes from memory once a tile (all of it unrolled: 213 us
      // became 236 at 8192 x 4096 x 4096).
#pragma unroll 1
      for (int i = 0; i < kTurns; i += kBatch) {
        float v[kBatch][V];
        uint32_t slot[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
          const int r = (i + u) * kRowsAtOnce + lane / kLanes;
          slot[u] = PRODUCT == kWeight ? 0 : __shfl(own_slot, r);
          const float *patch = (float *)(r < 32 ? lds0 : lds1) + (wave * 32 + r % 32) * kCols;
#pragma unroll
          for (int h = 0; h < V / 4; ++h) {
            const float4v q = *(const float4v *)(patch + ((piece + h) ^ (r & kTurn)) * 4);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[u][h * 4 + j] = q[j];
          }
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
          const int64_t out_row =
              PRODUCT == kWeight ? row0 + first + (i + u) * kRowsAtOnce + lane / kLanes : slot[u];
          if (PRODUCT == kWeight ? out_row < a.rows : slot[u] != NTC_PAD) {
            if constexpr (PRODUCT == kInput)
              if (a.written && col0 + wn == 0 && piece == 0) a.written[slot[u]] = 0;
            finish_some<T, PRODUCT, V>(a, expert, out_row, col0 + wn + piece * 4, v[u]);
          }
        }
      }
    };
    if (a.out_f32) leave(std::integral_constant<int, 4>());
    else leave(std::integral_constant<int, 8>());
    wave_shares();
  }
#endif
}

}  // namespace ntc
