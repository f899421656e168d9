// ntc_linear.hip -- linear layers over bins: operand layout, tiled products, gradients.
#include <initializer_list>

#include "ntc_linear_few.h"
#include "ntc_linear_tile.h"

namespace ntc {
namespace {

// ------------------------------------------------------------------ layout

int64_t round8(int64_t v) { return (v + 7) / 8 * 8; }
bool on16(const void *p) { return ((uintptr_t)p & 15) == 0; }
Divisor divisor(int32_t d) {
  uint32_t shift = 0;
  while ((1ll << shift) < d) ++shift;
  return {(uint32_t)(((1ull << (31 + shift)) + (uint32_t)d - 1) / (uint32_t)d), shift};
}
size_t round16(size_t v) { return (v + 15) / 16 * 16; }
int64_t item_rows(const ntc_linear_rows &r) {
  return (r.n + r.slots_per_row - 1) / r.slots_per_row;
}

// A workspace handed out from its start.
struct Space {
  char *base;
  size_t used = 0;
  void *take(size_t bytes) {
    void *p = base ? base + used : nullptr;
    used += round16(bytes);
    return p;
  }
};

// Eight values from `from`, those at and past `count` 0.
template <class T>
__device__ __forceinline__ void load8(const T *from, int count, bool wide, float (&to)[8]) {
  constexpr int kRun = 16 / sizeof(T);
  if (count >= 8) {
#pragma unroll
    for (int h = 0; h < 8 / kRun; ++h) {
      Run<T, kRun, false> r;
      if (wide) {
        const Run<T, kRun, true> w = *(const Run<T, kRun, true> *)(from + h * kRun);
#pragma unroll
        for (int j = 0; j < kRun; ++j) r.v[j] = w.v[j];
      } else {
        r = *(const Run<T, kRun, false> *)(from + h * kRun);
      }
#pragma unroll
      for (int j = 0; j < kRun; ++j) to[h * kRun + j] = (float)r.v[j];
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) to[j] = j < count ? (float)from[j] : 0.f;
  }
}

// rows x dim values to rows of round8(dim), the pad zero; a wave per row.
template <class T>
__global__ __launch_bounds__(kBlock) void lay_out(const T *from, int64_t stride, int64_t rows,
                                                  int32_t dim, bool wide, T *to) {
  const int64_t pitch = (dim + 7) / 8 * 8;
  for (int64_t row = (int64_t)blockIdx.x * kWavesPerBlock + threadIdx.x / 64; row < rows;
       row += (int64_t)gridDim.x * kWavesPerBlock)
    for (int32_t c = (threadIdx.x & 63) * 8; c < dim; c += 512) {
      float v[8];
      load8(from + row * stride + c, dim - c, wide, v);
      Run<T, 8, true> o;
#pragma unroll
      for (int j = 0; j < 8; ++j) o.v[j] = (T)v[j];
      *(Run<T, 8, true> *)(to + row * pitch + c) = o;
    }
}

// ---------------------------------------------------------------- gradients

__global__ __launch_bounds__(kBlock) void fill_u32(uint32_t *to, int64_t n, uint32_t value) {
  for (int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x; i < n;
       i += (int64_t)gridDim.x * kBlock)
    to[i] = value;
}

// dx[t] = sum over t's slots of their float32 parts, rounded once, where they were
// written; a wave per row, 16 bytes of a part a lane.  Bound by the parts' bytes.
template <class T>
__global__ __launch_bounds__(kBlock) void sum_parts(const float *parts, int64_t pitch,
                                                    const uint32_t *written, int64_t rows,
                                                    int32_t each, int64_t n, int32_t dim, T *dx,
                                                    int64_t stride) {
  for (int64_t t = (int64_t)blockIdx.x * kWavesPerBlock + threadIdx.x / 64; t < rows;
       t += (int64_t)gridDim.x * kWavesPerBlock)
    for (int32_t c = (threadIdx.x & 63) * 4; c < dim; c += 256) {
      float4v sum = {};
      const int32_t slots = (int32_t)min((int64_t)each, n - t * each);  // the last row's: fewer
#pragma unroll 4
      for (int32_t j = 0; j < slots; ++j)
        if (written[t * each + j] == 0) sum += *(const float4v *)(parts + (t * each + j) * pitch + c);
      T *to = dx + t * stride + c;
      if (c + 4 <= dim) {
        Run<T, 4, false> o;
#pragma unroll
        for (int j = 0; j < 4; ++j) o.v[j] = (T)sum[j];
        *(Run<T, 4, false> *)to = o;
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (c + j < dim) to[j] = (T)sum[j];
      }
    }
}

// Rows that no slot's product wrote become 0; a wave per row.
template <class T>
__global__ __launch_bounds__(kBlock) void clear_rows(const uint32_t *written, int64_t n, T *dx,
                                                     int64_t stride, int32_t dim) {
  const int lane = threadIdx.x & 63;
  for (int64_t s = (int64_t)blockIdx.x * kWavesPerBlock + threadIdx.x / 64; s < n;
       s += (int64_t)gridDim.x * kWavesPerBlock)
    if (written[s])
      for (int32_t c = lane; c < dim; c += 64) dx[s * stride + c] = (T)0.f;
}

// dz and the bias's gradient in one pass over dy: tiles of 64 slots of one expert and 512
// columns, a workgroup's four waves every fourth slot, 16 bytes a lane, two rows on
// their way.  dz = dy * act'(pre) is rounded to T (its one rounding: the products take
// 16-bit operands) and goes to rows of round8(dim), the pad zero; slots in no bin have
// none.  parts[tile][c] = sum of the tile's dz[s][c] before that rounding; bias_join adds
// an expert's tiles in order, without atomics.  Bound by the bytes of dy, pre and dz.
constexpr int kBiasLog = 6, kBiasTile = 1 << kBiasLog, kRowsAhead = 2;

struct GradArgs {
  const void *dy, *pre;
  int64_t dy_stride, pre_stride;
  int32_t activation;
  float slope;
  bool wide;    // rows start on 16 bytes
  void *dz;     // NULL: dz is dy
  float *parts; // NULL: not wanted
};

template <class T, class D>
__global__ __launch_bounds__(kBlock) void through_activation(TileArgs a, GradArgs g) {
  __shared__ uint32_t scratch[kWavesPerBlock];
  __shared__ TileSpot spot;
  __shared__ float sums[kWavesPerBlock][512];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t tile = blockIdx.x;
  uint32_t begin = tile * kBiasTile, end = a.n;
  if (a.perm) {
    uint32_t before, mine;
    if (tile >= count_tiles<kBlock>(a, kBiasLog, scratch, before, mine)) return;
    find_tile<kBlock>(a, kBiasLog, tile, before, mine, &spot);
    begin = spot.begin;
    end = spot.end;
  }
  end = min(end, begin + kBiasTile);
  const int c = (blockIdx.y * 64 + lane) * 8;
  const int64_t pitch = (a.rows + 7) / 8 * 8;
  float sum[8] = {};
  // this wave's slots: begin + wave + 4 r, lane r reads the r-th
  const uint32_t own = begin + wave + lane * kWavesPerBlock;
  const uint32_t slots = own < end ? (a.perm ? a.perm[own] : own) : NTC_PAD;
  for (int r = 0; r < kBiasTile / kWavesPerBlock; r += kRowsAhead) {
    float d[kRowsAhead][8], z[kRowsAhead][8];
#pragma unroll
    for (int u = 0; u < kRowsAhead; ++u) {
      const uint32_t s = read_lane(slots, r + u);
#pragma unroll
      for (int j = 0; j < 8; ++j) d[u][j] = 0.f;
      if (s < a.n && c < a.rows) {
        load8((const D *)g.dy + (int64_t)s * g.dy_stride + c, a.rows - c, g.wide, d[u]);
        if (g.activation != NTC_ACT_NONE)
          load8((const T *)g.pre + (int64_t)s * g.pre_stride + c, a.rows - c, g.wide, z[u]);
      }
    }
#pragma unroll
    for (int u = 0; u < kRowsAhead; ++u) {
      const uint32_t s = read_lane(slots, r + u);
      if (s < a.n && c < a.rows) {
        Run<T, 8, true> o;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (g.activation != NTC_ACT_NONE)
            d[u][j] *= activation_slope(z[u][j], g.activation, g.slope);
          o.v[j] = c + j < a.rows ? (T)d[u][j] : (T)0.f;
          sum[j] += d[u][j];  // 0 past the last column
        }
        if (g.dz) *(Run<T, 8, true> *)((T *)g.dz + (int64_t)s * pitch + c) = o;
      }
    }
  }
  if (!g.parts) return;
#pragma unroll
  for (int j = 0; j < 8; ++j) sums[wave][lane * 8 + j] = sum[j];
  __syncthreads();
  for (int i = threadIdx.x; i < 512; i += kBlock) {
    const int col = blockIdx.y * 512 + i;
    if (col < a.rows)
      g.parts[(int64_t)tile * a.rows + col] =
          (sums[0][i] + sums[1][i]) + (sums[2][i] + sums[3][i]);
  }
}

// there: the tiles that have parts; only bins that overlap would have more.
template <class T>
__global__ __launch_bounds__(kBlock) void bias_join(TileArgs a, const float *parts,
                                                    uint32_t there) {
  __shared__ uint32_t first;
  const int expert = blockIdx.y;
  uint32_t tiles = (a.n + kBiasTile - 1) / kBiasTile;
  if (threadIdx.x == 0) first = 0;
  __syncthreads();
  if (a.perm) {
    auto tiles_of = [&](int e) -> uint32_t {
      const uint32_t lo = min(a.bin_offset[e], a.perm_capacity);
      const uint32_t hi = min(a.bin_offset[e + 1], a.perm_capacity);
      return hi > lo ? (hi - lo + kBiasTile - 1) / kBiasTile : 0;
    };
    uint32_t before = 0;
    for (int e = threadIdx.x; e < expert; e += kBlock) before += tiles_of(e);
    if (before) atomicAdd(&first, before);  // whole numbers: any order
    tiles = tiles_of(expert);
  }
  __syncthreads();
  tiles = min(tiles, there - min(first, there));
  const int col = blockIdx.x * kBlock + threadIdx.x;
  if (col >= a.rows) return;
  const float *from = parts + (int64_t)first * a.rows + col;
  float sum = 0.f;
#pragma unroll 8
  for (uint32_t t = 0; t < tiles; ++t) sum += from[(int64_t)t * a.rows];
  const int64_t at = (int64_t)expert * a.rows + col;
  if (a.out_f32) ((float *)a.out)[at] = sum;
  else ((T *)a.out)[at] = (T)sum;
}

int64_t bias_tiles(const ntc_linear_layer &l, const ntc_linear_rows &r) {
  return (r.perm ? r.perm_capacity / kBiasTile + l.n_experts
                 : (r.n + kBiasTile - 1) / kBiasTile);
}

// ------------------------------------------------------------------- launches

uint32_t stride_grid(int64_t items, int per_block) {
  const int64_t blocks = (items + per_block - 1) / per_block;
  return (uint32_t)(blocks < 16384 ? blocks : 16384);
}

template <class T>
void lay_out_rows(const void *from, int64_t stride, int64_t rows, int32_t dim, void *to,
                  hipStream_t stream) {
  lay_out<T><<<stride_grid(rows, kWavesPerBlock), kBlock, 0, stream>>>(
      (const T *)from, stride, rows, dim, on16(from) && stride % 8 == 0, (T *)to);
}

// Rows take 8 elements at a time.
bool vec8(const void *p, int64_t stride, int bytes) {
  return !p || (((uintptr_t)p & (8 * bytes - 1)) == 0 && stride % 8 == 0);
}

void set_bins(TileArgs &t, const ntc_linear_layer &l, const ntc_linear_rows &r) {
  t.bin_offset = r.bin_offset;
  t.perm = r.perm;
  t.perm_capacity = (uint32_t)r.perm_capacity;
  t.n_experts = l.n_experts;
  t.n = (uint32_t)r.n;
  t.p_div = t.q_div = divisor(1);
}

// The operand's bytes reach past what a 32-bit offset does, counting up to four steps of 64
// rows past its end, which are asked for and read as 0.
bool far(int64_t rows, int64_t stride, int32_t width) {
  return (rows + 255) * stride * 2 + (int64_t)width * 2 >= 0xFFFFFFF0LL;
}

// How a product is launched.
struct Plan {
  Access access;
  int side;        // of a tile
  int rest;        // side of the tiles that the last, partly filled round is cut into, or 0
  int64_t blocks;
};
constexpr int64_t kMaxBlocks = 0xffffff;  // of 256 threads: 2^32 in a launch

Plan plan(Product product, const TileArgs &t) {
  const bool gather = t.perm || t.p_div.shift || t.q_div.shift;
  auto launched = [&](int64_t side) -> int64_t {
    const int64_t cols = (t.cols + side - 1) / side;
    if (product == kWeight)
      return ((t.rows + side - 1) / side * cols + 7) / 8 * 8 * t.n_experts;
    return (t.perm ? t.perm_capacity / side + t.n_experts : (t.n + side - 1) / side) * cols;
  };
  // offsets reach over a tile's rows, or over the whole operand
  const bool whole_p = gather || product == kWeight, whole_q = product != kForward;
  if ((whole_p && far(t.p_rows, t.p_stride, t.p_width)) ||
      (whole_q && far(t.q_rows, t.q_stride, t.q_width)))
    return {kFar, 128, 0, launched(128)};
  // The tile by what it costs on 256 CUs, in 128 x 128 tiles' worth of MFMA time: a 256
  // tile fills a CU, two 128 tiles share one at less of its rate (kernels alone, us with
  // 256 and 128, 8192 x 4096 x 4096: forward 211 and 240, input gradient 208 and 240, weight
  // gradient 197 and 232; forward of 32768 slots, 64 experts, 2048 to 1024: 190, its rest
  // among them, and 196), 64 tiles come to about half.  Small outputs take the smaller tile
  // that still gives every CU one.
  auto tiles = [&](int64_t side) -> int64_t {
    const int64_t half = (t.n_experts < (int64_t)t.n ? t.n_experts : (int64_t)t.n) / 2 + 1;
    const int64_t rows = product == kWeight ? ((t.rows + side - 1) / side) * t.n_experts
                         : t.perm           ? t.n / side + half
                                            : (t.n + side - 1) / side;
    return rows * ((t.cols + side - 1) / side);
  };
  auto rounds = [](int64_t count, int64_t at_once) { return (count + at_once - 1) / at_once; };
  const double pair = product == kForward && !gather ? 2.24 : 2.6;
  // A last round of 256 tiles at most half full is a launch of smaller tiles, where a round
  // outlasts a launch (10240 x 2048 outputs, us with it and without: contraction 1024
  // 53 and 51, 1536 70 and 70, 2048 87 and 88, 4096 151 and 161; 9000 slots of 4 experts,
  // 4096: 154 and 166).  Up to 48 tiles are cut into 64 x 64, more into 128 x 128 (contraction
  // 4096, us with either: 8 tiles 122 and 146, 48 148 and 155, 64 159 and 157, 128 207 and
  // 171); how many there are only the GPU knows with bins: 128 x 128 then.
  const int64_t over = tiles(256) % 256;
  const bool rest = product != kWeight && tiles(256) > 256 && t.contr >= 1536 &&
                    (t.perm || (over > 0 && over <= 128));
  const bool small = !t.perm && over <= 48;
  const double last = over == 0             ? 0
                      : !rest || over > 128 ? 4.0
                      : small               ? 0.5 * rounds(over * 16, 256)
                      : over <= 64          ? 1.4
                                            : pair;
  const double cost256 = 4.0 * (tiles(256) / 256) + last;
  const double cost128 = tiles(128) <= 256 ? 1.4 : pair * rounds(tiles(128), 512);
  const double cost64 = tiles(64) <= 256 ? 0.5 : 0.5 * rounds(tiles(64), 256);
  int side = cost64 < cost128 && cost64 < cost256 ? 64 : cost128 < cost256 ? 128 : 256;
  while (side < 256 && launched(side) > kMaxBlocks) side *= 2;
  return {gather ? kGather : kDense, side, !rest || side < 256 ? 0 : small ? 64 : 128,
          launched(side)};
}

template <class T, Product PRODUCT, Access ACCESS>
void start_tiles(TileArgs t, const Plan &p, hipStream_t stream) {
  const uint32_t blocks = (uint32_t)p.blocks;
  if (ACCESS == kFar || p.side == 128) {
    tile_product<T, PRODUCT, ACCESS, 128, 128><<<blocks, 256, 0, stream>>>(t);
    return;
  }
  if constexpr (ACCESS != kFar) {
    if (p.side == 64) {
      tile_product<T, PRODUCT, ACCESS, 64, 64><<<blocks, 256, 0, stream>>>(t);
      return;
    }
    if (p.rest) t.part = kWhole;
    tile_product<T, PRODUCT, ACCESS, 256, 256><<<blocks, 256, 0, stream>>>(t);
    t.part = kRest;
    if (p.rest == 64)  // 16 for each of up to 48
      tile_product<T, PRODUCT, ACCESS, 64, 64><<<768, 256, 0, stream>>>(t);
    else if (p.rest == 128)  // 4 for each of up to 128
      tile_product<T, PRODUCT, ACCESS, 128, 128><<<512, 256, 0, stream>>>(t);
  }
}

template <class T, Product PRODUCT>
void start_product(const TileArgs &t, hipStream_t stream) {
  const Plan p = plan(PRODUCT, t);
  if (p.access == kFar) start_tiles<T, PRODUCT, kFar>(t, p, stream);
  else if (p.access == kGather) start_tiles<T, PRODUCT, kGather>(t, p, stream);
  else start_tiles<T, PRODUCT, kDense>(t, p, stream);
}

// At most 16 rows an expert and tiles of 64 columns for less than half of the CUs: the
// contraction is what there is to share (4096 x 4096, weights in the last-level cache, us
// here and by 64 tiles: one row 7.6 and 13.3, 16 rows 10.2 and 13.4, 17 rows in two passes
// 11.5 and 13.7; 8192 x 4096, one row: 15.6 and 13.7.  Weights from memory: 9.0 and 18.9,
// 11.0 and 19.2, 16.6 and 19.4; 15.6 and 20.1).
bool few(const TileArgs &t) {
  const int64_t experts = t.n < (uint32_t)t.n_experts ? t.n : t.n_experts;
  return t.n <= 16 * experts && (t.cols + 63) / 64 * experts < 128;
}

template <class T>
void start_few(const TileArgs &t, hipStream_t stream) {
  const dim3 grid((uint32_t)((t.cols + 15) / 16), (uint32_t)t.n_experts);
  few_rows<T><<<grid, kFewWaves * 64, 0, stream>>>(t);
}

// Rows that don't start on 16 bytes, or lie so far apart that 256 of them leave the reach
// of a 32-bit offset, are laid out anew.
constexpr int64_t kMaxStride = 1 << 22;

bool lay_x(const ntc_linear_layer &l, const ntc_linear_rows &r) {
  return !on16(r.x) || r.x_stride % 8 || l.in_dim % 8 || r.x_stride > kMaxStride;
}
bool lay_weight(const ntc_linear_layer &l) { return !on16(l.weight) || l.in_dim % 8; }

// Layers whose launches don't fit are refused before anything is enqueued.
int fits(std::initializer_list<int64_t> blocks) {
  for (int64_t b : blocks)
    if (b > kMaxBlocks) return NTC_ERR_UNSUPPORTED;
  return NTC_OK;
}

template <class T>
int forward(const ntc_linear_layer &l, const ntc_linear_rows &r, const ntc_linear_epilogue &ep,
            void *y, int64_t y_stride, void *workspace, hipStream_t stream) {
  Space space{(char *)workspace};
  const int64_t in8 = round8(l.in_dim), xrows = item_rows(r);
  const int64_t wrows = (int64_t)l.n_experts * l.out_dim;
  void *x8 = lay_x(l, r) ? space.take(xrows * in8 * sizeof(T)) : nullptr;
  void *w8 = lay_weight(l) ? space.take(wrows * in8 * sizeof(T)) : nullptr;
  TileArgs t = {};
  set_bins(t, l, r);
  t.p = x8 ? x8 : r.x;
  t.p_stride = x8 ? in8 : r.x_stride;
  t.q = w8 ? w8 : l.weight;
  t.q_stride = in8;
  t.q_expert = in8 * l.out_dim;
  t.p_div = divisor(r.slots_per_row);
  t.cols = l.out_dim;
  t.contr = (int32_t)in8;
  t.p_rows = xrows;
  t.q_rows = l.out_dim;
  t.p_width = t.q_width = (int32_t)in8;
  t.out = y;
  t.out_stride = y_stride;
  t.out_f32 = ep.output_format == NTC_OUT_F32;
  t.bias = l.bias;
  t.activation = ep.activation;
  t.slope = ep.leaky_slope;
  t.residual = ep.residual;
  t.residual_stride = ep.residual_stride;
  t.pre = ep.pre;
  t.pre_stride = ep.pre_stride;
  const int to = type_bytes(ep.output_format);
  t.vec = l.out_dim % 8 == 0 && vec8(y, y_stride, to) && vec8(ep.residual, ep.residual_stride, to) &&
          vec8(ep.pre, ep.pre_stride, 2) && vec8(l.bias, 0, 2);
  if (!few(t)) {
    const int st = fits({plan(kForward, t).blocks});
    if (st != NTC_OK) return st;
  }
  if (x8) lay_out_rows<T>(r.x, r.x_stride, xrows, l.in_dim, x8, stream);
  if (w8) lay_out_rows<T>(l.weight, l.in_dim, wrows, l.in_dim, w8, stream);
  if (few(t)) start_few<T>(t, stream);
  else start_product<T, kForward>(t, stream);
  return hip_status(hipGetLastError());
}

bool needs_dz(const ntc_linear_layer &l, const ntc_linear_epilogue &ep,
              const ntc_linear_grads &g) {
  return ep.activation != NTC_ACT_NONE || g.dy_format != l.type || !on16(g.dy) ||
         g.dy_stride % 8 || l.out_dim % 8 || g.dy_stride > kMaxStride;
}

// The backward pass's workspace, handed out in this order.
struct BackwardSpace {
  void *dz, *x, *weight, *parts, *written, *bias;
  size_t bytes;
  BackwardSpace(const ntc_linear_layer &l, const ntc_linear_rows &r, const ntc_linear_epilogue &ep,
                const ntc_linear_grads &g, void *workspace) {
    Space s{(char *)workspace};
    const int64_t in8 = round8(l.in_dim), out8 = round8(l.out_dim);
    const bool any = r.n > 0;
    dz = x = weight = parts = written = bias = nullptr;
    if (any && needs_dz(l, ep, g)) dz = s.take(r.n * out8 * 2);
    if (any && g.dweight && lay_x(l, r)) x = s.take(item_rows(r) * in8 * 2);
    if (any && g.dx && lay_weight(l)) weight = s.take((int64_t)l.n_experts * l.out_dim * in8 * 2);
    // a slot's part of dx, and whether it has one
    if (any && g.dx && r.slots_per_row > 1) parts = s.take(r.n * in8 * 4);  // float32
    if (any && g.dx && (r.slots_per_row > 1 || r.perm))
      written = s.take(r.n * 4);
    if (any && g.dbias) bias = s.take(bias_tiles(l, r) * l.out_dim * 4);
    bytes = s.used;
  }
};

template <class T>
int backward(const ntc_linear_layer &l, const ntc_linear_rows &r, const ntc_linear_epilogue &ep,
             const ntc_linear_grads &g, void *workspace, hipStream_t stream) {
  const BackwardSpace ws(l, r, ep, g, workspace);
  const int64_t in8 = round8(l.in_dim), out8 = round8(l.out_dim), xrows = item_rows(r);
  const bool grad_f32 = g.grad_format == NTC_OUT_F32;
  TileArgs common = {};
  set_bins(common, l, r);
  common.p = ws.dz ? ws.dz : g.dy;
  common.p_stride = ws.dz ? out8 : g.dy_stride;
  common.p_rows = r.n;
  common.p_width = (int32_t)out8;

  TileArgs dx = common;
  dx.q = ws.weight ? ws.weight : l.weight;
  dx.q_stride = in8;
  dx.q_expert = in8 * l.out_dim;
  dx.q_rows = l.out_dim;
  dx.q_width = (int32_t)in8;
  dx.contr = (int32_t)out8;
  dx.cols = ws.parts ? (int32_t)in8 : l.in_dim;
  dx.out = ws.parts ? ws.parts : g.dx;
  dx.out_stride = ws.parts ? in8 : g.dx_stride;
  dx.out_f32 = ws.parts != nullptr;
  dx.written = (uint32_t *)ws.written;
  dx.vec = dx.cols % 8 == 0 && (ws.parts || vec8(g.dx, g.dx_stride, 2));

  TileArgs dw = common;
  dw.q = ws.x ? ws.x : r.x;
  dw.q_stride = ws.x ? in8 : r.x_stride;
  dw.q_div = divisor(r.slots_per_row);
  dw.q_rows = xrows;
  dw.q_width = (int32_t)in8;
  dw.rows = l.out_dim;
  dw.cols = l.in_dim;
  dw.out = g.dweight;
  dw.out_stride = l.in_dim;
  dw.out_expert = (int64_t)l.in_dim * l.out_dim;
  dw.out_f32 = grad_f32;
  dw.vec = l.in_dim % 8 == 0 && vec8(g.dweight, 0, grad_f32 ? 4 : 2);

  TileArgs db = common;
  db.rows = l.out_dim;
  db.out = g.dbias;
  db.out_f32 = grad_f32;
  if (r.n == 0) db.perm = nullptr;  // no tiles and no parts of them
  const dim3 parts((uint32_t)bias_tiles(l, r), (uint32_t)((l.out_dim + 511) / 512));

  const bool want_dx = g.dx && r.n > 0;
  const int st = fits({want_dx ? plan(kInput, dx).blocks : 0,
                       g.dweight ? plan(kWeight, dw).blocks : 0,
                       ws.dz || ws.bias ? bias_tiles(l, r) * parts.y : 0});
  if (st != NTC_OK) return st;

  if (ws.dz || ws.bias) {
    GradArgs ga = {g.dy, ep.pre, g.dy_stride, ep.pre_stride, ep.activation, ep.leaky_slope,
                   on16(g.dy) && g.dy_stride % 8 == 0 &&
                       (ep.activation == NTC_ACT_NONE || (on16(ep.pre) && ep.pre_stride % 8 == 0)),
                   ws.dz, (float *)ws.bias};
    if (g.dy_format == NTC_OUT_F32)
      through_activation<T, float><<<parts, kBlock, 0, stream>>>(db, ga);
    else
      through_activation<T, T><<<parts, kBlock, 0, stream>>>(db, ga);
  }
  if (want_dx) {
    if (ws.weight)
      lay_out_rows<T>(l.weight, l.in_dim, (int64_t)l.n_experts * l.out_dim, l.in_dim, ws.weight,
                      stream);
    if (ws.written)
      fill_u32<<<stride_grid(r.n, kBlock), kBlock, 0, stream>>>(dx.written, r.n, NTC_PAD);
    start_product<T, kInput>(dx, stream);
    if (ws.parts)
      sum_parts<T><<<stride_grid(xrows, kWavesPerBlock), kBlock, 0, stream>>>(
          (const float *)ws.parts, in8, dx.written, xrows, r.slots_per_row, r.n, l.in_dim,
          (T *)g.dx, g.dx_stride);
    else if (ws.written)
      clear_rows<T><<<stride_grid(r.n, kWavesPerBlock), kBlock, 0, stream>>>(
          dx.written, r.n, (T *)g.dx, g.dx_stride, l.in_dim);
  }
  if (g.dweight) {
    if (ws.x) lay_out_rows<T>(r.x, r.x_stride, xrows, l.in_dim, ws.x, stream);
    start_product<T, kWeight>(dw, stream);
  }
  if (g.dbias) {
    bias_join<T><<<dim3((uint32_t)((l.out_dim + kBlock - 1) / kBlock), (uint32_t)l.n_experts),
                   kBlock, 0, stream>>>(db, (const float *)ws.bias, parts.x);
  }
  return hip_status(hipGetLastError());
}

}  // namespace

size_t linear_workspace(const ntc_linear_layer &l, const ntc_linear_rows &r) {
  if (r.n == 0) return 0;
  Space s{nullptr};
  const int64_t in8 = round8(l.in_dim);
  if (lay_x(l, r)) s.take(item_rows(r) * in8 * 2);
  if (lay_weight(l)) s.take((int64_t)l.n_experts * l.out_dim * in8 * 2);
  return s.used;
}

int launch_linear(const ntc_linear_layer &l, const ntc_linear_rows &r,
                  const ntc_linear_epilogue &ep, void *y, int64_t y_stride, void *workspace,
                  hipStream_t stream) {
  return l.type == NTC_OUT_F16 ? forward<_Float16>(l, r, ep, y, y_stride, workspace, stream)
                               : forward<__bf16>(l, r, ep, y, y_stride, workspace, stream);
}

size_t linear_backward_workspace(const ntc_linear_layer &l, const ntc_linear_rows &r,
                                 const ntc_linear_epilogue &ep, const ntc_linear_grads &g) {
  return BackwardSpace(l, r, ep, g, nullptr).bytes;
}

int launch_linear_backward(const ntc_linear_layer &l, const ntc_linear_rows &r,
                           const ntc_linear_epilogue &ep, const ntc_linear_grads &g,
                           void *workspace, hipStream_t stream) {
  return l.type == NTC_OUT_F16 ? backward<_Float16>(l, r, ep, g, workspace, stream)
                               : backward<__bf16>(l, r, ep, g, workspace, stream);
}

}  // namespace ntc
