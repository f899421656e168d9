// ntc_linear_few.h -- linear layers of few rows: every weight is read once, straight from
// memory into MFMA operands.
#pragma once

#include "ntc_linear_tile.h"

namespace ntc {

typedef float float4x __attribute__((ext_vector_type(4)));

template <class T> struct Small;
template <> struct Small<_Float16> {
  static __device__ __forceinline__ float4x mfma(half8 a, half8 b, float4x c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
  }
};
template <> struct Small<__bf16> {
  static __device__ __forceinline__ float4x mfma(bf16x8 a, bf16x8 b, float4x c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
};

// A workgroup takes an expert's (blockIdx.y) 16 output columns (blockIdx.x) and its slots,
// 16 at a time.  Its waves share the contraction: wave w multiplies the blocks of 64
// values w, w + 8, ... (whole 128-byte lines of every weight row), and the partial sums
// meet in LDS, added in order.  Bound by the weights' bytes: with 8 waves of up to 16
// weight loads each a workgroup has 128 KB on their way (4096 x 4096, one row: 9.0 us from
// memory, 3.7 TB/s; 7.6 from the last-level cache).
constexpr int kFewWaves = 8;

template <class T>
__global__ __launch_bounds__(kFewWaves * 64) void few_rows(TileArgs a) {
  typedef typename Frag<T>::type F;
  __shared__ __align__(16) float part[kFewWaves][16][16];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int lr = lane & 15, lk = (lane >> 4) * 8;
  const int expert = blockIdx.y;
  const int col0 = blockIdx.x * 16;
  uint32_t begin = 0, end = a.n;
  if (a.perm) {
    begin = min(a.bin_offset[expert], a.perm_capacity);
    end = min(a.bin_offset[expert + 1], a.perm_capacity);
  }
  // columns that don't exist read the last one's weights
  const T *w_at = (const T *)a.q + (int64_t)expert * a.q_expert +
                  (int64_t)min(col0 + lr, a.cols - 1) * a.q_stride + lk;
  auto slot_at = [&](uint32_t pos) -> uint32_t {
    if (pos >= end) return NTC_PAD;
    const uint32_t s = a.perm ? a.perm[pos] : pos;
    return s < a.n ? s : NTC_PAD;
  };
  const int full = a.contr / 64;
  const int count = full > wave ? (full - 1 - wave) / kFewWaves + 1 : 0;

  for (uint32_t pos = begin; pos < end; pos += 16) {
    if (a.perm && a.perm[pos] == NTC_PAD) break;  // the bin's end is padding
    // slots that don't exist read the first row
    const uint32_t slot = slot_at(pos + lr);
    const T *x_at = (const T *)a.p +
                    (slot == NTC_PAD ? 0 : (int64_t)divided(slot, a.p_div) * a.p_stride) + lk;
    float4x acc = {};
    // `blocks` of this wave's whole blocks from the i-th on, all loads on their way before
    // the first product waits
    auto some = [&](auto blocks, int i) {
      constexpr int kBlocks = blocks.value;
      F wf[kBlocks][2], xf[kBlocks][2];
#pragma unroll
      for (int u = 0; u < kBlocks; ++u)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int k = (wave + (i + u) * kFewWaves) * 64 + h * 32;
          wf[u][h] = *(const F *)(w_at + k);
          xf[u][h] = *(const F *)(x_at + k);
        }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int u = 0; u < kBlocks; ++u)
#pragma unroll
        for (int h = 0; h < 2; ++h) acc = Small<T>::mfma(wf[u][h], xf[u][h], acc);
      __builtin_amdgcn_sched_barrier(0);
    };
    int i = 0;
#pragma unroll 1
    for (; i + 8 <= count; i += 8) some(std::integral_constant<int, 8>(), i);
    if (i + 4 <= count) some(std::integral_constant<int, 4>(), i), i += 4;
    if (i + 2 <= count) some(std::integral_constant<int, 2>(), i), i += 2;
    if (i < count) some(std::integral_constant<int, 1>(), i);
    if (a.contr % 64 && full % kFewWaves == wave) {  // the last, partial block
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int k = full * 64 + h * 32;
        const bool on = k + lk < a.contr;
        const F w = on ? *(const F *)(w_at + k) : F{};
        const F x = on ? *(const F *)(x_at + k) : F{};
        acc = Small<T>::mfma(w, x, acc);
      }
    }

    // lane: columns (lane >> 4) * 4 + 0..3 of row lr
    *(float4x *)&part[wave][lr][(lane >> 4) * 4] = acc;
    __syncthreads();
    if (threadIdx.x < 32) {
      const int r = threadIdx.x / 2, c = threadIdx.x % 2 * 8;
      const uint32_t s = slot_at(pos + r);
      if (s != NTC_PAD && col0 + c < a.cols) {
        float sum[8] = {};
#pragma unroll
        for (int w = 0; w < kFewWaves; ++w)
#pragma unroll
          for (int j = 0; j < 8; ++j) sum[j] += part[w][r][c + j];
        finish_some<T, kForward, 8>(a, expert, s, col0 + c, sum);
      }
    }
    __syncthreads();
  }
}

}  // namespace ntc
