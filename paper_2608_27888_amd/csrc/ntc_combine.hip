// ntc_combine.hip -- an item's k expert rows brought together, and the gradient.
#include "ntc_experts.h"

namespace ntc {
namespace {

// V values of T as one access of V * sizeof(T) bytes.
template <class T, int V>
struct alignas(sizeof(T) * V) Pack {
  T v[V];
};

__device__ __forceinline__ bool used(const uint32_t *ids, int64_t slot, uint32_t n_experts) {
  return !ids || ids[slot] < n_experts;
}

// A thread per V columns of an item.  Bound by bytes where rows take 16 at a time (8192 x 8
// rows of 2048 bf16 and a residual: 65 us, 5.2 TB/s); other widths and strides go element
// by element (rows of 2047: 223 us, 1.4 TB/s).
template <class T, int V>
__global__ __launch_bounds__(kBlock) void combine(CombineArgs a, uint32_t chunks) {
  typedef Pack<T, V> P;
  const uint64_t all = (uint64_t)a.n * chunks;
  for (uint64_t at = (uint64_t)blockIdx.x * kBlock + threadIdx.x; at < all;
       at += (uint64_t)gridDim.x * kBlock) {
    const int64_t t = (int64_t)(at / chunks);
    const int64_t col = (int64_t)(at % chunks) * V;
    float sum[V];
    if (a.residual) {
      const P r = *(const P *)((const T *)a.residual + t * a.residual_stride + col);
#pragma unroll
      for (int c = 0; c < V; ++c) sum[c] = (float)r.v[c];
    } else {
#pragma unroll
      for (int c = 0; c < V; ++c) sum[c] = 0.f;
    }
    for (int j = 0; j < a.k; ++j) {
      const int64_t s = t * a.k + j;
      if (!used(a.ids, s, a.n_experts)) continue;
      const float w = a.weights ? a.weights[s] : 1.f;
      const P r = *(const P *)((const T *)a.rows + s * a.rows_stride + col);
#pragma unroll
      for (int c = 0; c < V; ++c) sum[c] += w * (float)r.v[c];
    }
    P o;
#pragma unroll
    for (int c = 0; c < V; ++c) o.v[c] = (T)sum[c];
    *(P *)((T *)a.out + t * a.out_stride + col) = o;
  }
}

// A wave per slot.  Bound by bytes as well (8191 x 4 rows of 2056 fp16: 61 us, 5.0 TB/s;
// 8192 x 8 rows of 2047 bf16, element by element: 313 us, 1.8 TB/s).
template <class T, int V>
__global__ __launch_bounds__(kBlock) void combine_grad(CombineArgs a) {
  const int lane = threadIdx.x & 63;
  typedef Pack<T, V> P;
  const int64_t slots = a.n * a.k;
  for (int64_t s = (int64_t)blockIdx.x * kWavesPerBlock + threadIdx.x / 64; s < slots;
       s += (int64_t)gridDim.x * kWavesPerBlock) {
    const int64_t t = s / a.k;
    const bool on = used(a.ids, s, a.n_experts);
    const float w = a.weights && on ? a.weights[s] : 1.f;
    const T *d = (const T *)a.residual + t * a.residual_stride;
    const T *r = (const T *)a.rows + s * a.rows_stride;
    T *o = (T *)a.out + s * a.out_stride;
    float dot = 0.f;
    for (int col = lane * V; col < a.dim; col += 64 * V) {
      P dv = {}, ov = {};
      if (on) dv = *(const P *)(d + col);
      if (on && a.dweights) {
        const P rv = *(const P *)(r + col);
#pragma unroll
        for (int c = 0; c < V; ++c) dot += (float)dv.v[c] * (float)rv.v[c];
      }
      if (a.out) {
#pragma unroll
        for (int c = 0; c < V; ++c) ov.v[c] = on ? (T)(w * (float)dv.v[c]) : (T)0.f;
        *(P *)(o + col) = ov;
      }
    }
    if (a.dweights) {
      dot = sum_f32<64>(dot);
      if (lane == 0) a.dweights[s] = dot;
    }
  }
}

// 16-byte accesses where every row starts on 16 bytes and holds whole ones.
template <class T>
bool wide(const CombineArgs &a, const void *const *bases, const int64_t *strides, int count) {
  constexpr int V = 16 / sizeof(T);
  if (a.dim % V) return false;
  for (int i = 0; i < count; ++i)
    if (bases[i] && (((uintptr_t)bases[i] & 15) || strides[i] % V)) return false;
  return true;
}

// Workgroups of a grid whose threads go on to further work.
uint32_t strided(int64_t blocks) { return (uint32_t)(blocks < (1 << 22) ? blocks : 1 << 22); }

template <class T>
int start(const CombineArgs &a, hipStream_t stream) {
  constexpr int V = 16 / sizeof(T);
  const void *bases[] = {a.rows, a.residual, a.out};
  const int64_t strides[] = {a.rows_stride, a.residual_stride, a.out_stride};
  const bool w = wide<T>(a, bases, strides, 3);
  const uint32_t chunks = (uint32_t)(w ? a.dim / V : a.dim);
  const uint32_t blocks = strided((a.n * (int64_t)chunks + kBlock - 1) / kBlock);
  if (w) combine<T, V><<<blocks, kBlock, 0, stream>>>(a, chunks);
  else combine<T, 1><<<blocks, kBlock, 0, stream>>>(a, chunks);
  return hip_status(hipGetLastError());
}

template <class T>
int start_grad(const CombineArgs &a, hipStream_t stream) {
  constexpr int V = 16 / sizeof(T);
  const void *bases[] = {a.dweights ? a.rows : nullptr, a.residual, a.out};
  const int64_t strides[] = {a.rows_stride, a.residual_stride, a.out_stride};
  const bool w = wide<T>(a, bases, strides, 3);
  const uint32_t blocks = strided((a.n * a.k + kWavesPerBlock - 1) / kWavesPerBlock);
  if (w) combine_grad<T, V><<<blocks, kBlock, 0, stream>>>(a);
  else combine_grad<T, 1><<<blocks, kBlock, 0, stream>>>(a);
  return hip_status(hipGetLastError());
}

}  // namespace

int launch_combine(const CombineArgs &a, hipStream_t stream) {
  if (a.type == NTC_OUT_F16) return start<_Float16>(a, stream);
  if (a.type == NTC_OUT_BF16) return start<__bf16>(a, stream);
  return start<float>(a, stream);
}

int launch_combine_backward(const CombineArgs &a, hipStream_t stream) {
  if (a.type == NTC_OUT_F16) return start_grad<_Float16>(a, stream);
  if (a.type == NTC_OUT_BF16) return start_grad<__bf16>(a, stream);
  return start_grad<float>(a, stream);
}

}  // namespace ntc
