// ntc_route.hip -- routing of items to experts and its gradient.
#include <cfloat>

#include "ntc_experts.h"

namespace ntc {
namespace {

__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(_Float16 v) { return (float)v; }
__device__ __forceinline__ float widen(__bf16 v) { return (float)v; }

// A logit as it counts: -inf for NaN (never chosen), the largest float for +inf.
__device__ __forceinline__ float counted(float l) {
  l = l > -INFINITY ? l : -INFINITY;
  return fminf(l, FLT_MAX) + 0.f;  // + 0: -0 and 0 are equal
}

// Keys whose unsigned order is the value's; 0 is left for "not eligible".
__device__ __forceinline__ uint32_t key_of(float v) {
  const uint32_t u = __float_as_uint(v);
  return (u >> 31) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ uint64_t key_of(double v) {
  const uint64_t u = (uint64_t)__double_as_longlong(v + 0.0);
  return (u >> 63) ? ~u : u | 0x8000000000000000ull;
}

__device__ __forceinline__ float value_of(uint32_t key) {
  return __uint_as_float((key >> 31) ? key & 0x7fffffffu : ~key);
}
__device__ __forceinline__ double value_of(uint64_t key) {
  return __longlong_as_double((long long)((key >> 63) ? key & 0x7fffffffffffffffull : ~key));
}

template <int LANES>
__device__ __forceinline__ uint64_t max_key(uint64_t v) {
  const uint32_t hi = max_u32<LANES>((uint32_t)(v >> 32));
  const uint32_t lo = max_u32<LANES>((uint32_t)(v >> 32) == hi ? (uint32_t)v : 0u);
  return (uint64_t)hi << 32 | lo;
}

// For values of the choice: the float32 forms by the hardware's exponential and reciprocal.
__device__ __forceinline__ float exponential(float v) {
  return __builtin_amdgcn_exp2f(v * 1.44269504f);
}
__device__ __forceinline__ double exponential(double v) { return exp(v); }
__device__ __forceinline__ float reciprocal(float v) { return __builtin_amdgcn_rcpf(v); }
__device__ __forceinline__ double reciprocal(double v) { return 1.0 / v; }
template <int LANES>
__device__ __forceinline__ float sum_all(float v) { return sum_f32<LANES>(v); }
template <int LANES>
__device__ __forceinline__ double sum_all(double v) { return sum_f64<LANES>(v); }

template <int CTRL>
__device__ __forceinline__ float moved(float v) {
  return __uint_as_float(dpp<CTRL>(__float_as_uint(v)));
}
template <int CTRL>
__device__ __forceinline__ double moved(double v) {
  const uint64_t u = (uint64_t)__double_as_longlong(v);
  const uint64_t m = (uint64_t)dpp<CTRL>((uint32_t)(u >> 32)) << 32 | dpp<CTRL>((uint32_t)u);
  return __longlong_as_double((long long)m);
}

// The two largest of a value list, kept as values join it.
template <class V>
struct Best {
  V first = -INFINITY, second = -INFINITY;
  __device__ __forceinline__ void join(V f, V s) {
    const V low = first < f ? first : f;
    first = first < f ? f : first;
    second = second < s ? s : second;
    second = second < low ? low : second;
  }
  // sum of the `top` largest there are
  __device__ __forceinline__ V worth(int top) const {
    return top == 2 && second > (V)-INFINITY ? first + second : first;
  }
  // and of their sizes, which its rounding error goes by; -1 without any
  __device__ __forceinline__ V size(int top) const {
    if (!(first > (V)-INFINITY)) return -1;
    return fabs(first) + (top == 2 && second > (V)-INFINITY ? fabs(second) : (V)0);
  }
};

// How the groups' values are found: kNone (no groups), kLanes (a group is a power of two
// of lanes: folded across them), kShared (any other size: through LDS).
enum Groups { kNone, kLanes, kShared };

// What an item's lanes share in LDS.
template <int SLOTS, Groups GROUPS>
struct Shared {
  uint32_t id[NTC_MAX_CHOICES + 1];  // and the best that is left
  double value[GROUPS == kShared ? SLOTS : 1];
  uint64_t group[GROUPS == kShared ? SLOTS : 1];
  uint8_t keep[GROUPS == kShared ? SLOTS : 1];
};

// Float32 values whose order float64 might not share.  A softmax score is at most 1 and off
// by at most 30 roundings of 2^-24 (the sum of its exponentials has 22 of them), a sigmoid
// by 4; the value v with the bias by one more of its own: 2 (30 or 4) + 2 |v| roundings for
// two values, less than 2^-18 max(1, |v|), 2^-20 for sigmoids.  A key leaves out up to
// 15 * 2^-23 < 2^-19 of a value, downwards from both, so that the difference of two cut
// values is too large by less than one cut.
__device__ __forceinline__ float value_margin(bool softmax) { return softmax ? 0x1p-17f : 0x1p-18f; }
__device__ __forceinline__ bool too_close(float high, float low, float within) {
  return !(high - low > within * fmaxf(1.f, fmaxf(fabsf(high), fabsf(low))));
}
// How far a group's float32 value may be off: by those of its two summands and one
// rounding more, 2 (30 or 4) + 2 size roundings of 2^-24 (2^-18.1 or 2^-20.7 for sizes up to
// 1, 2^-23 of larger ones), where size is the sum of the summands' own sizes: large biases of
// opposite signs leave a small sum.
__device__ __forceinline__ float group_error(bool softmax, float size) {
  return (softmax ? 0x1p-17f : 0x1p-19f) * fmaxf(1.f, size);
}

// EPL values of `from` for the experts i EPL .., 0 past the last.
template <int EPL>
__device__ __forceinline__ void load_bias(const float *from, int i, int E, float (&b)[EPL]) {
  if (EPL >= 4 && E % EPL == 0 && ((uintptr_t)from & 15) == 0) {
#pragma unroll
    for (int h = 0; h < EPL / 4; ++h) {
      const float4v v = i * EPL < E ? *(const float4v *)(from + i * EPL + h * 4) : float4v{};
#pragma unroll
      for (int j = 0; j < 4; ++j) b[h * 4 + j] = v[j];
    }
  } else {
#pragma unroll
    for (int j = 0; j < EPL; ++j) b[j] = i * EPL + j < E ? from[i * EPL + j] : 0.f;
  }
}

// The values the choice looks at, -inf where an expert is not eligible, and with groups
// their values and which stay; V double by the written rule, V float near it.  `sure`:
// float32 could tell which groups stay.
template <class V, int LANES, int EPL, Groups GROUPS>
__device__ __forceinline__ void choice_values(const RouteArgs &a, const float (&l)[EPL], float top,
                                              int i, Shared<LANES * EPL, GROUPS> &mine,
                                              V (&value)[EPL], bool &sure) {
  const int lane = threadIdx.x & 63;
  const int E = a.n_experts;
  const bool softmax = a.opt.score == NTC_SCORE_SOFTMAX;
  const bool by_value = a.bias != nullptr;
  sure = true;
  // scores where the choice looks at them
  V v[EPL];
  if (by_value || (GROUPS != kNone && a.opt.group_top == 2)) {
    V sum = 0;
#pragma unroll
    for (int j = 0; j < EPL; ++j) {
      if (softmax) {
        v[j] = exponential((V)l[j] - (V)top);
        sum += v[j];
      } else {
        v[j] = reciprocal((V)1 + exponential(-(V)l[j]));
      }
    }
    if (softmax) {
      sum = reciprocal(sum_all<LANES>(sum));
#pragma unroll
      for (int j = 0; j < EPL; ++j) v[j] *= sum;
    }
    if (by_value) {
      float b[EPL];
      load_bias<EPL>(a.bias, i, E, b);
#pragma unroll
      for (int j = 0; j < EPL; ++j) v[j] += (V)b[j];
    }
  } else {
#pragma unroll
    for (int j = 0; j < EPL; ++j) v[j] = (V)l[j];
  }
#pragma unroll
  for (int j = 0; j < EPL; ++j) {
    const bool ok = l[j] > -INFINITY && v[j] > (V)-INFINITY;
    if (!ok) v[j] = -INFINITY;
    value[j] = ok && !by_value ? (V)l[j] : v[j];
  }

  if constexpr (GROUPS != kNone) {
    const int G = a.opt.n_groups, per = E / G, top_groups = a.opt.top_groups;
    const bool fuzzy = sizeof(V) == 4 && (by_value || a.opt.group_top == 2);
    // Keys of the least that a group that stays may be worth (inverted), and of the most that
    // one that goes may be.
    uint32_t in = 0, out = 0;
    auto ranked = [&](float own, float size, bool keep) {
      const float at = size < 0.f ? -INFINITY : fminf(fmaxf(own, -FLT_MAX), FLT_MAX);
      const float off = size < 0.f ? 0.f : fminf(group_error(softmax, size), FLT_MAX);
      if (keep) in = max(in, ~key_of(at - off));
      else out = max(out, key_of(at + off));
    };
    if constexpr (GROUPS == kLanes) {
      const int wide = per / EPL;  // lanes of a group
      Best<V> best;
#pragma unroll
      for (int j = 0; j < EPL; ++j) best.join(v[j], -INFINITY);
      if (wide > 1) best.join(moved<kXor1>(best.first), moved<kXor1>(best.second));
      if (wide > 2) best.join(moved<kXor2>(best.first), moved<kXor2>(best.second));
      if (wide > 4) best.join(moved<kHalfMirror>(best.first), moved<kHalfMirror>(best.second));
      if (wide > 8) best.join(moved<kMirror>(best.first), moved<kMirror>(best.second));
      if (LANES == 64 && wide > 16)
        best.join(__shfl_xor(best.first, 16), __shfl_xor(best.second, 16));
      if (LANES == 64 && wide > 32)
        best.join(__shfl_xor(best.first, 32), __shfl_xor(best.second, 32));
      const V own = best.worth(a.opt.group_top);
      const int g = i / wide;  // lanes past the last group hold no experts
      int better = 0;
      for (int h = 0; h < G; ++h) {
        const V other = __shfl(own, (lane & ~(LANES - 1)) + h * wide);
        better += other > own || (other == own && h < g);
      }
      const bool keep = better < top_groups;
      if (fuzzy && g < G) ranked((float)own, (float)best.size(a.opt.group_top), keep);
      if (!keep) {
#pragma unroll
        for (int j = 0; j < EPL; ++j) value[j] = -INFINITY;
      }
    } else {
#pragma unroll
      for (int j = 0; j < EPL; ++j) mine.value[i * EPL + j] = (double)v[j];
      wave_shares();
      for (int g = i; g < G; g += LANES) {
        Best<V> best;
        for (int e = g * per; e < (g + 1) * per; ++e) best.join((V)mine.value[e], -INFINITY);
        mine.group[g] = key_of((double)best.worth(a.opt.group_top));
        // the group's own values have been read, by this lane alone
        if (fuzzy) mine.value[g * per] = (double)best.size(a.opt.group_top);
      }
      wave_shares();
      for (int g = i; g < G; g += LANES) {
        const uint64_t own = mine.group[g];
        int better = 0;
        for (int h = 0; h < G; ++h) {
          const uint64_t other = mine.group[h];
          better += other > own || (other == own && h < g);
        }
        const bool keep = better < top_groups;
        mine.keep[g] = keep;
        if (fuzzy) ranked((float)value_of(own), (float)mine.value[g * per], keep);
      }
      wave_shares();
#pragma unroll
      for (int j = 0; j < EPL; ++j) {
        const int e = i * EPL + j;
        if (e < E && !mine.keep[e / per]) value[j] = -INFINITY;
      }
    }
    if (fuzzy) {
      in = max_u32<LANES>(in);
      out = max_u32<LANES>(out);
      if (in != 0 && out != 0 && value_of(out) > -INFINITY)
        sure = value_of(~in) > value_of(out);
    }
  }
}

// The choice of one item by LANES lanes, lane i holding the experts i EPL .. i EPL + EPL - 1:
// k rounds take the largest value left (its lowest lane, that lane's lowest expert: ties
// go to the lower index) and put the expert into its slot in LDS.  Returns how many were
// found.  This one by float32 keys whose last 4 bits hold the expert's place in its lane.
// What they leave out could matter where `sure` is false or, bit r of `pairs`, for the
// order of slots r and r + 1 (slot k: the best that is left; one behind it isn't looked
// at).  EXACT: the logits' type has no bits there, and the choice goes by logits.
template <int LANES, int EPL, Groups GROUPS, bool EXACT>
__device__ __forceinline__ int choose(const RouteArgs &a, const float (&l)[EPL], float top, int i,
                                      Shared<LANES * EPL, GROUPS> &mine, bool &sure,
                                      uint64_t &pairs) {
  static_assert(EPL <= 16, "");
  pairs = 0;
  const int lane = threadIdx.x & 63;
  const bool by_value = a.bias != nullptr;
  const float margin = value_margin(a.opt.score == NTC_SCORE_SOFTMAX);
  float value[EPL];
  choice_values<float, LANES, EPL, GROUPS>(a, l, top, i, mine, value, sure);
  uint32_t key[EPL];
#pragma unroll
  for (int j = 0; j < EPL; ++j)
    key[j] = value[j] > -INFINITY ? (key_of(value[j]) & ~15u) | (15 - j) : 0;
  int found = 0;
  uint32_t last = 0;
  for (int r = 0; r <= a.k; ++r) {  // one more: the best that is left
    uint32_t best = 0;
#pragma unroll
    for (int j = 0; j < EPL; ++j) best = max(best, key[j]);
    const uint32_t most = max_u32<LANES>(best >> 4);
    uint64_t holders = ballot(best >> 4 == most && most != 0);
    if (holders == 0) break;  // no item of the wave has an eligible expert left
    if (LANES == 16) holders = (holders >> (lane & 48)) & 0xffff;
    if constexpr (!EXACT) {
      if (last != 0 && most != 0 &&
          (by_value ? too_close(value_of(last << 4), value_of(most << 4), margin) : last == most))
        pairs |= 1ull << (r - 1);
      last = most;
    }
    found += holders != 0 && r < a.k;
    if (holders != 0 && i == __builtin_ctzll(holders)) {
      mine.id[r] = (uint32_t)(i * EPL + 15 - (int)(best & 15));
#pragma unroll
      for (int j = 0; j < EPL; ++j) key[j] = key[j] == best ? 0 : key[j];
    }
  }
  return found;
}

// The same by float64 values, every bit of them.
template <int LANES, int EPL, Groups GROUPS>
__device__ __forceinline__ int choose_exactly(const RouteArgs &a, const float (&l)[EPL], float top,
                                              int i, Shared<LANES * EPL, GROUPS> &mine) {
  const int lane = threadIdx.x & 63;
  double value[EPL];
  bool sure;
  choice_values<double, LANES, EPL, GROUPS>(a, l, top, i, mine, value, sure);
  uint64_t key[EPL];
#pragma unroll
  for (int j = 0; j < EPL; ++j) key[j] = value[j] > -INFINITY ? key_of(value[j]) : 0;
  int found = 0;
  for (int r = 0; r < a.k; ++r) {
    uint64_t best = 0;
#pragma unroll
    for (int j = 0; j < EPL; ++j) best = key[j] > best ? key[j] : best;
    const uint64_t most = max_key<LANES>(best);
    uint64_t holders = ballot(best == most && most != 0);
    if (holders == 0) break;
    if (LANES == 16) holders = (holders >> (lane & 48)) & 0xffff;
    found += holders != 0;
    if (holders != 0 && i == __builtin_ctzll(holders)) {
      int at = 0;
#pragma unroll
      for (int j = EPL - 1; j >= 0; --j)  // the lowest expert comes last
        if (key[j] == most) at = j;
#pragma unroll
      for (int j = 0; j < EPL; ++j)
        if (at == j) key[j] = 0;
      mine.id[r] = (uint32_t)(i * EPL + at);
    }
  }
  return found;
}

// V logits of T as one load.
template <class T, int EPL>
__device__ __forceinline__ void load_logits(const T *row, int i, int E, bool wide, bool live,
                                            float (&l)[EPL]) {
  constexpr int kRun = 16 / sizeof(T) < EPL ? 16 / sizeof(T) : EPL;
  struct alignas(kRun * sizeof(T)) Run {
    T v[kRun];
  };
#pragma unroll
  for (int j = 0; j < EPL; ++j) l[j] = -INFINITY;
  if (wide) {  // E is a multiple of EPL
    if (live && i * EPL < E) {
#pragma unroll
      for (int h = 0; h < EPL / kRun; ++h) {
        const Run r = *(const Run *)(row + i * EPL + h * kRun);
#pragma unroll
        for (int j = 0; j < kRun; ++j) l[h * kRun + j] = counted(widen(r.v[j]));
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < EPL; ++j)
      if (live && i * EPL + j < E) l[j] = counted(widen(row[i * EPL + j]));
  }
}

// Items are routed by LANES lanes each, up to 256 experts by 16 (four items a wave share
// every cross-lane step), more by a whole wave.  Bound by instruction issue: the rounds
// and, with a bias, the exponentials, which are float32 unless two values lie too close
// (16384 x 256, sigmoid, bias, 8 groups, kernel alone: 19.8 us; with float64 for the whole
// item wherever two of its slots are close 24, for all items 43).
template <class T, int LANES, int EPL, bool FUZZY, Groups GROUPS>
__global__ __launch_bounds__(kBlock) void route(RouteArgs a, bool wide) {
  constexpr int kItems = kBlock / LANES;  // per workgroup
  __shared__ Shared<LANES * EPL, GROUPS> shared[kItems];
  Shared<LANES * EPL, GROUPS> &mine = shared[threadIdx.x / LANES];
  const int i = threadIdx.x % LANES;
  const int E = a.n_experts;
  const bool softmax = a.opt.score == NTC_SCORE_SOFTMAX;
  for (int64_t first = (int64_t)blockIdx.x * kItems; first < a.n;
       first += (int64_t)gridDim.x * kItems) {
    const int64_t t = first + threadIdx.x / LANES;
    bool live = t < a.n;
    if (live && a.mask) live = a.mask[t] != 0;
    float l[EPL];
    load_logits<T, EPL>((const T *)a.logits + (live ? t : 0) * a.stride, i, E, wide, live, l);
    // the item's largest logit, for exponentials that don't overflow
    float top = -INFINITY;
#pragma unroll
    for (int j = 0; j < EPL; ++j) top = fmaxf(top, l[j]);
    top = fmaxf(max_f32<LANES>(top), -FLT_MAX);

    constexpr bool kExact = !FUZZY && sizeof(T) == 2;
    bool sure;
    uint64_t pairs;
    int found = choose<LANES, EPL, GROUPS, kExact>(a, l, top, i, mine, sure, pairs);
    if constexpr (!kExact) {
      // 16-bit logits themselves fit a key: equal ones are in the order of their indices
      if (sizeof(T) == 2 && !a.bias) pairs = 0;
      // Pairs of slots apart from one another are put in order by their own float64 values.
      // Softmax needs every expert's for that, and with the last slot more than the
      // runner-up might come before it.
      if (pairs & (pairs >> 1) || pairs >> (a.k - 1) || (pairs != 0 && softmax && a.bias))
        sure = false;
      wave_shares();
      if (pairs != 0 && sure)
        for (int r = i; r + 1 < a.k; r += LANES)
          if (pairs >> r & 1) {
            const uint32_t e = mine.id[r], f = mine.id[r + 1];
            auto exactly = [&](uint32_t of) -> double {
              const double at = (double)counted(widen(((const T *)a.logits)[t * a.stride + of]));
              return a.bias ? 1.0 / (1.0 + exp(-at)) + (double)a.bias[of] : at;
            };
            const double ve = exactly(e), vf = exactly(f);
            if (vf > ve || (vf == ve && f < e)) {
              mine.id[r] = f;
              mine.id[r + 1] = e;
            }
          }
      // items that float32 can't tell, one after the other by the whole wave
      constexpr int kEpl = EPL * LANES / 64;
      const int lane = threadIdx.x & 63;
      for (uint64_t left = ballot(!sure); left != 0;) {
        const int q = __builtin_ctzll(left) / LANES;
        left &= LANES == 64 ? 0 : ~(0xffffull << (q * 16));
        const int item = threadIdx.x / 64 * (64 / LANES) + q;
        float all[kEpl], most = -INFINITY;
        load_logits<T, kEpl>((const T *)a.logits + (first + item) * a.stride, lane, E, false, true,
                             all);
#pragma unroll
        for (int j = 0; j < kEpl; ++j) most = fmaxf(most, all[j]);
        most = fmaxf(max_f32<64>(most), -FLT_MAX);
        const int count = choose_exactly<64, kEpl, GROUPS>(a, all, most, lane, shared[item]);
        if (lane / LANES == q) found = count;
      }
    }
    wave_shares();
    // weights of the chosen; exponentials relative to the largest of the sum they go into
    float whole = 1.f, base = top;
    if (softmax && !a.opt.renormalize) {
      whole = 0.f;
#pragma unroll
      for (int j = 0; j < EPL; ++j) whole += expf(l[j] - top);
      whole = sum_f32<LANES>(whole);
    }
    // this lane's slots: every LANES-th from i on
    constexpr int kSlots = NTC_MAX_CHOICES / LANES;
    const int own = (a.k + LANES - 1) / LANES;
    float at[kSlots];
    uint32_t id[kSlots];
#pragma unroll
    for (int u = 0; u < kSlots; ++u) {
      const int r = i + u * LANES;
      at[u] = -INFINITY;
      id[u] = NTC_PAD;
      if (u < own && r < found) {
        id[u] = mine.id[r];
        at[u] = counted(widen(((const T *)a.logits)[t * a.stride + id[u]]));
      }
    }
    if (a.opt.renormalize) {
      base = -INFINITY;
#pragma unroll
      for (int u = 0; u < kSlots; ++u)
        if (u < own) base = fmaxf(base, softmax ? at[u] : fminf(at[u], 0.f));
      base = fmaxf(max_f32<LANES>(base), -FLT_MAX);
    } else if (!softmax) {
      base = 0.f;
    }
    float w[kSlots], sum = 0.f;
#pragma unroll
    for (int u = 0; u < kSlots; ++u)
      if (u < own) {  // sigmoid = exp(min(l, 0)) / (1 + exp(-|l|))
        w[u] = softmax ? expf(at[u] - base)
                       : expf(fminf(at[u], 0.f) - base) / (1.f + expf(-fabsf(at[u])));
        sum += w[u];  // 0 at empty slots
      }
    if (a.opt.renormalize) whole = sum_f32<LANES>(sum);
#pragma unroll
    for (int u = 0; u < kSlots; ++u) {
      const int r = i + u * LANES;
      if (u < own && t < a.n && r < a.k) {
        a.ids[t * a.k + r] = id[u];
        a.weights[t * a.k + r] = id[u] != NTC_PAD ? a.opt.scale * (w[u] / whole) : 0.f;
      }
    }
    wave_shares();
  }
}

// LANES lanes per item, lane i holding the experts i EPL .. in registers and, of the k
// slots, every LANES-th from i on: a weight's share p and the gradient d that reaches its
// logit directly.  Every expert then collects the d of its slots in ascending order, and
// with plain softmax weights -s_e sum(p g).  Bound by instruction issue: 480 vector
// instructions a wave of four items fill 78 % of the CUs' busy cycles (30001 x 128 bf16, 4
// slots: 9.2 us, where the bytes would take 3.1).
template <class T, int LANES, int EPL>
__global__ __launch_bounds__(kBlock) void route_grad(RouteArgs a, bool wide) {
  constexpr int kItems = kBlock / LANES;
  __shared__ uint32_t s_id[kItems][NTC_MAX_CHOICES];
  __shared__ float s_d[kItems][NTC_MAX_CHOICES];
  const int i = threadIdx.x % LANES, item = threadIdx.x / LANES;
  const int E = a.n_experts;
  const bool softmax = a.opt.score == NTC_SCORE_SOFTMAX, renorm = a.opt.renormalize != 0;
  const bool spread_all = softmax && !renorm;
  constexpr int kSlots = NTC_MAX_CHOICES / LANES;  // a lane's
  for (int64_t first = (int64_t)blockIdx.x * kItems; first < a.n;
       first += (int64_t)gridDim.x * kItems) {
    const int64_t t = first + item;
    const bool live = t < a.n;
    const T *row = (const T *)a.logits + (live ? t : 0) * a.stride;
    float l[EPL];
    float top = -INFINITY, all = 0.f;
    if (spread_all) {
      load_logits<T, EPL>(row, i, E, wide, live, l);
#pragma unroll
      for (int j = 0; j < EPL; ++j) top = fmaxf(top, l[j]);
      top = fmaxf(max_f32<LANES>(top), -FLT_MAX);
#pragma unroll
      for (int j = 0; j < EPL; ++j) {
        l[j] = expf(l[j] - top);  // from here on: the exponentials
        all += l[j];
      }
      all = sum_f32<LANES>(all);
    }
    // the slots: logit, gradient, share
    const int own = (a.k + LANES - 1) / LANES;  // of them in use
    float at[kSlots], g[kSlots], p[kSlots];
    uint32_t id[kSlots];
    float base = -INFINITY;
#pragma unroll
    for (int u = 0; u < kSlots; ++u) {
      if (u >= own) continue;
      const int r = i + u * LANES;
      id[u] = live && r < a.k ? a.ids[t * a.k + r] : NTC_PAD;
      at[u] = id[u] < (uint32_t)E ? counted(widen(row[id[u]])) : -INFINITY;
      if (!(at[u] > -INFINITY)) id[u] = NTC_PAD;
      g[u] = id[u] != NTC_PAD ? a.dweights[t * a.k + r] : 0.f;
      base = fmaxf(base, softmax ? at[u] : fminf(at[u], 0.f));
    }
    if (renorm) base = fmaxf(max_f32<LANES>(base), -FLT_MAX);
    else base = softmax ? top : 0.f;
    float sum = 0.f, back = 0.f;
#pragma unroll
    for (int u = 0; u < kSlots; ++u) {
      if (u >= own) continue;
      const float ex = expf(-fabsf(at[u]));
      p[u] = softmax ? expf(at[u] - base) : expf(fminf(at[u], 0.f) - base) / (1.f + ex);
      if (id[u] == NTC_PAD) p[u] = 0.f;
      sum += p[u];
    }
    if (renorm) sum = sum_f32<LANES>(sum);
    else sum = softmax ? all : 1.f;
#pragma unroll
    for (int u = 0; u < kSlots; ++u) {
      if (u >= own) continue;
      p[u] = id[u] != NTC_PAD ? p[u] / sum : 0.f;
      back += p[u] * g[u];
    }
    back = sum_f32<LANES>(back);
#pragma unroll
    for (int u = 0; u < kSlots; ++u) {
      if (u >= own) continue;
      const int r = i + u * LANES;
      const float ex = expf(-fabsf(at[u]));  // 1 - sigmoid is ex / (1 + ex) or 1 / (1 + ex)
      const float rest = softmax ? 1.f : (at[u] > 0.f ? ex : 1.f) / (1.f + ex);
      const float d = p[u] * (renorm ? g[u] - back : g[u]) * rest * a.opt.scale;
      if (r < a.k) {
        s_id[item][r] = id[u];
        s_d[item][r] = id[u] != NTC_PAD ? d : 0.f;
      }
    }
    wave_shares();
    // without an eligible expert the sum is 0, and so is every gradient
    const float spread = spread_all && all > 0.f ? back * a.opt.scale / all : 0.f;
#pragma unroll
    for (int j = 0; j < EPL; ++j) l[j] = spread_all ? -spread * l[j] : 0.f;
    for (int r = 0; r < a.k; ++r) {
      const uint32_t e = s_id[item][r];
      const float d = s_d[item][r];
#pragma unroll
      for (int j = 0; j < EPL; ++j)
        if (e == (uint32_t)(i * EPL + j)) l[j] += d;
    }
    if (live) {
      T *out = (T *)a.dlogits + t * a.dstride;
      constexpr int kRun = 16 / sizeof(T) < EPL ? 16 / sizeof(T) : EPL;
      struct alignas(kRun * sizeof(T)) Run {
        T v[kRun];
      };
      if (wide) {
        if (i * EPL < E) {
#pragma unroll
          for (int h = 0; h < EPL / kRun; ++h) {
            Run o;
#pragma unroll
            for (int j = 0; j < kRun; ++j) o.v[j] = (T)l[h * kRun + j];
            *(Run *)(out + i * EPL + h * kRun) = o;
          }
        }
      } else {
#pragma unroll
        for (int j = 0; j < EPL; ++j)
          if (i * EPL + j < E) out[i * EPL + j] = (T)l[j];
      }
    }
    wave_shares();
  }
}

// Rows hold whole runs of EPL experts on addresses that take them 16 bytes (or one run)
// at a time.
template <class T, int EPL>
bool runs(const void *base, int64_t stride, int32_t n_experts) {
  const int64_t bytes = EPL * sizeof(T) < 16 ? EPL * sizeof(T) : 16;
  return n_experts % EPL == 0 && ((uintptr_t)base & (bytes - 1)) == 0 &&
         stride * (int64_t)sizeof(T) % bytes == 0;
}

uint32_t item_blocks(int64_t n, int items) {
  const int64_t blocks = (n + items - 1) / items;
  return (uint32_t)(blocks < (1 << 20) ? blocks : 1 << 20);
}

template <class T, int LANES, int EPL, bool FUZZY>
int start_groups(const RouteArgs &a, bool wide, hipStream_t stream) {
  const dim3 grid(item_blocks(a.n, kBlock / LANES)), block(kBlock);
  const int per = a.n_experts / a.opt.n_groups;
  const int lanes = per / EPL;
  if (a.opt.top_groups == a.opt.n_groups)
    route<T, LANES, EPL, FUZZY, kNone><<<grid, block, 0, stream>>>(a, wide);
  else if (per % EPL == 0 && (lanes & (lanes - 1)) == 0)
    route<T, LANES, EPL, FUZZY, kLanes><<<grid, block, 0, stream>>>(a, wide);
  else
    route<T, LANES, EPL, FUZZY, kShared><<<grid, block, 0, stream>>>(a, wide);
  return hip_status(hipGetLastError());
}

template <class T, int LANES, int EPL>
int start(const RouteArgs &a, hipStream_t stream) {
  const bool wide = runs<T, EPL>(a.logits, a.stride, a.n_experts);
  if (a.dlogits) {
    const bool both = wide && runs<T, EPL>(a.dlogits, a.dstride, a.n_experts);
    route_grad<T, LANES, EPL>
        <<<item_blocks(a.n, kBlock / LANES), kBlock, 0, stream>>>(a, both);
    return hip_status(hipGetLastError());
  }
  const bool groups = a.opt.top_groups < a.opt.n_groups;
  if (a.bias || (groups && a.opt.group_top == 2))
    return start_groups<T, LANES, EPL, true>(a, wide, stream);
  return start_groups<T, LANES, EPL, false>(a, wide, stream);
}

template <class T>
int start_type(const RouteArgs &a, hipStream_t stream) {
  if (a.n_experts <= 64) return start<T, 16, 4>(a, stream);
  if (a.n_experts <= 128) return start<T, 16, 8>(a, stream);
  if (a.n_experts <= 256) return start<T, 16, 16>(a, stream);
  return start<T, 64, 16>(a, stream);
}

int start_any(const RouteArgs &a, hipStream_t stream) {
  if (a.type == NTC_OUT_F16) return start_type<_Float16>(a, stream);
  if (a.type == NTC_OUT_BF16) return start_type<__bf16>(a, stream);
  return start_type<float>(a, stream);
}

}  // namespace

int launch_route(const RouteArgs &a, hipStream_t stream) { return start_any(a, stream); }
int launch_route_backward(const RouteArgs &a, hipStream_t stream) { return start_any(a, stream); }

}  // namespace ntc
