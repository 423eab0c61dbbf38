// The draw of a token from a row of logits, at a temperature and under top-k, min-p and top-p, from a given uniform number.
//
//   w_v = exp((z_v - max z) / T);  tokens in falling order of z, equal ones in rising order;  the first k of them;  of these those with w >= min_p;  of these
//   the shortest run from the front whose mass reaches top_p of theirs;  of what is kept, in rising order of tokens, the first whose running mass passes
//   u times the kept mass
// A uniform number may fall next to a border between two tokens, so masses are float64 or whole numbers: w in units of 2^-s, s = 62 - log2 V, at most 52, whose
// sums are exact in any order (64-bit atomics in LDS give the same result whichever comes first).
//
// Two launches.  The first reads the logits once: maxima of groups of 64, and of units of 1024 the maximum, the mass at T and the sum of exponentials.  The second gives
// a workgroup to a row.  Without filters the unit and then the token are found from the units' masses; thresholds are found by their bits, eleven at a time from
// the top, with a histogram of counts or masses.
#include <algorithm>
#include <type_traits>

#include "umas_f32.h"
#include "umas_few.h"

namespace umas {
namespace {

typedef unsigned long long u64;
constexpr int kUnit = 1024, kGroup = 64, kGroupsPerUnit = kUnit / kGroup;
constexpr int kPerLane = kUnit / kWave;                       // logits of a unit that a lane holds
constexpr int kMaxSampleV = UMAS_MAX_SAMPLE_V;

// ------------------------------------------------------------------ weights
// 2^t for t <= 0, to 2^-47 of it: 2^n times the series of exp(f ln 2), |f| <= 1/2, whose first term left out is 6.3e-15.
__device__ __forceinline__ double exp2_of(double t) {
  if (!(t > -1000.0)) return 0.0;
  const double n = rint(t), f = t - n;
  double p = 4.4455382718708116e-10;                         // ln 2^k / k!, k = 11 .. 0
  p = fma(p, f, 7.0549116208011233e-09);
  p = fma(p, f, 1.0178086009239699e-07);
  p = fma(p, f, 1.3215486790144307e-06);
  p = fma(p, f, 1.5252733804059841e-05);
  p = fma(p, f, 1.5403530393381610e-04);
  p = fma(p, f, 1.3333558146428443e-03);
  p = fma(p, f, 9.6181291076284769e-03);
  p = fma(p, f, 5.5504108664821580e-02);
  p = fma(p, f, 2.4022650695910072e-01);
  p = fma(p, f, 6.9314718055994531e-01);
  p = fma(p, f, 1.0);
  return ldexp(p, static_cast<int>(n));
}
constexpr double kLog2e64 = 1.4426950408889634074;
// exp((z - top) / T) for z <= top.  Equal ones are 1 whatever they are, infinities among them.
__device__ __forceinline__ double weight_of(float z, float top, double inv_t) {
  if (z == top) return 1.0;
  return exp2_of((static_cast<double>(z) - static_cast<double>(top)) * inv_t * kLog2e64);
}
__device__ __forceinline__ uint32_t order_of(float z) {       // whole numbers in the order of the logits, one zero
  const uint32_t u = __float_as_uint(z + 0.f);
  return u ^ (static_cast<uint32_t>(static_cast<int32_t>(u) >> 31) | 0x80000000u);
}

struct Settings {                                            // numbers for all rows, or an array with one a row
  double temperature, top_p, min_p;
  int top_k;
  const float *temperature_of, *top_p_of, *min_p_of;
  const int32_t* top_k_of;
  __device__ __forceinline__ double t(int64_t row) const { return temperature_of ? temperature_of[row] : temperature; }
  __device__ __forceinline__ double p(int64_t row) const { return top_p_of ? top_p_of[row] : top_p; }
  __device__ __forceinline__ double m(int64_t row) const { return min_p_of ? min_p_of[row] : min_p; }
  __device__ __forceinline__ int k(int64_t row) const { return top_k_of ? top_k_of[row] : top_k; }
};
template <typename In>
struct Logits {
  const In* z;
  int64_t stride;
  int V, units;
  __device__ __forceinline__ const In* row(int64_t m) const { return z + m * stride; }
};
// What the first launch leaves, per row.
struct Summary {
  float *group, *unit;                                       // [rows][units * 16], [rows][units]: maxima; -infinity where nothing counts
  double *mass, *sum;                                        // [rows][units]: sum of w at T and of exp(z - max) at 1, relative to the unit's maximum
};

// ------------------------------------------------------------------ loads
// The lane's share of a unit: pieces of kRun tokens that lie next to each other, kRun * 64 tokens apart.  What is no number counts as -infinity, as what lies
// past the vocabulary.
template <typename In> constexpr int kRun = std::is_same<In, uint16_t>::value ? 8 : 4;
__device__ __forceinline__ float logit(float x) { return fmaxf(x, -INFINITY); }
__device__ __forceinline__ float logit(double x) { return fmaxf(static_cast<float>(x), -INFINITY); }
__device__ __forceinline__ float logit(uint16_t x) { return fmaxf(bf2f(x), -INFINITY); }
template <typename In>
__device__ __forceinline__ int token_of(int unit, int i) {    // of the lane's i-th logit
  return unit * kUnit + (i / kRun<In>) * (kRun<In> * kWave) + (threadIdx.x & 63) * kRun<In> + i % kRun<In>;
}
template <typename In>
__device__ __forceinline__ void load_unit(const In* __restrict__ z, int V, int unit, float (&x)[kPerLane]) {
  typedef uint32_t u32x4a __attribute__((ext_vector_type(4), aligned(2)));
  constexpr int R = kRun<In>;
#pragma unroll
  for (int i = 0; i < kPerLane; i += R) {
    const int v = token_of<In>(unit, i);
    if (v + R <= V) {
      if constexpr (std::is_same<In, double>::value) {
#pragma unroll
        for (int j = 0; j < R; ++j) x[i + j] = logit(z[v + j]);
      } else {
        const u32x4a w = *reinterpret_cast<const u32x4a*>(z + v);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if constexpr (R == 8) {
            x[i + 2 * j] = logit(__uint_as_float(w[j] << 16));
            x[i + 2 * j + 1] = logit(__uint_as_float(w[j] & 0xFFFF0000u));
          } else {
            x[i + j] = logit(__uint_as_float(w[j]));
          }
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < R; ++j) x[i + j] = v + j < V ? logit(z[v + j]) : -INFINITY;
    }
  }
}

// ------------------------------------------------------------------ first launch
constexpr int kOpenT = 256, kOpenUnits = kOpenT / kWave;
template <typename In>
__global__ void __launch_bounds__(kOpenT)
k_sample_open(Logits<In> L, Settings S, const int32_t* __restrict__ rowsel, int64_t c0, Summary out) {
  constexpr int R = kRun<In>, kLanes = kGroup / R;            // lanes to a group
  const int lane = threadIdx.x & 63, unit = blockIdx.x * kOpenUnits + (threadIdx.x >> 6);
  if (unit >= L.units) return;
  const int64_t m = blockIdx.y, row = rowsel ? rowsel[c0 + m] : c0 + m;
  float x[kPerLane];
  load_unit(L.row(m), L.V, unit, x);
  const int64_t at = m * L.units + unit;
  float top = -INFINITY;
#pragma unroll
  for (int i = 0; i < kPerLane; i += R) {
    float g = x[i];
#pragma unroll
    for (int j = 1; j < R; ++j) g = fmaxf(g, x[i + j]);
#pragma unroll
    for (int o = 1; o < kLanes; o <<= 1) g = fmaxf(g, __shfl_xor(g, o, kWave));
    if (lane % kLanes == 0) out.group[at * kGroupsPerUnit + i / R * R + lane / kLanes] = g;
    top = fmaxf(top, g);
  }
#pragma unroll
  for (int o = kLanes; o < kWave; o <<= 1) top = fmaxf(top, __shfl_xor(top, o, kWave));
  double mass = 0.0, sum = 0.0;
  if (top > -INFINITY) {
    const double t = S.t(row);
    const bool drawn = t > 0.0;
    const double inv_t = 1.0 / t;
    if (drawn)
#pragma unroll
      for (int i = 0; i < kPerLane; ++i) mass += weight_of(x[i], top, inv_t);
    if (drawn && t == 1.0) {
      sum = mass;
    } else {
      constexpr float kLog2e = 1.44269504088896341f;
#pragma unroll
      for (int i = 0; i < kPerLane; ++i) sum += static_cast<double>(x[i] == top ? 1.f : __builtin_amdgcn_exp2f((x[i] - top) * kLog2e));
    }
    mass = wave_sum(mass);
    sum = wave_sum(sum);
  }
  if (lane == 0) {
    out.unit[at] = top;
    out.mass[at] = mass;
    out.sum[at] = sum;
  }
}

// ------------------------------------------------------------------ second launch
constexpr int kRowT = 1024, kRowWaves = kRowT / kWave;
constexpr int kBins = 2048;
struct RowShared {
  u64 bins[kBins];
  u64 scan[17];
  double dscan[17];
  float fred[kRowWaves];
  u64 found_above, found_here;
  uint32_t found_bin;
  int found_id;
  u64 found_rest;
  double found_drest;
};
// The logits of a row, a unit to a wavefront at a time.
template <typename In>
struct RowSource {
  const In* z;
  int V, units;
  const float* unit_max;                                     // of the row
  RowShared& s;
  u64* s_unit;                                               // [units]
  // f(z, token) for every token with z > -infinity, and z >= lo; others may come
  template <class F>
  __device__ __forceinline__ void each(float lo, F f) const {
    for (int u = threadIdx.x >> 6; u < units; u += kRowWaves) {
      const float top = unit_max[u];
      if (!(top >= lo) || top == -INFINITY) continue;
      float x[kPerLane];
      load_unit(z, V, u, x);
#pragma unroll
      for (int i = 0; i < kPerLane; ++i)
        if (x[i] > -INFINITY) f(x[i], token_of<In>(u, i));
    }
  }
  // The first token, in rising order, at which the running sum of val passes `target`; -1: none.
  template <class F>
  __device__ __forceinline__ int first_beyond(float lo, F val, u64 target) const {
    for (int u = threadIdx.x >> 6; u < units; u += kRowWaves) {
      const float top = unit_max[u];
      u64 sum = 0;
      if (top >= lo && top > -INFINITY) {
        float x[kPerLane];
        load_unit(z, V, u, x);
#pragma unroll
        for (int i = 0; i < kPerLane; ++i)
          if (x[i] > -INFINITY) sum += val(x[i], token_of<In>(u, i));
        sum = wave_sum(sum);
      }
      if ((threadIdx.x & 63) == 0) s_unit[u] = sum;
    }
    __syncthreads();
    u64 before = 0;
    int unit = -1;
    if (threadIdx.x == 0) s.found_id = -1;
    for (int u0 = 0; u0 < units; u0 += kRowT) {
      const int u = u0 + threadIdx.x;
      const u64 mine = u < units ? s_unit[u] : 0;
      u64 total;
      const u64 excl = before + block_excl_scan(mine, s.scan, &total);
      if (excl <= target && target < excl + mine) {
        s.found_id = u;
        s.found_rest = target - excl;
      }
      before += total;
      __syncthreads();
      unit = s.found_id;
      if (unit >= 0) break;
    }
    if (unit < 0) return -1;
    const u64 rest = s.found_rest;
    const int v = unit * kUnit + threadIdx.x;
    const float x = v < V ? logit(z[v]) : -INFINITY;
    const u64 mine = x > -INFINITY ? val(x, v) : 0;
    u64 total;
    const u64 excl = block_excl_scan(mine, s.scan, &total);
    if (excl <= rest && rest < excl + mine) s.found_id = v;
    __syncthreads();
    const int id = s.found_id;
    __syncthreads();
    return id;
  }
};
template <class F>
__device__ __forceinline__ float block_reduce(float v, RowShared& s, F f) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = f(v, __shfl_xor(v, o, kWave));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s.fred[threadIdx.x >> 6] = v;
  __syncthreads();
  v = s.fred[0];
  for (int w = 1; w < kRowWaves; ++w) v = f(v, s.fred[w]);
  return v;
}
struct Border {
  uint32_t key;                                              // the order of a logit
  u64 above, here;                                           // sums over larger logits, and over those equal to it
};
// The logit at which the sum of val over the logits in falling order reaches `need`, 1 <= need <= the sum over all.
template <class Source, class F>
__device__ __forceinline__ Border border_of(const Source& src, RowShared& s, float lo, F val, u64 need) {
  Border b{0, 0, 0};
#pragma unroll 1
  for (int digit = 0; digit < 3; ++digit) {
    const int shift = digit == 0 ? 21 : digit == 1 ? 10 : 0, known = digit == 0 ? 32 : digit == 1 ? 21 : 10;
    const uint32_t mask = (1u << (known - shift)) - 1;
    for (int i = threadIdx.x; i < kBins; i += kRowT) s.bins[i] = 0;
    __syncthreads();
    src.each(lo, [&](float z, int id) {
      const uint32_t key = order_of(z);
      if (digit != 0 && (key ^ b.key) >> known) return;
      const u64 v = val(z, id);
      if (v) atomicAdd(&s.bins[(key >> shift) & mask], v);
    });
    __syncthreads();
    // from the largest bin down, two to a thread
    const int hi = kBins - 1 - 2 * static_cast<int>(threadIdx.x);
    const u64 x = s.bins[hi], y = s.bins[hi - 1];
    u64 total;
    const u64 above = b.above + block_excl_scan(x + y, s.scan, &total);
    if (above < need && need <= above + x) {
      s.found_bin = hi;
      s.found_above = above;
      s.found_here = x;
    } else if (above + x < need && need <= above + x + y) {
      s.found_bin = hi - 1;
      s.found_above = above + x;
      s.found_here = y;
    }
    __syncthreads();
    b.key |= s.found_bin << shift;
    b.above = s.found_above;
    b.here = s.found_here;
    __syncthreads();
  }
  return b;
}
template <class Source, class F>
__device__ __forceinline__ u64 total_of(const Source& src, RowShared& s, float lo, F val) {
  u64 sum = 0;
  src.each(lo, [&](float z, int id) { sum += val(z, id); });
  u64 total;
  block_excl_scan(sum, s.scan, &total);
  __syncthreads();
  return total;
}

struct SampleOut {
  int32_t* ids;
  float *logp, *logq;
};
struct Drawn {
  int id;
  double kept;                                               // the kept mass, in units of the largest weight
};
// What a row draws, from its logits and settings; some filter is on.
template <class Source>
__device__ __forceinline__ Drawn draw(const Source& src, RowShared& s, float top, double inv_t, int k, double p, double m, double u, int unit_bits) {
  const double one = ldexp(1.0, unit_bits);
  const float none = -INFINITY;
  auto w_of = [&](float z) {                                 // of the tokens that min_p leaves
    const double w = weight_of(z, top, inv_t);
    return w >= m ? static_cast<u64>(rint(w * one)) : u64{0};
  };
  uint32_t k_key = 0, p_key = 0;
  int k_tie = INT32_MAX, p_tie = INT32_MAX;                  // the last of the tokens at the border that is in
  if (k > 0) {
    const u64 have = total_of(src, s, none, [](float, int) { return u64{1}; });
    if (static_cast<u64>(k) < have) {
      const Border b = border_of(src, s, none, [](float, int) { return u64{1}; }, k);
      k_key = b.key;
      const u64 ties = k - b.above;
      if (ties < b.here) k_tie = src.first_beyond(none, [&](float z, int) { return u64{order_of(z) == k_key}; }, ties - 1);
    }
  }
  auto first_k = [&](float z, int id) {
    const uint32_t key = order_of(z);
    return key > k_key || (key == k_key && id <= k_tie);
  };
  auto w_k = [&](float z, int id) { return first_k(z, id) ? w_of(z) : u64{0}; };
  u64 mass = total_of(src, s, none, w_k);
  if (p < 1.0) {
    u64 need = static_cast<u64>(ceil(p * static_cast<double>(mass)));
    need = need < 1 ? 1 : need > mass ? mass : need;
    const Border b = border_of(src, s, none, w_k, need);
    p_key = b.key;
    const uint32_t bits = p_key & 0x80000000u ? p_key ^ 0x80000000u : ~p_key;
    const u64 w = w_of(__uint_as_float(bits)), ties = (need - b.above + w - 1) / w;
    mass = b.above + ties * w;
    if (ties * w < b.here)
      p_tie = src.first_beyond(none, [&](float z, int id) { return u64{order_of(z) == p_key && first_k(z, id)}; }, ties - 1);
  }
  u64 target = static_cast<u64>(u * static_cast<double>(mass));
  target = target < mass ? target : mass - 1;
  const int id = src.first_beyond(none, [&](float z, int id) {
    const uint32_t key = order_of(z);
    return key > p_key || (key == p_key && id <= p_tie) ? w_k(z, id) : u64{0};
  }, target);
  return Drawn{id, static_cast<double>(mass) / one};
}

template <typename In>
__global__ void __launch_bounds__(kRowT)
k_sample_row(Logits<In> L, Settings S, const int32_t* __restrict__ rowsel, int64_t c0, Summary A, const float* __restrict__ uniform, int unit_bits, SampleOut out) {
  extern __shared__ u64 s_unit[];
  __shared__ RowShared s;
  const int64_t m = blockIdx.x, row = rowsel ? rowsel[c0 + m] : c0 + m;
  const float* const unit_max = A.unit + m * L.units;
  const double *const mass_of = A.mass + m * L.units, *const sum_of = A.sum + m * L.units;
  const In* const z = L.row(m);
  float top = -INFINITY;
  for (int u = threadIdx.x; u < L.units; u += kRowT) top = fmaxf(top, unit_max[u]);
  top = block_reduce(top, s, [](float a, float b) { return fmaxf(a, b); });
  if (top == -INFINITY) {                                    // nothing to draw from
    if (threadIdx.x == 0) {
      out.ids[row] = -1;
      if (out.logp) out.logp[row] = 0.f;
      if (out.logq) out.logq[row] = 0.f;
    }
    return;
  }
  const double t = S.t(row), inv_t = 1.0 / t;
  int k = S.k(row);
  double p = S.p(row), mp = S.m(row);
  if (k >= L.V || k < 0) k = 0;
  if (!(p < 1.0)) p = 1.0;
  mp = mp > 0.0 ? fmin(mp, 1.0) : 0.0;
  double u = uniform[row];
  u = u > 0.0 ? fmin(u, 1.0) : 0.0;
  double sum = 0.0;                                          // of exp(z - top): the log-prob of the softmax itself
  for (int i = threadIdx.x; i < L.units; i += kRowT) sum += sum_of[i] * weight_of(unit_max[i], top, 1.0);
  block_excl_scan(sum, s.dscan, &sum);
  int id = -1;
  double kept = 1.0;
  if (!(t > 0.0)) {                                          // greedy: the first of the largest
    int first = INT32_MAX;
    for (int i = threadIdx.x; i < L.units; i += kRowT)
      if (unit_max[i] == top && i < first) first = i;
    first = -static_cast<int>(wave_max(-first));
    if (threadIdx.x == 0) s.found_id = INT32_MAX;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) atomicMin(&s.found_id, first);
    __syncthreads();
    const int unit = s.found_id;
    __syncthreads();
    if (threadIdx.x == 0) s.found_id = INT32_MAX;
    __syncthreads();
    const int v = unit * kUnit + threadIdx.x;
    if (v < L.V && logit(z[v]) == top) atomicMin(&s.found_id, v);
    __syncthreads();
    id = s.found_id;
  } else if (k == 0 && p == 1.0 && mp == 0.0) {              // no filter: by the units' masses
    double before = 0.0, total = 0.0;
    for (int i = threadIdx.x; i < L.units; i += kRowT) total += mass_of[i] * weight_of(unit_max[i], top, inv_t);
    block_excl_scan(total, s.dscan, &kept);
    const double target = u * kept;
    if (threadIdx.x == 0) s.found_id = -1;
    int unit = -1;
    for (int u0 = 0; u0 < L.units && unit < 0; u0 += kRowT) {
      const int i = u0 + threadIdx.x;
      const double mine = i < L.units ? mass_of[i] * weight_of(unit_max[i], top, inv_t) : 0.0;
      double all;
      const double excl = before + block_excl_scan(mine, s.dscan, &all);
      // the running sum of the unit's end as the next unit's start sees it; of several the first
      if (mine > 0.0 && excl + mine > target) atomicMin(reinterpret_cast<unsigned*>(&s.found_id), static_cast<unsigned>(i));
      __syncthreads();
      unit = s.found_id;
      if (i == unit) s.found_drest = target - excl;
      before += all;
      __syncthreads();
    }
    double rest = INFINITY;                                  // u = 1: the last token that has a weight
    if (unit >= 0) {
      rest = s.found_drest;
    } else {
      for (unit = L.units - 1; unit > 0 && !(mass_of[unit] * weight_of(unit_max[unit], top, inv_t) > 0.0);) --unit;
    }
    __syncthreads();
    if (threadIdx.x == 0) s.found_id = -1;
    const int v = unit * kUnit + threadIdx.x;
    const float x = v < L.V ? logit(z[v]) : -INFINITY;
    const double mine = x > -INFINITY ? weight_of(x, top, inv_t) : 0.0;
    double all;
    const double excl = block_excl_scan(mine, s.dscan, &all);
    if (mine > 0.0 && excl + mine > rest) atomicMin(reinterpret_cast<unsigned*>(&s.found_id), static_cast<unsigned>(v));
    __syncthreads();
    id = s.found_id;
    __syncthreads();
    if (id < 0) {                                            // the unit's sum, added up in another order, ends above the target: its last token
      if (mine > 0.0) atomicMax(&s.found_id, v);
      __syncthreads();
      id = s.found_id;
    }
  } else {
    const RowSource<In> src{z, L.V, L.units, unit_max, s, s_unit};
    const Drawn d = draw(src, s, top, inv_t, k, p, mp, u, unit_bits);
    id = d.id;
    kept = d.kept;
  }
  if (threadIdx.x != 0) return;
  out.ids[row] = id;
  const float zi = logit(z[id]);
  const double gap = zi == top ? 0.0 : static_cast<double>(zi) - static_cast<double>(top);
  if (out.logp) out.logp[row] = static_cast<float>(gap - log(sum));
  if (out.logq) out.logq[row] = t > 0.0 ? static_cast<float>((gap == 0.0 ? 0.0 : gap * inv_t) - log(kept)) : 0.f;
}
// what the call defines on rows that are not selected
__global__ void __launch_bounds__(256)
k_sample_clear(SampleOut out, int64_t n_rows) {
  const int64_t stride = static_cast<int64_t>(gridDim.x) * 256;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < n_rows; i += stride) {
    out.ids[i] = -1;
    if (out.logp) out.logp[i] = 0.f;
    if (out.logq) out.logq[i] = 0.f;
  }
}

// ------------------------------------------------------------------ logits of a head, row after row
template <class C>
__device__ __forceinline__ void plain_tile(const uint16_t* __restrict__ W, const uint16_t* __restrict__ H, int d, int V, const int32_t* __restrict__ rowsel,
                                           int64_t c0, int64_t mc, int tile_m, int tile_n, bool w_once, float* __restrict__ Z, int64_t Vp, uint16_t* lds) {
  constexpr int kPitch = C::WTM * 4 + 16, kStage = 16 * kPitch;   // a wavefront's sixteen rows on their way out
  static_assert(C::WM * C::WN * kStage <= Ring2Cfg<C>::LDS_BYTES, "the stages fit the tile buffers");
  const int m0 = tile_m * C::BM;
  const int64_t n0 = static_cast<int64_t>(tile_n) * C::BN;
  floatx4 acc[C::MI][C::NI];
  logit_tile<C>(W, H, d, V, rowsel, c0, mc, m0, n0, w_once, lds, acc);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave / C::WN, wn = wave % C::WN;
  char* const stage = reinterpret_cast<char*>(lds) + wave * kStage;
  __syncthreads();
  constexpr int kLanes = C::WTM / 4, kRows = kWave / kLanes;
  const int v = m0 + wm * C::WTM + lane % kLanes * 4;
#pragma unroll
  for (int j = 0; j < C::NI; ++j) {
#pragma unroll
    for (int i = 0; i < C::MI; ++i) *reinterpret_cast<floatx4*>(stage + (lane & 15) * kPitch + (i * 16 + (lane >> 4) * 4) * 4) = acc[i][j];
    __builtin_amdgcn_wave_barrier();
    const int64_t r0 = n0 + wn * C::WTN + j * 16 + lane / kLanes;
#pragma unroll
    for (int q = 0; q < 16 / kRows; ++q)
      if (r0 + q * kRows < mc)                               // past V: entries of the row's pitch that nobody reads
        *reinterpret_cast<floatx4*>(Z + (r0 + q * kRows) * Vp + v) = *reinterpret_cast<const floatx4*>(stage + (q * kRows + lane / kLanes) * kPitch + lane % kLanes * 16);
    __builtin_amdgcn_wave_barrier();
  }
  __syncthreads();
}
template <class C>
__device__ __forceinline__ void plain_tiles(const uint16_t* __restrict__ W, const uint16_t* __restrict__ H, int d, int V, const int32_t* __restrict__ rowsel, int64_t c0,
                                            int64_t mc, int tiles_m, int tiles_n, int panel, float* __restrict__ Z, int64_t Vp, uint16_t* lds, int halved) {
  const bool w_once = tiles_n == 1 && beyond_cache(d, V, kLogitsOnceBytes);
  for (int it = 0; it < kTilesPerWg; ++it) {
    int tile_m, tile_n;
    using Half = std::conditional_t<C::BN == HalfCfg::BN * 2, HalfCfg, HalfNarrowCfg>;
    const HalfTile h = half_tile<Half>(tiles_m, tiles_n, panel, halved, it, mc, &tile_m, &tile_n);
    if (h == HalfTile::kNone) continue;
    if (h == HalfTile::kHalf) plain_tile<Half>(W, H, d, V, rowsel, c0, mc, tile_m, tile_n, false, Z, Vp, lds);
    else plain_tile<C>(W, H, d, V, rowsel, c0, mc, tile_m, tile_n, w_once, Z, Vp, lds);
  }
}
__global__ void __launch_bounds__(Cfg::T)
k_sample_tiles(const uint16_t* __restrict__ W, const uint16_t* __restrict__ H, int d, int V, const int32_t* __restrict__ rowsel, int64_t c0, int64_t mc, int tiles_m,
               int tiles_n, int panel, int halved, float* __restrict__ Z, int64_t Vp) {
  __shared__ __attribute__((aligned(16))) uint16_t lds[kLogitLds / 2];
  plain_tiles<Cfg>(W, H, d, V, rowsel, c0, mc, tiles_m, tiles_n, panel, Z, Vp, lds, halved);
}
__global__ void __launch_bounds__(NarrowCfg::T)
k_sample_narrow(const uint16_t* __restrict__ W, const uint16_t* __restrict__ H, int d, int V, const int32_t* __restrict__ rowsel, int64_t c0, int64_t mc, int tiles_m,
                int halved, float* __restrict__ Z, int64_t Vp) {
  __shared__ __attribute__((aligned(16))) uint16_t lds[kNarrowLds / 2];
  plain_tiles<NarrowCfg>(W, H, d, V, rowsel, c0, mc, tiles_m, 1, kGN, Z, Vp, lds, halved);
}
template <int NI, int PPW>
__global__ void __launch_bounds__(kFewT)
k_sample_few(const uint16_t* __restrict__ W, const uint16_t* __restrict__ H, int d, int V, const int32_t* __restrict__ rowsel, int n_sel, int per, float* __restrict__ Z,
             int64_t stride) {
  few_logits<NI, PPW, false>(W, H, d, V, rowsel, n_sel, per, Z, stride, [](int, int, float, float, float, float) {});
}

// ------------------------------------------------------------------ host side
constexpr int64_t kSampleRows = 4096;                        // rows of a chunk: of given logits, ...
constexpr int64_t kHeadRows = 1024;                          // ... of a head, whose logits are kept on the way
struct SampleWs {
  Summary A;
  float* z;
  double* z64;
  char* room;
  size_t room_bytes;
  size_t bytes;
};
int units_of(int V) { return static_cast<int>(cdiv(V, kUnit)); }
void carve(Carver& c, SampleWs& w, int64_t rows, int V) {
  w = SampleWs{};
  const size_t units = static_cast<size_t>(rows) * units_of(V);
  w.A.group = c.take<float>(units * kGroupsPerUnit);
  w.A.unit = c.take<float>(units);
  w.A.mass = c.take<double>(units);
  w.A.sum = c.take<double>(units);
  w.bytes = c.off;
}
void carve(Carver& c, SampleWs& w, int64_t rows, int d, int V, umas_dtype dt) {
  carve(c, w, rows, V);
  if (dt == UMAS_BF16) {
    w.z = c.take<float>(rows <= few_rows(d) ? few_floats(rows, V) : static_cast<size_t>(rows) * round_up(V, 256));
  } else {
    w.z64 = c.take<double>(static_cast<size_t>(rows) * V);
    w.room_bytes = align_up(f32::score_room(rows, V));
    w.room = c.take<char>(w.room_bytes);
  }
  w.bytes = c.off;
}
size_t head_bytes(int64_t n_sel, int64_t cap, int d, int V, umas_dtype dt) {
  Carver c(nullptr);
  SampleWs w;
  carve(c, w, std::min(std::max<int64_t>(n_sel, 1), cap), d, V, dt);
  return w.bytes;
}
size_t logits_bytes(int64_t n_rows, int V) {
  Carver c(nullptr);
  SampleWs w;
  carve(c, w, std::min(std::max<int64_t>(n_rows, 1), kSampleRows), V);
  return w.bytes;
}
umas_status check_sampling(const umas_sampling* s, Settings* to, int V) {
  UMAS_REQUIRE(s, UMAS_EINVAL, "sampling must not be NULL");
  UMAS_REQUIRE(V <= kMaxSampleV, UMAS_ESHAPE, "V=%d exceeds %d", V, kMaxSampleV);
  UMAS_REQUIRE(s->temperature_of || s->temperature >= 0.0, UMAS_EINVAL, "temperature must be a number >= 0");
  UMAS_REQUIRE(s->top_p_of || (s->top_p >= 0.0 && s->top_p <= 1.0), UMAS_EINVAL, "top_p outside [0,1]");
  UMAS_REQUIRE(s->min_p_of || (s->min_p >= 0.0 && s->min_p <= 1.0), UMAS_EINVAL, "min_p outside [0,1]");
  UMAS_REQUIRE(s->top_k_of || s->top_k >= 0, UMAS_EINVAL, "top_k must be >= 0 (0: all)");
  *to = Settings{s->temperature, s->top_p, s->min_p, s->top_k, s->temperature_of, s->top_p_of, s->min_p_of, s->top_k_of};
  return UMAS_OK;
}
int bits_of(int V) {
  int b = 0;
  while ((int64_t{1} << b) < V) ++b;
  return std::min(52, 62 - b);
}
template <typename In>
umas_status sample_rows(const Logits<In>& L, const Settings& S, const int32_t* rowsel, int64_t c0, int64_t rows, const SampleWs& w, const float* u, const SampleOut& out,
                        hipStream_t st) {
  hipLaunchKernelGGL(k_sample_open<In>, dim3(cdiv(L.units, kOpenUnits), static_cast<unsigned>(rows)), dim3(kOpenT), 0, st, L, S, rowsel, c0, w.A);
  UMAS_LAUNCHED("k_sample_open");
  hipLaunchKernelGGL(k_sample_row<In>, dim3(static_cast<unsigned>(rows)), dim3(kRowT), L.units * sizeof(u64), st, L, S, rowsel, c0, w.A, u, bits_of(L.V), out);
  UMAS_LAUNCHED("k_sample_row");
  return UMAS_OK;
}

}  // namespace
}  // namespace umas

using namespace umas;

extern "C" size_t umas_sample_logits_workspace_bytes(int64_t n_rows, int32_t V) {
  if (n_rows < 0 || V < 1 || V > kMaxSampleV) return 0;
  return logits_bytes(n_rows, V);
}

extern "C" umas_status umas_sample_logits(const void* logits, umas_dtype dtype, int64_t n_rows, int32_t V, int64_t row_stride, const float* u,
                                          const umas_sampling* sampling, int32_t* ids, float* logp, float* logq, void* workspace, size_t workspace_bytes,
                                          void* hip_stream) {
  UMAS_REQUIRE(dtype == UMAS_F32 || dtype == UMAS_BF16, UMAS_EDTYPE, "dtype=%d is neither F32 nor BF16", static_cast<int>(dtype));
  UMAS_REQUIRE(n_rows >= 0, UMAS_EINVAL, "negative row count");
  UMAS_REQUIRE(V >= 1, UMAS_ESHAPE, "V=%d must be positive", V);
  Settings S;
  umas_status s = check_sampling(sampling, &S, V);
  if (s != UMAS_OK) return s;
  UMAS_REQUIRE(row_stride >= V || n_rows <= 1, UMAS_EINVAL, "row_stride=%lld is less than V=%d", static_cast<long long>(row_stride), V);
  UMAS_REQUIRE((logits && u && ids) || n_rows == 0, UMAS_EINVAL, "logits, u and ids must not be NULL");
  UMAS_REQUIRE(reinterpret_cast<uintptr_t>(logits) % (dtype == UMAS_BF16 ? 2 : 4) == 0, UMAS_EINVAL, "logits must be aligned to their type");
  s = check_ws(workspace, workspace_bytes, umas_sample_logits_workspace_bytes(n_rows, V));
  if (s != UMAS_OK) return s;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  prof_mark(st);
  Carver c(workspace);
  SampleWs w;
  carve(c, w, std::min(std::max<int64_t>(n_rows, 1), kSampleRows), V);
  for (int64_t c0 = 0; c0 < n_rows; c0 += kSampleRows) {
    const int64_t rows = std::min(kSampleRows, n_rows - c0);
    const SampleOut out{ids, logp, logq};
    if (dtype == UMAS_BF16)
      s = sample_rows(Logits<uint16_t>{static_cast<const uint16_t*>(logits) + c0 * row_stride, row_stride, V, units_of(V)}, S, nullptr, c0, rows, w, u, out, st);
    else
      s = sample_rows(Logits<float>{static_cast<const float*>(logits) + c0 * row_stride, row_stride, V, units_of(V)}, S, nullptr, c0, rows, w, u, out, st);
    if (s != UMAS_OK) return s;
  }
  return UMAS_OK;
}

extern "C" size_t umas_sample_tokens_workspace_bytes_min(int64_t n_sel, int32_t d, int32_t V, umas_dtype dtype) {
  if (n_sel < 0 || d < 1 || V < 1 || V > kMaxSampleV) return 0;
  return head_bytes(n_sel, 256, d, V, dtype);
}
extern "C" size_t umas_sample_tokens_workspace_bytes(int64_t n_sel, int32_t d, int32_t V, umas_dtype dtype) {
  if (n_sel < 0 || d < 1 || V < 1 || V > kMaxSampleV) return 0;
  return head_bytes(n_sel, kHeadRows, d, V, dtype);
}

extern "C" umas_status umas_sample_tokens(const void* H, const void* W, umas_dtype dtype, int64_t n_rows, int32_t d, int32_t V, const int32_t* rowsel, int64_t n_sel,
                                          const float* u, const umas_sampling* sampling, int32_t* ids, float* logp, float* logq, void* workspace,
                                          size_t workspace_bytes, void* hip_stream) {
  umas_status s = check_model_args(H, W, dtype, n_rows, d, V, ids, rowsel, n_sel);
  if (s != UMAS_OK) return s;
  Settings S;
  s = check_sampling(sampling, &S, V);
  if (s != UMAS_OK) return s;
  UMAS_REQUIRE(u || n_rows == 0, UMAS_EINVAL, "u must not be NULL");
  UMAS_REQUIRE(n_sel < (1LL << 31), UMAS_ESHAPE, "at most 2^31-1 selected rows");
  s = check_ws(workspace, workspace_bytes, umas_sample_tokens_workspace_bytes_min(n_sel, d, V, dtype));
  if (s != UMAS_OK) return s;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  prof_mark(st);
  const SampleOut out{ids, logp, logq};
  if (rowsel && n_rows > 0) {
    hipLaunchKernelGGL(k_sample_clear, dim3(static_cast<unsigned>(std::min<int64_t>(n_rows / 256 + 1, 1024))), dim3(256), 0, st, out, n_rows);
    UMAS_LAUNCHED("k_sample_clear");
  }
  if (n_sel == 0) return UMAS_OK;
  int64_t cap = std::min(n_sel, kHeadRows);
  while (cap > 256 && head_bytes(n_sel, cap, d, V, dtype) > workspace_bytes) cap = std::max<int64_t>(round_up(cap / 2, 256), 256);
  Carver c(workspace);
  SampleWs w;
  carve(c, w, cap, d, V, dtype);
  for (int64_t c0 = 0; c0 < n_sel; c0 += cap) {
    const int64_t rows = std::min(cap, n_sel - c0);
    if (dtype == UMAS_BF16) {
      const uint16_t *Wb = static_cast<const uint16_t*>(W), *Hb = static_cast<const uint16_t*>(H);
      int64_t stride = round_up(V, 256);
      if (cap <= few_rows(d)) {                              // one chunk
        const int parts = few_workgroups(V), per = few_per(V, parts);
        stride = static_cast<int64_t>(parts) * per * 16;
        with_few(d, rows, [&](auto ni, auto ppw) {
          hipLaunchKernelGGL((k_sample_few<decltype(ni)::value, decltype(ppw)::value>), dim3(parts), dim3(kFewT), 0, st, Wb, Hb, d, V, rowsel, static_cast<int>(rows), per,
                             w.z, stride);
        });
        UMAS_LAUNCHED("k_sample_few");
      } else if (rows <= NarrowCfg::BN) {
        const int tiles = static_cast<int>(cdiv(V, NarrowCfg::BM));
        const int halved = rows > HalfNarrowCfg::BN ? halved_tiles(tiles, 1, 2) : 0;
        hipLaunchKernelGGL(k_sample_narrow, score_grid(tiles, 1, kGN, halved), dim3(NarrowCfg::T), 0, st, Wb, Hb, d, V, rowsel, c0, rows, tiles, halved, w.z, stride);
        UMAS_LAUNCHED("k_sample_narrow");
      } else {
        const int tiles = static_cast<int>(cdiv(V, Cfg::BM)), tiles_n = static_cast<int>(cdiv(rows, Cfg::BN)), panel = row_panel(tiles_n, d);
        const int halved = halved_tiles(tiles, tiles_n);
        hipLaunchKernelGGL(k_sample_tiles, score_grid(tiles, tiles_n, panel, halved), dim3(Cfg::T), 0, st, Wb, Hb, d, V, rowsel, c0, rows, tiles, tiles_n, panel, halved, w.z,
                           stride);
        UMAS_LAUNCHED("k_sample_tiles");
      }
      s = sample_rows(Logits<float>{w.z, stride, V, units_of(V)}, S, rowsel, c0, rows, w, u, out, st);
    } else {
      const float* Hf = static_cast<const float*>(H) + (rowsel ? 0 : c0 * d);
      s = f32::score(static_cast<const float*>(W), Hf, d, V, rowsel ? rowsel + c0 : nullptr, rows, nullptr, w.room, w.room_bytes,
                     f32::ScoreOut{w.z64, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr}, st);
      if (s == UMAS_OK) s = sample_rows(Logits<double>{w.z64, V, V, units_of(V)}, S, rowsel, c0, rows, w, u, out, st);
    }
    if (s != UMAS_OK) return s;
  }
  return UMAS_OK;
}
