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
#include "umas_lanes.h"

namespace umas {
namespace {

typedef unsigned long long u64;
constexpr int kUnit = 1024, kGroup = 64, kGroupsPerUnit = kUnit / kGroup;
constexpr int kPerLane = kUnit / kWave;                       // logits of a unit that a lane holds
constexpr int kMaxSampleV = UMAS_MAX_SAMPLE_V;

// ------------------------------------------------------------------ weights
// exp((z - top) c), c = log2 e / T, for z <= top, as 2^n times a polynomial in the rest f, |f| <= 1/2: the interpolation of (2^f - 1) / f at eight Chebyshev nodes, times f, plus
// 1; off by 2.2e-12 of itself.  Whole and rest come from an addition that pushes the rest out of a float64, the power from an addition to the exponent's bits: the conversions and
// ldexp that the compiler would take for them cost four times a multiply-add each (39 million logits, with eleven coefficients, rint and ldexp 58 us).
// The largest logit's own weight is exactly 1, equal logits' weights are equal; below 2^-1000 is 2^-1000.
struct Weigh {
  double top, c;
  __device__ __forceinline__ double operator()(float z) const {
    constexpr double kPush = 6755399441055744.0;             // 3 * 2^51
    const double t = fmax((static_cast<double>(z) - top) * c, -1000.0);
    const double pushed = t + kPush, f = t - (pushed - kPush);
    double p = 1.3250805522890813e-06;
    p = fma(p, f, 1.530370071143596e-05);
    p = fma(p, f, 0.00015403475186508562);
    p = fma(p, f, 0.0013333478473685106);
    p = fma(p, f, 0.009618129135236166);
    p = fma(p, f, 0.05550410906325867);
    p = fma(p, f, 0.24022650695888503);
    p = fma(p, f, 0.6931471805568324);
    p = fma(p, f, 1.0);
    return __hiloint2double(__double2hiint(p) + (__double2loint(pushed) << 20), __double2loint(p));
  }
};
constexpr double kNoWeight = 1e-290;                          // what is no more than this is not drawn, u = 0 or not
constexpr double kLog2e64 = 1.4426950408889634074;
// A temperature whose inverse leaves no finite number: 0 times it has to stay 0.
__device__ __forceinline__ double scale_of(double t) { return fmin(kLog2e64 / t, 1e300); }
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
// Where the largest logit is +infinity: tokens that are as large share the mass, others have none.
__device__ __forceinline__ float or_none(float z, bool infinite) { return infinite ? (z == INFINITY ? 0.f : -INFINITY) : z; }
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
__device__ __forceinline__ double lanes_sum(double x) {       // of the wavefront, in every lane
  auto other = [](double v, auto j) {
    return __longlong_as_double(static_cast<long long>(lane_xor<decltype(j)::value>(static_cast<u64>(__double_as_longlong(v)))));
  };
  x += other(x, std::integral_constant<int, 1>());
  x += other(x, std::integral_constant<int, 2>());
  x += other(x, std::integral_constant<int, 4>());
  x += other(x, std::integral_constant<int, 8>());
  x += other(x, std::integral_constant<int, 16>());
  x += other(x, std::integral_constant<int, 32>());
  return x;
}
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
    const bool drawn = t > 0.0, infinite = top == INFINITY;
    if (infinite)
#pragma unroll
      for (int i = 0; i < kPerLane; ++i) x[i] = or_none(x[i], true);
    const float ref = infinite ? 0.f : top;
    if (drawn) {
      const Weigh w{ref, scale_of(t)};
#pragma unroll
      for (int i = 0; i < kPerLane; ++i) mass += w(x[i]);
      mass = lanes_sum(mass);
    }
    if (drawn && t == 1.0) {
      sum = mass;
    } else {
      constexpr float kLog2e = 1.44269504088896341f;
#pragma unroll
      for (int i = 0; i < kPerLane; ++i) sum += static_cast<double>(__builtin_amdgcn_exp2f((x[i] - ref) * kLog2e));
      sum = lanes_sum(sum);
    }
  }
  if (lane == 0) {
    out.unit[at] = top;
    out.mass[at] = mass;
    out.sum[at] = sum;
  }
}

// ------------------------------------------------------------------ second launch
constexpr int kBins = 2048;
constexpr int kTopRank = 64;
constexpr int kListCap = 4096, kRanked = 256;                // tokens of a list, and of one that is ordered by comparing all with all
constexpr int kGroupCap = 1024;
template <int T>
struct RowShared {
  u64 bins[kBins];                                           // masses or counts
  float list_z[kListCap];
  int list_id[kListCap];
  float top[T / kWave][kWave];
  u64 scan[17];
  double dscan[17];
  u64 found_above, found_here, found_rest;
  double found_drest;
  uint32_t found_bin;
  int found_id, n_list, n_groups;
};
// The logits of a row of T threads, a unit to a wavefront at a time.
template <typename In, int T>
struct RowSource {
  const In* z;
  int V, units;
  const float* unit_max;                                     // of the row
  bool infinite;                                             // its largest is
  __device__ __forceinline__ float at(int v) const { return v < V ? or_none(logit(z[v]), infinite) : -INFINITY; }
  // f(z, token) for every token with z > -infinity, and z >= lo; others may come.  `after` once a unit, by its wavefront, also where the unit has none
  template <class F, class G>
  __device__ __forceinline__ void each(float lo, F f, G after) const {
    for (int u = threadIdx.x >> 6; u < units; u += T / kWave) {
      const float top = unit_max[u];
      if (top >= lo && top > -INFINITY) {
        float x[kPerLane];
        load_unit(z, V, u, x);
#pragma unroll
        for (int i = 0; i < kPerLane; ++i) {
          const float zi = or_none(x[i], infinite);
          if (zi > -INFINITY) f(zi, token_of<In>(u, i));
        }
      }
      after(u);
    }
  }
  template <class F>
  __device__ __forceinline__ void each(float lo, F f) const { each(lo, f, [](int) {}); }
};
// Listed tokens [a, b).
template <int T>
struct ListSource {
  const RowShared<T>* s;
  int a, b;
  template <class F>
  __device__ __forceinline__ void each(float, F f) const {
    for (int i = a + static_cast<int>(threadIdx.x); i < b; i += T) f(s->list_z[i], s->list_id[i]);
  }
};
template <int T>
__device__ __forceinline__ u64 block_total(u64 v, RowShared<T>& s) {
  u64 total;
  block_excl_scan(v, s.scan, &total);
  __syncthreads();
  return total;
}
struct Border {
  uint32_t key;
  u64 above, here;                                           // sums over larger keys, and over those equal to it
};
// The key at which the sum of val over the keys in falling order reaches `need`, 1 <= need <= the sum over all.  Eleven bits at a time from the top; whole
// numbers, so that the order in which the additions come is nothing.
template <int T, class Source, class K, class F>
__device__ __forceinline__ Border border_of(const Source& src, RowShared<T>& s, float lo, K key_of, F val, u64 need) {
  constexpr int kEach = kBins / T;
  Border b{0, 0, 0};
#pragma unroll 1
  for (int digit = 0; digit < 3; ++digit) {
    const int shift = digit == 0 ? 21 : digit == 1 ? 10 : 0, known = digit == 0 ? 32 : digit == 1 ? 21 : 10;
    const uint32_t mask = (1u << (known - shift)) - 1;
    for (int i = threadIdx.x; i < kBins; i += T) s.bins[i] = 0;
    __syncthreads();
    src.each(lo, [&](float z, int id) {
      const uint32_t key = key_of(z, id);
      if (digit != 0 && (key ^ b.key) >> known) return;
      const u64 v = val(z, id);
      if (v) atomicAdd(&s.bins[(key >> shift) & mask], v);
    });
    __syncthreads();
    const int hi = kBins - 1 - kEach * static_cast<int>(threadIdx.x);   // from the largest bin down
    u64 sum = 0, total;
#pragma unroll
    for (int i = 0; i < kEach; ++i) sum += s.bins[hi - i];
    u64 above = b.above + block_excl_scan(sum, s.scan, &total);
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const u64 x = s.bins[hi - i];
      if (above < need && need <= above + x) {
        s.found_bin = static_cast<uint32_t>(hi - i);
        s.found_above = above;
        s.found_here = x;
      }
      above += x;
    }
    __syncthreads();
    b.key |= s.found_bin << shift;
    b.above = s.found_above;
    b.here = s.found_here;
    __syncthreads();
  }
  return b;
}

struct SampleOut {
  int32_t* ids;
  float *logp, *logq;
};
// A row's settings and what the first launch says about it.
struct RowDraw {
  float top;
  Weigh w;
  int k;                                                     // 0: none
  double p, m, u;                                            // p = 1, m = 0: none
  double all;                                                // the mass of all tokens, in units of the largest weight
  double one;                                                // 1 in units of the whole numbers
  __device__ __forceinline__ bool by_min() const { return m > 0.0; }
  __device__ __forceinline__ u64 whole(double x) const {     // x * one, one at most 2^51, rounded to nearest by the addition
    return static_cast<u64>(__double_as_longlong(fma(x, one, 4503599627370496.0))) & ((u64{1} << 52) - 1);
  }
  __device__ __forceinline__ u64 weight(float z) const {     // of the tokens that min_p leaves
    const double x = w(z);
    return x >= m ? whole(x) : u64{0};
  }
  __device__ __forceinline__ u64 share(double part, u64 of) const {   // the least whole number that reaches part of a mass
    const u64 n = static_cast<u64>(ceil(part * static_cast<double>(of)));
    return n < 1 ? 1 : n > of ? of : n;
  }
  __device__ __forceinline__ u64 target(u64 mass) const {
    const u64 t = static_cast<u64>(u * static_cast<double>(mass));
    return t < mass ? t : mass - 1;
  }
};
// Where what is kept ends: a token is in if its logit orders above the key, or at it with a token up to `tie`.
struct Cut {
  uint32_t key = 0;
  int tie = INT32_MAX;
  __device__ __forceinline__ bool in(float z, int id) const {
    const uint32_t o = order_of(z);
    return o > key || (o == key && id <= tie);
  }
};
struct Drawn {
  int id;
  u64 mass;                                                  // the kept one
};
// The cut after `need` of val, of which `each_one` at the border's logit; *mass: the sum of what is in.
template <int T, class Source, class F>
__device__ __forceinline__ Cut cut_at(const Source& src, RowShared<T>& s, float lo, F val, u64 need, u64* mass) {
  const Border b = border_of(src, s, lo, [](float z, int) { return order_of(z); }, val, need);
  Cut c;
  c.key = b.key;
  // how many of the tokens at the border, which have the same value each
  const u64 count = block_total([&] {
    u64 n = 0;
    src.each(lo, [&](float z, int id) { n += order_of(z) == b.key && val(z, id); });
    return n;
  }(), s);
  const u64 one = b.here / count, ties = (need - b.above + one - 1) / one;
  if (ties < count)                                          // the lowest tokens
    c.tie = static_cast<int>(~border_of(src, s, lo, [](float, int id) { return ~static_cast<uint32_t>(id); },
                                        [&](float z, int id) { return u64{order_of(z) == b.key && val(z, id)}; }, ties).key);
  *mass = b.above + ties * one;
  return c;
}
// The token at which the running mass of val, in rising order of tokens, passes `target`, which is less than all of it; unit_sum: the units' sums of val.
template <typename In, int T, class F>
__device__ __forceinline__ int token_beyond(const RowSource<In, T>& row, RowShared<T>& s, const u64* unit_sum, F val, u64 target) {
  u64 before = 0;
  if (threadIdx.x == 0) s.found_id = -1;
  int unit = -1;
  for (int u0 = 0; u0 < row.units && unit < 0; u0 += T) {
    const int u = u0 + threadIdx.x;
    const u64 mine = u < row.units ? unit_sum[u] : 0;
    u64 total;
    const u64 excl = before + block_excl_scan(mine, s.scan, &total);
    if (excl <= target && target < excl + mine) {
      s.found_id = u;
      s.found_rest = target - excl;
    }
    before += total;
    __syncthreads();
    unit = s.found_id;
  }
  u64 rest = s.found_rest;
  __syncthreads();
  constexpr int kEach = kUnit / T;
  const int v = unit * kUnit + static_cast<int>(threadIdx.x) * kEach;
  u64 mine[kEach], sum = 0, total;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const float x = row.at(v + i);
    mine[i] = x > -INFINITY ? val(x, v + i) : 0;
    sum += mine[i];
  }
  u64 excl = block_excl_scan(sum, s.scan, &total);
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    if (excl <= rest && rest < excl + mine[i]) s.found_id = v + i;
    excl += mine[i];
  }
  __syncthreads();
  return s.found_id;
}

// Any row, whatever its logits are: the thresholds by whole passes over it.
template <typename In, int T>
__device__ __noinline__ Drawn draw_by_passes(const RowSource<In, T>& row, RowShared<T>& s, u64* s_unit, const RowDraw& d) {
  const float none = -INFINITY;
  Cut first, run;
  u64 mass;
  if (d.k > 0) {
    u64 have = 0;
    row.each(none, [&](float, int) { ++have; });
    have = block_total(have, s);
    if (static_cast<u64>(d.k) < have) first = cut_at(row, s, none, [](float, int) { return u64{1}; }, static_cast<u64>(d.k), &mass);
  }
  auto of_first = [&](float z, int id) { return first.in(z, id) ? d.weight(z) : u64{0}; };
  mass = 0;
  row.each(none, [&](float z, int id) { mass += of_first(z, id); });
  mass = block_total(mass, s);
  if (d.p < 1.0) run = cut_at(row, s, none, of_first, d.share(d.p, mass), &mass);
  auto kept = [&](float z, int id) { return run.in(z, id) ? of_first(z, id) : u64{0}; };
  u64 sum = 0;
  row.each(none, [&](float z, int id) { sum += kept(z, id); }, [&](int u) {
    sum = wave_sum(sum);
    if ((threadIdx.x & 63) == 0) s_unit[u] = sum;
    sum = 0;
  });
  __syncthreads();
  return Drawn{token_beyond(row, s, s_unit, kept, d.target(mass)), mass};
}

// ---- the tokens in front
// A number that at least so many logits reach: the threads take the maximum over the row's groups in turn, and the rank-th largest of theirs is it.
template <int T>
__device__ __forceinline__ float front_bound(const float* __restrict__ group_max, int groups, RowShared<T>& s) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, rank = min(kTopRank, max(groups / 4, 1));
  float x = -INFINITY;
  for (int g = threadIdx.x; g < groups; g += T) x = fmaxf(x, group_max[g]);
  x = sorted_desc(x);
  s.top[wave][lane] = x;
  __syncthreads();
  x = s.top[0][lane];
#pragma unroll
  for (int w = 1; w < T / kWave; ++w) x = merged(x, s.top[w][lane]);
  __syncthreads();
  return __shfl(x, rank - 1, kWave);
}
// Lists the tokens with z >= bound; false: more than there is room for.
template <typename In, int T>
__device__ __forceinline__ bool list_front(const RowSource<In, T>& row, const float* __restrict__ group_max, float bound, RowShared<T>& s) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, groups = row.units * kGroupsPerUnit;
  int* const s_group = reinterpret_cast<int*>(s.bins);
  if (threadIdx.x == 0) s.n_list = s.n_groups = 0;
  __syncthreads();
  for (int g = threadIdx.x; g < groups; g += T) {
    const float x = group_max[g];
    if (x >= bound && x > -INFINITY) {
      const int at = atomicAdd(&s.n_groups, 1);
      if (at < kGroupCap) s_group[at] = g;
    }
  }
  __syncthreads();
  const int n = s.n_groups;
  if (n > kGroupCap) return false;
  constexpr int kAtOnce = 4;
  for (int i = wave; i < n; i += T / kWave * kAtOnce) {
    float x[kAtOnce];
    int id[kAtOnce];
#pragma unroll
    for (int q = 0; q < kAtOnce; ++q) {
      const int j = i + q * (T / kWave);
      id[q] = j < n ? s_group[j] * kGroup + lane : row.V;
      x[q] = row.at(id[q]);
    }
#pragma unroll
    for (int q = 0; q < kAtOnce; ++q) {
      const bool in = x[q] >= bound && x[q] > -INFINITY;
      const u64 m = __ballot(in);
      if (!m) continue;
      int at = 0;
      if (lane == 0) at = atomicAdd(&s.n_list, __popcll(m));
      at = __shfl(at, 0, kWave) + __popcll(m & ((u64{1} << lane) - 1));
      if (in && at < kListCap) {
        s.list_z[at] = x[q];
        s.list_id[at] = id[q];
      }
    }
  }
  __syncthreads();
  return s.n_list <= kListCap;
}
// What the listed tokens say, where they are enough: id -1 where they are not.  Each is compared with all of them, once by its logit and once by its number.
template <int T>
__device__ __forceinline__ Drawn draw_from_front(RowShared<T>& s, int n, float bound, bool all_listed, const RowDraw& d) {
  u64* const s_key = s.bins;                                 // [kRanked] each
  u64* const s_w = s.bins + kRanked;
  u64* const s_sorted = s.bins + 2 * kRanked;
  const int i = threadIdx.x;
  u64 key = 0, w = 0;
  if (i < n) {
    key = static_cast<u64>(order_of(s.list_z[i])) << 32 | (0xFFFFFFFFu - static_cast<uint32_t>(s.list_id[i]));
    w = d.weight(s.list_z[i]);
    s_key[i] = key;
  }
  __syncthreads();
  int rank = 0;
  if (i < n)
    for (int j = 0; j < n; ++j) rank += s_key[j] > key;
  const bool first = i < n && (d.k == 0 || rank < d.k);
  if (!first) w = 0;
  if (i < n) s_sorted[rank] = w;
  __syncthreads();
  u64 mass;
  const u64 ahead = block_excl_scan(i < n ? s_sorted[i] : 0, s.scan, &mass);   // of the i-th in falling order
  const bool whole = d.k > 0 || (d.by_min() && d.weight(bound) == 0) || all_listed;   // nothing that is not listed counts
  u64 need = mass;
  if (d.p < 1.0) {
    if (whole) need = d.share(d.p, mass);
    else {
      const double part = ceil(d.p * d.all * d.one);
      need = part < 1.0 ? 1 : static_cast<u64>(part);
    }
  }
  if ((d.k > n && !all_listed) || (!whole && (d.by_min() || d.p == 1.0 || need > mass))) return Drawn{-1, 0};
  if (i < n) {                                               // kept: whose front is shorter than what is needed
    if (ahead >= need) s_sorted[i] = 0;
    const u64 mine = s_sorted[i];
    if (mine && ahead + mine >= need) s.found_above = ahead + mine;
  }
  __syncthreads();
  mass = s.found_above;
  w = i < n ? s_sorted[rank] : 0;
  if (i < n) s_w[i] = w;
  __syncthreads();
  if (i < n && w) {
    u64 run = 0;
    const uint32_t mine = static_cast<uint32_t>(key);        // falls with the token
    for (int j = 0; j < n; ++j) run += static_cast<uint32_t>(s_key[j]) >= mine ? s_w[j] : 0;
    const u64 target = d.target(mass);
    if (target < run && run - w <= target) s.found_id = s.list_id[i];
  }
  __syncthreads();
  return Drawn{s.found_id, mass};
}

// ---- rows whose mass is spread
// The tokens below the front by their distance to it, in 1/64 of T: their counts say near which bin the border of top_p lies and in which exactly that of top_k.  A second
// pass sums what lies above for certain, by unit, and lists the tokens of the bins around; among those the borders are found as they are.  Where a border was not
// among the bins (id -1), or they hold too many, the row is gone through bit by bit.
constexpr double kBinsPerT = 64.0;
template <typename In, int T>
__device__ __forceinline__ Drawn draw_by_bins(const RowSource<In, T>& row, RowShared<T>& s, u64* s_unit, float bound, int n_front, double c, const RowDraw& d) {
  constexpr int kEach = kBins / T;
  uint32_t* const s_count = reinterpret_cast<uint32_t*>(s.bins);
  const float scale = static_cast<float>(fmin(c * (kBinsPerT / kLog2e64), 1e30));
  auto bin_of = [&](float z) { return static_cast<int>(fminf((bound - z) * scale, static_cast<float>(kBins - 1))); };
  // below this nothing counts: weights under min_p, or so small that all tokens together with them are not what top_p leaves out
  double least = d.by_min() ? d.m : d.k > 0 || d.p == 1.0 ? 0.0 : (1.0 - d.p) * d.all / row.V;
  float lo = -INFINITY;
  if (least > 0.0 && c > 0.0) {
    const double x = d.w.top + log2(least) / c;
    lo = static_cast<float>(x);
    lo -= fabsf(lo) * 1e-6f + 1e-30f;
  }
  for (int i = threadIdx.x; i < kBins; i += T) s_count[i] = 0;
  // the front's mass
  u64 front = 0;
  for (int i = threadIdx.x; i < n_front; i += T) front += d.weight(s.list_z[i]);
  front = block_total(front, s);
  row.each(lo, [&](float z, int) {
    if (z < bound && z >= lo) atomicAdd(&s_count[bin_of(z)], 1u);
  });
  __syncthreads();
  const double at_bound = d.w(bound), step = exp2(-1.0 / kBinsPerT * kLog2e64);
  u64 counts[kEach], n_mine = 0, n_all;
  double m_mine = 0.0, m_all, of[kEach];
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int b = static_cast<int>(threadIdx.x) * kEach + i;
    counts[i] = s_count[b];
    of[i] = at_bound * exp2(-(b + 0.5) / kBinsPerT * kLog2e64);
    n_mine += counts[i];
    m_mine += static_cast<double>(counts[i]) * of[i];
  }
  u64 n_before = block_excl_scan(n_mine, s.scan, &n_all);
  const double m_before = block_excl_scan(m_mine, s.dscan, &m_all);
  const double f_mass = static_cast<double>(front) / d.one;
  // the bin of the k-th token
  if (threadIdx.x == 0) {
    s.found_bin = kBins;
    s.found_drest = f_mass + m_all;
    s.found_rest = 0;
  }
  __syncthreads();
  const bool behind_counts = d.k == 0 || d.k > n_front;
  const u64 k_rest = d.k > n_front ? static_cast<u64>(d.k - n_front) : 0;   // places behind the front
  {
    u64 n = n_before;
    double m = m_before;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      if (d.k > 0 && n < k_rest && k_rest <= n + counts[i]) {
        s.found_bin = static_cast<uint32_t>(threadIdx.x * kEach + i);
        s.found_rest = k_rest - n;
        s.found_drest = f_mass + m + static_cast<double>(k_rest - n) * of[i];
      }
      n += counts[i];
      m += static_cast<double>(counts[i]) * of[i];
    }
  }
  __syncthreads();
  const int k_bin = static_cast<int>(s.found_bin);           // kBins: all are among the first k
  const u64 k_in_bin = s.found_rest;
  const double total = !d.by_min() && d.k == 0 ? d.all : s.found_drest;
  __syncthreads();
  // the bins around the border of top_p
  int b1 = 0, b2 = -1;
  if (d.p < 1.0 && behind_counts) {
    const double need = d.p * total - f_mass, off = 1e-3 * fabs(need) + 1e-6 * total;
    if (need + off > 0.0) {
      if (threadIdx.x == 0) s.found_id = s.n_groups = kBins - 1;
      __syncthreads();
      double m = m_before;
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const double next = m + static_cast<double>(counts[i]) * of[i];
        const int b = static_cast<int>(threadIdx.x) * kEach + i;
        if (need - off <= next) atomicMin(&s.found_id, b);
        if (need + off <= next) atomicMin(&s.n_groups, b);
        m = next;
      }
      __syncthreads();
      b1 = max(s.found_id - 1, 0);
      b2 = min(s.n_groups + 1, min(k_bin, kBins - 1));
      b1 = min(b1, b2);
    }
  }
  const bool by_p = d.p < 1.0;
  // tokens above b1 are in for certain; without top_p all that come before k_bin
  const int sure_end = by_p ? (b2 < 0 ? 0 : b1) : min(k_bin, kBins);
  const bool need_total = by_p && (d.k > 0 || d.by_min());   // the mass that top_p is of
  const int last = !behind_counts ? -1 : need_total || !by_p ? min(k_bin, kBins - 1) : b2;   // bins that matter
  if (threadIdx.x == 0) s.n_list = n_front;
  __syncthreads();
  u64 sure = 0, rest = 0, unit = 0;
  row.each(lo, [&](float z, int id) {
    if (!(z < bound && z >= lo)) return;
    const int b = bin_of(z);
    if (b > last) return;
    if (b == k_bin || (b >= b1 && b <= b2)) {
      const int at = atomicAdd(&s.n_list, 1);
      if (at < kListCap) {
        s.list_z[at] = z;
        s.list_id[at] = id;
      }
      return;
    }
    const u64 w = d.weight(z);
    if (b < sure_end) unit += w;
    else rest += w;
  }, [&](int u) {
    sure += unit;
    unit = wave_sum(unit);
    if ((threadIdx.x & 63) == 0) s_unit[u] = unit;
    unit = 0;
  });
  sure = block_total(sure, s);
  rest = block_total(rest, s);
  const int n_list = s.n_list;
  if (n_list > kListCap) return Drawn{-1, 0};
  // the first k: those in the bin of the k-th
  Cut first, run;
  const ListSource<T> listed{&s, 0, n_list}, front_list{&s, 0, n_front}, behind{&s, n_front, n_list};
  u64 mass;
  if (!behind_counts) first = cut_at(front_list, s, -INFINITY, [](float, int) { return u64{1}; }, static_cast<u64>(d.k), &mass);
  else if (k_bin < kBins) first = cut_at(behind, s, -INFINITY, [&](float z, int) { return u64{bin_of(z) == k_bin}; }, k_in_bin, &mass);
  auto of_first = [&](float z, int id) { return first.in(z, id) ? d.weight(z) : u64{0}; };
  auto sum_of = [&](const ListSource<T>& l) {
    u64 m = 0;
    l.each(-INFINITY, [&](float z, int id) { m += of_first(z, id); });
    return block_total(m, s);
  };
  const u64 in_front = sum_of(front_list), in_behind = sum_of(behind);
  mass = in_front + sure + in_behind + rest;
  bool sure_in = true;
  if (by_p) {
    u64 need = d.share(d.p, mass);
    if (!need_total) {
      const double part = ceil(d.p * d.all * d.one);
      need = part < 1.0 ? 1 : static_cast<u64>(part);
    }
    if (need <= in_front) {
      run = cut_at(front_list, s, -INFINITY, of_first, need, &mass);
      sure_in = false;
    } else {
      auto in_bins = [&](float z, int id) { return z < bound && bin_of(z) <= b2 ? of_first(z, id) : u64{0}; };
      u64 have = 0;
      behind.each(-INFINITY, [&](float z, int id) { have += in_bins(z, id); });
      have = block_total(have, s);
      if (need <= in_front + sure || need > in_front + sure + have) return Drawn{-1, 0};
      run = cut_at(behind, s, -INFINITY, in_bins, need - in_front - sure, &mass);
      mass += in_front + sure;
    }
  }
  auto kept = [&](float z, int id) { return run.in(z, id) ? of_first(z, id) : u64{0}; };
  if (!sure_in)
    for (int u = threadIdx.x; u < row.units; u += T) s_unit[u] = 0;
  __syncthreads();
  listed.each(-INFINITY, [&](float z, int id) {
    const u64 w = kept(z, id);
    if (w) atomicAdd(&s_unit[id / kUnit], w);
  });
  __syncthreads();
  return Drawn{token_beyond(row, s, s_unit, kept, d.target(mass)), mass};
}

// No filter: the unit from the units' masses, then the token.
template <typename In, int T, class Shared>
__device__ __forceinline__ Drawn draw_unfiltered(const RowSource<In, T>& row, Shared& s, const double* mass_of, const Weigh& w, double u, double all) {
  const double target = u * all;
  auto mass = [&](int i) { return mass_of[i] * w(or_none(row.unit_max[i], row.infinite)); };
  if (threadIdx.x == 0) s.found_id = -1;
  int unit = -1;
  double before = 0.0;
  for (int u0 = 0; u0 < row.units && unit < 0; u0 += T) {
    const int i = u0 + threadIdx.x;
    const double mine = i < row.units ? mass(i) : 0.0;
    double sum;
    const double excl = before + block_excl_scan(mine, s.dscan, &sum);
    if (mine > kNoWeight && excl + mine > target) atomicMin(reinterpret_cast<unsigned*>(&s.found_id), static_cast<unsigned>(i));
    __syncthreads();
    unit = s.found_id;
    if (i == unit) s.found_drest = target - excl;
    before += sum;
    __syncthreads();
  }
  double rest = INFINITY;                                    // u = 1: the last token that has a weight
  if (unit >= 0) {
    rest = s.found_drest;
  } else {
    for (unit = row.units - 1; unit > 0 && !(mass(unit) > kNoWeight);) --unit;
  }
  __syncthreads();
  if (threadIdx.x == 0) s.found_id = -1;
  constexpr int kEach = kUnit / T;
  const int v = unit * kUnit + static_cast<int>(threadIdx.x) * kEach;
  double mine[kEach], sum = 0.0, total;
  int last = -1;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const float x = row.at(v + i);
    mine[i] = x > -INFINITY ? w(x) : 0.0;
    if (!(mine[i] > kNoWeight)) mine[i] = 0.0;
    else last = v + i;
    sum += mine[i];
  }
  double run = block_excl_scan(sum, s.dscan, &total);
#pragma unroll
  for (int i = kEach - 1; i >= 0; --i) {                     // the thread's first that passes
    double to = run;
#pragma unroll
    for (int j = 0; j <= i; ++j) to += mine[j];
    if (mine[i] > 0.0 && to > rest) atomicMin(reinterpret_cast<unsigned*>(&s.found_id), static_cast<unsigned>(v + i));
  }
  __syncthreads();
  const int id = s.found_id;
  __syncthreads();
  if (id >= 0) return Drawn{id, 0};
  if (last >= 0) atomicMax(&s.found_id, last);               // the unit's sum, added up in another order, ends above the target: its last token
  __syncthreads();
  return Drawn{s.found_id, 0};
}
// Greedy: the lowest of the largest.
template <typename In, int T, class Shared>
__device__ __forceinline__ int largest(const RowSource<In, T>& row, Shared& s, float top) {
  if (threadIdx.x == 0) s.found_id = INT32_MAX;
  __syncthreads();
  for (int i = threadIdx.x; i < row.units; i += T)
    if (row.unit_max[i] == top) atomicMin(&s.found_id, i);
  __syncthreads();
  const int unit = s.found_id;
  __syncthreads();
  if (threadIdx.x == 0) s.found_id = INT32_MAX;
  __syncthreads();
  const float ref = or_none(top, row.infinite);
  for (int v = unit * kUnit + threadIdx.x; v < (unit + 1) * kUnit; v += T)
    if (row.at(v) == ref) atomicMin(&s.found_id, v);
  __syncthreads();
  return s.found_id;
}
struct PlainShared {
  float red[17];
  double dscan[17];
  double found_drest;
  int found_id;
};
// A workgroup to a row.  FILTERED: some row may have a filter.
template <typename In, int T, bool FILTERED>
__global__ void __launch_bounds__(T)
k_sample_row(Logits<In> L, Settings S, const int32_t* __restrict__ rowsel, int64_t c0, Summary A, const float* __restrict__ uniform, int unit_bits, SampleOut out) {
  extern __shared__ u64 s_unit[];                            // [units], FILTERED only
  __shared__ std::conditional_t<FILTERED, RowShared<T>, PlainShared> s;
  const int64_t m = blockIdx.x, row = rowsel ? rowsel[c0 + m] : c0 + m;
  const float* const unit_max = A.unit + m * L.units;
  const double *const mass_of = A.mass + m * L.units, *const sum_of = A.sum + m * L.units;
  const double t = S.t(row);
  double u = uniform[row];
  float top = -INFINITY;
  for (int i = threadIdx.x; i < L.units; i += T) top = fmaxf(top, unit_max[i]);
  {
    float* const red = reinterpret_cast<float*>(s.dscan);
    top = wave_max(top);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = top;
    __syncthreads();
    for (int w = 0; w < T / kWave; ++w) top = fmaxf(top, red[w]);
    __syncthreads();
  }
  if (top == -INFINITY) {                                    // nothing to draw from
    if (threadIdx.x == 0) {
      out.ids[row] = -1;
      if (out.logp) out.logp[row] = 0.f;
      if (out.logq) out.logq[row] = 0.f;
    }
    return;
  }
  const RowSource<In, T> src{L.row(m), L.V, L.units, unit_max, top == INFINITY};
  const float ref = or_none(top, src.infinite);
  const double c = scale_of(t);
  const Weigh w{ref, c}, w1{ref, kLog2e64};
  u = u > 0.0 ? fmin(u, 1.0) : 0.0;
  double sum = 0.0, all = 0.0;                               // of exp(z - top), for the log-prob of the softmax itself, and of the weights
  for (int i = threadIdx.x; i < L.units; i += T) {
    const float x = or_none(unit_max[i], src.infinite);
    sum += sum_of[i] * w1(x);
    all += mass_of[i] * w(x);
  }
  block_excl_scan(sum, s.dscan, &sum);
  block_excl_scan(all, s.dscan, &all);
  int id;
  double kept = all;
  if (!(t > 0.0)) {
    id = largest(src, s, top);
  } else if constexpr (!FILTERED) {
    id = draw_unfiltered(src, s, mass_of, w, u, all).id;
  } else {
    int k = S.k(row);
    double p = S.p(row), mp = S.m(row);
    if (k >= L.V || k < 0) k = 0;
    p = p < 1.0 ? fmax(p, 0.0) : 1.0;
    mp = mp > 0.0 ? fmin(mp, 1.0) : 0.0;
    if (k == 0 && p == 1.0 && mp == 0.0) {
      id = draw_unfiltered(src, s, mass_of, w, u, all).id;
    } else {
      const RowDraw d{ref, w, k, p, mp, u, all, ldexp(1.0, unit_bits)};
      const float* const group_max = A.group + m * L.units * kGroupsPerUnit;
      const int groups = L.units * kGroupsPerUnit;
      float bound = src.infinite ? -INFINITY : L.V <= kRanked ? -INFINITY : front_bound<T>(group_max, groups, s);
      Drawn got{-1, 0};
      if (src.infinite) {
        got = draw_by_passes<In, T>(src, s, s_unit, d);
      } else {
        const bool listed = list_front(src, group_max, bound, s);
        const int n = listed ? s.n_list : 0;
        __syncthreads();
        if (listed && n <= kRanked) got = draw_from_front(s, n, bound, bound == -INFINITY, d);
        if (!listed) bound = INFINITY;
        if (got.id < 0 && bound > -INFINITY && listed) got = draw_by_bins(src, s, s_unit, bound, n, c, d);
        if (got.id < 0) got = draw_by_passes<In, T>(src, s, s_unit, d);
      }
      id = got.id;
      kept = static_cast<double>(got.mass) / d.one;
    }
  }
  if (threadIdx.x != 0) return;
  out.ids[row] = id;
  const float zi = src.at(id);
  const double gap = zi == ref ? 0.0 : static_cast<double>(zi) - static_cast<double>(ref);
  if (out.logp) out.logp[row] = static_cast<float>(gap - log(sum));
  if (out.logq) out.logq[row] = t > 0.0 ? static_cast<float>(gap * (c / kLog2e64) - log(kept)) : 0.f;
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
  return std::min(51, 62 - b);
}
constexpr int kRowT = 1024, kPlainT = 256;
template <typename In>
umas_status sample_rows(const Logits<In>& L, const Settings& S, const int32_t* rowsel, int64_t c0, int64_t rows, const SampleWs& w, const float* u, const SampleOut& out,
                        hipStream_t st) {
  hipLaunchKernelGGL(k_sample_open<In>, dim3(cdiv(L.units, kOpenUnits), static_cast<unsigned>(rows)), dim3(kOpenT), 0, st, L, S, rowsel, c0, w.A);
  UMAS_LAUNCHED("k_sample_open");
  const bool plain = !S.top_k_of && !S.top_p_of && !S.min_p_of && S.min_p == 0.0 && S.top_p == 1.0 && (S.top_k == 0 || S.top_k >= L.V);
  const bool greedy = !S.temperature_of && S.temperature == 0.0;
  if (plain || greedy) hipLaunchKernelGGL((k_sample_row<In, kPlainT, false>), dim3(static_cast<unsigned>(rows)), dim3(kPlainT), 0, st, L, S, rowsel, c0, w.A, u, 0, out);
  else
    hipLaunchKernelGGL((k_sample_row<In, kRowT, true>), dim3(static_cast<unsigned>(rows)), dim3(kRowT), L.units * sizeof(u64), st, L, S, rowsel, c0, w.A, u, bits_of(L.V), out);
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
