// The draw of a token from a row of logits, at a temperature and under top-k, min-p and top-p, from a given uniform number.
//
//   w_v = exp((z_v - max z) / T);  tokens in falling order of z, equal ones in rising order;  the first k of them;  of these those with w >= min_p;  of these
//   the shortest run from the front whose mass reaches top_p of theirs;  of what is kept, in rising order of tokens, the first whose running mass passes
//   u times the kept mass
// A uniform number may fall next to a border between two tokens, so masses are float64 where nothing is filtered, and else whole numbers: w in units of 2^-s, s = min(51, 62 - log2 V),
// whose sums are exact in any order (64-bit atomics in LDS give the same result whichever comes first).
//
// The first launch, k_sample_open, is the one pass over all logits: maxima of groups of 64, and of units of 1024 the maximum, the sum of exponentials and, where all tokens' mass decides,
// that mass in float64.  From memory that is a read at 5.6 TB/s (400 float32 rows of 151 936: 43 us); where float64 exponentials count, a wavefront first reads its
// two units and then computes, one after the other: 777 float32 rows of 50 001 39 us, of which reading 156 MB is 25 and fifteen float64 instructions a logit, of 5.4 cycles each, are 20.
// The second, k_sample_row, gives a workgroup to a row.  Without filters the unit and then the token are found from the units' masses.  Else the front is listed: the tokens that the
// 64th largest of the threads' group maxima bounds, or all that min_p leaves; up to 512 of them decide by themselves if nothing behind them can count (13 us for a row of 152 064, 14.5 for 256).
// Rows that are spread, whose border lies behind the front, go through four more launches over the chip: counts of the tokens by their distance to the front (k_sample_count), from these the
// thresholds between which a border lies (k_sample_bracket), the sums above and lists between them (k_sample_sums), and the border and token from those (k_sample_flat): 11, 10,
// 28 and 25 us for what is spread among 256 rows.  A single row does all of it in the second launch.  Where lists overflow, with floods of equal logits, thresholds are found bit by bit, eleven
// at a time from the top, with a histogram of counts or masses (draw_by_passes): right for every row, and slow.
#include <float.h>

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
// The largest logit's own weight is exactly 1, equal logits' weights are equal; below 2^-1000 is 2^-1000, nearly: logits are held up to the first float32 number whose weight is no
// more than that, in float32, which costs a third of a float64 maximum.  (Where that one is not below the largest itself the temperature is so low that c may as well be what takes
// the next number below the largest to 2^-1000.)  At low temperatures numbers that lie next to each other are hundreds of powers of two apart and that number's own power may be 2^-2000:
// the power is held up as well, a whole number's maximum, or it would run over into the sign.
// The maximum of two numbers in one instruction (fmaxf makes both quiet first).
__device__ __forceinline__ float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ __forceinline__ float next_below(float x) {        // of a finite one
  const uint32_t u = __float_as_uint(x);
  return x == 0.f ? __uint_as_float(0x80000001u) : __uint_as_float(x > 0.f ? u - 1 : u + 1);
}
struct Weigh {
  static constexpr int kLeastPower = -1000;
  double top, c;
  float least;
  __device__ __forceinline__ Weigh(float largest, double c_) : top(largest) {
    const float below = next_below(largest);
    c = fmax(fmin(c_, static_cast<double>(1000.f * __builtin_amdgcn_rcpf(largest - below))), 1e-30);   // (a temperature without end: all are 1 but those of -infinity)
    least = fminf(fmaxf(largest - 1000.f * __builtin_amdgcn_rcpf(static_cast<float>(fmin(c, 1e38))), -3e38f), below);
    if ((static_cast<double>(least) - top) * c > kLeastPower) least = next_below(least);   // rounded towards the largest
  }
  __device__ __forceinline__ float next_above() const {      // the largest logit's next number
    const float x = static_cast<float>(top);
    const uint32_t u = __float_as_uint(x);
    return x == 0.f ? __uint_as_float(1u) : __uint_as_float(x > 0.f ? u + 1 : u - 1);
  }
  __device__ __forceinline__ double operator()(float z) const {
    constexpr double kPush = 6755399441055744.0;             // 3 * 2^51
    const double t = (static_cast<double>(larger(z, least)) - top) * c;
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
    const int power = max(__double2loint(pushed), kLeastPower);
    return __hiloint2double(__double2hiint(p) + static_cast<int>(static_cast<uint32_t>(power) << 20), __double2loint(p));
  }
};
constexpr double kNoWeight = 1e-290;                          // what is no more than this is not drawn, u = 0 or not
constexpr double kLog2e64 = 1.4426950408889634074;
// log x of 1 <= x: the float32 one and a step of Newton's, whose error is half the square of what that one is off by.  (The library's took 3 us of a row.)
__device__ __forceinline__ double log_of(double x) {
  const float y = __logf(static_cast<float>(x));
  return static_cast<double>(y) + (x * Weigh(0.f, kLog2e64)(-y) - 1.0);   // (the largest is 0, as y >= 0)
}
// 2^t, nearly: for estimates.
__device__ __forceinline__ double exp2_near(double t) { return static_cast<double>(__builtin_amdgcn_exp2f(static_cast<float>(t))); }
// Rounded by itself, where what it is added to may differ from one kernel to the next.
__device__ __forceinline__ double product(double a, double b) {
#pragma clang fp contract(off)
  return a * b;
}
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
  // the mass of all tokens decides: they are drawn from, or top_p is a part of it
  __device__ __forceinline__ bool of_all(int64_t row, int V) const {
    const int first = k(row);
    return t(row) > 0.0 && (first <= 0 || first >= V) && !(m(row) > 0.0);
  }
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
  float* ref;                                                // [rows][units]: what the sums are relative to, the larger maximum of two units
  double *mass, *sum;                                        // [rows][units]: sum of w at T and of exp(z - ref) at 1
};

// ------------------------------------------------------------------ loads
// The lane's share of a unit: pieces of kRun tokens that lie next to each other, kRun * 64 tokens apart.  What is no number counts as -infinity, as what lies
// past the vocabulary.
template <typename In> constexpr int kRun = std::is_same<In, uint16_t>::value ? 8 : 4;
__device__ __forceinline__ float logit(float x) { return x == x ? x : -INFINITY; }
__device__ __forceinline__ float logit(double x) { return logit(static_cast<float>(x)); }
__device__ __forceinline__ float logit(uint16_t x) { return logit(bf2f(x)); }
// Where the largest logit is +infinity, or the type's lowest number, which has none below it: tokens that are as large share the mass, others have none.
struct Extreme {
  float top;
  bool is;
  __device__ __forceinline__ explicit Extreme(float t) : top(t), is(t == INFINITY || t == -FLT_MAX) {}
  __device__ __forceinline__ float operator()(float z) const { return is ? (z == top ? 0.f : -INFINITY) : z; }
};
template <typename In>
__device__ __forceinline__ int token_of(int unit, int i) {    // of the lane's i-th logit
  return unit * kUnit + (i / kRun<In>) * (kRun<In> * kWave) + (threadIdx.x & 63) * kRun<In> + i % kRun<In>;
}
template <typename In>
__device__ __forceinline__ void load_unit(const In* __restrict__ z, int V, int unit, float (&x)[kPerLane]) {   // as they are, numbers or not
  typedef uint32_t u32x4a __attribute__((ext_vector_type(4), aligned(2)));
  constexpr int R = kRun<In>;
  if ((unit + 1) * kUnit <= V) {
#pragma unroll
    for (int i = 0; i < kPerLane; i += R) {
      const int v = token_of<In>(unit, i);
      if constexpr (std::is_same<In, double>::value) {
#pragma unroll
        for (int j = 0; j < R; ++j) x[i + j] = static_cast<float>(z[v + j]);
      } else {
        const u32x4a w = *reinterpret_cast<const u32x4a*>(z + v);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if constexpr (R == 8) {
            x[i + 2 * j] = __uint_as_float(w[j] << 16);
            x[i + 2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
          } else {
            x[i + j] = __uint_as_float(w[j]);
          }
        }
      }
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < kPerLane; ++i) {
    const int v = token_of<In>(unit, i);
    x[i] = v < V ? logit(z[v]) : -INFINITY;
  }
}

// ------------------------------------------------------------------ first launch
// A wavefront takes two units, whose largest logit is found and whose sums are exchanged together.
constexpr int kOpenT = 256, kOpenPairs = kOpenT / kWave;
template <typename In>
__device__ __forceinline__ float group_maxima(const float (&x)[kPerLane], float (&g)[kPerLane / kRun<In>]) {   // ... and the lane's
  constexpr int R = kRun<In>;
  float top = -INFINITY;
#pragma unroll
  for (int i = 0; i < kPerLane; i += R) {
    float m = x[i];
#pragma unroll
    for (int j = 1; j < R; ++j) m = larger(m, x[i + j]);
    m = larger(m, lane_xor<1>(m));
    m = larger(m, lane_xor<2>(m));
    m = larger(m, lane_xor<4>(m));
    if constexpr (kGroup / R > 8) m = larger(m, lane_xor<8>(m));
    g[i / R] = m;
    top = larger(top, m);
  }
  if constexpr (kGroup / R <= 8) top = larger(top, lane_xor<8>(top));
  top = larger(top, lane_xor<16>(top));
  return larger(top, lane_xor<32>(top));
}
// Of two numbers, summed over the wavefront: the first in the lower half's lanes, the second in the upper half's.
__device__ __forceinline__ double halves_sum(double a, double b) {
  const bool upper = threadIdx.x & 32;
  const double mine = upper ? b : a, other = upper ? a : b;
  double x = mine + bits_of(lane_xor<32>(bits_in(other)), double());
  x += bits_of(lane_xor<1>(bits_in(x)), double());
  x += bits_of(lane_xor<2>(bits_in(x)), double());
  x += bits_of(lane_xor<4>(bits_in(x)), double());
  x += bits_of(lane_xor<8>(bits_in(x)), double());
  return x + bits_of(lane_xor<16>(bits_in(x)), double());
}
template <typename In>
__global__ void __launch_bounds__(kOpenT, 8)
k_sample_open(Logits<In> L, Settings S, const int32_t* __restrict__ rowsel, int64_t c0, Summary out, int* __restrict__ count) {
  constexpr int R = kRun<In>, kLanes = kGroup / R;            // lanes to a group
  const int lane = threadIdx.x & 63, u0 = 2 * (blockIdx.x * kOpenPairs + static_cast<int>(threadIdx.x >> 6));
  if (count && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *count = 0;
  if (u0 >= L.units) return;
  const int64_t m = blockIdx.y, row = rowsel ? rowsel[c0 + m] : c0 + m;
  float x[2][kPerLane], g[2][kPerLane / R], top[2];
  load_unit(L.row(m), L.V, u0, x[0]);
  load_unit(L.row(m), L.V, u0 + 1, x[1]);                    // of one that does not exist: nothing
#pragma unroll
  for (int p = 0; p < 2; ++p) top[p] = group_maxima<In>(x[p], g[p]);
  if (!(top[0] == top[0] && top[1] == top[1])) {             // some are no number: as if they were -infinity
#pragma unroll
    for (int p = 0; p < 2; ++p) {
#pragma unroll
      for (int i = 0; i < kPerLane; ++i) x[p][i] = logit(x[p][i]);
      top[p] = group_maxima<In>(x[p], g[p]);
    }
  }
  const int64_t at = m * L.units + u0;
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    if (u0 + p >= L.units) continue;
#pragma unroll
    for (int i = 0; i < kPerLane / R; ++i)
      if (lane % kLanes == 0) out.group[(at + p) * kGroupsPerUnit + i * R + lane / kLanes] = g[p][i];
  }
  const float most = larger(top[0], top[1]);
  double mass[2] = {0.0, 0.0}, sum[2] = {0.0, 0.0};
  if (most > -INFINITY) {
    // float64 exponentials only where they count: 256 bf16 rows of 152 064 with settings of their own 40 -> 25.6 us, 400 float32 rows under min_p 53 -> 43
    const double t = S.t(row);
    const bool drawn = S.of_all(row, L.V);
    const Extreme extreme(most);
    if (extreme.is)
#pragma unroll
      for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int i = 0; i < kPerLane; ++i) x[p][i] = extreme(x[p][i]);
    const float ref = extreme(most);
    if (drawn) {
      const Weigh w(ref, scale_of(t));
#pragma unroll
      for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int i = 0; i < kPerLane; ++i) mass[p] += w(x[p][i]);
      mass[0] = halves_sum(mass[0], mass[1]);
    }
    if (drawn && t == 1.0) {
      sum[0] = mass[0];
    } else {
      constexpr float kLog2e = 1.44269504088896341f;
#pragma unroll
      for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int i = 0; i < kPerLane; ++i) sum[p] += static_cast<double>(__builtin_amdgcn_exp2f((x[p][i] - ref) * kLog2e));
      sum[0] = halves_sum(sum[0], sum[1]);
    }
  }
  if (lane % 32 != 0 || u0 + lane / 32 >= L.units) return;
  out.unit[at + lane / 32] = lane == 0 ? top[0] : top[1];
  out.ref[at + lane / 32] = most;
  out.mass[at + lane / 32] = mass[0];
  out.sum[at + lane / 32] = sum[0];
}

// ------------------------------------------------------------------ second launch
constexpr int kBins = 2048, kCounts = 4096;                  // of eleven bits of a key, and of distances to the front
constexpr int kTopRank = 64;
constexpr int kListCap = 4096, kRanked = 512, kCompared = 128;   // tokens of a list, of one that decides by itself, and of one that is ordered by comparing all with all
constexpr int kGroupCap = 1024;
// Sums and scans over a workgroup of T threads: what the wavefronts have goes through one of two buffers in turn, so that one barrier is enough.  Float64 numbers that are taken T at a time, in
// their order, each time onto what there is so far, are added up in the same order whatever T is: one after the other the sums of 64.
template <int T>
struct Block {
  static constexpr int W = T / kWave;
  u64 (*buf)[2][W];                                          // [2], of two numbers a wavefront
  int turn = 0;
  __device__ __forceinline__ explicit Block(u64 (*b)[2][W]) : buf(b) {}
  template <class V>
  __device__ __forceinline__ V scan(V v, V* total, V from = V()) {   // exclusive, from a number on, which *total has in it
    const int wave = threadIdx.x >> 6;
    const V incl = lanes_scan(v);
    u64(&to)[W] = buf[turn][0];
    turn ^= 1;
    if ((threadIdx.x & 63) == 63) to[wave] = bits_in(incl);
    __syncthreads();
    V before = from, all = from;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const V x = umas::bits_of(to[w], V());
      before += w < wave ? x : V();
      all += x;
    }
    *total = all;
    return before + (incl - v);
  }
  template <class V>
  __device__ __forceinline__ void add(V& a, V& b, V x, V y) {   // all threads' x and y onto a and b
    x = lanes_sum(x);
    y = lanes_sum(y);
    u64(&to)[2][W] = buf[turn];
    turn ^= 1;
    if ((threadIdx.x & 63) == 0) {
      to[0][threadIdx.x >> 6] = bits_in(x);
      to[1][threadIdx.x >> 6] = bits_in(y);
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < W; ++w) {
      a += umas::bits_of(to[0][w], V());
      b += umas::bits_of(to[1][w], V());
    }
  }
  template <class V>
  __device__ __forceinline__ void sum(V& a, V& b) {
    const V x = a, y = b;
    a = b = V();
    add(a, b, x, y);
  }
  template <class V>
  __device__ __forceinline__ V sum(V a) {
    V b = V();
    sum(a, b);
    return a;
  }
  __device__ __forceinline__ float max(float v) {
    v = wave_max(v);
    u64(&to)[W] = buf[turn][0];
    turn ^= 1;
    if ((threadIdx.x & 63) == 0) to[threadIdx.x >> 6] = __float_as_uint(v);
    __syncthreads();
#pragma unroll
    for (int w = 0; w < W; ++w) v = larger(v, __uint_as_float(static_cast<uint32_t>(to[w])));
    return v;
  }
};
// LIST: tokens that are listed; ALL: with their weights, and the units' sums.
template <int T, int LIST = kListCap, bool ALL = true>
struct RowShared {
  static constexpr int kList = LIST;
  u64 block[2][2][T / kWave];
  u64 bins[kBins];                                           // masses or counts
  u64 list_w[ALL ? LIST : 1];
  u64 unit[ALL ? kMaxSampleV / kUnit : 1];
  float list_z[LIST];
  int list_id[LIST];
  float top[4][kWave];
  int rank[kRanked];
  u64 found_above, found_here, found_rest;
  double found_drest;
  uint32_t found_bin;
  int found_id, n_list, n_groups, n_members[3];
};
// A row's settings and what the first launch says about it.
struct RowDraw {
  float top;
  Weigh w;
  int k;                                                     // 0: none
  double p, m, u;                                            // p = 1, m = 0: none
  double all;                                                // the mass of all tokens, in units of the largest weight
  double one;                                                // 1 in units of the whole numbers
  int id_bits;                                               // of a token's number
  __device__ __forceinline__ bool by_min() const { return m > 0.0; }
  // x * one, one at most 2^51, rounded to nearest by the addition of 2^52, whose bits are kNothing; of a weight that min_p does not leave nothing
  static constexpr u64 kNothing = 0x4330000000000000ull;
  __device__ __forceinline__ u64 bits(double x) const { return static_cast<u64>(__double_as_longlong(fma(x >= m ? x : 0.0, one, 4503599627370496.0))); }
  __device__ __forceinline__ u64 weight(float z) const { return bits(w(z)) - kNothing; }
  __device__ __forceinline__ u64 share(double part, u64 of) const {   // the least whole number that reaches part of a mass
    const u64 n = static_cast<u64>(ceil(part * static_cast<double>(of)));
    return n < 1 ? 1 : n > of ? of : n;
  }
  // What the kept run has to reach, of whole numbers that add up to `mass`: top_p's part of them, or without top_k and min_p of all tokens' float64 mass.  (That is known before any
  // whole number; it holds what rounds to none of them as well, so that the whole numbers may fall short of it.)  Every way to a row's token takes it from here.
  __device__ __forceinline__ u64 needed(u64 mass) const {
    if (!(p < 1.0)) return mass;
    if (k > 0 || by_min()) return share(p, mass);
    const double part = ceil(p * all * one);
    return part < 1.0 ? 1 : static_cast<u64>(part);
  }
  __device__ __forceinline__ u64 target(u64 mass) const {
    const u64 t = static_cast<u64>(u * static_cast<double>(mass));
    return t < mass ? t : mass - 1;
  }
};
// The logits of a row of T threads, a unit to a wavefront at a time.
template <typename In, int T>
struct RowSource {
  const In* z;
  int V, units;
  const float* unit_max;                                     // of the row
  Extreme extreme;
  __device__ __forceinline__ float at(int v) const { return static_cast<unsigned>(v) < static_cast<unsigned>(V) ? extreme(logit(z[v])) : -INFINITY; }   // -1: no token
  // f(z, token, weight()) for every token with z > -infinity, and z >= lo; others may come.  `after` once a unit, by its wavefront, also where the unit has none
  template <class F, class G>
  __device__ __forceinline__ void each(float lo, const RowDraw& d, F f, G after) const {
    for (int u = threadIdx.x >> 6; u < units; u += T / kWave) {
      const float top = unit_max[u];
      if ((extreme.is || top >= lo) && top > -INFINITY) {
        float x[kPerLane];
        load_unit(z, V, u, x);
#pragma unroll
        for (int i = 0; i < kPerLane; ++i) {
          const float zi = extreme(logit(x[i]));
          if (zi > -INFINITY) f(zi, token_of<In>(u, i), [&] { return d.weight(zi); });
          if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);  // sixteen weights at once take more registers than there are
        }
      }
      after(u);
    }
  }
  template <class F>
  __device__ __forceinline__ void each(float lo, const RowDraw& d, F f) const { each(lo, d, f, [](int) {}); }
};
// Listed tokens [a, b).
template <int T>
struct ListSource {
  const RowShared<T>* s;
  int a, b;
  template <class F>
  __device__ __forceinline__ void each(float, const RowDraw&, F f) const {
    for (int i = a + static_cast<int>(threadIdx.x); i < b; i += T) f(s->list_z[i], s->list_id[i], [&] { return s->list_w[i]; });
  }
};
struct Border {
  uint32_t key;
  u64 above, here;                                           // sums over larger keys, and over those equal to it
};
// The key at which the sum of val over the keys in falling order reaches `need`, 1 <= need <= the sum over all; keys of `known` bits.  Eleven
// bits at a time from the top; whole numbers, so that the order in which the additions come is nothing.
template <int T, class Source, class K, class F>
__device__ __forceinline__ Border border_of(const Source& src, RowShared<T>& s, Block<T>& all, float lo, const RowDraw& d, K key_of, F val, u64 need, int known) {
  constexpr int kEach = kBins / T;
  Border b{0, 0, 0};
#pragma unroll 1
  while (known > 0) {
    const int shift = max(known - 11, 0);
    const uint32_t mask = (1u << (known - shift)) - 1;
    for (int i = threadIdx.x; i < kBins; i += T) s.bins[i] = 0;
    __syncthreads();
    src.each(lo, d, [&](float z, int id, auto w) {
      const uint32_t key = key_of(z, id);
      if (known < 32 && (key ^ b.key) >> known) return;
      const u64 v = val(z, id, w);
      if (v) atomicAdd(&s.bins[(key >> shift) & mask], v);
    });
    __syncthreads();
    const int hi = kBins - 1 - kEach * static_cast<int>(threadIdx.x);   // from the largest bin down
    u64 sum = 0, total;
#pragma unroll
    for (int i = 0; i < kEach; ++i) sum += s.bins[hi - i];
    u64 above = b.above + all.scan(sum, &total);
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
    known = shift;
    __syncthreads();
  }
  return b;
}

struct SampleOut {
  int32_t* ids;
  float *logp, *logq;
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
__device__ __forceinline__ float logit_at(uint32_t order) { return __uint_as_float(order & 0x80000000u ? order ^ 0x80000000u : ~order); }
// Where the orders of logits lie: from base on, as many bits.
struct Span {
  uint32_t base = 0;
  int bits = 32;
};
// The cut after `need` of val, which is the same for equal logits or 0; *mass: the sum of what is in.
template <int T, class Source, class F>
__device__ __forceinline__ Cut cut_at(const Source& src, RowShared<T>& s, Block<T>& all, float lo, const RowDraw& d, F val, u64 need, u64* mass, Span span = Span()) {
  Border b = border_of(src, s, all, lo, d, [&](float z, int) { return order_of(z) - span.base; }, val, need, span.bits);
  b.key += span.base;
  Cut c;
  c.key = b.key;
  // how many tokens lie at the border
  u64 count = 0;
  src.each(lo, d, [&](float z, int id, auto w) { count += order_of(z) == b.key && val(z, id, w); });
  count = all.sum(count);
  const u64 one = b.here / count, ties = (need - b.above + one - 1) / one;
  if (ties < count) {                                        // the lowest of them
    const int last = (1 << d.id_bits) - 1;
    c.tie = last - static_cast<int>(border_of(src, s, all, lo, d, [&](float, int id) { return static_cast<uint32_t>(last - id); },
                                              [&](float z, int id, auto w) { return u64{order_of(z) == b.key && val(z, id, w)}; }, ties, d.id_bits).key);
  }
  *mass = b.above + ties * one;
  return c;
}
// The token at which the running mass of val, in rising order of tokens, passes `target`, which is less than all of it; unit_sum: the units' sums of val.
template <typename In, int T, class F>
__device__ __forceinline__ int token_beyond(const RowSource<In, T>& row, RowShared<T>& s, Block<T>& all, const u64* unit_sum, F val, u64 target) {
  u64 before = 0;
  if (threadIdx.x == 0) s.found_id = -1;
  int unit = -1;
  for (int u0 = 0; u0 < row.units && unit < 0; u0 += T) {
    const int u = u0 + threadIdx.x;
    const u64 mine = u < row.units ? unit_sum[u] : 0;
    u64 total;
    const u64 excl = before + all.scan(mine, &total);
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
  u64 excl = all.scan(sum, &total);
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
__device__ __noinline__ Drawn draw_by_passes(RowSource<In, T> row, RowShared<T>* shared, int turn, u64* s_unit, RowDraw d) {
  RowShared<T>& s = *shared;
  Block<T> all(s.block);
  all.turn = turn;
  const float none = -INFINITY;
  Cut first, run;
  u64 mass;
  auto one = [](float, int, auto) { return u64{1}; };
  if (d.k > 0) {
    u64 have = 0;
    row.each(none, d, [&](float, int, auto) { ++have; });
    have = all.sum(have);
    if (static_cast<u64>(d.k) < have) first = cut_at(row, s, all, none, d, one, static_cast<u64>(d.k), &mass);
  }
  auto of_first = [&](float z, int id, auto w) { return first.in(z, id) ? w() : u64{0}; };
  mass = 0;
  row.each(none, d, [&](float z, int id, auto w) { mass += of_first(z, id, w); });
  mass = all.sum(mass);
  if (d.p < 1.0) run = cut_at(row, s, all, none, d, of_first, min(d.needed(mass), mass), &mass);
  auto kept = [&](float z, int id, auto w) { return run.in(z, id) ? of_first(z, id, w) : u64{0}; };
  u64 sum = 0;
  row.each(none, d, [&](float z, int id, auto w) { sum += kept(z, id, w); }, [&](int u) {
    sum = lanes_sum(sum);
    if ((threadIdx.x & 63) == 0) s_unit[u] = sum;
    sum = 0;
  });
  __syncthreads();
  return Drawn{token_beyond(row, s, all, s_unit, [&](float z, int id) { return kept(z, id, [&] { return d.weight(z); }); }, d.target(mass)), mass};
}

// ---- the tokens in front
// A number that at least so many logits reach: the threads of four wavefronts take the maximum over the row's groups in turn, and the rank-th largest of theirs is it.
// (All sixteen, whose lists everybody merges: 5 us more of a row.)
constexpr int kBoundT = 256;
template <int T, class Shared>
__device__ __forceinline__ float front_bound(const float* __restrict__ group_max, int groups, Shared& s) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, rank = min(kTopRank, groups / 8);
  if (wave < kBoundT / kWave) {
    float x = -INFINITY;
    for (int g = threadIdx.x; g < groups / 4; g += 4 * kBoundT) {   // four groups that lie next to each other; a row's are a multiple of sixteen
      floatx4 y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        y[i] = g + i * kBoundT < groups / 4 ? reinterpret_cast<const floatx4*>(group_max)[g + i * kBoundT] : floatx4{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
      for (int i = 0; i < 4; ++i) x = larger(x, larger(larger(y[i][0], y[i][1]), larger(y[i][2], y[i][3])));
    }
    s.top[wave][lane] = sorted_desc(x);
  }
  __syncthreads();
  if (wave == 0) {
    float x = merged(merged(s.top[0][lane], s.top[1][lane]), merged(s.top[2][lane], s.top[3][lane]));
    s.top[0][lane] = x;
  }
  __syncthreads();
  return s.top[0][rank - 1];
}
// Lists the tokens with z >= bound; false: they lie in more than so many groups, or are more than there is room for.
template <typename In, int T, class Shared>
__device__ __forceinline__ bool list_front(const RowSource<In, T>& row, const float* __restrict__ group_max, float bound, int most_groups, Shared& s) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, groups = row.units * kGroupsPerUnit;
  int* const s_group = reinterpret_cast<int*>(s.bins);
  if (threadIdx.x == 0) s.n_list = s.n_groups = 0;
  __syncthreads();
  for (int g = threadIdx.x; g < groups / 4; g += T) {
    const floatx4 x = reinterpret_cast<const floatx4*>(group_max)[g];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (x[i] >= bound && x[i] > -INFINITY) {
        const int at = atomicAdd(&s.n_groups, 1);
        if (at < kGroupCap) s_group[at] = g * 4 + i;
      }
  }
  __syncthreads();
  const int n = s.n_groups;
  if (n > most_groups) return false;
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
      if (in && at < Shared::kList) {
        s.list_z[at] = x[q];
        s.list_id[at] = id[q];
      }
    }
  }
  __syncthreads();
  return s.n_list <= Shared::kList;
}
// What the listed tokens say, where they are enough: id -1 where they are not.  `complete`: no other token has a weight, so that a top_k beyond them keeps them all (24 rows of 152 064
// under top_k 50 and min_p 0.05, of which few tokens are left, 15 us; gone through as if others might count 57).  Up to 128 tokens: each is compared with all of them, once by its logit and once by its number, by
// the threads that it has: of 1024 sixteen for up to 64 tokens, eight for up to 128.
template <int T, class Shared>
__device__ __forceinline__ Drawn draw_from_front(Shared& s, Block<T>& all, int n, bool complete, const RowDraw& d) {
  u64* const s_key = s.bins;                                 // [kCompared] each
  u64* const s_w = s.bins + kCompared;
  u64* const s_sorted = s.bins + 2 * kCompared;
  u64* const s_run = s.bins + 3 * kCompared;
  static_assert(4 * kCompared <= kBins && kCompared <= T, "a thread at the least to a token");
  int* const s_rank = s.rank;
  const int of = n <= kWave ? kWave : kCompared, parts = T / of;
  const int i = threadIdx.x & (of - 1), part = threadIdx.x / of;   // a part to whole wavefronts
  const bool one = part == 0 && i < n;                       // the token's own thread
  u64 w = 0;
  if (part == 0) {
    s_key[i] = i < n ? static_cast<u64>(order_of(s.list_z[i])) << 32 | (0xFFFFFFFFu - static_cast<uint32_t>(s.list_id[i])) : 0;
    s_rank[i] = 0;
    s_run[i] = 0;
    if (i < n) w = d.weight(s.list_z[i]);
  }
  if (threadIdx.x == 0) s.found_id = -1;
  __syncthreads();
  const u64 key = s_key[i];
  const int j0 = part * (of / parts), j1 = min(j0 + of / parts, n);
  if (i < n && j0 < j1) {
    int rank = 0;
#pragma unroll 8
    for (int j = j0; j < j1; ++j) rank += s_key[j] > key;
    atomicAdd(&s_rank[i], rank);
  }
  __syncthreads();
  const int rank = s_rank[i];
  if (!one || (d.k > 0 && rank >= d.k)) w = 0;
  if (one) s_sorted[rank] = w;
  __syncthreads();
  u64 mass;
  const u64 here = one ? s_sorted[i] : 0, ahead = all.scan(here, &mass);   // of the i-th in falling order
  const bool whole = d.k > 0 || complete;                    // nothing that is not listed counts
  u64 need = d.needed(mass);
  if (whole) need = min(need, mass);
  if ((d.k > n && !complete) || (!whole && (d.by_min() || d.p == 1.0 || need > mass))) return Drawn{-1, 0};
  if (one) {                                                 // kept: whose front is shorter than what is needed
    if (ahead >= need) s_sorted[i] = 0;
    else if (here && ahead + here >= need) s.found_above = ahead + here;
  }
  __syncthreads();
  mass = s.found_above;
  if (one) s_w[i] = w = s_sorted[rank];
  __syncthreads();
  const uint32_t mine = static_cast<uint32_t>(key);          // falls with the token
  if (i < n && j0 < j1) {
    u64 run = 0;
#pragma unroll 8
    for (int j = j0; j < j1; ++j) run += static_cast<uint32_t>(s_key[j]) >= mine ? s_w[j] : 0;
    if (run) atomicAdd(&s_run[i], run);
  }
  __syncthreads();
  if (one && w) {
    const u64 run = s_run[i], target = d.target(mass);
    if (target < run && run - w <= target) s.found_id = s.list_id[i];
  }
  __syncthreads();
  return Drawn{s.found_id, mass};
}
// ... and up to 512: a border, or the token, is found among the sums of 512 runs of logits, or of tokens, and then among those of its run.  (Comparing all with all, a 400 rows' launch
// with fronts of up to 512 took 48 us, the last step by runs 39; all by runs takes 4 us less of the call's 424.)
template <int T, class Shared>
__device__ __forceinline__ Drawn draw_from_long_front(Shared& s, Block<T>& all, int n, float bound, bool complete, const RowDraw& d) {
  u64* const s_key = s.bins;                                 // [kRanked] each
  u64* const s_w = s.bins + kRanked;
  u64* const s_mass = s.bins + 2 * kRanked;
  int* const s_member = reinterpret_cast<int*>(s.bins + 3 * kRanked);
  int* const s_count = s.rank;
  static_assert(4 * kRanked <= kBins && kRanked <= T, "a thread at the least to a token, and to a run");
  const int i = threadIdx.x;
  const bool one = i < n;
  if (i < kRanked) s_count[i] = s_mass[i] = 0;
  if (i < 3) s.n_members[i] = 0;
  if (i == 0) {
    s.found_id = -1;
    s.found_here = 0;
  }
  __syncthreads();
  const float z = one ? s.list_z[i] : 0.f, range = bound > -INFINITY ? d.top - bound : 40.f / static_cast<float>(d.w.c);
  const int id = one ? s.list_id[i] : 0, run = static_cast<int>(fminf((d.top - z) * (kRanked / range), kRanked - 1.f));   // falling logits; what is no number is the last one's
  const u64 key = static_cast<u64>(order_of(z)) << 32 | (0xFFFFFFFFu - static_cast<uint32_t>(id));
  u64 w = one ? d.weight(z) : 0;
  if (one) {
    s_key[i] = key;
    atomicAdd(&s_count[run], 1);
    if (w) atomicAdd(&s_mass[run], w);
  }
  __syncthreads();
  u64 mass, count, in_run = i < kRanked ? s_mass[i] : 0;
  const u64 n_run = i < kRanked ? s_count[i] : 0, n_before = all.scan(n_run, &count), before = all.scan(in_run, &mass);
  if (d.k > 0 && d.k < n) {
    const u64 k = static_cast<u64>(d.k);
    if (n_before < k && k <= n_before + n_run) {
      s.found_bin = i;
      s.found_rest = n_before;
      s.found_above = before;
    }
    __syncthreads();
    const int border = static_cast<int>(s.found_bin);
    const bool member = one && run == border;
    if (member) s_member[atomicAdd(&s.n_members[0], 1)] = i;
    __syncthreads();
    if (member) {
      u64 rank = s.found_rest;
      for (int m = 0; m < s.n_members[0]; ++m) rank += s_key[s_member[m]] > key;
      if (rank >= k) w = 0;
      else if (w) atomicAdd(&s.found_here, w);
    } else if (run > border) {
      w = 0;
    }
    __syncthreads();
    in_run = i < border ? in_run : i == border ? s.found_here : 0;
    mass = s.found_above + s.found_here;
  }
  const bool whole = d.k > 0 || complete;                    // nothing that is not listed counts
  u64 need = d.needed(mass);
  if (whole) need = min(need, mass);
  if ((d.k > n && !complete) || (!whole && (d.by_min() || d.p == 1.0 || need > mass))) return Drawn{-1, 0};
  if (need < mass) {
    if (before < need && need <= before + in_run) {
      s.found_bin = i;
      s.found_rest = before;
    }
    if (one) s_w[i] = w;
    __syncthreads();
    const int border = static_cast<int>(s.found_bin);
    const bool member = one && w && run == border;
    if (member) s_member[atomicAdd(&s.n_members[1], 1)] = i;
    __syncthreads();
    if (member) {
      u64 ahead = s.found_rest;
      for (int m = 0; m < s.n_members[1]; ++m) ahead += s_key[s_member[m]] > key ? s_w[s_member[m]] : 0;
      if (ahead >= need) w = 0;
      else if (ahead + w >= need) s.found_above = ahead + w;
    } else if (run > border) {
      w = 0;
    }
    __syncthreads();
    mass = s.found_above;
  }
  // in rising order of tokens
  if (i < kRanked) s_mass[i] = 0;
  if (one) s_w[i] = w;
  __syncthreads();
  const u64 target = d.target(mass);
  const int part = id >> max(d.id_bits - 9, 0);
  static_assert(kRanked == 1 << 9, "runs of tokens");
  if (w) atomicAdd(&s_mass[part], w);
  __syncthreads();
  u64 total;
  const u64 in_part = i < kRanked ? s_mass[i] : 0, ahead = all.scan(in_part, &total);
  if (ahead <= target && target < ahead + in_part) {
    s.found_bin = i;
    s.found_rest = ahead;
  }
  __syncthreads();
  const bool member = w && part == static_cast<int>(s.found_bin);
  if (member) s_member[atomicAdd(&s.n_members[2], 1)] = i;
  __syncthreads();
  if (member) {
    u64 upto = s.found_rest;
    for (int m = 0; m < s.n_members[2]; ++m) upto += static_cast<uint32_t>(s_key[s_member[m]]) >= static_cast<uint32_t>(key) ? s_w[s_member[m]] : 0;
    if (target < upto && upto - w <= target) s.found_id = id;
  }
  __syncthreads();
  return Drawn{s.found_id, mass};
}

// ---- rows whose mass is spread
// The tokens below the front by their distance to it, in 1/128 of T, at most 1/128: their counts say near which bin the border of top_p lies and in which exactly that of top_k.  A second
// pass sums what lies above for certain, by unit, and lists the tokens of the bins around; among those the borders are found as they are.  Where a border was not
// among the bins, or they hold too many, the row is gone through bit by bit.
constexpr float kCountsPerOne = 128.f;
struct Binning {
  float bound, lo, scale;                                    // of tokens with lo <= z < bound; bins to a difference of 1
  __device__ __forceinline__ Binning(float bound_, const RowDraw& d, int V) : bound(bound_), lo(-INFINITY) {
    const double c = d.w.c;
    scale = kCountsPerOne * fminf(static_cast<float>(c / kLog2e64), 1.f);
    // below lo nothing counts: weights under min_p, or so small that all tokens together with them are not what top_p leaves out
    const double least = d.by_min() ? d.m : d.k > 0 || d.p == 1.0 ? 0.0 : (1.0 - d.p) * d.all / V;
    if (least > 0.0) lo = least_logit(d, least);
  }
  // A logit that is below all whose weight is `least` or more, but not far.
  __device__ __forceinline__ static float least_logit(const RowDraw& d, double least) {
    const float z = static_cast<float>(d.w.top + static_cast<double>(__log2f(static_cast<float>(least))) / d.w.c * (1.0 + 1e-6));
    return z - (fabsf(z) * 1e-6f + static_cast<float>(1e-5 / d.w.c));
  }
  __device__ __forceinline__ bool has(float z) const { return z < bound && z >= lo && z > -INFINITY; }
  __device__ __forceinline__ float place(float z) const { return fminf((bound - z) * scale, static_cast<float>(kCounts - 1)); }
  __device__ __forceinline__ int bin(float z) const { return static_cast<int>(place(z)); }
  // The largest logit of the bins from b on: found by its bits, as what bin() rounds to is what counts.
  __device__ __forceinline__ float edge(int b) const {
    if (b >= kCounts) return -INFINITY;
    uint32_t below = order_of(-INFINITY), above = order_of(bound);   // bin(below) >= b, and that of above is not (or is the bound)
    while (above - below > 1) {
      const uint32_t mid = below + (above - below) / 2;
      if (bin(logit_at(mid)) >= b) below = mid;
      else above = mid;
    }
    return logit_at(below);
  }
};
// What counts, between thresholds.
struct Bracket {
  float sure;                                                // above it tokens are in for certain
  float list;                                                // from sure down to here, exclusive, lies the border of top_p
  float k_from, k_to;                                        // from k_from down to k_to, exclusive, lies the k-th token (-infinity: all are among the first k)
  float last;                                                // what is not above it counts for nothing
  u64 k_in_bin;                                              // places from k_from down
  __device__ __forceinline__ bool lists(float z) const { return (z <= sure && z > list) || (z <= k_from && z > k_to); }
  __device__ __forceinline__ static Span span(float from, float to) {   // of the logits from `from` down to `to`, exclusive
    Span a;
    a.base = order_of(to) + 1;
    a.bits = max(32 - __clz(static_cast<int>(order_of(from) - a.base)), 1);
    return a;
  }
};
// First pass, of the units [u0, u1).  s_off: where in the bin, in 256ths, one of its tokens lies.  (Of bf16 logits a bin holds few values, at temperatures near 1 all in the same place
// of theirs: with the bins' middles taken for it thresholds were half a bin off, and flat rows were gone through bit by bit, 64 of 152 064 under top_p 516 us in place of 99.)
template <typename In, int T>
__device__ __forceinline__ void count_bins(const RowSource<In, T>& row, const Binning& q, int u0, int u1, uint32_t* s_count, uint8_t* s_off) {
  for (int u = u0 + static_cast<int>(threadIdx.x >> 6); u < u1; u += T / kWave) {
    const float most = row.unit_max[u];
    if (!(most >= q.lo) || most == -INFINITY) continue;
    float x[kPerLane];
    load_unit(row.z, row.V, u, x);
#pragma unroll
    for (int i = 0; i < kPerLane; ++i)
      if (q.has(x[i])) {
        const float at = q.place(x[i]);
        const int b = static_cast<int>(at);
        atomicAdd(&s_count[b], 1u);
        s_off[b] = static_cast<uint8_t>((at - static_cast<float>(b)) * 256.f);   // whichever comes last: thresholds may differ by it, the border that is found between them does not
      }
  }
}
// A bin of a part in 32 bits: fewer than 2^24 tokens, and their place.
constexpr int kOffShift = 24;
static_assert(kMaxSampleV < 1 << kOffShift, "a bin holds a vocabulary");
// counts: this thread's bins, kCounts / T of them from threadIdx.x * kCounts / T on, and places: the sums of where their tokens lie.
template <int T, class Shared>
__device__ __forceinline__ Bracket bracket_of(const uint32_t (&counts)[kCounts / T], const uint32_t (&places)[kCounts / T], Shared& s, Block<T>& all, const Binning& q, u64 front, int n_front, const RowDraw& d) {
  constexpr int kEach = kCounts / T;
  const double at_bound = d.w(q.bound), per_bin = -d.w.c / q.scale;   // the power of 2 that a bin takes from a weight
  u64 n_mine = 0, n_all;
  double m_mine = 0.0, m_all, of[kEach];
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int b = static_cast<int>(threadIdx.x) * kEach + i;
    const float place = (static_cast<float>(places[i]) * __builtin_amdgcn_rcpf(fmaxf(static_cast<float>(counts[i]), 1.f)) + 0.5f) * (1.f / 256);
    of[i] = b < kCounts - 1 ? at_bound * exp2_near((b + static_cast<double>(place)) * per_bin) : 0.0;   // (what is further away, under a mask, weighs nothing, or the thresholds do not hold)
    n_mine += counts[i];
    m_mine += static_cast<double>(counts[i]) * of[i];
  }
  const u64 n_before = all.scan(n_mine, &n_all);
  const double m_before = all.scan(m_mine, &m_all);
  const double f_mass = static_cast<double>(front) / d.one;
  if (threadIdx.x == 0) {
    s.found_bin = kCounts;
    s.found_drest = f_mass + m_all;
    s.found_rest = 0;
    s.found_id = s.n_groups = kCounts - 1;
  }
  __syncthreads();
  if (d.k > 0) {                                             // the bin of the k-th token; all of the front are among the first k
    const u64 k_rest = static_cast<u64>(d.k - n_front);
    u64 n = n_before;
    double m = m_before;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      if (n < k_rest && k_rest <= n + counts[i]) {
        s.found_bin = threadIdx.x * kEach + i;
        s.found_rest = k_rest - n;
        s.found_drest = f_mass + m + static_cast<double>(k_rest - n) * of[i];
      }
      n += counts[i];
      m += static_cast<double>(counts[i]) * of[i];
    }
    __syncthreads();
  }
  int k_bin = static_cast<int>(s.found_bin);
  // the last bin holds all that is further away, a mask's lowest numbers among it: where that weighs nothing it does not matter which of it are among the first k
  if (k_bin == kCounts - 1 && d.weight(q.edge(k_bin)) == 0) k_bin = kCounts;
  const double total = !d.by_min() && d.k == 0 ? d.all : s.found_drest;   // what top_p is of, nearly
  int b1 = 0, b2 = -1;
  const double need = d.p * total - f_mass, off = (5e-4 + per_bin * per_bin / 16) * fabs(need) + 1e-6 * total;   // (logits of a bin are not all in one place)
  if (d.p < 1.0 && need + off > 0.0) {
    int from = kCounts - 1, to = kCounts - 1;                    // the thread's first bin that reaches the lower end, and the upper one
    double m = m_before + m_mine;
#pragma unroll
    for (int i = kEach - 1; i >= 0; --i) {
      const int b = static_cast<int>(threadIdx.x) * kEach + i;
      if (need - off <= m) from = b;
      if (need + off <= m) to = b;
      m -= static_cast<double>(counts[i]) * of[i];
    }
    from = -wave_max(-from);
    to = -wave_max(-to);
    if ((threadIdx.x & 63) == 0) {
      atomicMin(&s.found_id, from);
      atomicMin(&s.n_groups, to);
    }
    __syncthreads();
    b2 = min(s.n_groups + 1, min(k_bin, kCounts - 1));
    b1 = min(max(s.found_id - 1, 0), b2);
  }
  // the thresholds, a lane to each
  const int lane = threadIdx.x & 63, bin = lane == 0 ? b1 : lane == 1 ? b2 + 1 : lane == 2 ? k_bin : min(k_bin + 1, kCounts);
  const float edge = q.edge(bin);
  const float e1 = __shfl(edge, 0, kWave), e2 = __shfl(edge, 1, kWave);
  Bracket r;
  r.k_from = __shfl(edge, 2, kWave);
  r.k_to = __shfl(edge, 3, kWave);
  r.k_in_bin = s.found_rest;
  const bool by_p = d.p < 1.0, total_open = d.k > 0 || d.by_min();
  r.sure = !by_p ? r.k_from : b2 < 0 ? INFINITY : e1;
  r.list = !by_p ? r.k_from : b2 < 0 ? INFINITY : e2;
  r.last = total_open || !by_p ? r.k_to : r.list;
  __syncthreads();
  return r;
}
// Second pass, of the units [u0, u1): the sum of what is in for certain of every unit, of all units what else top_p may be of, and the list.
// The sums are of the bits of x + 2^52, x a weight as a whole number: without a mask, 2^52's own bits are taken off the sixteen at the end.
template <typename In, int T>
__device__ __forceinline__ void sum_units(const RowSource<In, T>& row, const Binning& q, const Bracket& r, const RowDraw& d, int u0, int u1, u64* unit_sum, float* list_z,
                                          int* list_id, int* n_list, int room, u64& sure, u64& rest) {
  const bool total_open = d.p < 1.0 && (d.k > 0 || d.by_min());
  for (int u = u0 + static_cast<int>(threadIdx.x >> 6); u < u1; u += T / kWave) {
    u64 unit = 0;
    const float most = row.unit_max[u];
    if (most >= q.lo && most > -INFINITY) {
      float x[kPerLane];
      load_unit(row.z, row.V, u, x);
      uint32_t mask = 0;                                     // of what the lane lists
#pragma unroll
      for (int i = 0; i < kPerLane; ++i) {
        const bool has = q.has(x[i]), list = has && r.lists(x[i]);
        if (list) mask |= 1u << i;
        const float z = has && !list && x[i] > r.last ? x[i] : -INFINITY;   // a weight of nothing
        if (!__ballot(z > -INFINITY)) {
          unit += RowDraw::kNothing;
          if (total_open) rest += RowDraw::kNothing;
        } else if (!total_open) {
          unit += d.bits(d.w(z > r.sure ? z : -INFINITY));
        } else {
          const u64 w = d.bits(d.w(z));
          unit += z > r.sure ? w : RowDraw::kNothing;
          rest += z > r.sure ? RowDraw::kNothing : w;
        }
      }
      unit -= kPerLane * RowDraw::kNothing;
      if (total_open) rest -= kPerLane * RowDraw::kNothing;
      if (__ballot(mask)) {                                  // one place for all that a wavefront lists of a unit
        const int mine = __popc(mask), upto = static_cast<int>(lanes_scan(static_cast<u64>(mine)));
        int at = 0;
        if ((threadIdx.x & 63) == 63) at = atomicAdd(n_list, upto);
        at = __shfl(at, 63, kWave) + upto - mine;
#pragma unroll
        for (int i = 0; i < kPerLane; ++i)
          if (mask >> i & 1) {
            if (at < room) {
              list_z[at] = x[i];
              list_id[at] = token_of<In>(u, i);
            }
            ++at;
          }
      }
      sure += unit;
      unit = lanes_sum(unit);
    }
    if ((threadIdx.x & 63) == 0) unit_sum[u] = unit;
  }
}
// From the lists and sums, in LDS: the borders, and the token.  id -1: the border of top_p lies elsewhere.
template <typename In, int T>
__device__ __forceinline__ Drawn draw_listed(const RowSource<In, T>& row, RowShared<T>& s, Block<T>& all, u64* s_unit, const Binning& q, const Bracket& r, int n_front, int n_list,
                                             u64 sure, u64 rest, const RowDraw& d) {
  Cut first, run;
  const ListSource<T> listed{&s, 0, n_list}, front_list{&s, 0, n_front}, behind{&s, n_front, n_list};
  for (int i = threadIdx.x; i < n_list; i += T) s.list_w[i] = d.weight(s.list_z[i]);
  __syncthreads();
  u64 mass;
  const float none = -INFINITY;
  if (r.k_from > -INFINITY)
    first = cut_at(behind, s, all, none, d, [&](float z, int, auto) { return u64{z <= r.k_from && z > r.k_to}; }, r.k_in_bin, &mass, Bracket::span(r.k_from, r.k_to));
  auto of_first = [&](float z, int id, auto w) { return first.in(z, id) ? w() : u64{0}; };
  auto in_bins = [&](float z, int id, auto w) { return z <= r.sure && z > r.list ? of_first(z, id, w) : u64{0}; };
  u64 in_front = 0, in_behind = 0, have = 0, other = 0;
  front_list.each(none, d, [&](float, int, auto w) { in_front += w(); });
  behind.each(none, d, [&](float z, int id, auto w) { in_behind += of_first(z, id, w); have += in_bins(z, id, w); });
  all.sum(in_front, in_behind);
  all.sum(have, other);
  mass = in_front + sure + in_behind + rest;
  if (d.p < 1.0) {
    const u64 need = d.needed(mass);
    if (need <= in_front) {
      run = cut_at(front_list, s, all, none, d, [](float, int, auto w) { return w(); }, need, &mass);
      for (int u = threadIdx.x; u < row.units; u += T) s_unit[u] = 0;
    } else {
      if (need <= in_front + sure || need > in_front + sure + have) return Drawn{-1, 0};
      run = cut_at(behind, s, all, none, d, in_bins, need - in_front - sure, &mass, Bracket::span(r.sure, r.list));
      mass += in_front + sure;
    }
  }
  auto kept = [&](float z, int id, auto w) { return run.in(z, id) ? of_first(z, id, w) : u64{0}; };
  __syncthreads();
  listed.each(none, d, [&](float z, int id, auto w) {
    const u64 x = kept(z, id, w);
    if (x) atomicAdd(&s_unit[id / kUnit], x);
  });
  __syncthreads();
  return Drawn{token_beyond(row, s, all, s_unit, [&](float z, int id) { return kept(z, id, [&] { return d.weight(z); }); }, d.target(mass)), mass};
}

// The least of the lanes' numbers that is not negative into *to, which all but the first such lane of a wavefront leave alone: numbers rise with the lanes.
__device__ __forceinline__ void first_of(int* to, int mine) {
  const u64 have = __ballot(mine >= 0);
  if (have && (threadIdx.x & 63) == static_cast<unsigned>(__ffsll(static_cast<long long>(have)) - 1)) atomicMin(reinterpret_cast<unsigned*>(to), static_cast<unsigned>(mine));
}
// No filter: the unit from the units' masses, then the token.  A row alone, or one whose settings lie in arrays, has another T than others: the sums' order does not depend on it.
template <typename In, int T, class Shared>
__device__ __forceinline__ Drawn draw_unfiltered(const RowSource<In, T>& row, Shared& s, Block<T>& block, const float* ref_of, const double* mass_of, const Weigh& w, double u, double all) {
  const double target = product(u, all);
  auto mass = [&](int i) { return product(mass_of[i], w(row.extreme(ref_of[i]))); };
  if (threadIdx.x == 0) s.found_id = -1;
  int unit = -1;
  double before = 0.0;
  for (int u0 = 0; u0 < row.units && unit < 0; u0 += T) {
    const int i = u0 + threadIdx.x;
    const double mine = i < row.units ? mass(i) : 0.0;
    double upto;
    const double excl = block.scan(mine, &upto, before);
    first_of(&s.found_id, mine > kNoWeight && excl + mine > target ? i : -1);
    __syncthreads();
    unit = s.found_id;
    if (i == unit) s.found_drest = target - excl;
    before = upto;
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
  constexpr int kEach = 4;                                   // by as many threads as that takes
  static_assert(T >= kUnit / kEach, "a unit's tokens have their threads");
  const bool has = threadIdx.x < kUnit / kEach;
  const int v = unit * kUnit + static_cast<int>(threadIdx.x) * kEach;
  double mine[kEach], sum = 0.0, total;
  int last = -1;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const float x = has ? row.at(v + i) : -INFINITY;
    mine[i] = x > -INFINITY ? w(x) : 0.0;
    if (!(mine[i] > kNoWeight)) mine[i] = 0.0;
    else last = v + i;
    sum += mine[i];
  }
  double run = block.scan(sum, &total);
  int passes = -1;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    run += mine[i];
    if (passes < 0 && mine[i] > 0.0 && run > rest) passes = v + i;
  }
  first_of(&s.found_id, passes);
  __syncthreads();
  const int id = s.found_id;
  __syncthreads();
  if (id >= 0) return Drawn{id, 0};
  if (last >= 0) atomicMax(&s.found_id, last);               // u = 1, or the unit's sum, added up in another order, ends above the target: its last token
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
  const float ref = row.extreme(top);
  for (int v = unit * kUnit + threadIdx.x; v < (unit + 1) * kUnit; v += T)
    if (row.at(v) == ref) atomicMin(&s.found_id, v);
  __syncthreads();
  return s.found_id;
}
template <int T>
struct PlainShared {
  u64 block[2][2][T / kWave];
  double found_drest;
  int found_id;
};
template <int T>
struct BinShared {
  u64 block[2][2][T / kWave];
  u64 found_rest;
  double found_drest;
  uint32_t found_bin;
  int found_id, n_groups;
};
// What the kernels of a row have in common: its largest logit, sums and settings.
struct RowCalls {
  Settings S;
  const int32_t* rowsel;
  int64_t c0;
  Summary A;
  const float* uniform;
  SampleOut out;
  int unit_bits;
};
template <typename In, int T>
__device__ __forceinline__ RowSource<In, T> row_source(const Logits<In>& L, const RowCalls& C, int64_t m, float top) {
  return RowSource<In, T>{L.row(m), L.V, L.units, C.A.unit + m * L.units, Extreme(top)};
}
__device__ __forceinline__ RowDraw row_draw(const RowCalls& C, int64_t row, float ref, double t, double u, double all, int V) {
  RowDraw d{ref, Weigh(ref, scale_of(t)), C.S.k(row), C.S.p(row), C.S.m(row), u, all, ldexp(1.0, C.unit_bits), 32 - __clz(V - 1)};
  if (d.k >= V || d.k < 0) d.k = 0;
  d.p = d.p < 1.0 ? fmax(d.p, 0.0) : 1.0;
  d.m = d.m > 0.0 ? fmin(d.m, 1.0) : 0.0;
  return d;
}
__device__ __forceinline__ double row_uniform(const RowCalls& C, int64_t row) {
  const double u = C.uniform[row];
  return u > 0.0 ? fmin(u, 1.0) : 0.0;
}
// By one thread.  zi, ref: the token's logit and the largest, sum: of exp(z - ref); kept: the mass that it was drawn from.
__device__ __forceinline__ void write_drawn(const SampleOut& out, int64_t row, int id, float zi, float ref, double sum, double t, double kept) {
  out.ids[row] = id;
  const double gap = zi == ref ? 0.0 : static_cast<double>(zi) - static_cast<double>(ref);
  if (out.logp) out.logp[row] = static_cast<float>(gap - log_of(sum));
  if (out.logq) out.logq[row] = t > 0.0 ? static_cast<float>(gap / t - log_of(kept)) : 0.f;
}
// A row that its front did not decide, on its way through the launches behind.
struct RowState {
  int bins;                                                  // bins serve; else it is gone through bit by bit
  float top, bound;
  int n_front, n_list;
  double all, sum;
  u64 front, rest;
  Bracket bracket;
};
struct FlatWs {
  int* count;                                                // of such rows, cleared by the first launch
  int* order;                                                // [rows]: their numbers, as they came
  RowState* state;                                           // [rows]
  uint32_t* counts;                                          // [rows][parts][kCounts]
  u64* unit_sum;                                             // [rows][units]
  float* list_z;                                             // [rows][kListCap]
  int* list_id;
  int parts;
};
enum class Filter { kNone, kSome, kSomeInOne };              // no row has one; rows may have; ... and the launch does all of a row

// A workgroup to a row.
template <typename In, int T, Filter FILTER>
__global__ void __launch_bounds__(T)
k_sample_row(Logits<In> L, RowCalls C, FlatWs F) {
  __shared__ std::conditional_t<FILTER == Filter::kNone, PlainShared<T>, std::conditional_t<FILTER == Filter::kSome, RowShared<T, 2 * kRanked, false>, RowShared<T>>> s;
  const int64_t m = blockIdx.x, row = C.rowsel ? C.rowsel[C.c0 + m] : C.c0 + m;
  const float* const unit_max = C.A.unit + m * L.units;
  const float* const ref_of = C.A.ref + m * L.units;
  const double *const mass_of = C.A.mass + m * L.units, *const sum_of = C.A.sum + m * L.units;
  const double t = C.S.t(row), u = row_uniform(C, row);
  float top = -INFINITY;
  for (int i = threadIdx.x; i < L.units; i += T) top = larger(top, unit_max[i]);
  Block<T> block(s.block);
  top = block.max(top);
  if (top == -INFINITY) {                                    // nothing to draw from
    if (threadIdx.x == 0) {
      C.out.ids[row] = -1;
      if (C.out.logp) C.out.logp[row] = 0.f;
      if (C.out.logq) C.out.logq[row] = 0.f;
    }
    return;
  }
  const RowSource<In, T> src = row_source<In, T>(L, C, m, top);
  const float ref = src.extreme(top);
  const Weigh w(ref, scale_of(t)), w1(ref, kLog2e64);
  double sum = 0.0, all = 0.0;                               // of exp(z - top), for the log-prob of the softmax itself, and of the weights
  for (int u0 = 0; u0 < L.units; u0 += T) {
    const int i = u0 + threadIdx.x;
    double mine = 0.0, mass = 0.0;
    if (i < L.units) {
      const float x = src.extreme(ref_of[i]);
      mine = product(sum_of[i], w1(x));
      mass = product(mass_of[i], w(x));
    }
    block.add(sum, all, mine, mass);
  }
  int id;
  double kept = all;
  if (!(t > 0.0)) {
    id = largest(src, s, top);
  } else if constexpr (FILTER == Filter::kNone) {
    id = draw_unfiltered(src, s, block, ref_of, mass_of, w, u, all).id;
  } else {
    const RowDraw d = row_draw(C, row, ref, t, u, all, L.V);
    if (d.k == 0 && d.p == 1.0 && d.m == 0.0) {
      id = draw_unfiltered(src, s, block, ref_of, mass_of, w, u, all).id;
    } else {
      const float* const group_max = C.A.group + m * L.units * kGroupsPerUnit;
      float bound = -INFINITY;                               // up to as many as can be ordered: all of them
      Drawn got{-1, 0};
      int n = 0;
      if (!src.extreme.is) {
        // under min_p what is not below its border is all that counts, where that is not too much
        bool listed = false;
        if (d.by_min()) {
          const float least = Binning::least_logit(d, d.m);
          listed = list_front(src, group_max, least, kRanked, s) && s.n_list <= kRanked;
          __syncthreads();
          if (listed) bound = least;
        }
        if (!listed) {
          if (L.V > kRanked) bound = front_bound<T>(group_max, L.units * kGroupsPerUnit, s);
          listed = list_front(src, group_max, bound, kGroupCap, s);
        }
        n = s.n_list;
        __syncthreads();
        const bool complete = bound == -INFINITY || (d.by_min() && d.weight(bound) == 0);
        if (listed && n <= kCompared) got = draw_from_front(s, block, n, complete, d);
        else if (listed && n <= kRanked) got = draw_from_long_front(s, block, n, bound, complete, d);
        if (!listed || n > kRanked) {                        // many that are alike: no front, bins from the largest on
          n = 0;
          bound = INFINITY;
        }
      }
      if (got.id < 0) {
        const bool bins = !src.extreme.is && bound > -INFINITY;
        if (bound == INFINITY) bound = d.w.next_above();
        u64 front = 0;
        for (int i = threadIdx.x; i < n; i += T) front += d.weight(s.list_z[i]);
        front = block.sum(front);
        if constexpr (FILTER == Filter::kSome) {
          for (int i = threadIdx.x; i < n; i += T) {
            F.list_z[m * kListCap + i] = s.list_z[i];
            F.list_id[m * kListCap + i] = s.list_id[i];
          }
          if (threadIdx.x == 0) {
            F.order[atomicAdd(F.count, 1)] = static_cast<int>(m);
            F.state[m] = RowState{bins ? 1 : 0, top, bound, n, n, all, sum, front, 0, Bracket{}};
          }
          return;
        } else {
          if (bins) {
            const Binning q(bound, d, L.V);
            uint32_t* const s_count = reinterpret_cast<uint32_t*>(s.bins);
            uint8_t* const s_off = reinterpret_cast<uint8_t*>(s.list_w);
            static_assert(kCounts * 4 <= sizeof(s.bins) && kCounts <= sizeof(s.list_w), "counts and places");
            for (int i = threadIdx.x; i < kCounts; i += T) s_count[i] = 0;
            __syncthreads();
            count_bins(src, q, 0, L.units, s_count, s_off);
            __syncthreads();
            uint32_t counts[kCounts / T], places[kCounts / T];
#pragma unroll
            for (int i = 0; i < kCounts / T; ++i) {
              const int b = threadIdx.x * (kCounts / T) + i;
              counts[i] = s_count[b];
              places[i] = counts[i] ? counts[i] * s_off[b] : 0;
            }
            __syncthreads();
            const Bracket r = bracket_of<T>(counts, places, s, block, q, front, n, d);
            if (threadIdx.x == 0) s.n_list = n;
            __syncthreads();
            u64 sure = 0, rest = 0;
            sum_units(src, q, r, d, 0, L.units, s.unit, s.list_z, s.list_id, &s.n_list, kListCap, sure, rest);
            block.sum(sure, rest);
            if (s.n_list <= kListCap) got = draw_listed(src, s, block, s.unit, q, r, n, s.n_list, sure, rest, d);
            __syncthreads();
          }
          if (got.id < 0) got = draw_by_passes<In, T>(src, &s, block.turn, s.unit, d);
        }
      }
      id = got.id;
      kept = static_cast<double>(got.mass) / d.one;
    }
  }
  if (threadIdx.x == 0) write_drawn(C.out, row, id, src.at(id), ref, sum, t, kept);
}
// Rows that are spread, a part of the units to a workgroup: the counts, ...  (A row's last workgroup to find out what they say would need a fence, whose
// writing back of the caches took the launch from 17 us to 165.)
template <typename In, int T>
__global__ void __launch_bounds__(T)
k_sample_count(Logits<In> L, RowCalls C, FlatWs F) {
  __shared__ uint32_t s_count[kCounts];
  __shared__ uint8_t s_off[kCounts];
  if (static_cast<int>(blockIdx.y) >= *F.count) return;
  const int64_t m = F.order[blockIdx.y];
  RowState& state = F.state[m];
  if (!state.bins) return;
  const int64_t row = C.rowsel ? C.rowsel[C.c0 + m] : C.c0 + m;
  const RowSource<In, T> src = row_source<In, T>(L, C, m, state.top);
  const RowDraw d = row_draw(C, row, state.top, C.S.t(row), 0.0, state.all, L.V);
  const Binning q(state.bound, d, L.V);
  for (int i = threadIdx.x; i < kCounts; i += T) s_count[i] = 0;
  __syncthreads();
  count_bins(src, q, L.units * static_cast<int>(blockIdx.x) / F.parts, L.units * static_cast<int>(blockIdx.x + 1) / F.parts, s_count, s_off);
  __syncthreads();
  uint32_t* const to = F.counts + (m * F.parts + blockIdx.x) * kCounts;
  for (int i = threadIdx.x; i < kCounts; i += T) to[i] = s_count[i] ? s_count[i] | static_cast<uint32_t>(s_off[i]) << kOffShift : 0;
}
// ... what they say, ...
template <int T>
__global__ void __launch_bounds__(T)
k_sample_bracket(RowCalls C, FlatWs F, int V) {
  constexpr int kEach = kCounts / T;
  __shared__ BinShared<T> s;
  if (static_cast<int>(blockIdx.x) >= *F.count) return;
  const int64_t m = F.order[blockIdx.x];
  RowState& state = F.state[m];
  if (!state.bins) return;
  const int64_t row = C.rowsel ? C.rowsel[C.c0 + m] : C.c0 + m;
  const RowDraw d = row_draw(C, row, state.top, C.S.t(row), 0.0, state.all, V);
  const Binning q(state.bound, d, V);
  uint32_t counts[kEach] = {}, places[kEach] = {};
  auto take = [&](int i, uint32_t x) {
    const uint32_t n = x & ((1u << kOffShift) - 1);
    counts[i] += n;
    places[i] += n * (x >> kOffShift);
  };
  static_assert(kEach % 4 == 0, "sixteen bytes at a time");
  constexpr int kAtOnce = 4;                                 // parts under way
  for (int p = 0; p < F.parts; p += kAtOnce) {
    uint4 x[kAtOnce][kEach / 4];
#pragma unroll
    for (int b = 0; b < kAtOnce; ++b)
#pragma unroll
      for (int i = 0; i < kEach / 4; ++i)
        x[b][i] = p + b < F.parts ? reinterpret_cast<const uint4*>(F.counts + (m * F.parts + p + b) * kCounts + threadIdx.x * kEach)[i] : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
    for (int b = 0; b < kAtOnce; ++b)
#pragma unroll
      for (int i = 0; i < kEach / 4; ++i) {
        take(4 * i, x[b][i].x);
        take(4 * i + 1, x[b][i].y);
        take(4 * i + 2, x[b][i].z);
        take(4 * i + 3, x[b][i].w);
      }
  }
  Block<T> block(s.block);
  const Bracket r = bracket_of<T>(counts, places, s, block, q, state.front, state.n_front, d);
  if (threadIdx.x == 0) state.bracket = r;
}
// ... then the sums and lists, ...
constexpr int kSumUnits = 4, kSumList = 2048;               // of a workgroup (24 float32 rows of 152 064 under top_p with 2, 4, 8 and 16: 60.4, 59.7, 65.0 and 75.9 us)
template <typename In, int T>
__global__ void __launch_bounds__(T, 4)
k_sample_sums(Logits<In> L, RowCalls C, FlatWs F) {
  __shared__ u64 s_block[2][2][T / kWave];
  __shared__ float s_z[kSumList];
  __shared__ int s_id[kSumList];
  __shared__ int s_n, s_at;
  if (static_cast<int>(blockIdx.y) >= *F.count) return;
  const int64_t m = F.order[blockIdx.y];
  RowState& state = F.state[m];
  if (!state.bins) return;
  const int64_t row = C.rowsel ? C.rowsel[C.c0 + m] : C.c0 + m;
  const RowSource<In, T> src = row_source<In, T>(L, C, m, state.top);
  const RowDraw d = row_draw(C, row, state.top, C.S.t(row), 0.0, state.all, L.V);
  Block<T> block(s_block);
  if (threadIdx.x == 0) s_n = 0;
  __syncthreads();
  u64 sure = 0, rest = 0;
  const int u0 = blockIdx.x * kSumUnits;
  sum_units(src, Binning(state.bound, d, L.V), state.bracket, d, u0, min(u0 + kSumUnits, L.units), F.unit_sum + m * L.units, s_z, s_id, &s_n, kSumList, sure, rest);
  rest = block.sum(rest);
  // the workgroup's list behind the others' (by every wavefront for itself it took twice the launch: all wait at one address)
  const int n = s_n;
  if (threadIdx.x == 0) {
    s_at = n > 0 ? atomicAdd(&state.n_list, n <= kSumList ? n : kListCap + 1) : 0;   // more than there is room for: the row's list is full
    if (rest) atomicAdd(&state.rest, rest);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < min(n, kSumList); i += T) {
    const int at = s_at + i;
    if (at < kListCap) {
      F.list_z[m * kListCap + at] = s_z[i];
      F.list_id[m * kListCap + at] = s_id[i];
    }
  }
}
// ... and the token, a workgroup to a row.
template <typename In, int T>
__global__ void __launch_bounds__(T)
k_sample_flat(Logits<In> L, RowCalls C, FlatWs F) {
  __shared__ RowShared<T> s;
  if (static_cast<int>(blockIdx.x) >= *F.count) return;
  const int64_t m = F.order[blockIdx.x];
  const RowState& state = F.state[m];
  const int64_t row = C.rowsel ? C.rowsel[C.c0 + m] : C.c0 + m;
  const RowSource<In, T> src = row_source<In, T>(L, C, m, state.top);
  const float ref = src.extreme(state.top);
  const double t = C.S.t(row);
  const RowDraw d = row_draw(C, row, ref, t, row_uniform(C, row), state.all, L.V);
  Block<T> block(s.block);
  Drawn got{-1, 0};
  const int n = state.n_list;
  if (state.bins && n <= kListCap) {
    for (int i = threadIdx.x; i < n; i += T) {
      s.list_z[i] = F.list_z[m * kListCap + i];
      s.list_id[i] = F.list_id[m * kListCap + i];
    }
    u64 sure = 0;
    for (int i = threadIdx.x; i < L.units; i += T) sure += s.unit[i] = F.unit_sum[m * L.units + i];
    sure = block.sum(sure);
    got = draw_listed(src, s, block, s.unit, Binning(state.bound, d, L.V), state.bracket, state.n_front, n, sure, state.rest, d);
    __syncthreads();
  }
  if (got.id < 0) got = draw_by_passes<In, T>(src, &s, block.turn, s.unit, d);
  if (threadIdx.x == 0) write_drawn(C.out, row, got.id, src.at(got.id), ref, state.sum, t, static_cast<double>(got.mass) / d.one);
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
constexpr int64_t kSampleRows = 1024;                        // rows of a chunk
// A single row: its workgroup does all of it, 19 us in place of 24 of 152 064 logits where the front decides, 155 in place of 56 where it does not, which has to be so for one draw in
// twenty to weigh as much.  Of four rows any may be spread: 156 and 58 us.
constexpr int64_t kRowsInOne = 1;
struct SampleWs {
  Summary A;
  FlatWs flat;
  float* z;
  double* z64;
  char* room;
  size_t room_bytes;
  size_t bytes;
};
// Workgroups to a row that is spread, of as many rows; 0: the row's own does all of it.
int flat_parts(int64_t rows) { return rows <= kRowsInOne ? 0 : static_cast<int>(std::min<int64_t>(std::max<int64_t>(2048 / rows, 4), 16)); }
int units_of(int V) { return static_cast<int>(cdiv(V, kUnit)); }
void carve(Carver& c, SampleWs& w, int64_t rows, int V) {
  w = SampleWs{};
  const size_t units = static_cast<size_t>(rows) * units_of(V);
  w.A.group = c.take<float>(units * kGroupsPerUnit);
  w.A.unit = c.take<float>(units);
  w.A.ref = c.take<float>(units);
  w.A.mass = c.take<double>(units);
  w.A.sum = c.take<double>(units);
  w.flat.parts = flat_parts(rows);
  if (w.flat.parts > 0) {
    w.flat.count = c.take<int>(1);
    w.flat.order = c.take<int>(rows);
    w.flat.state = c.take<RowState>(rows);
    w.flat.counts = c.take<uint32_t>(static_cast<size_t>(std::min(rows * 16, std::max<int64_t>(2048, rows * 4))) * kCounts);   // as many as any count of rows up to it takes
    w.flat.unit_sum = c.take<u64>(units);
    w.flat.list_z = c.take<float>(static_cast<size_t>(rows) * kListCap);
    w.flat.list_id = c.take<int>(static_cast<size_t>(rows) * kListCap);
  }
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
constexpr int kRowT = 1024, kOneT = 512, kPlainT = 256, kFlatT = 512, kSumT = 256;
template <typename In>
umas_status sample_rows(const Logits<In>& L, const Settings& S, const int32_t* rowsel, int64_t c0, int64_t rows, const SampleWs& w, const float* u, const SampleOut& out,
                        hipStream_t st) {
  const unsigned n = static_cast<unsigned>(rows);
  hipLaunchKernelGGL(k_sample_open<In>, dim3(cdiv(L.units, 2 * kOpenPairs), n), dim3(kOpenT), 0, st, L, S, rowsel, c0, w.A, w.flat.parts > 0 ? w.flat.count : nullptr);
  UMAS_LAUNCHED("k_sample_open");
  const bool plain = !S.top_k_of && !S.top_p_of && !S.min_p_of && S.min_p == 0.0 && S.top_p == 1.0 && (S.top_k == 0 || S.top_k >= L.V);
  const bool greedy = !S.temperature_of && S.temperature == 0.0;
  const RowCalls C{S, rowsel, c0, w.A, u, out, bits_of(L.V)};
  if (plain || greedy) {
    hipLaunchKernelGGL((k_sample_row<In, kPlainT, Filter::kNone>), dim3(n), dim3(kPlainT), 0, st, L, C, w.flat);
    UMAS_LAUNCHED("k_sample_row");
    return UMAS_OK;
  }
  // the front decides where it holds the first k, or all that min_p leaves, but for rows of many equal logits: no launches for others, which cost 4 us each where there is nothing for them to do
  // (bf16 rows of 152 064 under top_k 20: 2 rows 18 us and with them 23.5, 24 rows 18.7 and 24.5, 256 rows 33 and 41, 1024 rows 116 and 124; float32 the same differences)
  const bool decided = !S.top_k_of && S.top_k >= 1 && S.top_k <= std::min(kTopRank, L.units * kGroupsPerUnit / 8);
  if (w.flat.parts == 0 || decided) {
    hipLaunchKernelGGL((k_sample_row<In, kOneT, Filter::kSomeInOne>), dim3(n), dim3(kOneT), 0, st, L, C, w.flat);
    UMAS_LAUNCHED("k_sample_row");
    return UMAS_OK;
  }
  const dim3 parts(w.flat.parts, n);
  hipLaunchKernelGGL((k_sample_row<In, kRowT, Filter::kSome>), dim3(n), dim3(kRowT), 0, st, L, C, w.flat);
  UMAS_LAUNCHED("k_sample_row");
  hipLaunchKernelGGL((k_sample_count<In, kFlatT>), parts, dim3(kFlatT), 0, st, L, C, w.flat);
  UMAS_LAUNCHED("k_sample_count");
  hipLaunchKernelGGL((k_sample_bracket<kFlatT>), dim3(n), dim3(kFlatT), 0, st, C, w.flat, L.V);
  UMAS_LAUNCHED("k_sample_bracket");
  hipLaunchKernelGGL((k_sample_sums<In, kSumT>), dim3(cdiv(L.units, kSumUnits), n), dim3(kSumT), 0, st, L, C, w.flat);
  UMAS_LAUNCHED("k_sample_sums");
  hipLaunchKernelGGL((k_sample_flat<In, kFlatT>), dim3(n), dim3(kFlatT), 0, st, L, C, w.flat);
  UMAS_LAUNCHED("k_sample_flat");
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
  return head_bytes(n_sel, kSampleRows, d, V, dtype);
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
  int64_t cap = std::min(n_sel, kSampleRows);
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
