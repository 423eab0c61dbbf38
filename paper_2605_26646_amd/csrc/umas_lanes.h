// Exchanges between the lanes of a wavefront by moves of the vector unit, and sorting networks of 64 made of them.
#pragma once

#include "umas_common.h"

namespace umas {
namespace {

// The value of lane ^ J, J a power of two or 63: moves of the vector unit.  (Through LDS, which a __shfl_xor is, an exchange waits for a round trip of it.)
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t x) { return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), CTRL, 0xF, 0xF, true)); }
template <int J>
__device__ __forceinline__ uint32_t lane_xor(uint32_t x) {
  const int lane = threadIdx.x & 63;
  if constexpr (J == 1) return dpp<0xB1>(x);
  else if constexpr (J == 2) return dpp<0x4E>(x);
  else if constexpr (J == 4) return dpp<0x1B>(dpp<0x141>(x));   // ^ 7, ^ 3
  else if constexpr (J == 8) return dpp<0x128>(x);
  else if constexpr (J == 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);   // of every two groups of sixteen: twice the first, twice the second
    return lane & 16 ? r[0] : r[1];
  } else if constexpr (J == 32) {
    const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return lane & 32 ? r[0] : r[1];
  } else {
    static_assert(J == 63, "");
    return lane_xor<32>(lane_xor<16>(dpp<0x140>(x)));
  }
}
template <int J>
__device__ __forceinline__ float lane_xor(float x) { return __uint_as_float(lane_xor<J>(__float_as_uint(x))); }
template <int J>
__device__ __forceinline__ unsigned long long lane_xor(unsigned long long x) {
  return static_cast<unsigned long long>(lane_xor<J>(static_cast<uint32_t>(x >> 32))) << 32 | lane_xor<J>(static_cast<uint32_t>(x));
}
__device__ __forceinline__ unsigned long long either(bool larger, unsigned long long x, unsigned long long y) { return (x > y) == larger ? x : y; }
__device__ __forceinline__ float either(bool larger, float x, float y) { return larger ? fmaxf(x, y) : fminf(x, y); }
// A list of 64, one to a lane, that falls and then rises, or the like of it in runs of 2 J: falling in runs of K, rising in every second of them.
template <int K, int J = K / 2, class T>
__device__ __forceinline__ T order_runs(T x) {
  const int lane = threadIdx.x & 63;
  x = either(((lane & J) == 0) == ((lane & K) == 0), x, lane_xor<J>(x));
  if constexpr (J > 1) return order_runs<K, J / 2>(x);
  else return x;
}
template <int K = 2, class T>
__device__ __forceinline__ T sorted_desc(T x) {
  x = order_runs<K>(x);
  if constexpr (K < kWave) return sorted_desc<K * 2>(x);
  else return x;
}
// The 64 largest of two falling lists, falling.
template <class T>
__device__ __forceinline__ T merged(T x, T y) { return order_runs<kWave>(either(true, x, lane_xor<63>(y))); }

// Sums over the wavefront in 32 or 64 bits, by moves of the vector unit as well: of all lanes, and of the lanes up to the own one.
__device__ __forceinline__ double bits_of(unsigned long long x, double) { return __longlong_as_double(static_cast<long long>(x)); }
__device__ __forceinline__ unsigned long long bits_of(unsigned long long x, unsigned long long) { return x; }
__device__ __forceinline__ unsigned long long bits_in(double x) { return static_cast<unsigned long long>(__double_as_longlong(x)); }
__device__ __forceinline__ unsigned long long bits_in(unsigned long long x) { return x; }
template <class T>
__device__ __forceinline__ T lanes_sum(T x) {                 // double, unsigned long long
  x += bits_of(lane_xor<1>(bits_in(x)), T());
  x += bits_of(lane_xor<2>(bits_in(x)), T());
  x += bits_of(lane_xor<4>(bits_in(x)), T());
  x += bits_of(lane_xor<8>(bits_in(x)), T());
  x += bits_of(lane_xor<16>(bits_in(x)), T());
  x += bits_of(lane_xor<32>(bits_in(x)), T());
  return x;
}
// What the lane gets from another one, 0 where there is none: CTRL of DPP, in the rows of 16 lanes that ROWS names.
template <int CTRL, int ROWS>
__device__ __forceinline__ unsigned long long moved(unsigned long long x) {
  const uint32_t lo = static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), CTRL, ROWS, 0xF, false));
  const uint32_t hi = static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x >> 32), CTRL, ROWS, 0xF, false));
  return static_cast<unsigned long long>(hi) << 32 | lo;
}
template <class T>
__device__ __forceinline__ T lanes_scan(T x) {                // inclusive
  x += bits_of(moved<0x111, 0xF>(bits_in(x)), T());           // one, two, four, eight lanes up in a row of 16
  x += bits_of(moved<0x112, 0xF>(bits_in(x)), T());
  x += bits_of(moved<0x114, 0xF>(bits_in(x)), T());
  x += bits_of(moved<0x118, 0xF>(bits_in(x)), T());
  x += bits_of(moved<0x142, 0xA>(bits_in(x)), T());           // a row's last lane to the next row, then the half's to the other half
  x += bits_of(moved<0x143, 0xC>(bits_in(x)), T());
  return x;
}

}  // namespace
}  // namespace umas
