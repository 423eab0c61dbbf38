// Root-mean-square norm in front of a head: s = x + r, i = 1 / sqrt(mean s^2 + eps), y = s i g, and its backward pass.
//
//   forward   a row stays in registers between its sum of squares and what is written: one read of x and r, one write of s and y
//   8 bits    c = max_j |y_j| / 448 (448 is the largest e4m3 number), q_j = e4m3(y_j / c): a second reduction over the same registers.  y_j / c = 448 s_j gain_j / max_k |s_k gain_k|
//             does not depend on i, and is taken without it: of bf16 the products are exact, so that the quotient is rounded once to float32, and nothing that lies next to a border of
//             e4m3 falls to the other side.  (About one in 2500 lies on one; with y_j and c themselves, both rounded, a fifth of
//             these went to the uneven side, others with another number of rows.)
//   backward  with a_j = dy_j g_j:  dx = i (a - s i^2/d sum_k a_k s_k) + ds,  dg = sum over rows of dy s i
// All of it is bound by memory: four arrays of n d elements each way.
#include <algorithm>
#include <type_traits>

#include "umas_logits.h"

namespace umas {
namespace {

constexpr int kNT = 256;                                     // threads of a workgroup
constexpr int kMaxNormD = 16384;

// 16 bytes of a row; rows of float32 of any width start at multiples of 4 bytes only, which a 16-byte load may here
typedef uint32_t u32x4u __attribute__((ext_vector_type(4), aligned(4)));
template <typename T> struct Piece;
template <> struct Piece<uint16_t> {
  static constexpr int N = 8;
  __device__ static __forceinline__ void unpack(const u32x4u& v, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(v[i] << 16);
      x[2 * i + 1] = __uint_as_float(v[i] & 0xFFFF0000u);
    }
  }
  __device__ static __forceinline__ u32x4u pack(const float (&x)[8]) {
    return u32x4u{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])};
  }
};
template <> struct Piece<float> {
  static constexpr int N = 4;
  __device__ static __forceinline__ void unpack(const u32x4u& v, float (&x)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(v[i]);
  }
  __device__ static __forceinline__ u32x4u pack(const float (&x)[4]) {
    return u32x4u{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
  }
};
// Piece p of a row of d elements; of the last one only what exists (float32, d no multiple of 4).
template <typename T>
__device__ __forceinline__ u32x4u load_piece(const T* row, int p, int d) {
  constexpr int N = Piece<T>::N;
  if (std::is_same<T, uint16_t>::value || (p + 1) * N <= d) return *reinterpret_cast<const u32x4u*>(row + p * N);
  u32x4u v = {0u, 0u, 0u, 0u};
  for (int i = 0; i < d - p * N; ++i) v[i] = reinterpret_cast<const uint32_t*>(row)[p * N + i];
  return v;
}
template <typename T>
__device__ __forceinline__ void store_piece(T* row, int p, int d, const u32x4u& v) {
  constexpr int N = Piece<T>::N;
  if (std::is_same<T, uint16_t>::value || (p + 1) * N <= d) {
    *reinterpret_cast<u32x4u*>(row + p * N) = v;
    return;
  }
  for (int i = 0; i < d - p * N; ++i) reinterpret_cast<uint32_t*>(row)[p * N + i] = v[i];
}
// Over the T threads of a row: a wavefront, or the workgroup.
template <int T, class F>
__device__ __forceinline__ float row_reduce(float v, float* s, F f) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = f(v, __shfl_xor(v, o, kWave));
  if constexpr (T == kNT) {
    __syncthreads();                                         // s may still be read from the reduction before
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
    __syncthreads();
    v = s[0];
#pragma unroll
    for (int w = 1; w < kNT / kWave; ++w) v = f(v, s[w]);
  }
  return v;
}
__device__ __forceinline__ float add(float a, float b) { return a + b; }
// largest, and not a number where one of the two is none
__device__ __forceinline__ float most(float a, float b) { return a >= b ? a : b >= a ? b : a + b; }

struct NormArgs {
  const void *x, *residual, *gain;
  int64_t n;
  int d;
  float eps;
  void *hidden, *y;
  uint8_t* q;
  float *scale, *inv_rms;
};
template <typename E, int T, int NV, bool QUANT>
__global__ void __launch_bounds__(kNT)
k_rms_norm(NormArgs A) {
  constexpr int N = Piece<E>::N, kRows = kNT / T;
  __shared__ float s_red[kNT / kWave];
  const int t = threadIdx.x % T, pieces = (A.d + N - 1) / N;
  // a row to a workgroup or wavefront, and more only where there are more than a grid holds
  for (int64_t row = static_cast<int64_t>(blockIdx.x) * kRows + threadIdx.x / T; row < A.n; row += static_cast<int64_t>(gridDim.x) * kRows) {
    const E* const x = static_cast<const E*>(A.x) + row * A.d;
    const E* const r = A.residual ? static_cast<const E*>(A.residual) + row * A.d : nullptr;
    E* const hidden = A.hidden ? static_cast<E*>(A.hidden) + row * A.d : nullptr;
    u32x4u v[NV], g[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) v[k] = t + k * T < pieces ? load_piece(x, t + k * T, A.d) : u32x4u{0u, 0u, 0u, 0u};
    if (r) {
      u32x4u w[NV];
#pragma unroll
      for (int k = 0; k < NV; ++k) w[k] = t + k * T < pieces ? load_piece(r, t + k * T, A.d) : u32x4u{0u, 0u, 0u, 0u};
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        float a[N], b[N];
        Piece<E>::unpack(v[k], a);
        Piece<E>::unpack(w[k], b);
#pragma unroll
        for (int i = 0; i < N; ++i) a[i] += b[i];
        v[k] = Piece<E>::pack(a);                              // the norm is of the sum as it is stored
        if (hidden && t + k * T < pieces) store_piece(hidden, t + k * T, A.d, v[k]);
      }
    }
#pragma unroll
    for (int k = 0; k < NV; ++k) g[k] = t + k * T < pieces ? load_piece(static_cast<const E*>(A.gain), t + k * T, A.d) : u32x4u{0u, 0u, 0u, 0u};
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      float a[N];
      Piece<E>::unpack(v[k], a);
#pragma unroll
      for (int i = 0; i < N; ++i) sum = fmaf(a[i], a[i], sum);
    }
    sum = row_reduce<T>(sum, s_red, add);
    const float inv = 1.f / sqrtf(sum / static_cast<float>(A.d) + A.eps);
    // in 8 bits, inv's power of 2 in its place, which rounds nothing and keeps products where y is
    const float by = QUANT ? __uint_as_float(__float_as_uint(inv) & 0x7F800000u) : inv;
    if (A.inv_rms && t == 0) A.inv_rms[row] = inv;
    float c = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      float a[N], b[N];
      Piece<E>::unpack(v[k], a);
      Piece<E>::unpack(g[k], b);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        a[i] = a[i] * by * b[i];
        if constexpr (QUANT) c = most(c, fabsf(a[i]));
      }
      if constexpr (!QUANT)
        if (t + k * T < pieces) store_piece(static_cast<E*>(A.y) + row * A.d, t + k * T, A.d, Piece<E>::pack(a));
    }
    if constexpr (QUANT) {
      float top = row_reduce<T>(c, s_red, most);
      c = top > 0.f ? top * (inv / by) / 448.f : top;
      if (c == 0.f) {                                          // a row of zeros
        c = 1.f;
        top = INFINITY;
      }
      if (c == INFINITY) c = top = NAN;                        // an infinite gain, or a product beyond float32: no scale brings the row into 8 bits
      if (t == 0) A.scale[row] = c;
      uint8_t* const q = A.q + row * A.d;
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        if (t + k * T >= pieces) continue;
        float a[N], b[N];
        Piece<E>::unpack(v[k], a);
        Piece<E>::unpack(g[k], b);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          a[i] = a[i] * by * b[i] * 0.875f / top * 512.f;      // 448 = 7/8 of 512: nothing runs over, and of bf16 nothing rounds but the quotient
          // of float32, 7/8 of the largest one may round up; what is no number stays none
          if constexpr (std::is_same<E, float>::value) a[i] = a[i] > 448.f ? 448.f : a[i] < -448.f ? -448.f : a[i];
        }
        uint32_t w[N / 4];
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
          int p = __builtin_amdgcn_cvt_pk_fp8_f32(a[4 * i], a[4 * i + 1], 0, false);
          p = __builtin_amdgcn_cvt_pk_fp8_f32(a[4 * i + 2], a[4 * i + 3], p, true);
          w[i] = static_cast<uint32_t>(p);
        }
        const int at = (t + k * T) * N;
        if (std::is_same<E, uint16_t>::value) {
          typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
          if constexpr (N == 8) *reinterpret_cast<u32x2*>(q + at) = u32x2{w[0], w[1]};
        } else {
          for (int i = 0; i < 4 && at + i < A.d; ++i) q[at + i] = static_cast<uint8_t>(w[0] >> (8 * i));
        }
      }
    }
  }
}

// ------------------------------------------------------------------ backward
// T threads to a row, up to two pieces each, so that a row, the next one on its way, and the columns' share of dg over all rows that the threads do stay in
// registers at four wavefronts to a SIMD.  A workgroup's shares meet in LDS, the workgroups' in k_norm_gain, both in a fixed order.  A row whose dy is 0 throughout
// adds nothing, whatever it holds.
struct NormBackArgs {
  const void *dy, *hidden, *gain;
  const float* inv_rms;
  const void* dhidden;
  int64_t n;
  int d;
  void* dx;
  float* part;                                               // [gridDim.x][d]
};
template <int T> constexpr int kBackT = T < 256 ? 256 : T;   // threads of a workgroup
template <typename E, int NV, bool THROUGH>
struct BackRow {
  u32x4u y[NV], h[NV], th[THROUGH ? NV : 1];
  float inv;
  template <int T>
  __device__ __forceinline__ void load(const NormBackArgs& A, int64_t row, int t, int pieces) {
    const u32x4u none = {0u, 0u, 0u, 0u};
    if (row >= A.n) {                                        // nothing to add, nothing to write
#pragma unroll
      for (int k = 0; k < NV; ++k) y[k] = none;
      return;
    }
    const int64_t at = row * A.d;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int p = t + k * T;
      const bool in = p < pieces;
      y[k] = in ? load_piece(static_cast<const E*>(A.dy) + at, p, A.d) : none;
      h[k] = in ? load_piece(static_cast<const E*>(A.hidden) + at, p, A.d) : none;
      if constexpr (THROUGH) th[k] = in ? load_piece(static_cast<const E*>(A.dhidden) + at, p, A.d) : none;
    }
    inv = A.inv_rms[row];
  }
};
template <typename E, int T, int NV, bool THROUGH>
__global__ void __launch_bounds__(kBackT<T>)
k_norm_back(NormBackArgs A) {
  constexpr int N = Piece<E>::N, B = kBackT<T>, kRows = B / T, kWaves = T / kWave;
  __shared__ float2 s_red[2][B / kWave];
  __shared__ float s_part[kRows == 1 ? 1 : B * 4];
  const int t = threadIdx.x % T, slot = threadIdx.x / T, pieces = (A.d + N - 1) / N;
  float dg[NV][N];
  u32x4u gain[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    gain[k] = t + k * T < pieces ? load_piece(static_cast<const E*>(A.gain), t + k * T, A.d) : u32x4u{0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < N; ++i) dg[k][i] = 0.f;
  }
  const int64_t step = static_cast<int64_t>(gridDim.x) * kRows;
  int64_t row = static_cast<int64_t>(blockIdx.x) * kRows + slot;
  constexpr bool kAhead = T < 1024;                          // the next row on its way: of 1024 threads there are no registers for it
  BackRow<E, NV, THROUGH> at, next;
  if constexpr (kAhead) at.template load<T>(A, row, t, pieces);
  int turn = 0;
  for (int64_t first = static_cast<int64_t>(blockIdx.x) * kRows; first < A.n; first += step, row += step, turn ^= 1) {   // the workgroup's rows together
    if constexpr (kAhead) next.template load<T>(A, row + step, t, pieces);
    else at.template load<T>(A, row, t, pieces);
    float dot = 0.f, some = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      float a[N], b[N], g[N];
      Piece<E>::unpack(at.y[k], a);
      Piece<E>::unpack(at.h[k], b);
      Piece<E>::unpack(gain[k], g);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        dot = fmaf(a[i] * g[i], b[i], dot);
        if (!(a[i] == 0.f)) some = 1.f;
      }
    }
    dot = row_reduce<kWave>(dot, nullptr, add);
    some = __ballot(some != 0.f) ? 1.f : 0.f;
    if constexpr (T > kWave) {                               // one barrier a row: the next row's sums go to the other buffer
      if ((threadIdx.x & 63) == 0) s_red[turn][threadIdx.x >> 6] = make_float2(dot, some);
      __syncthreads();
      dot = some = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float2 v = s_red[turn][slot * kWaves + w];
        dot += v.x;
        some += v.y;
      }
    }
    if (row < A.n) {
      const float m = dot * at.inv * at.inv / static_cast<float>(A.d);
      E* const dx = static_cast<E*>(A.dx) + row * A.d;
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        if (t + k * T >= pieces) continue;
        float a[N], b[N], g[N], o[N];
        Piece<E>::unpack(at.y[k], a);
        Piece<E>::unpack(at.h[k], b);
        Piece<E>::unpack(gain[k], g);
        if constexpr (THROUGH) Piece<E>::unpack(at.th[k], o);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float v = some != 0.f ? at.inv * (a[i] * g[i] - b[i] * m) : 0.f;
          if (some != 0.f) dg[k][i] = fmaf(a[i], b[i] * at.inv, dg[k][i]);
          if constexpr (THROUGH) o[i] += v;
          else o[i] = v;
        }
        store_piece(dx, t + k * T, A.d, Piece<E>::pack(o));
      }
    }
    if constexpr (kAhead) at = next;
  }
  float* const part = A.part + static_cast<int64_t>(blockIdx.x) * A.d;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    if constexpr (kRows == 1) {
#pragma unroll
      for (int i = 0; i < N; ++i)
        if ((t + k * T) * N + i < A.d) part[(t + k * T) * N + i] = dg[k][i];
    } else {
#pragma unroll
      for (int i0 = 0; i0 < N; i0 += 4) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) s_part[threadIdx.x * 4 + i] = dg[k][i0 + i];
        __syncthreads();
        if (threadIdx.x < T) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float v = s_part[threadIdx.x * 4 + i];
#pragma unroll
            for (int w = 1; w < kRows; ++w) v += s_part[(w * T + threadIdx.x) * 4 + i];
            if ((t + k * T) * N + i0 + i < A.d) part[(t + k * T) * N + i0 + i] = v;
          }
        }
      }
    }
  }
}
// dg from the workgroups' shares: a workgroup to 64 columns, sixteen threads to a share, eight loads of a thread under way.
constexpr int kGainT = 1024;
__global__ void __launch_bounds__(kGainT)
k_norm_gain(const float* __restrict__ part, int parts, int d, int accumulate, float* __restrict__ dgain) {
  constexpr int kShares = kGainT / 16, kAtOnce = 8;
  typedef float floatx4u __attribute__((ext_vector_type(4), aligned(4)));
  __shared__ floatx4 s[kShares][16];
  const int q = threadIdx.x & 15, w = threadIdx.x >> 4, col = blockIdx.x * kWave + q * 4;
  floatx4 v = {0.f, 0.f, 0.f, 0.f};
  for (int p = w; p < parts; p += kShares * kAtOnce) {
    floatx4u x[kAtOnce];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const float* const from = part + static_cast<int64_t>(p + i * kShares) * d + col;
      x[i] = floatx4u{0.f, 0.f, 0.f, 0.f};
      if (p + i * kShares < parts) {
        if (col + 4 <= d) x[i] = *reinterpret_cast<const floatx4u*>(from);
        else
          for (int j = 0; j < d - col; ++j) x[i][j] = from[j];
      }
    }
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) v += floatx4{x[i][0], x[i][1], x[i][2], x[i][3]};
  }
  s[w][q] = v;
#pragma unroll
  for (int o = kShares / 2; o > 0; o >>= 1) {
    __syncthreads();
    if (w < o) s[w][q] = v = v + s[w + o][q];
  }
  if (w != 0) return;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (col + j < d) dgain[col + j] = accumulate ? dgain[col + j] + v[j] : v[j];
}

// ------------------------------------------------------------------ host side
// launch(T, NV): threads to a row and pieces to a thread.  One piece: a wavefront, whatever the number of rows (bf16, 512 columns with a residual: 2000 rows 3.2 us, by workgroups
// 4.3, 40 000 rows 26 and 40).  Up to four: a workgroup while rows are few (2048 columns: 64 rows 3.3 and 2.9 us, in 8 bits 4.7 and 3.6; 1000 rows 4.5 and 4.2; 2000 as
// fast; 4000 rows 11.0 and 12.9, 40 000 rows 113 and 116).  More: a workgroup (4096 columns: 500 rows 5.2 and 4.3 us, 8000 rows 39.2 and 40.3, in 8 bits 41.0 and 37.2).
constexpr int64_t kWideRows = 2048;
template <class Launch>
void with_width(int pieces, int64_t rows, Launch launch) {
  auto go = [&](auto t) {
    constexpr int T = decltype(t)::value;
    const int nv = static_cast<int>(cdiv(pieces, T));
    if (nv <= 1) launch(t, std::integral_constant<int, 1>());
    else if (nv <= 2) launch(t, std::integral_constant<int, 2>());
    else if (nv <= 4) launch(t, std::integral_constant<int, 4>());
    else if constexpr (T == kNT) {
      if (nv <= 8) launch(t, std::integral_constant<int, 8>());
      else launch(t, std::integral_constant<int, 16>());
    }
  };
  if (pieces > 4 * kWave || (pieces > kWave && rows <= kWideRows)) go(std::integral_constant<int, kNT>());
  else go(std::integral_constant<int, kWave>());
}
// ... of the backward pass: two pieces, from 2048 on (float32, 16 384 columns are 4096 pieces) four
template <class Launch>
void with_back(int pieces, Launch launch) {
  auto go = [&](auto t, auto nv) { launch(t, nv); };
  using One = std::integral_constant<int, 1>;
  using Two = std::integral_constant<int, 2>;
  if (pieces <= 64) go(std::integral_constant<int, 64>(), One());
  else if (pieces <= 128) go(std::integral_constant<int, 64>(), Two());
  else if (pieces <= 256) go(std::integral_constant<int, 128>(), Two());
  else if (pieces <= 512) go(std::integral_constant<int, 256>(), Two());
  else if (pieces <= 1024) go(std::integral_constant<int, 512>(), Two());
  else if (pieces <= 2048) go(std::integral_constant<int, 1024>(), Two());
  else go(std::integral_constant<int, 1024>(), std::integral_constant<int, 4>());
}
constexpr unsigned kNormGrid = 1u << 23;                     // threads of a launch are counted in 32 bits
constexpr int kNormParts = 1024;                             // shares of dg at most (back_parts)
umas_status check_norm(umas_dtype dt, int64_t n, int d) {
  UMAS_REQUIRE(dt == UMAS_F32 || dt == UMAS_BF16, UMAS_EDTYPE, "dtype=%d is neither F32 nor BF16", static_cast<int>(dt));
  UMAS_REQUIRE(n >= 0, UMAS_EINVAL, "negative row count");
  UMAS_REQUIRE(d >= 1 && d <= kMaxNormD, UMAS_ESHAPE, "d=%d outside [1,%d]", d, kMaxNormD);
  UMAS_REQUIRE(dt != UMAS_BF16 || d % 8 == 0, UMAS_ESHAPE, "bf16 needs d %% 8 == 0 (d=%d)", d);
  UMAS_REQUIRE(n < (1LL << 31), UMAS_ESHAPE, "at most 2^31-1 rows");
  return UMAS_OK;
}
bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }
umas_status norm(const NormArgs& A, umas_dtype dt, hipStream_t st) {
  UMAS_REQUIRE(!(A.eps < 0.f) && A.eps < INFINITY, UMAS_EINVAL, "eps must be a number >= 0");
  UMAS_REQUIRE(A.gain, UMAS_EINVAL, "gain must not be NULL");
  UMAS_REQUIRE((A.x && (A.y || (A.q && A.scale))) || A.n == 0, UMAS_EINVAL, "x and the output must not be NULL");
  UMAS_REQUIRE(!A.residual == !A.hidden || A.n == 0, UMAS_EINVAL, "residual and hidden go together");
  for (const void* p : {A.x, A.residual, A.gain, static_cast<const void*>(A.hidden), static_cast<const void*>(A.y), static_cast<const void*>(A.q)})
    UMAS_REQUIRE(aligned16(p), UMAS_EINVAL, "x, residual, gain, hidden and the output must be 16-byte aligned");
  prof_mark(st);
  if (A.n == 0) return UMAS_OK;
  auto run = [&](auto e) {
    using E = decltype(e);
    with_width(static_cast<int>(cdiv(A.d, Piece<E>::N)), A.n, [&](auto t, auto nv) {
      const dim3 grid(std::min(cdiv(A.n, kNT / decltype(t)::value), kNormGrid));
      if (A.q) hipLaunchKernelGGL((k_rms_norm<E, decltype(t)::value, decltype(nv)::value, true>), grid, dim3(kNT), 0, st, A);
      else hipLaunchKernelGGL((k_rms_norm<E, decltype(t)::value, decltype(nv)::value, false>), grid, dim3(kNT), 0, st, A);
    });
  };
  if (dt == UMAS_BF16) run(uint16_t{});
  else run(float{});
  UMAS_LAUNCHED("k_rms_norm");
  return UMAS_OK;
}
// Workgroups of the backward pass, each of which leaves a share of dg.  A row of 4 KB and more keeps enough loads under way for one to a compute unit, and every other one costs
// its share: 39 224 bf16 rows of 2048 with 256, 512 and 1024 of them 116, 124 and 143 us, 20 000 of 4096 117, 125 and 144, 10 000 of 8192 127, 134 and 146, 2000 of 2048 13.2, 14.8 and 18.7;
// shorter rows 30 000 of 512 33, 27.4 and 28, 100 000 of 256 83, 55 and 44.5; float32, whose rows of up to 16 KB want two, 10 000 of 2048 79, 65 and 69, 4000 of 8192
// 105, 108.
int back_parts(int64_t n, int rows_at_once, umas_dtype dt, int d) {
  const int64_t bytes = static_cast<int64_t>(d) * (dt == UMAS_BF16 ? 2 : 4);
  const int64_t most = bytes < 1024 ? 1024 : bytes < 4096 || (dt == UMAS_F32 && bytes <= 16384) ? 512 : 256;
  return static_cast<int>(std::min<int64_t>(cdiv(std::max<int64_t>(n, 1), rows_at_once), most));
}

}  // namespace
}  // namespace umas

using namespace umas;

extern "C" umas_status umas_rms_norm(const void* x, const void* residual, const void* gain, umas_dtype dtype, int64_t n_rows, int32_t d, float eps,
                                     void* hidden, void* y, float* inv_rms, void* hip_stream) {
  umas_status s = check_norm(dtype, n_rows, d);
  if (s != UMAS_OK) return s;
  return norm(NormArgs{x, residual, gain, n_rows, d, eps, hidden, y, nullptr, nullptr, inv_rms}, dtype, static_cast<hipStream_t>(hip_stream));
}

extern "C" umas_status umas_rms_norm_quantized(const void* x, const void* residual, const void* gain, umas_dtype dtype, int64_t n_rows, int32_t d, float eps,
                                               void* hidden, uint8_t* q, float* scale, float* inv_rms, void* hip_stream) {
  umas_status s = check_norm(dtype, n_rows, d);
  if (s != UMAS_OK) return s;
  UMAS_REQUIRE((q && scale) || n_rows == 0, UMAS_EINVAL, "q and scale must not be NULL");
  return norm(NormArgs{x, residual, gain, n_rows, d, eps, hidden, nullptr, q, scale, inv_rms}, dtype, static_cast<hipStream_t>(hip_stream));
}

extern "C" size_t umas_rms_norm_workspace_bytes(int64_t n_rows, int32_t d) {
  if (n_rows < 0 || d < 1 || d > kMaxNormD) return 0;
  return align_up(static_cast<size_t>(std::min<int64_t>(std::max<int64_t>(n_rows, 1), kNormParts)) * d * sizeof(float));
}

extern "C" umas_status umas_rms_norm_bwd(const void* dy, const void* hidden, const void* gain, const float* inv_rms, const void* dhidden, umas_dtype dtype,
                                         int64_t n_rows, int32_t d, int32_t accumulate_dgain, void* dx, float* dgain, void* workspace,
                                         size_t workspace_bytes, void* hip_stream) {
  umas_status s = check_norm(dtype, n_rows, d);
  if (s != UMAS_OK) return s;
  UMAS_REQUIRE(gain && dgain, UMAS_EINVAL, "gain and dgain must not be NULL");
  UMAS_REQUIRE((dy && hidden && inv_rms && dx) || n_rows == 0, UMAS_EINVAL, "dy, hidden, inv_rms and dx must not be NULL");
  for (const void* p : {dy, hidden, gain, dhidden, static_cast<const void*>(dx)})
    UMAS_REQUIRE(aligned16(p), UMAS_EINVAL, "dy, hidden, gain, dhidden and dx must be 16-byte aligned");
  s = check_ws(workspace, workspace_bytes, umas_rms_norm_workspace_bytes(n_rows, d));
  if (s != UMAS_OK) return s;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  prof_mark(st);
  int parts = 0;
  if (n_rows > 0) {
    NormBackArgs A{dy, hidden, gain, inv_rms, dhidden, n_rows, d, dx, static_cast<float*>(workspace)};
    auto run = [&](auto e) {
      using E = decltype(e);
      with_back(static_cast<int>(cdiv(d, Piece<E>::N)), [&](auto t, auto nv) {
        constexpr int T = decltype(t)::value, NV = decltype(nv)::value;
        parts = back_parts(n_rows, kBackT<T> / T, dtype, d);
        if (dhidden) hipLaunchKernelGGL((k_norm_back<E, T, NV, true>), dim3(parts), dim3(kBackT<T>), 0, st, A);
        else hipLaunchKernelGGL((k_norm_back<E, T, NV, false>), dim3(parts), dim3(kBackT<T>), 0, st, A);
      });
    };
    if (dtype == UMAS_BF16) run(uint16_t{});
    else run(float{});
    UMAS_LAUNCHED("k_norm_back");
  }
  hipLaunchKernelGGL(k_norm_gain, dim3(cdiv(d, kWave)), dim3(kGainT), 0, st, static_cast<const float*>(workspace), parts, d, accumulate_dgain, dgain);
  UMAS_LAUNCHED("k_norm_gain");
  return UMAS_OK;
}
