// Logits of a few rows (up to 32, 64 at d <= 2048) that are to be read again: the product is bound by reading W once.
#pragma once

#include <float.h>

#include <type_traits>

#include "umas_logits.h"

namespace umas {
namespace {

// W streams past rows that stay in registers (the loop and what bounds it: k_score_few).  A thread has one place of every block of 16 entries of its
// workgroup's part of the vocabulary, `per` blocks.  The logits are summed over the wavefronts in a fixed order; they collect in LDS, 64 KB of them, and leave
// together: memory operations are counted in order, and a store in every step has the loads of W behind it wait for it (one row of 2048 129 us in place
// of 110, 24 rows of 3584 247 in place of 199).
// Logit v of row n goes to Z[n * stride + v], up to the end of the workgroups' parts.  From V on lies what no logit is: -infinity, and a thread that has none emits the lowest
// number, or with ENTROPY, where products with it have to stay finite, kMasked for both.
// emit(n, place, m, most, s, t): the thread's maximum, and
// for its row's part of the vocabulary the maximum, sum exp(z - most) and, with ENTROPY, sum exp(z - most) z.
template <int NI, int PPW, bool ENTROPY, class Emit>
__device__ __forceinline__ void few_logits(const uint16_t* __restrict__ W, const uint16_t* __restrict__ H, int d, int V, const int32_t* __restrict__ rowsel, int n_sel, int per,
                                           float* __restrict__ Z, int64_t stride, Emit emit) {
  constexpr float kNone = ENTROPY ? kMasked : -INFINITY, kFirst = ENTROPY ? kMasked : -FLT_MAX;
  constexpr int MB = PPW <= 4 && NI <= 2 ? 2 : 1;            // blocks of 16 vocabulary entries per step
  constexpr int NL = (NI + 1) / 2;                           // logits per thread and block
  constexpr int kHold = 64 / NI, kHoldPitch = kHold * 16 + 16;   // blocks that collect, floats of a row of them (16 more: banks)
  __shared__ __attribute__((aligned(16))) float s_z[2][kFewWaves][MB][NI][16][16];   // [.][wavefront][block][.][row][entry]
  __shared__ __attribute__((aligned(16))) float s_out[NI * 16 * kHoldPitch];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int piece = (lane >> 4) * 8;
  bf16x8 hf[PPW][2][NI];
#pragma unroll
  for (int p = 0; p < PPW; ++p)
#pragma unroll
    for (int q = 0; q < 2; ++q)
#pragma unroll
      for (int j = 0; j < NI; ++j) {
        const int n = min(j * 16 + (lane & 15), n_sel - 1), k = (p * kFewWaves + wave) * 64 + q * 32 + piece;
        const int64_t row = rowsel ? rowsel[n] : n;
        const uint4 v = k < d ? *reinterpret_cast<const uint4*>(H + row * d + k) : make_uint4(0u, 0u, 0u, 0u);
        hf[p][q][j] = __builtin_bit_cast(bf16x8, v);
      }
  const int blocks = (V + 15) / 16;
  const int b0 = static_cast<int>(blockIdx.x) * per, b1 = min(b0 + per, blocks);
  uint4 w[MB][PPW][2];
  bool past[2];                                              // the last piece's columns that do not exist
#pragma unroll
  for (int q = 0; q < 2; ++q) past[q] = ((PPW - 1) * kFewWaves + wave) * 64 + q * 32 + piece >= d;
  auto load = [&](int b, int p, int q, int i) {              // past the hidden size: some entry of the row, cleared where it is used
    const int v = min((b + i) * 16 + (lane & 15), V - 1), k = min((p * kFewWaves + wave) * 64 + q * 32 + piece, d - 8);
    w[i][p][q] = *reinterpret_cast<const uint4*>(W + static_cast<int64_t>(v) * d + k);
  };
  if (b0 < b1)
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int p = 0; p < PPW; ++p) { load(b0, p, 0, i); load(b0, p, 1, i); }
  const bool mine = tid < NI * 256;
  const int my_n = (tid >> 4) & 15, my_v = tid & 15;
  float m[NL], s[NL], t[NL];
#pragma unroll
  for (int l = 0; l < NL; ++l) {
    m[l] = kFirst;
    s[l] = t[l] = 0.f;
  }
  int first = b0;                                            // of the blocks that collect
  auto leave = [&](int end) {                                // a wavefront to a row
    __syncthreads();
    for (int n = wave; n < n_sel; n += kFewWaves) {
      float* const z = Z + n * stride + static_cast<int64_t>(first) * 16;
      for (int c = lane * 4; c < (end - first) * 16; c += kWave * 4)
        *reinterpret_cast<floatx4*>(z + c) = *reinterpret_cast<const floatx4*>(s_out + n * kHoldPitch + c);
    }
    __syncthreads();
    first = end;
  };
  int buf = 0;
  for (int b = b0; b < b1; b += MB, buf ^= 1) {
    floatx4 acc[MB][NI];
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int j = 0; j < NI; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
    const int nb = b + MB < b1 ? b + MB : b;                 // past the range: loaded again, not used
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int p = 0; p < PPW; ++p)
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          const bf16x8 a = __builtin_bit_cast(bf16x8, p == PPW - 1 && past[q] ? make_uint4(0u, 0u, 0u, 0u) : w[i][p][q]);
#pragma unroll
          for (int j = 0; j < NI; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, hf[p][q][j], acc[i][j], 0, 0, 0);
          load(nb, p, q, i);
        }
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int j = 0; j < NI; ++j) *reinterpret_cast<floatx4*>(&s_z[buf][wave][i][j][lane & 15][(lane >> 4) * 4]) = acc[i][j];
    __syncthreads();
    if (mine) {
#pragma unroll
      for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int l = 0; l < NL; ++l) {
          float z = 0.f;
#pragma unroll
          for (int k = 0; k < kFewWaves; ++k) z += s_z[buf][k][i][2 * l + (tid >> 8)][my_n][my_v];
          if ((b + i) * 16 + my_v >= V || b + i >= b1) z = kNone;
          s_out[((2 * l + (tid >> 8)) * 16 + my_n) * kHoldPitch + (b + i - first) * 16 + my_v] = z;
          const float gap = z - m[l], e = __expf(-fabsf(gap));  // one exponential: of the smaller relative to the larger
          s[l] = gap > 0.f ? fmaf(s[l], e, 1.f) : s[l] + e;
          if constexpr (ENTROPY) t[l] = gap > 0.f ? fmaf(t[l], e, z) : fmaf(e, z, t[l]);
          m[l] = fmaxf(m[l], z);
        }
    }
    if (b + MB - first == kHold) leave(b + MB);
  }
  if (first < b1) leave(min(b0 + per, (b1 - first + MB - 1) / MB * MB + first));
#pragma unroll
  for (int l = 0; l < NL; ++l) {
    float most = m[l];                                       // of the row's sixteen threads, which are neighbours
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) most = fmaxf(most, __shfl_xor(most, o, kWave));
    const float e = __expf(m[l] - most);
    float sum = s[l] * e, sum_z = ENTROPY ? t[l] * e : 0.f;
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) {
      sum += __shfl_xor(sum, o, kWave);
      if constexpr (ENTROPY) sum_z += __shfl_xor(sum_z, o, kWave);
    }
    const int n = (2 * l + (tid >> 8)) * 16 + my_n;
    if (mine && n < n_sel) emit(n, my_v, m[l], most, sum, sum_z);
  }
}

// ------------------------------------------------------------------ host side
constexpr int kFewMostTiles = 512;
inline int few_workgroups(int V) { return std::min(std::min(device_cus(), kFewMostTiles), static_cast<int>(cdiv(V, 16))); }
// blocks of 16 entries to a workgroup; steps of two blocks end in them
inline int few_per(int V, int workgroups) { return static_cast<int>(round_up(cdiv(cdiv(V, 16), workgroups), 2)); }
// floats of Z with any number of workgroups
inline size_t few_floats(int64_t rows, int V) { return static_cast<size_t>(rows) * (round_up(V, 256) + 3 * kFewMostTiles * 16); }
// launch(NI, PPW) with the instance for these rows
template <class Launch>
void with_few(int d, int64_t rows, Launch launch) {
  auto by_rows = [&](auto ppw) {
    if constexpr (decltype(ppw)::value <= 4)
      if (rows > 32) return launch(std::integral_constant<int, 4>(), ppw);
    if (rows <= 16) launch(std::integral_constant<int, 1>(), ppw);
    else launch(std::integral_constant<int, 2>(), ppw);
  };
  switch (few_pieces(d)) {
    case 1: return by_rows(std::integral_constant<int, 1>());
    case 2: return by_rows(std::integral_constant<int, 2>());
    case 3: return by_rows(std::integral_constant<int, 3>());
    case 4: return by_rows(std::integral_constant<int, 4>());
    case 5: return by_rows(std::integral_constant<int, 5>());
    case 6: return by_rows(std::integral_constant<int, 6>());
    case 7: return by_rows(std::integral_constant<int, 7>());
    default: return by_rows(std::integral_constant<int, 8>());
  }
}

}  // namespace
}  // namespace umas
