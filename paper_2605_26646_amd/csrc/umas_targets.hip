// Teaching a head from targets: softmax cross entropy of given tokens and distillation from a teacher's largest logits, each with its gradient to hidden
// states and head.
//
// Both are one computation with k targets a row (cross entropy: one, of mass 1).  For a selected row i with z = W h_i, lse = log sum_v exp z_v, targets
// (v_j, t_j) of mass T = sum t_j and weight w_i, over norm rows:
//   cross entropy  l_i = lse - z_y + c lse^2          distillation  l_i = sum_j t_j (log t_j - z_{v_j} + lse)
//   loss = sum_i w_i l_i / norm,  g = w_i / norm,  dz_v = g (a' p_v - t_v),  p = softmax(z),  a' = T + 2 c lse,  dH = dz W,  dW = dz^T H
// The dense part of dz is a row factor times the softmax, so one product of logits serves both directions, as in the policy update: the scoring pass
// leaves E = bf16(exp(z - r_i)) behind, r_i the largest logit among the row's targets, which a gather of k dot products finds beforehand and which is
// never far above the row's logsumexp.  What is left is f = g a' exp(r - lse) as a row factor (folded into dH's rows and into the copy of H that dW reads)
// and k entries a row, which are written over their numerators before the gradient products:
//   E[i, v_j] = bf16((a' p - t) / (a' exp(r - lse))) = bf16(exp(lse - r) (p - t / a'))
// so the sparse part costs k two-byte stores a row and no pass of its own over dH or dW.
//
// What bounds it: the products.  16 384 rows of 2048 against 151 936: the scores 7.82 ms (1.30 PFLOP/s), both gradients 14.9 ms (1.37 PFLOP/s), all else 0.11 ms;
// 4096 rows 2.02 and 3.81 ms and 0.20 (64 targets a row).  Fewer rows are bound by W and dW, which have to be read twice and written: 203 rows of 3584 against
// 152 064, 3.3 GB and 1.0 TFLOP of whole blocks: 0.94 ms.
//
// Roundings to bf16: an entry of E (relative error up to 2^-8; the sum of exponentials and the logsumexp are float32 and do not see it), the scaled
// copy of H, and the results.  A row of dW that a single row of H makes carries all three: dW is off by 0.0024 to 0.0029 of its norm, where
// rounding the result alone is 0.0017 (one target a row: 300 rows 0.0028, 1500 0.0024, 8192 0.0019; 64 targets: 2000 rows 0.0029, 4096 0.0027 to 0.0029, with 20 targets 0.0024).  Up to
// 256 rows (two roundings, see below) 0.0022 to 0.0024.  dH, whose factor undoes what its targets' entries lost, 0.0017 (one target) to 0.0021.
#include <float.h>

#include "umas_f32.h"
#include "umas_few.h"
#include "umas_gradients.h"

namespace umas {
namespace {

// What a row is taught.
struct Targets {
  const int32_t* ids;      // [n_rows][k]; a place whose token does not exist does not count
  const float* logits;     // [n_rows][k] the teacher's, NULL: cross entropy, mass 1 for the one token
  const float* lse;        // [n_rows] the teacher's, NULL: the k places are all there is
  int k;
};
struct Teach {
  Targets t;
  const int32_t* rowsel;
  int64_t n_sel;
  int V, d;
  const float* weight;     // [n_rows] or NULL: 1
  float norm, z_coef;
};
__device__ __forceinline__ float exp_of(float x) { return expf(x); }
__device__ __forceinline__ double exp_of(double x) { return exp(x); }
// A lane's target of a row, its mass (0: does not count) and the mass of the row; every lane of a wavefront calls it.  Real: float or, where sums
// are in float64, double.
template <class Real>
struct Place {
  int id;
  Real t, mass;
};
template <class Real>
__device__ __forceinline__ Place<Real> place_of(const Targets& T, int V, int64_t row) {
  const int lane = threadIdx.x & 63;
  const bool in = lane < T.k;
  const int id = in ? T.ids[row * T.k + lane] : -1;
  bool have = id >= 0 && id < V;
  Real t;
  if (!T.logits) {
    t = have ? Real(1) : Real(0);
  } else {
    const float l = have ? T.logits[row * T.k + lane] : -INFINITY;
    have = have && l > -INFINITY;                            // no number: does not count
    const float m = wave_max(have ? l : -INFINITY);
    t = have ? exp_of(Real(l) - Real(m)) : Real(0);
    if (T.lse) t = have ? t * exp_of(Real(m) - Real(T.lse[row])) : Real(0);
    else { const Real s = wave_sum(t); t = have ? t / s : Real(0); }
  }
  return Place<Real>{id, t, wave_sum(t)};
}
// Mass of the lane's token over all places that name it.
template <class Real>
__device__ __forceinline__ Real mass_of_token(int k, int id, Real t) {
  Real s = 0;
  for (int j = 0; j < k; ++j) {
    const Real tj = __shfl(t, j, kWave);
    if (__shfl(id, j, kWave) == id) s += tj;
  }
  return s;
}
// g of the row: 0 where nothing is taught
__device__ __forceinline__ float row_weight(const Teach& A, int64_t row, bool taught) { return taught ? (A.weight ? A.weight[row] : 1.f) : 0.f; }
// a', the factor of the dense part; the sparse part is divided by it, T / a'.  With the penalty it can come to 0 beside a mass that does not (a negative logsumexp):
// then it is kept off 0 by what is below the rounding of either part.  Without, it is the mass, however little that is: a teacher may give e^-40 to its places.
template <class Real>
__device__ __forceinline__ Real dense_factor(Real mass, float z_coef, Real lse) { return z_coef != 0.f ? mass + 2 * Real(z_coef) * lse : mass; }
__device__ __forceinline__ float dense_divisor(float mass, float z_coef, float lse) {
  const float a = dense_factor(mass, z_coef, lse);
  return fabsf(a) < 1e-10f * mass ? 1e-10f * mass : a;
}

// ------------------------------------------------------------------ what a call leaves per row, compact, in selection order
struct RowArrays {
  float* lse;
  float* ent;
  float* l;                // the row's loss without its weight
  float* w;                // its weight, 0 where nothing is taught
  float* a;                // g a' for the blocks that are computed once more
  float* zero;             // zeros
  float* cref;             // r
  float* sc;               // f
  uint16_t* entries;       // [n_sel][k] (up to kFewTaught rows)
  float* zt;               // [n_sel][k] logits of the targets
  float* tt;               // [n_sel][k] their masses, all places of a token added up
  float* mass;
};
struct OpenArgs {
  Teach A;
  const uint16_t *H, *W;
  RowArrays R;
  int32_t* flags;
  int n_flags;
  LiveArgs live;           // of the first chunk
  uint32_t* dH;            // cleared, with the row outputs, where rows are left out; else NULL
  int64_t dh_words;
  float* row_out;
  int64_t n_rows;
  int share;               // wavefronts to a row: 1 or 4
};
// One wavefront (four) per selected row: the targets' masses, their logits (dot products of float32 sums), the row's reference.  The first workgroup clears
// the flags and lays out the chunk, others clear what the call defines everywhere.  Bound by the rows of W: 4096 rows with 64 targets of 4 KB each 150 us (7.2 TB/s, a part of it
// from the caches; a wavefront to a row, whose sixteen turns are one behind the other, 184).  16 384 rows with one target 32 us (a wavefront to a row).
constexpr int kAtOnce = 4;   // targets whose rows of W are under way together
__global__ void __launch_bounds__(256)
k_target_open(OpenArgs O) {
  if (blockIdx.x == 0) {
    for (int i = threadIdx.x; i < O.n_flags; i += 256) O.flags[i] = 0;
    live_scan(O.live, static_cast<int>(threadIdx.x) < O.live.nblk);
    return;
  }
  const Teach& A = O.A;
  const int64_t blk = static_cast<int64_t>(blockIdx.x) - 1, nb = static_cast<int64_t>(gridDim.x) - 1;
  if (O.dH) {
    const int64_t stride = nb * 256;
    for (int64_t i = blk * 256 + threadIdx.x; i < O.dh_words; i += stride) O.dH[i] = 0u;
    for (int64_t i = blk * 256 + threadIdx.x; i < O.n_rows; i += stride) O.row_out[i] = 0.f;
  }
  // `share` wavefronts to a row: their numbers in the row, its targets dealt out among them
  __shared__ float s_z[4][kWave];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, k = A.t.k, share = O.share, mine = wave % share;
  for (int64_t n0 = blk * (4 / share); n0 < A.n_sel; n0 += nb * (4 / share)) {
    const int64_t n = min(n0 + wave / share, A.n_sel - 1);
    const int64_t row = A.rowsel ? A.rowsel[n] : n;
    const Place<float> P = place_of<float>(A.t, A.V, row);
    const uint4* h = reinterpret_cast<const uint4*>(O.H + row * A.d);
    float z = 0.f;
    const unsigned long long share_of = share == 4 ? 0x1111111111111111ull << mine : ~0ull;
    unsigned long long left = __ballot(P.t != 0.f) & share_of;   // NaN counts
    while (left) {
      int j[kAtOnce];
      const uint4* w[kAtOnce];
      float s[kAtOnce];
#pragma unroll
      for (int b = 0; b < kAtOnce; ++b) {
        j[b] = left ? __ffsll(static_cast<long long>(left)) - 1 : j[b - (b > 0)];
        left &= left - 1;
        w[b] = reinterpret_cast<const uint4*>(O.W + static_cast<int64_t>(__shfl(P.id, j[b], kWave)) * A.d);
        s[b] = 0.f;
      }
      for (int c = lane; c < A.d / 8; c += kWave) {
        float x[8];
        bf16x8_to_f32(h[c], x);
#pragma unroll
        for (int b = 0; b < kAtOnce; ++b) {
          float y[8];
          bf16x8_to_f32(w[b][c], y);
#pragma unroll
          for (int q = 0; q < 8; ++q) s[b] = fmaf(x[q], y[q], s[b]);
        }
      }
#pragma unroll
      for (int b = 0; b < kAtOnce; ++b) {
        const float sum = wave_sum(s[b]);
        if (lane == j[b]) z = sum;
      }
    }
    if (share == 4) {
      __syncthreads();                                       // (the row before)
      s_z[wave][lane] = z;
      __syncthreads();
      z = s_z[lane & 3][lane];
      if (wave != 0) continue;
    } else if (n0 + wave >= A.n_sel) {
      continue;
    }
    const bool taught = P.mass > 0.f || P.mass != P.mass;
    const float top = wave_max(P.t != 0.f ? z : -INFINITY), ts = mass_of_token(k, P.id, P.t);
    if (lane < k) {
      O.R.zt[n * k + lane] = z;
      O.R.tt[n * k + lane] = P.t != 0.f ? ts : 0.f;
    }
    if (lane == 0) {
      O.R.cref[n] = taught ? top : 1e30f;                    // every numerator of a row that teaches nothing is 0
      O.R.w[n] = row_weight(A, row, taught);
      O.R.mass[n] = P.mass;
      O.R.zero[n] = 0.f;
    }
  }
}

// ------------------------------------------------------------------ statistics
struct StatArgs {
  int64_t n_sel;
  const int32_t *rowsel, *role;
  const float *l, *w, *ent, *lse, *mass;
  float norm;
  umas_target_stats* stats;
};
// The model's record (k = 0) or a role's, a workgroup of T threads to each, next to others that do something else; sums in float64, in an order that does
// not depend on scheduling.
template <int T>
__device__ __forceinline__ void target_stats(const StatArgs& S, int k, double* smem) {
  constexpr int kRows = 4;                                   // loads of as many rows are under way
  constexpr int kSums = 7;
  double v[kSums] = {}, sum[kSums];
  for (int64_t n0 = threadIdx.x; n0 < S.n_sel; n0 += kRows * T) {
    float l[kRows], w[kRows], ent[kRows], lse[kRows], mass[kRows];
    bool in[kRows];
#pragma unroll
    for (int q = 0; q < kRows; ++q) {
      const int64_t n = n0 + q * T, at = n < S.n_sel ? n : n0;
      l[q] = S.l[at]; w[q] = S.w[at]; ent[q] = S.ent[at]; lse[q] = S.lse[at]; mass[q] = S.mass[at];
      in[q] = n < S.n_sel && (k == 0 || S.role[S.rowsel ? S.rowsel[at] : at] == k - 1);
    }
#pragma unroll
    for (int q = 0; q < kRows; ++q) {
      if (!in[q]) continue;
      // a row of weight 0 counts in the means of entropy and logsumexp while they are numbers: its hidden state may be anything
      const bool taught = mass[q] != 0.f, counts = taught && (w[q] != 0.f || (fabsf(ent[q]) < INFINITY && fabsf(lse[q]) < INFINITY));
      v[0] += w[q] != 0.f ? static_cast<double>(w[q]) * static_cast<double>(l[q]) : 0.0;
      v[1] += static_cast<double>(w[q]);
      v[2] += counts ? static_cast<double>(ent[q]) : 0.0;
      v[3] += counts ? static_cast<double>(lse[q]) : 0.0;
      v[4] += 1.0;
      v[5] += taught ? 0.0 : 1.0;
      v[6] += counts ? 1.0 : 0.0;
    }
  }
#pragma unroll
  for (int j = 0; j < kSums; ++j) sum[j] = block_sum<double>(v[j], smem);
  if (threadIdx.x != 0) return;
  umas_target_stats s;
  s.loss = sum[4] > 0 ? static_cast<float>(sum[0] / (k == 0 ? static_cast<double>(S.norm) : sum[4])) : 0.f;
  s.weight_mean = sum[4] > 0 ? static_cast<float>(sum[1] / sum[4]) : 0.f;
  s.entropy_mean = sum[6] > 0 ? static_cast<float>(sum[2] / sum[6]) : 0.f;
  s.lse_mean = sum[6] > 0 ? static_cast<float>(sum[3] / sum[6]) : 0.f;
  s.n_scored = static_cast<int64_t>(sum[4]);
  s.n_ignored = static_cast<int64_t>(sum[5]);
  S.stats[k] = s;
}
__global__ void __launch_bounds__(256)
k_target_stats(StatArgs S) {
  __shared__ double smem[32];
  target_stats<256>(S, static_cast<int>(blockIdx.x), smem);
}

// ------------------------------------------------------------------ bf16: scores that keep the numerators
__global__ void __launch_bounds__(Cfg::T)
k_target_tiles(const uint16_t* __restrict__ W, const uint16_t* __restrict__ H, int d, int V, const int32_t* __restrict__ rowsel, int64_t c0, int64_t mc,
               int tiles_m, int tiles_n, int panel, int halved, float4* __restrict__ partial, int64_t n_pad, const float* __restrict__ cref,
               uint16_t* __restrict__ E, int64_t Vp, int32_t* __restrict__ flags, const int32_t* __restrict__ cidx) {
  __shared__ __attribute__((aligned(16))) uint16_t lds[kLogitLds / 2];
  score_tiles<Leave::kNumerators, Cfg>(W, H, d, V, rowsel, c0, mc, nullptr, tiles_m, tiles_n, panel, partial, n_pad, KeepArgs{cref, E, Vp, flags, cidx, nullptr}, lds, halved);
}
// ... where the rows end in the first half of a tile of 256
__global__ void __launch_bounds__(Cfg::T)
k_target_tiles_end(const uint16_t* __restrict__ W, const uint16_t* __restrict__ H, int d, int V, const int32_t* __restrict__ rowsel, int64_t c0, int64_t mc,
                   int tiles_m, int tiles_n, int panel, int halved, float4* __restrict__ partial, int64_t n_pad, const float* __restrict__ cref,
                   uint16_t* __restrict__ E, int64_t Vp, int32_t* __restrict__ flags, const int32_t* __restrict__ cidx) {
  __shared__ __attribute__((aligned(16))) uint16_t lds[kLogitLds / 2];
  score_tiles<Leave::kNumerators, Cfg, true>(W, H, d, V, rowsel, c0, mc, nullptr, tiles_m, tiles_n, panel, partial, n_pad, KeepArgs{cref, E, Vp, flags, cidx, nullptr}, lds, halved);
}
// ------------------------------------------------------------------ bf16: rows
// Eight rows to a workgroup, a wavefront to each, which asks for what it needs of its row; then all of them merge the rows' parts (a load covers the eight rows of
// eight parts), and a wavefront goes on with its row: its loss and factor, its k entries of the operand, its scaled copy of H.  Bound by the parts (16 bytes a row and tile) and
// the copy: 16 384 rows of 2048 against 151 936 57 us (5.1 TB/s), 4096 rows 24 (a workgroup of four wavefronts to four rows 66 and 30), 1111 rows of 1096 10 us, which is latency.
constexpr int kRowsT = 512;
struct MergedRows {
  float lse[8], ent[8], sum[8];
};
__device__ __forceinline__ void merge_rows(const float4* __restrict__ partial, int parts, int64_t n_pad, int64_t n0, bool live, MergedRows& out) {
  __shared__ float4 s_part[kRowsT / kWave][8];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  constexpr int kParts = kRowsT / 8;
  Part p{kNegInf, 0.f, 0.f};
  if (live)
    for (int t0 = threadIdx.x >> 3; t0 < parts; t0 += 4 * kParts) {
      float4 q[4];
#pragma unroll
      for (int k = 0; k < 4; ++k)
        q[k] = t0 + k * kParts < parts ? partial[static_cast<int64_t>(t0 + k * kParts) * n_pad + n0 + (lane & 7)] : make_float4(kNegInf, 0.f, 0.f, 0.f);
#pragma unroll
      for (int k = 0; k < 4; ++k) p = part_merge(p, Part{q[k].x, q[k].y, q[k].z});
    }
#pragma unroll
  for (int o = 8; o < kWave; o <<= 1) p = part_merge(p, Part{__shfl_xor(p.m, o, kWave), __shfl_xor(p.s, o, kWave), __shfl_xor(p.t, o, kWave)});
  if (lane < 8) s_part[wave][lane] = make_float4(p.m, p.s, p.t, 0.f);
  __syncthreads();
  if (threadIdx.x < 8) {
    p = Part{kNegInf, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kRowsT / kWave; ++w) {
      const float4 q = s_part[w][threadIdx.x];
      p = part_merge(p, Part{q.x, q.y, q.z});
    }
    const float lse = p.m + logf(p.s);
    out.lse[threadIdx.x] = lse;
    out.ent[threadIdx.x] = lse - p.t / p.s;
    out.sum[threadIdx.x] = p.s;
  }
  __syncthreads();
}
// one wavefront: bf16(f h) into the column blocks that dW reads; zeros, whatever h is, for f = 0
__device__ __forceinline__ void copy_row(const uint16_t* __restrict__ H, int64_t row, int d, float f, uint16_t* __restrict__ Hs, int64_t mcp, int64_t mp) {
  const uint4* h = reinterpret_cast<const uint4*>(H + row * d);
  for (int c = threadIdx.x & 63; c < d / 8; c += kWave) {
    float x[8];
    bf16x8_to_f32(h[c], x);
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (f != 0.f) v = make_uint4(pack_bf16x2(x[0] * f, x[1] * f), pack_bf16x2(x[2] * f, x[3] * f), pack_bf16x2(x[4] * f, x[5] * f), pack_bf16x2(x[6] * f, x[7] * f));
    reinterpret_cast<uint4*>(Hs + (static_cast<int64_t>(c >> 5) * mcp + mp) * 256)[c & 31] = v;
  }
}
struct RowsArgs {
  Teach A;
  const uint16_t* H;
  RowArrays R;
  const float4* partial;
  int tiles_m;
  int64_t n_pad, c0, rows;
  const int32_t *flags, *cidx;
  uint16_t* E;
  int64_t tiles_v;
  uint16_t* Hs;            // NULL: dW is not wanted
  int64_t mcp;
  float* row_out;
};
// (a' p - t) / (a' exp(r - lse)); p near 1 is taken as 1 + expm1, so that a confident row's difference keeps its digits
__device__ __forceinline__ float target_entry(float z, float lse, float r, float t, float a) {
  const float lp = z - lse, q = t / a;
  return __expf(lse - r) * (lp > -0.7f ? expm1f(lp) + (1.f - q) : __expf(lp) - q);
}
// A row's entries are rounded to bf16.  dH's row factor is taken as what makes them, times it, what they were (least squares; one target: exactly), as
// they and not the dense part make most of the row's dH: 60 rows of 2048 with ten targets dH off by 0.0028 of its norm without it, its own rounding
// being 0.0017; with it 270 rows with eight targets 0.0019.  (Not so dW's, where a dense entry of few rows stands by itself and would carry the shift.)
__device__ __forceinline__ float rounding_shift(float e, uint16_t rounded) {
  const float most = wave_max(fabsf(e));
  if (!(most > 0.f)) return 1.f;
  const float x = e / most, y = bf2f(rounded) / most, xy = wave_sum(x * y), yy = wave_sum(y * y);
  return yy > 0.f ? xy / yy : 1.f;
}
__device__ __forceinline__ bool is_finite(float x) { return fabsf(x) < INFINITY; }
// sign and exponent of a number (of the smallest normal one for numbers below it); no number for infinities and no numbers
__device__ __forceinline__ float power_below(float x) {
  return fabsf(x) < FLT_MIN ? copysignf(FLT_MIN, x) : __uint_as_float(__float_as_uint(x) & 0xff800000u);
}
__global__ void __launch_bounds__(kRowsT)
k_target_rows(RowsArgs O) {
  __shared__ MergedRows s_rows;
  const Teach& A = O.A;
  const int lane = threadIdx.x & 63, q = threadIdx.x >> 6, k = A.t.k;
  const int64_t m0 = static_cast<int64_t>(blockIdx.x) * 8, m = m0 + q, n = O.c0 + min(m, O.rows - 1);
  const int64_t row = A.rowsel ? A.rowsel[n] : n;
  const int blk = O.cidx[n >> 8], flag = O.flags[n >> 8];
  const float w = O.R.w[n], mass = O.R.mass[n], r = O.R.cref[n];
  const bool in = lane < k, taught = mass > 0.f || mass != mass;   // (not by r, which is what a target's logit happens to be, infinity among others)
  const int id = in ? A.t.ids[row * k + lane] : -1;
  const float z = in ? O.R.zt[n * k + lane] : 0.f, ts = in ? O.R.tt[n * k + lane] : 0.f, t = A.t.logits ? place_of<float>(A.t, A.V, row).t : 0.f;
  merge_rows(O.partial, O.tiles_m, O.n_pad, O.c0 + m0, m0 + (lane & 7) < O.rows, s_rows);
  if (m >= O.rows) return;
  const float lse = s_rows.lse[q], g = w / A.norm, a = dense_divisor(mass, A.z_coef, lse);
  float l = 0.f, out = 0.f, f = 0.f;
  if (taught) {
    if (!A.t.logits) {
      out = __shfl(z, 0, kWave) - lse;
      l = A.z_coef != 0.f ? fmaf(A.z_coef * lse, lse, -out) : -out;
    } else {
      out = l = wave_sum(t != 0.f ? t * (logf(t) - (z - lse)) : 0.f);
    }
    f = g != 0.f ? (flag ? 1.f : g * a * __expf(r - lse)) : 0.f;
  }
  const bool put = f != 0.f && !flag && ts != 0.f;
  const float e = put ? target_entry(z, lse, r, ts, a) : 0.f;
  const uint16_t rounded = f2bf(e);
  const float shift = rounding_shift(e, rounded);
  if (lane == 0) {
    O.R.lse[n] = taught ? lse : 0.f;
    O.R.ent[n] = taught ? s_rows.ent[q] : 0.f;
    O.R.l[n] = l;
    O.R.a[n] = g != 0.f ? g * a : 0.f;
    O.R.sc[n] = f * shift;
    if (O.row_out) O.row_out[row] = out;
  }
  uint16_t* const Erow = O.E + blk_offset(blk, 0, O.tiles_v) + (m & 255) * 256;
  if (f != 0.f) {
    if (put) Erow[static_cast<int64_t>(id >> 8) * kBlkElems + (id & 255)] = rounded;
  } else if (!is_finite(s_rows.sum[q]) || (taught && !is_finite(lse))) {
    // a row that teaches nothing may hold anything: its numerators must not be multiplied; the last row's stand in those behind it as well
    const int64_t rows = m == O.rows - 1 ? (m & ~int64_t{63}) + 64 - m : 1;
    for (int64_t i = 0; i < rows; ++i)
      for (int64_t vb = 0; vb < O.tiles_v; ++vb) *reinterpret_cast<uint2*>(Erow + i * 256 + vb * kBlkElems + lane * 4) = make_uint2(0u, 0u);
  }
  if (O.Hs) copy_row(O.H, row, A.d, f, O.Hs, O.mcp, static_cast<int64_t>(blk) * 256 + (m & 255));
}

// ------------------------------------------------------------------ bf16: one block of rows
// Up to 256 rows the scores leave their logits in float32 instead: 6 bytes a logit more to write and read, of which there are few here, in place of the
// gather, the references and what they may not serve for.  The operand is then made from the logits, D = bf16(dz / u), u the power of two below the row's factor g a': the copy of
// H that dW reads is u h, which is exact, so that dW has the roundings of D and of the result.  (Few rows are where it shows: a row of dW is one
// row's entry times its hidden state.  203 rows of 3584 dW off by 0.0022 of its norm, by the way of more rows 0.0027, for 940 us in place of
// 909; from a whole block on the logits would cost more than that.)
constexpr uint16_t kNoEntry = 0xFFFF;                        // a place that does not count
__global__ void __launch_bounds__(Cfg::T)
k_target_logits(const uint16_t* __restrict__ W, const uint16_t* __restrict__ H, int d, int V, const int32_t* __restrict__ rowsel, int64_t n_sel,
                const int32_t* __restrict__ ids, int tiles_m, int halved, float4* __restrict__ partial, int64_t n_pad, float* __restrict__ Z, int64_t Vp) {
  __shared__ __attribute__((aligned(16))) uint16_t lds[kLogitLds / 2];
  score_tiles<Leave::kLogits, Cfg>(W, H, d, V, rowsel, 0, n_sel, ids, tiles_m, 1, kGN, partial, n_pad, KeepArgs{nullptr, nullptr, Vp, nullptr, nullptr, Z}, lds, halved);
}
__global__ void __launch_bounds__(NarrowCfg::T)
k_target_logits_narrow(const uint16_t* __restrict__ W, const uint16_t* __restrict__ H, int d, int V, const int32_t* __restrict__ rowsel, int64_t n_sel,
                       const int32_t* __restrict__ ids, int tiles_m, int halved, float4* __restrict__ partial, int64_t n_pad, float* __restrict__ Z, int64_t Vp) {
  __shared__ __attribute__((aligned(16))) uint16_t lds[kNarrowLds / 2];
  score_tiles<Leave::kLogits, NarrowCfg, true>(W, H, d, V, rowsel, 0, n_sel, ids, tiles_m, 1, kGN, partial, n_pad, KeepArgs{nullptr, nullptr, Vp, nullptr, nullptr, Z}, lds, halved);
}
template <int NI, int PPW>
__global__ void __launch_bounds__(kFewT)
k_target_logits_few(const uint16_t* __restrict__ W, const uint16_t* __restrict__ H, int d, int V, const int32_t* __restrict__ rowsel, int n_sel, int per,
                    float4* __restrict__ partial, int64_t n_pad, float* __restrict__ Z, int64_t stride) {
  few_logits<NI, PPW, true>(W, H, d, V, rowsel, n_sel, per, Z, stride, [&](int n, int place, float, float most, float s, float t) {
    if (place == 0) partial[static_cast<int64_t>(blockIdx.x) * n_pad + n] = make_float4(most, s, t, 0.f);
  });
}
// Where the block's logits lie: rows of `stride`, or (0) blocks of 256 x 256.
struct KeptLogits {
  const float* z;
  int64_t stride;
  __device__ __forceinline__ const float* at(int64_t n, int blk, int c) const { return z + (stride ? n * stride + blk * 256 : blk * kBlkElems + n * 256) + c; }
};
// The first workgroup lays the block out, `clearing` of them clear what the call defines everywhere, the others do eight rows each.  12 us for 60 to 256 rows: a
// few dependent reads (rows one after the other in a workgroup of four wavefronts: 22).
struct FewArgs {
  Teach A;
  const uint16_t* H;
  RowArrays R;
  float* y;                // [rows] g a' over its power of two; 0 for a row without a gradient
  uint16_t* entries;       // [rows][k] the targets' entries of the operand
  const float4* partial;
  int tiles_m;
  int64_t n_pad;
  KeptLogits Z;
  uint16_t* Hs;
  int64_t mcp;
  float* row_out;
  LiveArgs live;
  unsigned clearing;
  uint32_t* dH;
  int64_t dh_words, n_rows;
};
__global__ void __launch_bounds__(kRowsT)
k_target_few(FewArgs F) {
  __shared__ MergedRows s_rows;
  const Teach& A = F.A;
  const int lane = threadIdx.x & 63, q = threadIdx.x >> 6, k = A.t.k;
  if (blockIdx.x == 0) {
    live_scan(F.live, static_cast<int>(threadIdx.x) < F.live.nblk);
    return;
  }
  if (blockIdx.x <= F.clearing) {
    const int64_t stride = static_cast<int64_t>(F.clearing) * kRowsT, i0 = static_cast<int64_t>(blockIdx.x - 1) * kRowsT + threadIdx.x;
    for (int64_t i = i0; i < F.dh_words; i += stride) F.dH[i] = 0u;
    if (F.row_out)
      for (int64_t i = i0; i < F.n_rows; i += stride) F.row_out[i] = 0.f;
    return;
  }
  const int64_t m0 = (static_cast<int64_t>(blockIdx.x) - 1 - F.clearing) * 8, n = min(m0 + q, A.n_sel - 1);
  const int64_t row = A.rowsel ? A.rowsel[n] : n;
  const Place<float> P = place_of<float>(A.t, A.V, row);
  const bool taught = P.mass != 0.f;                         // (a mass that is no number is the caller's)
  const float w = row_weight(A, row, taught), g = w / A.norm, ts = mass_of_token(k, P.id, P.t);
  const float z = P.t != 0.f ? *F.Z.at(n, P.id >> 8, P.id & 255) : 0.f;
  merge_rows(F.partial, F.tiles_m, F.n_pad, m0, m0 + (lane & 7) < A.n_sel, s_rows);
  if (m0 + q >= A.n_sel) return;
  const float lse = s_rows.lse[q], a = dense_divisor(P.mass, A.z_coef, lse);
  float l = 0.f, out = 0.f;
  if (taught) {
    if (!A.t.logits) {
      out = __shfl(z, 0, kWave) - lse;
      l = A.z_coef != 0.f ? fmaf(A.z_coef * lse, lse, -out) : -out;
    } else {
      out = l = wave_sum(P.t != 0.f ? P.t * (logf(P.t) - (z - lse)) : 0.f);
    }
  }
  const float f = g != 0.f ? g * a : 0.f, unit = f != 0.f ? power_below(f) : 0.f, y = f != 0.f ? f / unit : 0.f;
  const float e = f != 0.f && P.t != 0.f ? y * target_entry(z, lse, lse, ts, a) : 0.f;
  const uint16_t rounded = f2bf(e);
  const float shift = rounding_shift(e, rounded);
  if (lane < k) F.entries[n * k + lane] = P.t != 0.f ? rounded : kNoEntry;
  if (lane == 0) {
    F.R.lse[n] = taught ? lse : 0.f;
    F.R.ent[n] = taught ? s_rows.ent[q] : 0.f;
    F.R.l[n] = l;
    F.R.w[n] = w;
    F.R.mass[n] = P.mass;
    F.R.sc[n] = unit * shift;
    F.y[n] = y;
    F.R.a[n] = out;                                          // to row_out by who comes next: others clear it now
  }
  if (F.Hs) copy_row(F.H, row, A.d, unit, F.Hs, F.mcp, n);
}
// 32 rows of a block of 256 entries to a workgroup; rows up to the next multiple of 64 are zeros.  203 rows against 152 064 35 us for 191 MB (5.4 TB/s).
constexpr int kTurnedRows = 32;
__global__ void __launch_bounds__(256)
k_target_turn(KeptLogits Z, int V, const float* __restrict__ lse, const float* __restrict__ scale, const uint16_t* __restrict__ entries, Targets T,
              const int32_t* __restrict__ rowsel, int64_t n_sel, uint16_t* __restrict__ D, const float* __restrict__ out, float* __restrict__ row_out, int tiles_v, StatArgs S) {
  if (static_cast<int>(blockIdx.x) >= tiles_v) {             // the statistics
    __shared__ double smem[32];
    if (blockIdx.y == 0) target_stats<256>(S, static_cast<int>(blockIdx.x) - tiles_v, smem);
    return;
  }
  if (blockIdx.x == 0 && row_out && threadIdx.x < kTurnedRows) {
    const int64_t n = static_cast<int64_t>(blockIdx.y) * kTurnedRows + threadIdx.x;
    if (n < n_sel) row_out[rowsel ? rowsel[n] : n] = out[n];
  }
  const int64_t at = static_cast<int64_t>(blockIdx.x) * kBlkElems;
  const int r = static_cast<int>(blockIdx.y) * kTurnedRows + (threadIdx.x >> 3), c = (threadIdx.x & 7) * 8;
  const float y = r < n_sel ? scale[r] : 0.f, l2 = r < n_sel ? lse[r] * 1.44269504088896341f : 0.f;
  float4 z[4][2];
  if (y != 0.f)
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int q = 0; q < 2; ++q) z[i][q] = *reinterpret_cast<const float4*>(Z.at(r, blockIdx.x, i * 64 + c + q * 4));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint4 o = make_uint4(0u, 0u, 0u, 0u);
    if (y != 0.f) {
      const int left = V - static_cast<int>(blockIdx.x) * 256 - i * 64 - c;   // entries from V on: 0, whatever lies there
      auto p = [&](float x, int e) { return e < left ? __builtin_amdgcn_exp2f(fmaf(x, 1.44269504088896341f, -l2)) * y : 0.f; };
      o = make_uint4(pack_bf16x2(p(z[i][0].x, 0), p(z[i][0].y, 1)), pack_bf16x2(p(z[i][0].z, 2), p(z[i][0].w, 3)), pack_bf16x2(p(z[i][1].x, 4), p(z[i][1].y, 5)),
                     pack_bf16x2(p(z[i][1].z, 6), p(z[i][1].w, 7)));
    }
    *reinterpret_cast<uint4*>(D + at + r * 256 + i * 64 + c) = o;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < kTurnedRows * T.k; i += 256) {
    const int64_t n = static_cast<int64_t>(blockIdx.y) * kTurnedRows + i / T.k;
    if (n >= n_sel || scale[n] == 0.f) continue;
    const int id = T.ids[(rowsel ? rowsel[n] : n) * T.k + i % T.k];
    const uint16_t e = entries[n * T.k + i % T.k];
    if (e != kNoEntry && id >> 8 == static_cast<int>(blockIdx.x)) D[at + n * 256 + (id & 255)] = e;
  }
}
// Blocks in which some logit lies far above its row's reference: dz is computed once more, its k entries on the way out.  Without any 9 to 20 us, in which the
// statistics are summed beside.
struct PutTargets {
  const int32_t *rowsel, *ids;
  int k;
  const float *zt, *tt, *lse, *a, *w;
  float norm;
  __device__ __forceinline__ void operator()(char* staged, int64_t n, int v0, int width) const {
    const float g = n < 0 ? 0.f : w[n] / norm;
    if (g == 0.f) {                                          // whatever its logits are
      for (int i = 0; i < width * 2; i += 4) *reinterpret_cast<uint32_t*>(staged + i) = 0u;
      return;
    }
    const int32_t* id = ids + (rowsel ? rowsel[n] : n) * k;
    for (int j = 0; j < k; ++j) {
      const int v = id[j] - v0;
      const float t = tt[n * k + j];
      if (v < 0 || v >= width || t == 0.f) continue;
      const uint16_t e = f2bf(fmaf(a[n], __expf(zt[n * k + j] - lse[n]), -g * t));
      __builtin_memcpy(staged + v * 2, &e, 2);
    }
  }
};
__global__ void __launch_bounds__(Cfg::T)
k_target_flagged(const uint16_t* __restrict__ W, const uint16_t* __restrict__ H, int d, int V, const int32_t* __restrict__ rowsel, int64_t c0, int64_t mc,
                 const float* __restrict__ zero, PutTargets put, int tiles_m, int tiles_n, uint16_t* __restrict__ dZ, int64_t Vp,
                 const int32_t* __restrict__ flags, const int32_t* __restrict__ cidx, StatArgs S) {
  __shared__ __attribute__((aligned(16))) uint16_t lds[kLogitLds / 2];
  if (blockIdx.x >= kFlaggedGrid) {                          // the statistics, behind the last chunk's rows
    target_stats<Cfg::T>(S, static_cast<int>(blockIdx.x) - kFlaggedGrid, reinterpret_cast<double*>(lds));
    return;
  }
  for (int tile_n = 0; tile_n < tiles_n; ++tile_n) {
    const int out_blk = cidx[(c0 >> 8) + tile_n];
    if (!flags[(c0 >> 8) + tile_n]) continue;                // the same for every thread of the grid
    for (int tile_m = blockIdx.x; tile_m < tiles_m; tile_m += kFlaggedGrid)
      dz_tile(tile_m, tile_n, W, H, d, V, rowsel, c0, mc, put, put.lse, put.a, zero, dZ, Vp, out_blk, lds);
  }
}

// ------------------------------------------------------------------ bf16: the two gradient products (umas_gradients.h)
struct GradientArgs {
  const uint16_t* E;
  int64_t Vp, mcp;
  const uint16_t *W, *Hs;
  int d, V, tiles_v, tiles_d;
  DhSlices sl;
  int tiles_r;
  LiveInfo* info;
  const int32_t* blk_orig;
  uint16_t* dH;
  int accumulate;
  const int32_t* rowsel;
  int64_t c0, rows;
  const float* sc;
};
__global__ void __launch_bounds__(Cfg::T)
k_target_gemm(GradientArgs G, float* __restrict__ dW) {
  __shared__ __attribute__((aligned(16))) uint16_t lds[MixedLdsBytes<Cfg>::value / 2];
  gemm_dh_dw<false, float>(G.E, 1, G.Vp, G.mcp, G.W, G.Hs, G.d, G.V, G.tiles_v, G.tiles_d, G.sl, G.tiles_r, G.info, G.blk_orig, G.dH, dW, G.accumulate,
                           G.rowsel, G.c0, G.rows, nullptr, nullptr, G.sc, lds);
}
__global__ void __launch_bounds__(Cfg::T)
k_target_gemm_bf16(GradientArgs G, uint16_t* __restrict__ dW) {
  __shared__ __attribute__((aligned(16))) uint16_t lds[MixedLdsBytes<Cfg>::value / 2];
  gemm_dh_dw<false, uint16_t>(G.E, 1, G.Vp, G.mcp, G.W, G.Hs, G.d, G.V, G.tiles_v, G.tiles_d, G.sl, G.tiles_r, G.info, G.blk_orig, G.dH, dW, G.accumulate,
                              G.rowsel, G.c0, G.rows, nullptr, nullptr, G.sc, lds);
}
__global__ void __launch_bounds__(ShortCfg::T, 2)
k_target_dw_short(GradientArgs G, int tiles_n, float* __restrict__ dW) {
  __shared__ __attribute__((aligned(16))) char lds[kShortLds];
  dw_short<float>(G.E, 1, G.Vp, G.mcp, G.Hs, G.d, G.V, G.tiles_v, tiles_n, G.info, dW, G.accumulate, lds);
}
__global__ void __launch_bounds__(ShortCfg::T, 2)
k_target_dw_short_bf16(GradientArgs G, int tiles_n, uint16_t* __restrict__ dW) {
  __shared__ __attribute__((aligned(16))) char lds[kShortLds];
  dw_short<uint16_t>(G.E, 1, G.Vp, G.mcp, G.Hs, G.d, G.V, G.tiles_v, tiles_n, G.info, dW, G.accumulate, lds);
}
// dW of bf16 from the float32 sums of several chunks: rounded once
__global__ void __launch_bounds__(256)
k_target_round(const float* __restrict__ sums, uint16_t* __restrict__ dW, int64_t n8, int accumulate) {
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < n8; i += static_cast<int64_t>(gridDim.x) * 256) {
    float4 lo = reinterpret_cast<const float4*>(sums)[2 * i], hi = reinterpret_cast<const float4*>(sums)[2 * i + 1];
    uint4* const at = reinterpret_cast<uint4*>(dW) + i;
    if (accumulate) {
      float x[8];
      bf16x8_to_f32(*at, x);
      lo.x += x[0]; lo.y += x[1]; lo.z += x[2]; lo.w += x[3];
      hi.x += x[4]; hi.y += x[5]; hi.z += x[6]; hi.w += x[7];
    }
    *at = make_uint4(pack_bf16x2(lo.x, lo.y), pack_bf16x2(lo.z, lo.w), pack_bf16x2(hi.x, hi.y), pack_bf16x2(hi.z, hi.w));
  }
}

// The sum of the slices of dH.
struct ReduceArgs {
  unsigned rows_pad;
  DhSlices sl;
  int tiles_r, tiles_d, d;
  const LiveInfo* info;
  const int32_t* blk_orig;
  uint16_t* dH;
  const int32_t* rowsel;
  int64_t c0, rows;
  const float* sc;
};
__global__ void __launch_bounds__(256)
k_target_reduce(ReduceArgs C) {
  dh_reduce<false>(blockIdx.x % C.rows_pad, blockIdx.x / C.rows_pad, C.sl, C.tiles_r, C.tiles_d, nullptr, C.d, C.info, C.blk_orig, C.dH, C.rowsel, C.c0, C.rows,
                   nullptr, nullptr, C.sc);
}

// ------------------------------------------------------------------ float32, sums in float64
// The scores keep the float64 logits of a chunk of rows (see k_score_f32) and leave the statistics of parts of the vocabulary; then a workgroup of a row and part
// of the vocabulary merges the row's parts and takes its targets for itself, and turns its share of the logits into dz, the first one of the row leaving what else
// there is to say of it; then the gradient products, of rows of H that are zeros where nothing is taught.
struct DzArgsF32 {
  Teach A;
  const float* H;
  RowArrays R;
  const double* z;                        // [rows][V], of the chunk
  const f32::Stat* part;
  int splits;
  int64_t c0, rows;
  int per_wg;
  float *dz, *h_rows, *row_out;           // h_rows: of the chunk, NULL: no dW
};
__global__ void __launch_bounds__(256)
k_target_dz_f32(DzArgsF32 D) {
  const Teach& A = D.A;
  const int lane = threadIdx.x & 63, k = A.t.k, V = A.V;
  const int64_t m = blockIdx.y, n = D.c0 + m, row = A.rowsel ? A.rowsel[n] : n;
  f32::Stat a = f32::empty_stat();
  for (int p = lane; p < D.splits; p += kWave) a = f32::merge(a, D.part[p * D.rows + m]);
  if (a.s == 0.0) a = f32::Stat{-INFINITY, 0.0, 0.0, 0.0, 0.0};
  const double most = wave_max(a.m), e = a.s == 0.0 ? 0.0 : exp(a.m - most), s = wave_sum(a.s * e);
  const double lse = most + log(s), ent = lse - wave_sum(a.t * e) / s;
  const Place<double> P = place_of<double>(A.t, V, row);
  const bool taught = P.mass != 0.0;
  const float w = row_weight(A, row, taught);
  const double g = static_cast<double>(w) / static_cast<double>(A.norm), f = g * dense_factor(P.mass, A.z_coef, lse);
  const double ts = mass_of_token(k, P.id, P.t), z = P.t != 0.0 ? D.z[m * V + P.id] : 0.0;
  const int v0 = blockIdx.x * D.per_wg, v1 = min(v0 + D.per_wg, V);
  for (int vb = v0; vb < v1; vb += 1024)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int v = vb + q * 256 + threadIdx.x;
      if (v < v1) D.dz[m * V + v] = g != 0.0 ? static_cast<float>(f * exp(D.z[m * V + v] - lse)) : 0.f;
    }
  __syncthreads();
  if (threadIdx.x < kWave && P.t != 0.0 && g != 0.0 && P.id >= v0 && P.id < v1) D.dz[m * V + P.id] = static_cast<float>(f * exp(z - lse) - g * ts);
  if (blockIdx.x != 0) return;
  if (D.h_rows)
    for (int c = threadIdx.x; c < A.d; c += 256) D.h_rows[m * A.d + c] = w != 0.f ? D.H[row * A.d + c] : 0.f;
  if (threadIdx.x >= kWave) return;
  double l = 0.0, out = 0.0;
  if (taught && !A.t.logits) {
    out = __shfl(z, 0, kWave) - lse;
    l = -out + static_cast<double>(A.z_coef) * lse * lse;
  } else if (taught) {
    out = l = wave_sum(P.t != 0.0 ? P.t * (log(P.t) - (z - lse)) : 0.0);
  }
  if (lane != 0) return;
  D.R.l[n] = static_cast<float>(l);
  D.R.w[n] = w;
  D.R.mass[n] = static_cast<float>(P.mass);
  D.R.lse[n] = taught ? static_cast<float>(lse) : 0.f;
  D.R.ent[n] = taught ? static_cast<float>(ent) : 0.f;
  if (D.row_out) D.row_out[row] = static_cast<float>(out);
}

// ------------------------------------------------------------------ host side
struct Ws {
  float4* partial;
  RowArrays R;
  int32_t *flags, *blk_cidx, *blk_orig;
  LiveInfo* live;
  char* chunk;
  size_t fixed_bytes;
};
void carve(Carver& c, Ws& w, int64_t n_sel, int d, int V, int k, umas_dtype dt) {
  const int64_t n_pad = round_up(n_sel > 0 ? n_sel : 1, Cfg::BN), tiles_m = (V + Cfg::BM - 1) / Cfg::BM;
  const bool bf = dt == UMAS_BF16;
  w = Ws{};
  if (bf) w.partial = c.take<float4>(std::max(static_cast<size_t>(tiles_m) * n_pad, n_sel <= 64 ? static_cast<size_t>(kFewMostTiles) * 64 : 0));
  for (float** p : {&w.R.lse, &w.R.ent, &w.R.l, &w.R.w, &w.R.a, &w.R.zero, &w.R.cref, &w.R.sc, &w.R.mass}) *p = c.take<float>(n_pad);
  if (bf) {
    w.R.zt = c.take<float>(static_cast<size_t>(n_pad) * k);
    w.R.tt = c.take<float>(static_cast<size_t>(n_pad) * k);
    w.R.entries = reinterpret_cast<uint16_t*>(w.R.tt);       // one or the other
    w.flags = c.take<int32_t>(cdiv(n_pad, 256));
    w.blk_cidx = c.take<int32_t>(cdiv(n_pad, 256));
    w.blk_orig = c.take<int32_t>(cdiv(n_pad, 256));
    w.live = c.take<LiveInfo>(1);
  }
  w.chunk = c.base ? c.base + c.off : nullptr;
  w.fixed_bytes = c.off;
}
// A block of rows keeps its float32 logits; dH's partial sums take their place later.
constexpr int64_t kFewTaught = 256;
size_t few_bytes(int64_t n_sel, int V, umas_dtype dt) { return dt == UMAS_BF16 && n_sel <= kFewTaught ? std::max(static_cast<size_t>(256) * round_up(V, 256), few_floats(64, V) + 256) * sizeof(float) : 0; }
// float32 sums of dW where it is bf16 and comes from several chunks
size_t sum_bytes(int d, int V, int dW_type) { return dW_type == UMAS_BF16 ? align_up(static_cast<size_t>(V) * d * sizeof(float)) : 0; }
// float32: a chunk's dz, its rows of H, its float64 logits and the statistics of their parts.  256 MiB of logits to a chunk, what the memory-side cache holds,
// is as many as it takes to fill the chip.
size_t f32_bytes(int64_t mc, int d, int V) {
  return align_up(static_cast<size_t>(mc) * V * sizeof(float)) + align_up(static_cast<size_t>(mc) * d * sizeof(float)) +
         align_up(static_cast<size_t>(mc) * V * sizeof(double)) + align_up(static_cast<size_t>(f32::part_plan(mc, V).splits) * mc * sizeof(f32::Stat));
}
int64_t f32_rows(int64_t n_sel, int V) {
  const int64_t fit = static_cast<int64_t>((size_t{256} << 20) / (static_cast<size_t>(V) * sizeof(double)));
  return std::min(std::max<int64_t>(n_sel, 1), std::min(std::max<int64_t>(fit, 256), kF32ChunkRows));
}
bool sizes_ok(int64_t n_sel, int d, int V, int k, int dW_type) {
  return n_sel >= 0 && d >= 1 && V >= 1 && k >= 1 && k <= UMAS_MAX_TOP && dW_type >= UMAS_NO_DW && dW_type <= UMAS_BF16;
}
size_t least_bytes(int64_t n_sel, int d, int V, int k, umas_dtype dt, int dW_type) {
  if (!sizes_ok(n_sel, d, V, k, dW_type)) return 0;
  Carver c(nullptr);
  Ws w;
  carve(c, w, n_sel, d, V, k, dt);
  const int64_t all = std::max<int64_t>(n_sel, 1), mc = std::min<int64_t>(all, 256);
  if (dt == UMAS_F32) return c.off + f32_bytes(std::min<int64_t>(all, 32), d, V);
  const size_t chunked = chunk_bytes(mc, d, V, dt) + (n_sel > 256 ? sum_bytes(d, V, dW_type) : 0);
  // the sums of chunks can take more than one chunk of all rows
  return c.off + (all <= kMaxChunkRows ? std::min(chunked, chunk_bytes(all, d, V, dt)) : chunked) + few_bytes(all, V, dt);
}
size_t full_bytes(int64_t n_sel, int d, int V, int k, umas_dtype dt, int dW_type) {
  if (!sizes_ok(n_sel, d, V, k, dW_type)) return 0;
  Carver c(nullptr);
  Ws w;
  carve(c, w, n_sel, d, V, k, dt);
  if (dt == UMAS_F32) return c.off + f32_bytes(f32_rows(n_sel, V), d, V);
  int64_t mc = std::max<int64_t>(n_sel, 1);
  size_t sums = 0;
  if (mc > kMaxChunkRows) {
    const int64_t nchunk = (mc + kMaxChunkRows - 1) / kMaxChunkRows;
    mc = round_up((mc + nchunk - 1) / nchunk, 256);
    sums = sum_bytes(d, V, dW_type);
  }
  // (a frozen head: room for what plan_dh_alone may want, up to four rounds of pieces)
  const size_t parts = dW_type == UMAS_NO_DW ? std::min<size_t>(static_cast<size_t>(dh_tiles(mc, d)) * cdiv(V, 256), 1024) * (256 * 256 * sizeof(float)) : full_part_bytes(n_sel, mc, d, V);
  return c.off + chunk_bytes(mc, d, V, dt) + std::max(parts, few_bytes(mc, V, dt)) + sums;
}

struct Call {
  const void *H, *W;
  umas_dtype dt;
  int64_t n_rows;
  int32_t d, V;
  Targets t;
  const int32_t* rowsel;
  int64_t n_sel;
  const float* weight;
  const int32_t* tok_role;
  int32_t n_roles;
  float z_coef;
  int32_t accumulate_dW;
  int64_t norm_rows;
  umas_target_stats* stats;
  float* row_out;
  void *dH, *dW;
  int32_t dW_type;
  void* workspace;
  size_t workspace_bytes;
  hipStream_t st;
};
umas_status check_call(const Call& a) {
  umas_status s = check_model_args(a.H, a.W, a.dt, a.n_rows, a.d, a.V, a.t.ids, a.rowsel, a.n_sel);
  if (s != UMAS_OK) return s;
  UMAS_REQUIRE(a.t.k >= 1 && a.t.k <= UMAS_MAX_TOP, UMAS_ESHAPE, "k=%d outside [1,%d]", a.t.k, UMAS_MAX_TOP);
  UMAS_REQUIRE(a.dH || a.n_rows == 0, UMAS_EINVAL, "dH must not be NULL");
  UMAS_REQUIRE(a.stats, UMAS_EINVAL, "stats must not be NULL");
  UMAS_REQUIRE(a.n_roles >= 0 && a.n_roles <= UMAS_MAX_ROLES, UMAS_ESHAPE, "n_roles=%d outside [0,%d]", a.n_roles, UMAS_MAX_ROLES);
  UMAS_REQUIRE(a.tok_role || a.n_roles == 0, UMAS_EINVAL, "tok_role is NULL but n_roles > 0");
  UMAS_REQUIRE(a.dW_type == UMAS_F32 || (a.dW_type == UMAS_BF16 && a.dt == UMAS_BF16) || a.dW_type == UMAS_NO_DW, UMAS_EDTYPE,
               "dW_type=%d: float32, the type of the head, or none", a.dW_type);
  UMAS_REQUIRE((a.dW != nullptr) == (a.dW_type != UMAS_NO_DW), UMAS_EINVAL, "dW must be NULL with UMAS_NO_DW and only then");
  UMAS_REQUIRE(a.dW_type != UMAS_BF16 || reinterpret_cast<uintptr_t>(a.dW) % 16 == 0, UMAS_EINVAL, "a dW of bf16 must be 16-byte aligned");
  UMAS_REQUIRE(a.z_coef >= 0.f && a.z_coef < INFINITY, UMAS_EINVAL, "z_coef=%g must be finite and not negative", static_cast<double>(a.z_coef));
  UMAS_REQUIRE(a.n_sel < (1LL << 31), UMAS_ESHAPE, "at most 2^31-1 selected rows");
  UMAS_REQUIRE(a.norm_rows == 0 || a.norm_rows >= a.n_sel, UMAS_EINVAL, "norm_rows=%lld must be 0 or at least n_sel=%lld",
               static_cast<long long>(a.norm_rows), static_cast<long long>(a.n_sel));
  return check_ws(a.workspace, a.workspace_bytes, least_bytes(a.n_sel, a.d, a.V, a.t.k, a.dt, a.dW_type));
}
StatArgs stat_args(const Call& a, const Ws& w, float norm) {
  return StatArgs{a.n_sel, a.rowsel, a.tok_role, w.R.l, w.R.w, w.R.ent, w.R.lse, w.R.mass, norm, a.stats};
}

umas_status run_f32(const Call& a, const Ws& w, const Teach& A) {
  hipStream_t st = a.st;
  const float *H = static_cast<const float*>(a.H), *W = static_cast<const float*>(a.W);
  const size_t room = a.workspace_bytes - w.fixed_bytes;
  const int64_t n = a.n_sel;
  int64_t mc = f32_rows(n, a.V);
  while (mc > 32 && f32_bytes(mc, a.d, a.V) > room) mc = std::max<int64_t>(mc / 2, 32);
  const f32::PartPlan plan = f32::part_plan(mc, a.V);   // of every chunk
  for (int64_t c0 = 0; c0 < n; c0 += mc) {
    const int64_t rows = std::min(mc, n - c0);
    Carver c(w.chunk);
    float* const dz = c.take<float>(static_cast<size_t>(rows) * a.V);
    float* const h_rows = c.take<float>(static_cast<size_t>(rows) * a.d);
    double* const z = c.take<double>(static_cast<size_t>(rows) * a.V);
    f32::Stat* const part = c.take<f32::Stat>(static_cast<size_t>(plan.splits) * rows);
    ClearArgs clear{};
    unsigned n_clear = 0;                    // in rows of the grid
    if (a.rowsel && c0 == 0) {
      clear = ClearArgs{{reinterpret_cast<uint32_t*>(a.row_out), static_cast<uint32_t*>(a.dH), nullptr}, {a.n_rows, a.n_rows * a.d, 0}};
      const unsigned wg = cdiv(static_cast<size_t>(a.n_rows) * a.d, 2048);
      n_clear = cdiv(std::min(wg, 1024u), cdiv(rows, plan.side));
    }
    const f32::ScoreOut out{z, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr};
    const float* const Hc = a.rowsel ? H : H + c0 * a.d;
    const dim3 grid(cdiv(rows, plan.side), plan.splits + n_clear);
    auto score = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, grid, dim3(f32::kWaves * kWave), 0, st, W, Hc, a.d, a.V, a.rowsel ? a.rowsel + c0 : nullptr, rows, nullptr, part, out, plan.splits,
                         clear);
    };
    if (plan.side == f32::kTile) score(f32::k_score_f32<true, 2>);
    else score(f32::k_score_f32<true, 1>);
    UMAS_LAUNCHED("k_score_f32");
    const unsigned wgs = cdiv(2048, static_cast<size_t>(rows)), most = cdiv(a.V, 1024);      // eight workgroups to a compute unit
    const int per_wg = static_cast<int>(cdiv(most, std::min(wgs, most))) * 1024;
    hipLaunchKernelGGL(k_target_dz_f32, dim3(cdiv(a.V, per_wg), static_cast<unsigned>(rows)), dim3(256), 0, st,
                       DzArgsF32{A, H, w.R, z, part, plan.splits, c0, rows, per_wg, dz, a.dW ? h_rows : nullptr, a.row_out});
    UMAS_LAUNCHED("k_target_dz_f32");
    f32::launch_gradients(f32::GradArgs{dz, W, H, a.d, a.V, a.rowsel, c0, static_cast<int>(rows), a.accumulate_dW || c0 > 0 ? 1 : 0,
                                        static_cast<float*>(a.dH), static_cast<float*>(a.dW), 0, 0, 0, h_rows}, f32::StatArgs{}, st);
    UMAS_LAUNCHED("k_target_gradients_f32");
  }
  hipLaunchKernelGGL(k_target_stats, dim3(1 + a.n_roles), dim3(256), 0, st, stat_args(a, w, A.norm));
  UMAS_LAUNCHED("k_target_stats");
  return UMAS_OK;
}

umas_status run_bf16(const Call& a, const Ws& w, const Teach& A) {
  hipStream_t st = a.st;
  const uint16_t *H = static_cast<const uint16_t*>(a.H), *W = static_cast<const uint16_t*>(a.W);
  const int64_t n_sel = a.n_sel, Vp = round_up(a.V, 256);
  const int d = a.d, V = a.V, tiles_v = static_cast<int>(Vp / 256), tiles_d = (d + 255) / 256;
  size_t room = a.workspace_bytes - w.fixed_bytes;
  // chunks of rows as the workspace allows; a dW of bf16 that comes from several has its sums in front of them
  int64_t mc = std::min(n_sel, kMaxChunkRows);
  const bool chunked = n_sel > kMaxChunkRows || chunk_bytes(mc, d, V, UMAS_BF16) > room;
  float* sums = nullptr;
  char* chunk = w.chunk;
  if (chunked && a.dW_type == UMAS_BF16) {
    sums = reinterpret_cast<float*>(chunk);
    chunk += sum_bytes(d, V, UMAS_BF16);
    room -= sum_bytes(d, V, UMAS_BF16);
  }
  if (chunked) {
    if (chunk_bytes(mc, d, V, UMAS_BF16) > room) mc = std::max<int64_t>(static_cast<int64_t>(room / chunk_bytes(256, d, V, UMAS_BF16)), 1) * 256;
    const int64_t nchunk = (n_sel + mc - 1) / mc;
    mc = std::min(mc, round_up((n_sel + nchunk - 1) / nchunk, 256));
  }
  UMAS_REQUIRE(chunk_bytes(std::min(mc, n_sel), d, V, UMAS_BF16) <= room, UMAS_EWORKSPACE, "workspace cannot hold one chunk of %lld rows", static_cast<long long>(mc));
  const bool no_dw = a.dW_type == UMAS_NO_DW;
  const StatArgs stats = stat_args(a, w, A.norm);
  auto plan = [&](int64_t rows, DhSlices* sl) {             // as in the policy update: partial sums behind the chunk's operands or in the place of the scores' parts
    const size_t used = chunk_bytes(rows, d, V, UMAS_BF16), behind = room > used ? room - used : 0;
    const size_t front = static_cast<size_t>(reinterpret_cast<char*>(w.R.lse) - reinterpret_cast<char*>(w.partial));
    const size_t have = std::max(behind, front);
    const GradPlan p = no_dw ? GradPlan{plan_dh_alone(static_cast<int64_t>(cdiv(rows, 256)) * tiles_d, tiles_v, device_cus(), have), false}
                             : plan_gradients(n_sel, rows, d, V, slices_dh(n_sel, mc, d) ? have : 0);
    *sl = DhSlices{p.dh.slices, p.dh.voc_blks, behind > front ? reinterpret_cast<float*>(chunk + used) : reinterpret_cast<float*>(w.partial)};
    return p.dw_apart;
  };
  auto live_args = [&](int64_t c0, int64_t rows, int slices, bool dw_apart) {
    return LiveArgs{static_cast<int>(c0 >> 8), static_cast<int>(cdiv(rows, 256)), rows, 1, dw_apart || no_dw ? 0 : tiles_v, tiles_d, Vp, slices, nullptr,
                    w.blk_cidx, w.blk_orig, w.live};
  };
  for (int64_t c0 = 0; c0 < n_sel; c0 += mc) {
    const int64_t rows = std::min(mc, n_sel - c0), mcp = round_up(rows, 256);
    const int tiles_r = static_cast<int>(mcp / 256), panel = row_panel(tiles_r, d), halved = halved_tiles(tiles_v, tiles_r);
    uint16_t* const E = reinterpret_cast<uint16_t*>(chunk);
    uint16_t* const Hs = no_dw ? nullptr : reinterpret_cast<uint16_t*>(chunk + align_up(static_cast<size_t>(mcp) * Vp * 2));
    DhSlices sl;
    const bool dw_apart = plan(rows, &sl);
    const LiveArgs live = live_args(c0, rows, sl.n, dw_apart);
    const bool few = n_sel <= kFewTaught;
    const bool narrow = n_sel <= NarrowCfg::BN;
    const int64_t n_pad = n_sel <= few_rows(d) ? 64 : round_up(n_sel, narrow ? NarrowCfg::BN : Cfg::BN);
    if (few) {
      float* const Z = reinterpret_cast<float*>(chunk + chunk_bytes(rows, d, V, UMAS_BF16));
      KeptLogits kept{Z, 0};
      int parts = tiles_v;
      if (n_sel <= few_rows(d)) {
        parts = few_workgroups(V);
        const int per = few_per(V, parts);
        kept.stride = static_cast<int64_t>(parts) * per * 16;
        with_few(d, n_sel, [&](auto ni, auto ppw) {
          hipLaunchKernelGGL((k_target_logits_few<decltype(ni)::value, decltype(ppw)::value>), dim3(parts), dim3(kFewT), 0, st, W, H, d, V, a.rowsel,
                             static_cast<int>(n_sel), per, w.partial, n_pad, Z, kept.stride);
        });
        UMAS_LAUNCHED("k_target_logits_few");
      } else if (narrow) {
        parts = static_cast<int>(Vp / NarrowCfg::BM);
        // (the pass of 128 rows of 2048 490 -> 482 us, of 106 of 1344 against 138 057 314 -> 308, 100 of 3584 equal)
        const int halved = n_sel > HalfNarrowCfg::BN ? halved_tiles(parts, 1, 2) : 0;
        hipLaunchKernelGGL(k_target_logits_narrow, score_grid(parts, 1, kGN, halved), dim3(NarrowCfg::T), 0, st, W, H, d, V, a.rowsel, n_sel,
                           a.t.ids, parts, halved, w.partial, n_pad, Z, Vp);
        UMAS_LAUNCHED("k_target_logits_narrow");
      } else {
        hipLaunchKernelGGL(k_target_logits, score_grid(tiles_v, 1, kGN, halved), dim3(Cfg::T), 0, st, W, H, d, V, a.rowsel, n_sel, a.t.ids, tiles_v, halved, w.partial,
                           n_pad, Z, Vp);
        UMAS_LAUNCHED("k_target_logits");
      }
      const unsigned clearing = a.rowsel ? 128 : 0;
      hipLaunchKernelGGL(k_target_few, dim3(1 + clearing + cdiv(n_sel, 8)), dim3(kRowsT), 0, st,
                         FewArgs{A, H, w.R, w.R.cref, w.R.entries, w.partial, parts, n_pad, kept, Hs, mcp, a.row_out, live, clearing, static_cast<uint32_t*>(a.dH),
                                 a.n_rows * static_cast<int64_t>(d) / 2, a.n_rows});
      UMAS_LAUNCHED("k_target_few");
      hipLaunchKernelGGL(k_target_turn, dim3(tiles_v + 1 + a.n_roles, static_cast<unsigned>(round_up(n_sel, 64) / kTurnedRows)), dim3(256), 0, st, kept, V, w.R.lse, w.R.cref, w.R.entries, A.t,
                         a.rowsel, n_sel, E, w.R.a, a.row_out, tiles_v, stats);
      UMAS_LAUNCHED("k_target_turn");
    } else if (c0 == 0) {
      const int share = a.t.k > 4 ? 4 : 1;
      const OpenArgs O{A, H, W, w.R, w.flags, static_cast<int>(cdiv(n_sel, 256)), live, a.rowsel ? static_cast<uint32_t*>(a.dH) : nullptr,
                       a.n_rows * static_cast<int64_t>(d) / 2, a.row_out, a.row_out ? a.n_rows : 0, share};
      hipLaunchKernelGGL(k_target_open, dim3(1 + std::min<unsigned>(std::max<unsigned>(cdiv(n_sel, 4 / share), a.rowsel ? 1024 : 1), 8192)), dim3(256), 0, st, O);
      UMAS_LAUNCHED("k_target_open");
    } else {
      hipLaunchKernelGGL(k_live_scan, dim3(1), dim3(512), 0, st, live);
      UMAS_LAUNCHED("k_live_scan");
    }
    if (!few) {
      // (half a tile less of 17 is 2 %, of 64 what the other loop costs)
      const bool ends = rows % Cfg::BN != 0 && rows % Cfg::BN <= HalfCfg::BN && tiles_r <= 32;
      hipLaunchKernelGGL(ends ? k_target_tiles_end : k_target_tiles, score_grid(tiles_v, tiles_r, panel, halved), dim3(Cfg::T), 0, st, W, H, d, V, a.rowsel, c0, rows, tiles_v, tiles_r,
                         panel, halved, w.partial, n_pad, w.R.cref, E, Vp, w.flags, w.blk_cidx);
      UMAS_LAUNCHED("k_target_tiles");
      hipLaunchKernelGGL(k_target_rows, dim3(cdiv(rows, 8)), dim3(kRowsT), 0, st,
                         RowsArgs{A, H, w.R, w.partial, tiles_v, n_pad, c0, rows, w.flags, w.blk_cidx, E, tiles_v, Hs, mcp, a.row_out});
      UMAS_LAUNCHED("k_target_rows");
      const PutTargets put{a.rowsel, a.t.ids, a.t.k, w.R.zt, w.R.tt, w.R.lse, w.R.a, w.R.w, A.norm};
      hipLaunchKernelGGL(k_target_flagged, dim3(kFlaggedGrid + (c0 + rows >= n_sel ? 1 + a.n_roles : 0)), dim3(Cfg::T), 0, st, W, H, d, V, a.rowsel, c0, rows, w.R.zero, put, tiles_v, tiles_r, E, Vp,
                         w.flags, w.blk_cidx, stats);
      UMAS_LAUNCHED("k_target_flagged");
    }
    const int add = c0 > 0 || (a.accumulate_dW && !sums) ? 1 : 0;
    const GradientArgs G{E, Vp, mcp, W, Hs, d, V, tiles_v, tiles_d, sl, tiles_r, w.live, w.blk_orig, static_cast<uint16_t*>(a.dH), add, a.rowsel, c0, rows, w.R.sc};
    const unsigned grid = static_cast<unsigned>(round_up(device_cus(), 8));
    if (sums || a.dW_type == UMAS_F32) hipLaunchKernelGGL(k_target_gemm, dim3(grid), dim3(Cfg::T), 0, st, G, sums ? sums : static_cast<float*>(a.dW));
    else hipLaunchKernelGGL(k_target_gemm_bf16, dim3(grid), dim3(Cfg::T), 0, st, G, static_cast<uint16_t*>(a.dW));
    UMAS_LAUNCHED("k_target_gemm");
    if (dw_apart) {
      const int tiles_n = (d + ShortCfg::BN - 1) / ShortCfg::BN;
      const dim3 g2(static_cast<unsigned>(round_up(static_cast<int64_t>(tiles_v) * tiles_n, 8)));
      if (sums || a.dW_type == UMAS_F32) hipLaunchKernelGGL(k_target_dw_short, g2, dim3(ShortCfg::T), 0, st, G, tiles_n, sums ? sums : static_cast<float*>(a.dW));
      else hipLaunchKernelGGL(k_target_dw_short_bf16, g2, dim3(ShortCfg::T), 0, st, G, tiles_n, static_cast<uint16_t*>(a.dW));
      UMAS_LAUNCHED("k_target_dw_short");
    }
    if (sl.n > 1) {
      hipLaunchKernelGGL(k_target_reduce, dim3(static_cast<unsigned>(mcp) * cdiv(d, 1024)), dim3(256), 0, st,
                         ReduceArgs{static_cast<unsigned>(mcp), sl, tiles_r, tiles_d, d, w.live, w.blk_orig, static_cast<uint16_t*>(a.dH), a.rowsel, c0, rows, w.R.sc});
      UMAS_LAUNCHED("k_target_reduce");
    }
  }
  if (sums) {
    const int64_t n8 = static_cast<int64_t>(V) * d / 8;
    hipLaunchKernelGGL(k_target_round, dim3(static_cast<unsigned>(std::min<int64_t>((n8 + 255) / 256, 8192))), dim3(256), 0, st, sums,
                       static_cast<uint16_t*>(a.dW), n8, a.accumulate_dW ? 1 : 0);
    UMAS_LAUNCHED("k_target_round");
  }
  return UMAS_OK;
}

umas_status run(const Call& a) {
  umas_status s = check_call(a);
  if (s != UMAS_OK) return s;
  hipStream_t st = a.st;
  prof_mark(st);
  Carver c(a.workspace);
  Ws w;
  carve(c, w, a.n_sel, a.d, a.V, a.t.k, a.dt);
  const float norm = static_cast<float>(a.norm_rows > 0 ? a.norm_rows : a.n_sel > 0 ? a.n_sel : 1);
  const Teach A{a.t, a.rowsel, a.n_sel, a.V, a.d, a.weight, norm, a.z_coef};
  if (a.n_sel == 0) {
    const size_t esz = a.dt == UMAS_BF16 ? 2 : 4, dw = static_cast<size_t>(a.V) * a.d * (a.dW_type == UMAS_BF16 ? 2 : 4);
    UMAS_HIP(clear_bytes(st, a.n_rows > 0 ? a.dH : nullptr, static_cast<size_t>(a.n_rows) * a.d * esz, a.row_out, static_cast<size_t>(a.n_rows) * 4,
                         a.accumulate_dW ? nullptr : a.dW, dw));
    hipLaunchKernelGGL(k_target_stats, dim3(1 + a.n_roles), dim3(256), 0, st, stat_args(a, w, norm));
    UMAS_LAUNCHED("k_target_stats");
    return UMAS_OK;
  }
  return a.dt == UMAS_F32 ? run_f32(a, w, A) : run_bf16(a, w, A);
}

}  // namespace
}  // namespace umas

using namespace umas;

extern "C" size_t umas_cross_entropy_workspace_bytes_min(int64_t n_sel, int32_t d, int32_t V, umas_dtype dtype, int32_t dW_type) {
  return least_bytes(n_sel, d, V, 1, dtype, dW_type);
}
extern "C" size_t umas_cross_entropy_workspace_bytes(int64_t n_sel, int32_t d, int32_t V, umas_dtype dtype, int32_t dW_type) {
  return full_bytes(n_sel, d, V, 1, dtype, dW_type);
}
extern "C" size_t umas_distill_workspace_bytes_min(int64_t n_sel, int32_t d, int32_t V, int32_t k, umas_dtype dtype, int32_t dW_type) {
  return least_bytes(n_sel, d, V, k, dtype, dW_type);
}
extern "C" size_t umas_distill_workspace_bytes(int64_t n_sel, int32_t d, int32_t V, int32_t k, umas_dtype dtype, int32_t dW_type) {
  return full_bytes(n_sel, d, V, k, dtype, dW_type);
}

extern "C" umas_status umas_cross_entropy_fwd_bwd(const void* H, const void* W, umas_dtype dtype, int64_t n_rows, int32_t d, int32_t V, const int32_t* ids,
                                                  const int32_t* rowsel, int64_t n_sel, const float* weight, const int32_t* tok_role, int32_t n_roles,
                                                  float z_coef, int32_t accumulate_dW, int64_t norm_rows, umas_target_stats* stats, float* logp, void* dH,
                                                  void* dW, int32_t dW_type, void* workspace, size_t workspace_bytes, void* hip_stream) {
  return run(Call{H, W, dtype, n_rows, d, V, Targets{ids, nullptr, nullptr, 1}, rowsel, n_sel, weight, tok_role, n_roles, z_coef,
                  accumulate_dW, norm_rows, stats, logp, dH, dW, dW_type, workspace, workspace_bytes, static_cast<hipStream_t>(hip_stream)});
}

extern "C" umas_status umas_distill_fwd_bwd(const void* H, const void* W, umas_dtype dtype, int64_t n_rows, int32_t d, int32_t V, const int32_t* top_ids,
                                            const float* top_logits, int32_t k, const float* teacher_lse, const int32_t* rowsel, int64_t n_sel,
                                            const float* weight, const int32_t* tok_role, int32_t n_roles, int32_t accumulate_dW, int64_t norm_rows,
                                            umas_target_stats* stats, float* kl, void* dH, void* dW, int32_t dW_type, void* workspace,
                                            size_t workspace_bytes, void* hip_stream) {
  UMAS_REQUIRE(top_logits || n_rows == 0, UMAS_EINVAL, "top_logits must not be NULL");
  static const float none = 0.f;           // no rows: anything but NULL, which stands for cross entropy
  return run(Call{H, W, dtype, n_rows, d, V, Targets{top_ids, top_logits ? top_logits : &none, teacher_lse, k}, rowsel, n_sel, weight,
                  tok_role, n_roles, 0.f, accumulate_dW, norm_rows, stats, kl, dH, dW, dW_type, workspace, workspace_bytes,
                  static_cast<hipStream_t>(hip_stream)});
}
