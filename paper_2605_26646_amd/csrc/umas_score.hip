// LM-head scoring, the clipped PPO surrogate and the backward through the LM head.
//
// Scoring ("old log probabilities", paragraph "Advantage computation and policy evaluation"):
// for every selected row z = W h, lse = log sum exp z, logp = z[y] - lse, entropy = lse -
// sum softmax(z) z.  The bf16 path computes 256x256 logit tiles with MFMA and reduces each tile
// to per-row (max, sum exp, sum exp*z, taken logit) in registers; logits never leave the chip.
// Update (paragraph "Model-specific updates and synchronization", PPO after Schulman et al.
// 2017): ratio = exp(logp - logp_old), L = max(-A ratio, -A clip(ratio)), g = dL/dlogp, then
// dH = dz W and dW = dz^T H with dz = g (onehot - softmax) run as MFMA GEMMs over a bf16 operand
// [rows, vocabulary] held in a bounded chunk buffer; W is read as it lies, of H dW reads a copy of the chunk's rows
// in column blocks (operands that are not K-contiguous go through transposing LDS reads); the one-hot part (one term
// per row) is added in float32.
// Without an entropy bonus the dense part of dz is a row factor times the softmax, so the scoring pass of
// the update itself leaves that operand behind: E = bf16(exp(z - z_y)), the softmax numerators relative to
// the taken token's logit, and the row factor -g exp(z_y - lse) is applied where dH is written and folded
// into the copy of H that dW reads; the logits are computed once.  With an entropy bonus the
// scoring pass leaves the float32 logits behind, which one pass over them turns into dz; in a workspace without room
// for them, for narrow heads (and for blocks of rows whose logits spread too far for E) dz is recomputed tile by tile from H, W and lse.
// The float32 path, for small shapes, carries its sums in float64 (umas_f32.h).
#include <mutex>

#include "umas_f32.h"
#include "umas_gradients.h"

namespace umas {
namespace {

// (kernel templates whose bodies use buffer resources do not get their host stubs emitted: plain kernels)
__global__ void __launch_bounds__(Cfg::T)
k_score_tiles(const uint16_t* __restrict__ W, const uint16_t* __restrict__ H, int d, int V,
              const int32_t* __restrict__ rowsel, int64_t n_sel, const int32_t* __restrict__ ids,
              int tiles_m, int tiles_n, int panel, int halved, float4* __restrict__ partial, int64_t n_pad) {
  __shared__ __attribute__((aligned(16))) uint16_t lds[kLogitLds / 2];
  score_tiles<Leave::kNothing, Cfg>(W, H, d, V, rowsel, 0, n_sel, ids, tiles_m, tiles_n, panel, partial, n_pad, KeepArgs{}, lds, halved);
}
__global__ void __launch_bounds__(NarrowCfg::T)
k_score_narrow(const uint16_t* __restrict__ W, const uint16_t* __restrict__ H, int d, int V,
               const int32_t* __restrict__ rowsel, int64_t n_sel, const int32_t* __restrict__ ids,
               int tiles_m, int tiles_n, int panel, float4* __restrict__ partial, int64_t n_pad) {
  __shared__ __attribute__((aligned(16))) uint16_t lds[kNarrowLds / 2];
  score_tiles<Leave::kNothing, NarrowCfg>(W, H, d, V, rowsel, 0, n_sel, ids, tiles_m, tiles_n, panel, partial, n_pad, KeepArgs{}, lds);
}
__global__ void __launch_bounds__(Cfg::T)
k_score_keep_tiles(const uint16_t* __restrict__ W, const uint16_t* __restrict__ H, int d, int V,
                   const int32_t* __restrict__ rowsel, int64_t c0, int64_t mc, const int32_t* __restrict__ ids,
                   int tiles_m, int tiles_n, int panel, int halved, float4* __restrict__ partial, int64_t n_pad,
                   const float* __restrict__ cref, uint16_t* __restrict__ E, int64_t Vp, int32_t* __restrict__ flags,
                   const int32_t* __restrict__ cidx) {
  __shared__ __attribute__((aligned(16))) uint16_t lds[kLogitLds / 2];
  score_tiles<Leave::kNumerators, Cfg>(W, H, d, V, rowsel, c0, mc, ids, tiles_m, tiles_n, panel, partial, n_pad, KeepArgs{cref, E, Vp, flags, cidx, nullptr}, lds, halved);
}
// ... and what an update of so few rows keeps: half rows of half blocks of the operand, whose other rows are never read (100 rows of 3584 270 -> 211
// us; the update, with shorter sums for dW and half the products for dH, 1000 -> 887, of 2048 608 -> 518).
__global__ void __launch_bounds__(NarrowCfg::T)
k_score_keep_narrow(const uint16_t* __restrict__ W, const uint16_t* __restrict__ H, int d, int V,
                    const int32_t* __restrict__ rowsel, int64_t n_sel, const int32_t* __restrict__ ids,
                    int tiles_m, float4* __restrict__ partial, int64_t n_pad, const float* __restrict__ cref, uint16_t* __restrict__ E, int64_t Vp,
                    int32_t* __restrict__ flags, const int32_t* __restrict__ cidx) {
  __shared__ __attribute__((aligned(16))) uint16_t lds[kNarrowLds / 2];
  score_tiles<Leave::kNumerators, NarrowCfg>(W, H, d, V, rowsel, 0, n_sel, ids, tiles_m, 1, kGN, partial, n_pad, KeepArgs{cref, E, Vp, flags, cidx, nullptr}, lds);
}
__global__ void __launch_bounds__(Cfg::T)
k_score_logits(const uint16_t* __restrict__ W, const uint16_t* __restrict__ H, int d, int V,
               const int32_t* __restrict__ rowsel, int64_t c0, int64_t mc, const int32_t* __restrict__ ids,
               int tiles_m, int tiles_n, int panel, int halved, float4* __restrict__ partial, int64_t n_pad, float* __restrict__ Z, int64_t Vp) {
  __shared__ __attribute__((aligned(16))) uint16_t lds[kLogitLds / 2];
  score_tiles<Leave::kLogits, Cfg>(W, H, d, V, rowsel, c0, mc, ids, tiles_m, tiles_n, panel, partial, n_pad, KeepArgs{nullptr, nullptr, Vp, nullptr, nullptr, Z}, lds, halved);
}

// ------------------------------------------------------------------ bf16: a few rows
// Up to 32 selected rows (64 up to d = 2048): the pass is bound by reading W once, and a 256x256 tile with most of its columns empty spends
// its time filling and draining.  Here the rows of H stay in registers and W streams past them: the eight wavefronts of a
// workgroup split the hidden dimension (each takes PPW pieces of 64, next to each other across the wavefronts, so that a
// row of W is read in whole lines), a wavefront holds its pieces of up to 16 NI rows as MFMA operands for the whole kernel
// and walks a contiguous range of the vocabulary MB blocks of 16 entries at a time, W going straight to registers; a
// piece's registers are loaded again for the next step as soon as they have been used, so that 8 KB and more are in flight
// per wavefront all the time.  The eight partial logits meet in LDS (one barrier a step, two buffers), and every thread
// keeps the softmax statistics of one (row, place in the block of 16) over its workgroup's whole range.  One workgroup per
// compute unit; partials [workgroup][row].
// 24 rows of 2048 (3584) against 151 936: 256x256 tiles 183 (279) us, this kernel 117 (199) us = 5.3 (5.5) TB/s of W; 64
// rows of 2048 182 -> 122 us.
template <int NI, int PPW>
__global__ void __launch_bounds__(kFewT)
k_score_few(const uint16_t* __restrict__ W, const uint16_t* __restrict__ H, int d, int V, const int32_t* __restrict__ rowsel, int n_sel,
            const int32_t* __restrict__ ids, float4* __restrict__ partial, int n_pad) {
  constexpr int MB = PPW <= 4 && NI <= 2 ? 2 : 1;            // blocks of 16 vocabulary entries per step
  constexpr int NL = (NI + 1) / 2;                           // logits per thread and block
  __shared__ __attribute__((aligned(16))) float s_z[2][kFewWaves][MB][NI][16][16];   // [.][wavefront][block][.][row][entry]
  __shared__ float4 s_part[NI * 16][16];
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
  // this workgroup's blocks of 16 vocabulary entries
  const int blocks = (V + 15) / 16;
  const int per = (blocks + static_cast<int>(gridDim.x) - 1) / static_cast<int>(gridDim.x);
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
  // thread -> (row, place): statistics of the logits of that row at that place of every block
  const bool mine = tid < NI * 256;
  const int my_n = (tid >> 4) & 15, my_v = tid & 15;
  int y[NL];
  float m[NL], s[NL], t[NL], zy[NL];
#pragma unroll
  for (int l = 0; l < NL; ++l) {
    const int n = (2 * l + (tid >> 8)) * 16 + my_n;
    y[l] = mine && n < n_sel ? ids[rowsel ? rowsel[n] : n] : -1;
    // kMasked as in the tiles: against a maximum of -infinity a logit of -infinity makes the sums NaN, and the merge drops
    // a partial whose maximum a NaN logit has left there
    m[l] = kMasked; s[l] = t[l] = zy[l] = 0.f;
  }
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
          // zeros of H alone would not do: their product with a weight that is not finite is NaN
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
          const int v = (b + i) * 16 + my_v;
          if (v < V && b + i < b1) {
            if (v == y[l]) zy[l] = z;
            const float gap = z - m[l], e = __expf(-fabsf(gap));  // one exponential: of the smaller relative to the larger
            if (gap > 0.f) { s[l] = fmaf(s[l], e, 1.f); t[l] = fmaf(t[l], e, z); m[l] = z; }
            else { s[l] += e; t[l] = fmaf(e, z, t[l]); }
          }
        }
    }
  }
#pragma unroll
  for (int l = 0; l < NL; ++l)
    if (mine) s_part[(2 * l + (tid >> 8)) * 16 + my_n][my_v] = make_float4(m[l], s[l], t[l], zy[l]);
  __syncthreads();
  if (tid < NI * 16) {
    Part p{kNegInf, 0.f, 0.f};
    float z = 0.f;
    for (int k = 0; k < 16; ++k) {
      const float4 q = s_part[tid][k];
      p = part_merge(p, Part{q.x, q.y, q.z});
      z += q.w;
    }
    partial[static_cast<int64_t>(blockIdx.x) * n_pad + tid] = make_float4(p.m, p.s, p.t, z);
  }
}

template <bool SPLIT>
__global__ void __launch_bounds__(256)
k_score_finalize(const float4* __restrict__ partial, int tiles_m, int64_t n_pad, int64_t n_begin,
                 int64_t n_end, const float* __restrict__ zy_c, const int32_t* __restrict__ rowsel,
                 const int32_t* __restrict__ ids, int V,
                 float* __restrict__ logp_c, float* __restrict__ lse_c, float* __restrict__ ent_c,
                 float* __restrict__ logp, float* __restrict__ lse, float* __restrict__ entropy) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t n = n_begin + (SPLIT ? static_cast<int64_t>(blockIdx.x) : static_cast<int64_t>(blockIdx.x) * 4 + wave) * 8 + (lane & 7);
  Part p;
  float zy;
  if (!merge_parts<SPLIT>(partial, tiles_m, n_pad, n, n < n_end, p, zy)) return;
  if (zy_c) zy = zy_c[n];                                   // taken logits computed beforehand
  const int64_t row = rowsel ? rowsel[n] : n;
  const int y = ids[row];
  const RowScore r = row_score(p, zy, y >= 0 && y < V);
  if (logp_c) { logp_c[n] = r.logp; lse_c[n] = r.lse; ent_c[n] = r.entropy; }
  if (logp) logp[row] = r.logp;
  if (lse) lse[row] = r.lse;
  if (entropy) entropy[row] = r.entropy;
}

// ------------------------------------------------------------------ clipped surrogate
// Per selected row its surrogate, and what the backward needs of it; per block of rows the sums of the statistics for the model and for
// each role.
__global__ void __launch_bounds__(kRowBlock)
k_ppo_rows(Surrogate S, int64_t n_begin, int64_t n_end, const float* __restrict__ logp_c, const float* __restrict__ ent_c,
           float k_ent, int label_apart, const float* __restrict__ lse_c, float* __restrict__ g_c,
           float* __restrict__ a_c, float* __restrict__ kz_c, double* __restrict__ blk_stats) {
  extern __shared__ double s_acc[];   // [wavefronts][(1+n_roles) * kStat]
  const int n_roles = S.n_roles, nacc = (1 + n_roles) * kStat;
  const int lane = threadIdx.x & (kWave - 1);
  double* const w_acc = s_acc + threadIdx.x / kWave * nacc;
  for (int i = lane; i < nacc; i += kWave) w_acc[i] = 0.0;
  __builtin_amdgcn_wave_barrier();
  SurrogateRow R{0.f, 0.f, 0.f, 0.f, 0.f, -1, false};
  const int64_t n = n_begin + static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x;   // n_begin is a multiple of the block size
  if (n < n_end) {
    const int64_t row = S.rowsel ? S.rowsel[n] : n;
    const int y = S.ids[row];
    const bool ok = y >= 0 && y < S.V;
    const float lp = ok ? logp_c[n] : 0.f, en = ok ? ent_c[n] : 0.f;
    R = surrogate_row(S, row, ok, lp, en);
    // With label_apart the taken token's column is left out of the dense (bf16) part of dz and g_c carries all of
    // dz[n, y] = g (1 - p_y) + k_ent p_y (log p_y + entropy) in float32: for a confident token g and g p_y nearly
    // cancel, and the rounding of a bf16 g p_y would be as large as what is left.
    g_c[n] = label_apart && ok ? fmaf(R.g, -expm1f(lp), k_ent * __expf(lp) * (lp + en)) : R.g;
    // coefficients of the backward's dense part dz = p (a + kz z): -g from the surrogate, the rest from the
    // entropy bonus k_ent p (log p + entropy); a row with an invalid id has neither
    a_c[n] = ok ? -R.g + k_ent * (en - lse_c[n]) : 0.f;
    kz_c[n] = ok ? k_ent : 0.f;
  }
  const float L = R.L, clipped = R.clipped, en = R.en, kl = R.kl;
  const int role = R.role, valid = R.valid;
  // Sums over the wavefront's rows, the model's and then each role's that occurs among them (usually one or two); the
  // wavefronts' sums are added in a fixed order.  (256 threads adding to six float64 words by atomics took 18 us.)
  const unsigned long long in = __ballot(n < n_end);
  auto sum_into = [&](unsigned long long group, double* acc) {
    const bool mine = (group >> lane) & 1;
    const double sl = wave_sum(mine ? static_cast<double>(L) : 0.0), se = wave_sum(mine ? static_cast<double>(en) : 0.0);
    const double sk = wave_sum(mine ? static_cast<double>(kl) : 0.0);
    const int c = __popcll(__ballot(mine && clipped != 0.f)), bad = __popcll(__ballot(mine && !valid));
    if (lane == 0) { acc[0] = sl; acc[1] = c; acc[2] = se; acc[3] = sk; acc[4] = __popcll(group); acc[5] = bad; }
  };
  sum_into(in, w_acc);
  unsigned long long left = in & __ballot(role >= 0 && role < n_roles);
  while (left) {                                              // the same for every lane
    const int r = __shfl(role, __ffsll(static_cast<long long>(left)) - 1, kWave);
    const unsigned long long group = left & __ballot(role == r);
    sum_into(group, w_acc + (1 + r) * kStat);
    left &= ~group;
  }
  __syncthreads();
  const int64_t blk = n_begin / kRowBlock + blockIdx.x;
  for (int i = threadIdx.x; i < nacc; i += blockDim.x) {
    double v = 0.0;
    for (int w = 0; w < kRowBlock / kWave; ++w) v += s_acc[w * nacc + i];
    blk_stats[blk * nacc + i] = v;
  }
}

// The record of the model (k = 0) or of a role, a workgroup to each.
__device__ __forceinline__ void
ppo_stats(int k, int nblk, int n_roles, float entropy_coef, int64_t norm_rows, const double* __restrict__ blk_stats,
            umas_loss_stats* __restrict__ stats) {
  __shared__ double smem[32];
  const int nacc = (1 + n_roles) * kStat;
  double v[kStat] = {}, sum[kStat];
  for (int b = threadIdx.x; b < nblk; b += blockDim.x)
#pragma unroll
    for (int j = 0; j < kStat; ++j) v[j] += blk_stats[static_cast<int64_t>(b) * nacc + k * kStat + j];
#pragma unroll
  for (int j = 0; j < kStat; ++j) sum[j] = block_sum<double>(v[j], smem);
  if (threadIdx.x != 0) return;
  stats[k] = loss_stats(sum, k, entropy_coef, norm_rows);
}

// The same from the rows, where they are few and k_rows_few has left no sums.
__device__ __forceinline__ void ppo_stats_by_row(int k, const Surrogate& S, int64_t n_sel, float entropy_coef, int64_t norm_rows, const float* __restrict__ logp_c,
                                                 const float* __restrict__ ent_c, umas_loss_stats* __restrict__ stats) {
  __shared__ double smem[32];
  double v[kStat] = {}, sum[kStat];
  for (int64_t n = threadIdx.x; n < n_sel; n += blockDim.x) {
    const int64_t row = S.rowsel ? S.rowsel[n] : n;
    const int y = S.ids[row];
    const SurrogateRow R = surrogate_row(S, row, y >= 0 && y < S.V, logp_c[n], ent_c[n]);
    if (k > 0 && R.role != k - 1) continue;
    v[0] += static_cast<double>(R.L);
    v[1] += R.clipped != 0.f ? 1.0 : 0.0;
    v[2] += static_cast<double>(R.en);
    v[3] += static_cast<double>(R.kl);
    v[4] += 1.0;
    v[5] += R.valid ? 0.0 : 1.0;
  }
#pragma unroll
  for (int j = 0; j < kStat; ++j) sum[j] = block_sum<double>(v[j], smem);
  if (threadIdx.x != 0) return;
  stats[k] = loss_stats(sum, k, entropy_coef, norm_rows);
}

// What opens the keeping update, in one launch: the first nblk workgroups mark the live blocks of 256 selected rows and
// clear their flags, the others take the rows' references and clear what the call defines everywhere (logp_new when rows
// are left out, dH), each its share.  Up to kFewBlocks blocks in one chunk the first workgroup alone marks them and packs them as well, under the
// others' work (203 rows of 3584 1025 -> 1018 us, 2000 of 2048 3137 -> 3099).
constexpr int kFewBlocks = 8;
struct OpenArgs {
  const uint16_t* H;
  const uint16_t* W;
  int d, V;
  const int32_t* rowsel;
  int64_t n_sel;
  const int32_t* ids;
  const float* adv;
  int nblk;
  int32_t* blk_live;
  int32_t* flags;
  float* cref;
  uint32_t* dH;          // n_rows * d bf16 as words
  int64_t dh_words;
  float* logp_new;       // NULL: nothing to clear
  int64_t n_rows;
  int pack;              // few blocks: nblk is 1, the blocks are live.nblk
  LiveArgs live;
};
// ------------------------------------------------------------------ bf16: row references and row factors of the keeping pass
__global__ void __launch_bounds__(256)
k_update_open(OpenArgs A) {
  if (A.pack && blockIdx.x == 0) {
    float adv[kFewBlocks];
#pragma unroll
    for (int b = 0; b < kFewBlocks; ++b) {
      const int64_t n = b * 256 + threadIdx.x;
      adv[b] = n < A.n_sel ? A.adv[A.rowsel ? A.rowsel[n] : n] : 0.f;
    }
    int live = 0;
#pragma unroll
    for (int b = 0; b < kFewBlocks; ++b) {
      const int any = __syncthreads_or(adv[b] != 0.f);
      if (static_cast<int>(threadIdx.x) == b && b < A.live.nblk) {
        live = any || A.live.all_live;
        A.flags[b] = 0;
      }
    }
    live_scan(A.live, live);
    return;
  }
  if (static_cast<int>(blockIdx.x) < A.nblk) {
    const int64_t n = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    const int live = n < A.n_sel && A.adv[A.rowsel ? A.rowsel[n] : n] != 0.f;
    const int any = __syncthreads_or(live);
    if (threadIdx.x == 0) {
      A.blk_live[blockIdx.x] = any;
      A.flags[blockIdx.x] = 0;
    }
    return;
  }
  const int64_t blk = static_cast<int64_t>(blockIdx.x) - A.nblk, nb = static_cast<int64_t>(gridDim.x) - A.nblk;
  {
    const int64_t n4 = A.dh_words / 4, stride = nb * 256;
    uint4* const p = reinterpret_cast<uint4*>(A.dH);
    if (reinterpret_cast<uintptr_t>(p) % 16 == 0) {
      for (int64_t i = blk * 256 + threadIdx.x; i < n4; i += stride) p[i] = make_uint4(0u, 0u, 0u, 0u);
      for (int64_t i = 4 * n4 + blk * 256 + threadIdx.x; i < A.dh_words; i += stride) A.dH[i] = 0u;
    } else {
      for (int64_t i = blk * 256 + threadIdx.x; i < A.dh_words; i += stride) A.dH[i] = 0u;
    }
    if (A.logp_new)
      for (int64_t i = blk * 256 + threadIdx.x; i < A.n_rows; i += stride) A.logp_new[i] = 0.f;
  }
  // cref[n] = h_n . W[y_n], the taken token's logit (never above the row's logsumexp); NaN for an invalid id.
  // One wavefront per selected row.
  const int lane = threadIdx.x & 63;
  for (int64_t n = blk * 4 + threadIdx.x / kWave; n < A.n_sel; n += nb * 4) {
    const int64_t row = A.rowsel ? A.rowsel[n] : n;
    const int y = A.ids[row];
    if (y < 0 || y >= A.V) {
      if (lane == 0) A.cref[n] = NAN;
      continue;
    }
    const uint4* h = reinterpret_cast<const uint4*>(A.H + row * A.d);
    const uint4* w = reinterpret_cast<const uint4*>(A.W + static_cast<int64_t>(y) * A.d);
    float s = 0.f;
    for (int k = lane; k < A.d / 8; k += kWave) {
      float a[8], b[8];
      bf16x8_to_f32(h[k], a);
      bf16x8_to_f32(w[k], b);
#pragma unroll
      for (int j = 0; j < 8; ++j) s = fmaf(a[j], b[j], s);
    }
    s = wave_sum(s);
    if (lane == 0) A.cref[n] = s;
  }
}
// Row factor sc[n] = a_n exp(c_n - lse_n) of dz = sc E, and Hs[n - c0, :] = bf16(sc[n] h_n), the operand dW reads, in
// column blocks [d / 256][mcp][256].
// Rows of a flagged block get factor 1: their dz comes complete from the recomputing kernel.  The entry of the
// taken token is cleared in the [rows, V] operand (see k_ppo_rows).
struct KeptRows {
  const uint16_t* H;
  int d, V;
  uint16_t* E;
  int64_t tiles_v;
  const float* cref;
  const int32_t* flags;
  const int32_t* cidx;
  float* sc;
  uint16_t* Hs;
  int64_t mcp;
};
// blk: place of the row's block among the live ones
__device__ __forceinline__ float kept_factor(int blk, int flag, float cref, float a, float lse) {
  if (blk < 0) return 0.f;                                   // a dead block: no row of it has a gradient
  if (flag) return 1.f;
  return a != 0.f ? a * __expf(cref - lse) : 0.f;            // a = 0: invalid id (reference NaN) or no gradient
}
// one wavefront; m: the row's place in the chunk, n: in the selection
__device__ __forceinline__ void kept_row(const KeptRows& K, int64_t m, int64_t n, int blk, int64_t row, int y, float f) {
  const int lane = threadIdx.x & 63;
  if (lane == 0) K.sc[n] = f;
  if (blk < 0) return;
  const int64_t mp = static_cast<int64_t>(blk) * 256 + (m & 255);   // row in the packed operands
  if (lane == 0 && y >= 0 && y < K.V)                        // the taken token's column goes through g_c in float32
    K.E[blk_offset(blk, y >> 8, K.tiles_v) + (m & 255) * 256 + (y & 255)] = 0;
  const uint4* h = reinterpret_cast<const uint4*>(K.H + row * K.d);
  for (int k = lane; k < K.d / 8; k += kWave) {
    uint4* o = reinterpret_cast<uint4*>(K.Hs + (static_cast<int64_t>(k >> 5) * K.mcp + mp) * 256);   // column block k / 32 of the row
    float x[8];
    bf16x8_to_f32(h[k], x);
    uint4 v;
    v.x = pack_bf16x2(x[0] * f, x[1] * f);
    v.y = pack_bf16x2(x[2] * f, x[3] * f);
    v.z = pack_bf16x2(x[4] * f, x[5] * f);
    v.w = pack_bf16x2(x[6] * f, x[7] * f);
    o[k & 31] = v;
  }
}
__global__ void __launch_bounds__(256)
k_keep_rows(KeptRows K, const int32_t* __restrict__ rowsel, int64_t c0, int64_t rows, const int32_t* __restrict__ ids, const float* __restrict__ lse_c,
            const float* __restrict__ a_c) {
  const int64_t m = static_cast<int64_t>(blockIdx.x) * (blockDim.x / kWave) + threadIdx.x / kWave;
  if (m >= rows) return;
  const int64_t n = c0 + m, row = rowsel ? rowsel[n] : n;
  // what the row needs is asked for together (place, flag and reference one after the other: 3738 rows of 2048 11.9 us, like this 11.55)
  const int blk = K.cidx[n >> 8], flag = K.flags[n >> 8];
  const float a = a_c[n], lse = lse_c[n], cref = K.cref[n];
  kept_row(K, m, n, blk, row, ids[row], kept_factor(blk, flag, cref, a, lse));
}
// Few rows (one chunk of up to kFewBlocks blocks): k_score_finalize, k_ppo_rows and k_keep_rows in one launch, eight rows to a workgroup; the statistics are left
// to k_update_close, which goes over the rows once more.  Bound by its chain of loads, as the three were: update of 203 rows of 1096 against 50 001 191.6 and
// 184.5 us, 60 rows of 1024 against 151 936 271 and 266, 500 of 512 against 30 001 138.9 and 126.7, 2000 270.3 and 262.2, 2000 of 2048 against 151 936
// 3218 and 3194, of 3584 against 50 001 1875 and 1868.
struct RowsArgs {
  const float4* partial;
  int tiles_m;
  int64_t n_pad, n_sel;
  Surrogate S;
  float *logp_c, *lse_c, *ent_c, *logp_new, *g_c, *a_c, *kz_c;
  KeptRows K;
};
__global__ void __launch_bounds__(256)
k_rows_few(RowsArgs A) {
  __shared__ float s_f[8];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t n0 = static_cast<int64_t>(blockIdx.x) * 8, n = n0 + (lane & 7);
  Part p;
  float zy;
  if (merge_parts<true>(A.partial, A.tiles_m, A.n_pad, n, n < A.n_sel, p, zy)) {
    const int64_t row = A.S.rowsel ? A.S.rowsel[n] : n;
    const int y = A.S.ids[row];
    const bool ok = y >= 0 && y < A.S.V;
    const float cref = A.K.cref[n];
    const RowScore r = row_score(p, cref, ok);
    const SurrogateRow R = surrogate_row(A.S, row, ok, r.logp, r.entropy);
    const float a = ok ? -R.g : 0.f;
    A.logp_c[n] = r.logp;
    A.lse_c[n] = r.lse;
    A.ent_c[n] = r.entropy;
    if (A.logp_new) A.logp_new[row] = r.logp;
    A.g_c[n] = ok ? R.g * -expm1f(r.logp) : R.g;             // all of dz[n, y] (see k_ppo_rows)
    A.a_c[n] = a;                                            // for the blocks that are computed once more
    A.kz_c[n] = 0.f;
    s_f[lane] = kept_factor(A.K.cidx[n >> 8], A.K.flags[n >> 8], cref, a, r.lse);
  }
  __syncthreads();
#pragma unroll
  for (int k = wave; k < 8; k += 4) {
    if (n0 + k >= A.n_sel) continue;
    const int64_t row = A.S.rowsel ? A.S.rowsel[n0 + k] : n0 + k;
    kept_row(A.K, n0 + k, n0 + k, A.K.cidx[(n0 + k) >> 8], row, A.S.ids[row], s_f[k]);
  }
}

__global__ void __launch_bounds__(Cfg::T)
k_dz_tiles(const uint16_t* __restrict__ W, const uint16_t* __restrict__ H, int d, int V,
           const int32_t* __restrict__ rowsel, int64_t c0, int64_t mc,
           const float* __restrict__ lse_c, const float* __restrict__ a_c, const float* __restrict__ kz_c,
           int tiles_m, int tiles_n, int panel, uint16_t* __restrict__ dZ, int64_t Vp) {
  __shared__ __attribute__((aligned(16))) uint16_t lds[kLogitLds / 2];
  for (int it = 0; it < kTilesPerWg; ++it) {     // a workgroup walks the same place of kTilesPerWg consecutive tile groups
    int tile_m, tile_n;
    if (!tile_coords<kGM, kGN>(tiles_m, tiles_n, panel, &tile_m, &tile_n, it, kTilesPerWg)) continue;
    dz_tile(tile_m, tile_n, W, H, d, V, rowsel, c0, mc, LeaveRows{}, lse_c, a_c, kz_c, dZ, Vp, tile_n, lds);
  }
}
// The same tiles for the blocks of 256 rows that the keeping scoring pass has flagged, and only those: a fixed,
// small grid walks (flagged block, vocabulary tile) pairs, so that the usual case of no flag costs next to nothing.
__global__ void __launch_bounds__(Cfg::T)
k_dz_flagged(const uint16_t* __restrict__ W, const uint16_t* __restrict__ H, int d, int V,
             const int32_t* __restrict__ rowsel, int64_t c0, int64_t mc, const int32_t* __restrict__ ids,
             const float* __restrict__ lse_c, const float* __restrict__ a_c, const float* __restrict__ kz_c,
             int tiles_m, int tiles_n, uint16_t* __restrict__ dZ, int64_t Vp, const int32_t* __restrict__ flags,
             const int32_t* __restrict__ cidx) {
  __shared__ __attribute__((aligned(16))) uint16_t lds[kLogitLds / 2];
  for (int tile_n = 0; tile_n < tiles_n; ++tile_n) {
    const int out_blk = cidx[(c0 >> 8) + tile_n];
    if (!flags[(c0 >> 8) + tile_n] || out_blk < 0) continue;        // the same for every thread of the grid
    for (int tile_m = blockIdx.x; tile_m < tiles_m; tile_m += gridDim.x)
      dz_tile(tile_m, tile_n, W, H, d, V, rowsel, c0, mc, ClearTaken{rowsel, ids}, lse_c, a_c, kz_c, dZ, Vp, out_blk, lds);
  }
}

// dz from the logits that k_score_logits has left, in place: a block of 256 x 256 floats becomes bf16 in its first half (so
// the operand's blocks lie two block lengths apart).  A workgroup turns one block, 32 rows at a time, a row to a wavefront's
// load; a group of rows is written once all wavefronts have what lies there and in front of it in registers, and the
// next one is on its way meanwhile.  Bound by the 6 bytes a logit that are read and written: 16 100 rows against 151 936 in 2.75
// ms (5.3 TB/s).  With the logits stored (1.05 ms more for the scoring pass) instead of computed twice, and so these two in place
// of 7.6 ms of k_dz_tiles, that update takes 27.0 ms in two chunks instead of 30.2; 203 rows of 3584 1.21 instead of 1.43.
constexpr int kTurnRows = 32, kTurnWaves = 4, kRowsPerWave = kTurnRows / kTurnWaves;
__global__ void __launch_bounds__(kTurnWaves * kWave)
k_dz_from_logits(float* Z, int tiles_v, int64_t c0, int64_t mc, const float* __restrict__ lse_c, const float* __restrict__ a_c,
                 const float* __restrict__ kz_c) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t n0 = static_cast<int64_t>(blockIdx.x / tiles_v) * 256;     // chunk-relative
  float* const blk = Z + static_cast<int64_t>(blockIdx.x) * kBlkElems;
  uint16_t* const out = reinterpret_cast<uint16_t*>(blk);
  floatx4 z[2][kRowsPerWave];
  auto fetch = [&](int g, floatx4 (&x)[kRowsPerWave]) {
#pragma unroll
    for (int r = 0; r < kRowsPerWave; ++r) {
      const int row = g * kTurnRows + wave * kRowsPerWave + r;
      x[r] = floatx4{0.f, 0.f, 0.f, 0.f};
      if (n0 + row < mc) x[r] = __builtin_nontemporal_load(reinterpret_cast<const floatx4*>(blk + row * 256 + lane * 4));
    }
  };
  fetch(0, z[0]);
#pragma unroll
  for (int g = 0; g < 256 / kTurnRows; ++g) {
    // this group has arrived: its registers are taken as used here, or the loads could sink below the barrier and meet what
    // another wavefront has written there
#pragma unroll
    for (int r = 0; r < kRowsPerWave; ++r) asm volatile("" : "+v"(z[g & 1][r]) : : "memory");
    __syncthreads();
    if (g + 1 < 256 / kTurnRows) fetch(g + 1, z[(g + 1) & 1]);
#pragma unroll
    for (int r = 0; r < kRowsPerWave; ++r) {
      const int row = g * kTurnRows + wave * kRowsPerWave + r;
      float l2 = 1e30f, a = 0.f, kz = 0.f;                                 // rows past the chunk: 0
      if (n0 + row < mc) {
        l2 = lse_c[c0 + n0 + row] * 1.44269504088896341f;
        a = a_c[c0 + n0 + row];
        kz = kz_c[c0 + n0 + row];
      }
      float dz[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float x = z[g & 1][r][k];
        dz[k] = __builtin_amdgcn_exp2f(fmaf(x, 1.44269504088896341f, -l2)) * fmaf(kz, x, a);
      }
      *reinterpret_cast<uint2*>(out + row * 256 + lane * 4) = make_uint2(pack_bf16x2(dz[0], dz[1]), pack_bf16x2(dz[2], dz[3]));
    }
  }
}

// What the gradient products need besides dZ: the taken token's entry of every row is cleared (that column goes through
// g_c in float32, see k_ppo_rows), and the row of H goes to the operand that dW reads, in the column blocks of k_keep_rows.
// One wavefront per row.  (dW reading the rows through the selection: two kinds of loads in flight, whose waits have to be
// for all of them, 16 100 rows of 2048: both products 16.3 ms, with the copy, 25 us, 14.9.)
__global__ void __launch_bounds__(256)
k_dz_rows(const uint16_t* __restrict__ H, int d, int V, const int32_t* __restrict__ rowsel, int64_t c0, int64_t rows,
          const int32_t* __restrict__ ids, uint16_t* __restrict__ dZ, int64_t tiles_v, int blk_pitch, uint16_t* __restrict__ Hs, int64_t mcp) {
  const int lane = threadIdx.x & 63;
  const int64_t m = static_cast<int64_t>(blockIdx.x) * (blockDim.x / kWave) + threadIdx.x / kWave;
  if (m >= rows) return;
  const int64_t row = rowsel ? rowsel[c0 + m] : c0 + m;
  const int y = ids[row];
  if (lane == 0 && y >= 0 && y < V) dZ[blk_offset(m >> 8, y >> 8, tiles_v) * blk_pitch + (m & 255) * 256 + (y & 255)] = 0;
  const uint4* h = reinterpret_cast<const uint4*>(H + row * d);
  for (int k = lane; k < d / 8; k += kWave) reinterpret_cast<uint4*>(Hs + (static_cast<int64_t>(k >> 5) * mcp + m) * 256)[k & 31] = h[k];
}

// (the bodies and what bounds them: umas_gradients.h)
__global__ void __launch_bounds__(ShortCfg::T, 2)
k_dw_short(const uint16_t* __restrict__ dZ, int blk_pitch, int64_t Vp, int64_t mcp, const uint16_t* __restrict__ Hs, int d, int V, int tiles_v,
           int tiles_n, const LiveInfo* __restrict__ info, float* __restrict__ dW, int accumulate) {
  __shared__ __attribute__((aligned(16))) char lds[kShortLds];
  dw_short<float>(dZ, blk_pitch, Vp, mcp, Hs, d, V, tiles_v, tiles_n, info, dW, accumulate, lds);
}
__global__ void __launch_bounds__(Cfg::T)
k_gemm_dh_dw(const uint16_t* __restrict__ dZ, int blk_pitch, int64_t Vp, int64_t mcp, const uint16_t* __restrict__ W,
             const uint16_t* __restrict__ Hs, int d, int V, int tiles_v,
             int tiles_d, DhSlices sl, int tiles_r, LiveInfo* __restrict__ info, const int32_t* __restrict__ blk_orig,
             uint16_t* __restrict__ dH, float* __restrict__ dW, int accumulate, const int32_t* __restrict__ rowsel,
             int64_t c0, int64_t rows, const int32_t* __restrict__ ids, const float* __restrict__ g_c,
             const float* __restrict__ sc) {
  __shared__ __attribute__((aligned(16))) uint16_t lds[MixedLdsBytes<Cfg>::value / 2];
  gemm_dh_dw<true, float>(dZ, blk_pitch, Vp, mcp, W, Hs, d, V, tiles_v, tiles_d, sl, tiles_r, info, blk_orig, dH, dW, accumulate, rowsel, c0, rows, ids, g_c, sc, lds);
}

// One-hot part of dW: dW[y_n, :] += g_n h_n for every selected row, in float32.  Rows that took the same token add
// into the same dW row, hence atomics - and token frequencies are skewed (a seventh of the rows of a Zipf(1.1) batch
// took the most frequent token), so adding row by row queues thousands of atomics on the same cache lines.  A
// workgroup therefore takes kOneHotRows consecutive selected rows and adds them up by token first: the first row of
// every token in the group is its leader; a wavefront sums the leader and its followers in registers, 2048 columns at
// a time (16-byte loads, a lane owning eight consecutive columns of each of four pieces), turns every piece through
// its corner of LDS so that consecutive lanes hold consecutive columns, and issues one atomic per element of the sum.
// A wavefront needs about a microsecond per token, so with few groups each is worked on by several workgroups; and the
// most frequent token's rows are a chain of loads, so they come four at a time (203 rows of 3584 37 -> 27 us, 725 of 2048 27 -> 20).
constexpr int kOneHotRows = 128;
constexpr int kOneHotPieces = 4;                    // pieces of 512 columns a wavefront holds at a time
constexpr int kOneHotAhead = 4;                     // rows a wavefront loads together
static_assert(kOneHotRows == 2 * kWave, "the rows of a token are two ballots");
__device__ __forceinline__ void
dw_onehot(int group, int part, int parts, const uint16_t* __restrict__ H, int d, const int32_t* __restrict__ rowsel, int64_t n_sel,
          const int32_t* __restrict__ ids, const float* __restrict__ g_c, float* __restrict__ dW) {
  __shared__ __attribute__((aligned(16))) int32_t s_id[kOneHotRows];   // token of the row, -1 when the row adds nothing
  __shared__ float s_g[kOneHotRows];
  __shared__ int64_t s_row[kOneHotRows];
  __shared__ int32_t s_leader[kOneHotRows];         // the group's leaders, compacted
  __shared__ int32_t s_n_leader[kOneHotRows / kWave];
  __shared__ float s_turn[256 / kWave][8 * kWave];  // one piece per wavefront, in column order
  const int tid = threadIdx.x, lane = tid & 63, wave = tid / kWave;
  if (tid < kOneHotRows) {
    const int64_t n = static_cast<int64_t>(group) * kOneHotRows + tid;
    float g = 0.f;
    int64_t row = 0;
    int32_t id = -1;
    if (n < n_sel) {
      g = g_c[n];                                  // 0: clipped rows, zero advantage, invalid ids
      row = rowsel ? rowsel[n] : n;
      if (g != 0.f) id = ids[row];
    }
    s_id[tid] = id; s_g[tid] = g; s_row[tid] = row;
  }
  __syncthreads();
  bool leader = false;
  if (tid < kOneHotRows) {
    const int32_t id = s_id[tid];
    int earlier = 0;                                // rows of the group in front of this one with its token
#pragma unroll 8
    for (int u = 0; u < kOneHotRows; u += 4) {
      const int4 o = *reinterpret_cast<const int4*>(s_id + u);
      earlier += (o.x == id && u < tid) + (o.y == id && u + 1 < tid) + (o.z == id && u + 2 < tid) + (o.w == id && u + 3 < tid);
    }
    leader = id >= 0 && earlier == 0;
  }
  const unsigned long long leaders = __ballot(leader);       // listed in row order: every workgroup of the group has the same list
  if (lane == 0 && wave < kOneHotRows / kWave) s_n_leader[wave] = __popcll(leaders);
  __syncthreads();
  int n_leader = 0, before = 0;
#pragma unroll
  for (int k = 0; k < kOneHotRows / kWave; ++k) { before += k < wave ? s_n_leader[k] : 0; n_leader += s_n_leader[k]; }
  if (leader) s_leader[before + __popcll(leaders & ((1ull << lane) - 1))] = tid;
  __syncthreads();
  float* turn = s_turn[wave];
  // the group's tokens are spread over the wavefronts of `parts` workgroups
  for (int li = wave + part * (256 / kWave); li < n_leader; li += 256 / kWave * parts) {
    const int32_t id = s_id[s_leader[li]];
    float* dst = dW + static_cast<int64_t>(id) * d;
    unsigned long long same[kOneHotRows / kWave];   // the rows of the group that took this token
#pragma unroll
    for (int k = 0; k < kOneHotRows / kWave; ++k) same[k] = __ballot(s_id[lane + kWave * k] == id);
    for (int c0 = 0; c0 < d; c0 += kOneHotPieces * 8 * kWave) {   // d is a multiple of 8: a lane's eight columns are all inside or all outside
      float acc[kOneHotPieces][8];
#pragma unroll
      for (int q = 0; q < kOneHotPieces; ++q)
#pragma unroll
        for (int k = 0; k < 8; ++k) acc[q][k] = 0.f;
      unsigned long long lo = same[0], hi = same[1];
      while (lo | hi) {                               // kOneHotAhead rows are in flight together
        uint4 hv[kOneHotAhead][kOneHotPieces];
        float g[kOneHotAhead];
#pragma unroll
        for (int b = 0; b < kOneHotAhead; ++b) {
          g[b] = 0.f;
          if (!(lo | hi)) {
#pragma unroll
            for (int q = 0; q < kOneHotPieces; ++q) hv[b][q] = make_uint4(0u, 0u, 0u, 0u);
            continue;
          }
          const int u = lo ? __ffsll(static_cast<long long>(lo)) - 1 : kWave + __ffsll(static_cast<long long>(hi)) - 1;
          if (lo) lo &= lo - 1; else hi &= hi - 1;
          const uint16_t* h = H + s_row[u] * d;
          g[b] = s_g[u];
#pragma unroll
          for (int q = 0; q < kOneHotPieces; ++q) {
            const int c = c0 + (q * kWave + lane) * 8;
            hv[b][q] = c < d ? *reinterpret_cast<const uint4*>(h + c) : make_uint4(0u, 0u, 0u, 0u);
          }
        }
#pragma unroll
        for (int b = 0; b < kOneHotAhead; ++b)
#pragma unroll
          for (int q = 0; q < kOneHotPieces; ++q) {
            const uint32_t w4[4] = {hv[b][q].x, hv[b][q].y, hv[b][q].z, hv[b][q].w};
#pragma unroll
            for (int k2 = 0; k2 < 4; ++k2) {
              acc[q][2 * k2] += g[b] * bf2f(static_cast<uint16_t>(w4[k2] & 0xFFFFu));
              acc[q][2 * k2 + 1] += g[b] * bf2f(static_cast<uint16_t>(w4[k2] >> 16));
            }
          }
      }
#pragma unroll
      for (int q = 0; q < kOneHotPieces; ++q) {
        const int cq = c0 + q * 8 * kWave;           // first column of the piece
        if (cq >= d) break;
        // column cq + 8 lane + k sits in this lane's acc[q][k]; after the turn, lane l adds columns cq + 64 k + l
        *reinterpret_cast<float4*>(turn + 8 * lane) = make_float4(acc[q][0], acc[q][1], acc[q][2], acc[q][3]);
        *reinterpret_cast<float4*>(turn + 8 * lane + 4) = make_float4(acc[q][4], acc[q][5], acc[q][6], acc[q][7]);
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int c = cq + kWave * k + lane;
          if (c < d) unsafeAtomicAdd(dst + c, turn[kWave * k + lane]);
        }
        __builtin_amdgcn_wave_barrier();
      }
    }
  }
}

// What is left of an update when its products are there, in one launch, as none of it needs the other: the one-hot part of dW,
// the statistics, and the sum of the slices of dH.  The longest first: it is chains of loads, which the sum's bytes hide behind.
// 203 rows of 3584 against 152 064: launches of 18 to 23, 5 and 12 us, in one 24 to 27.
struct CloseArgs {
  unsigned onehot_groups, onehot_parts;   // workgroups of dw_onehot; 0: none
  const uint16_t* H;
  int d;
  const int32_t* rowsel;
  int64_t n_sel;
  const int32_t* ids;
  const float* g_c;
  float* dW;
  unsigned n_stats;                       // workgroups of ppo_stats; 0: none
  int nblk, n_roles;
  float entropy_coef;
  int64_t norm_rows;
  const double* blk_stats;                // NULL: from the rows
  Surrogate S;
  const float *logp_c, *ent_c;
  umas_loss_stats* stats;
  unsigned reduce_rows, reduce_pieces;    // workgroups of dh_reduce; 0: none
  DhSlices sl;
  int tiles_r, tiles_d;
  const uint16_t* W;
  const LiveInfo* info;
  const int32_t* blk_orig;
  uint16_t* dH;
  int64_t c0, rows;
  const float* sc;
};
__global__ void __launch_bounds__(256)
k_update_close(CloseArgs A) {
  unsigned i = blockIdx.x;
  if (i < A.onehot_groups * A.onehot_parts) {
    dw_onehot(i % A.onehot_groups, i / A.onehot_groups, A.onehot_parts, A.H, A.d, A.rowsel, A.n_sel, A.ids, A.g_c, A.dW);
    return;
  }
  i -= A.onehot_groups * A.onehot_parts;
  if (i < A.n_stats) {
    if (A.blk_stats) ppo_stats(i, A.nblk, A.n_roles, A.entropy_coef, A.norm_rows, A.blk_stats, A.stats);
    else ppo_stats_by_row(i, A.S, A.n_sel, A.entropy_coef, A.norm_rows, A.logp_c, A.ent_c, A.stats);
    return;
  }
  i -= A.n_stats;
  dh_reduce<true>(i % A.reduce_rows, i / A.reduce_rows, A.sl, A.tiles_r, A.tiles_d, A.W, A.d, A.info, A.blk_orig, A.dH, A.rowsel, A.c0, A.rows,
            A.ids, A.g_c, A.sc);
}

// ------------------------------------------------------------------ host side
struct ScoreWs {
  float4* partial;   // [tiles_m][n_pad]
  float* logp_c;
  float* lse_c;
  float* ent_c;
};
size_t carve_score(Carver& c, ScoreWs& w, int64_t n_sel, int V, umas_dtype dt, bool compact) {
  const int64_t n_pad = round_up(n_sel > 0 ? n_sel : 1, Cfg::BN);
  const int64_t tiles_m = (V + Cfg::BM - 1) / Cfg::BM;
  w.partial = dt == UMAS_BF16 ? c.take<float4>(static_cast<size_t>(tiles_m) * n_pad) : nullptr;
  w.logp_c = w.lse_c = w.ent_c = nullptr;
  if (compact) {
    w.logp_c = c.take<float>(n_pad);
    w.lse_c = c.take<float>(n_pad);
    w.ent_c = c.take<float>(n_pad);
  }
  return c.off;
}

struct PpoWs {
  ScoreWs score;
  float* g_c;
  float* a_c;        // per selected row: coefficients of the backward's dense part
  float* kz_c;
  float* cref;       // keeping pass: per selected row, the reference of E and the row factor of dz = sc E
  float* sc;
  double* rest;      // float32 path, in place of these two: sum of the probabilities of the tokens not taken
  int32_t* flags;    // keeping pass: blocks of 256 selected rows whose dz must be recomputed
  int32_t* blk_live; // per block of 256 selected rows: some row has a gradient
  int32_t* blk_cidx; // its place among the live blocks of its chunk, -1 for a dead one
  int32_t* blk_orig; // per chunk: live block -> block of the chunk
  LiveInfo* live;    // of the chunk in work
  double* blk_stats;
  char* chunk;       // rest of the workspace: dZ (or E) [mcp, Vp], then the scaled copy of the chunk's rows of H
  size_t fixed_bytes;
};
// The float32 update keeps the logits (float64) of all its rows where that is no more than 1 GiB.  Storing and reading them costs the same
// at every hidden size, a second product costs by it: below 64 columns up to 128 MiB, which the memory-side cache holds together with
// dz, below 32 up to 32 MiB.  Update on new rows, computed twice / kept: 500 rows of 8 against 8000 (30 MiB) 179 / 180 us, 2000 (122) 278 /
// 298, 4000 of 16 against 4000 262 / 279, 1843 of 33 against 8001 359 / 346, 1000 of 40 against 16 000 446 / 458 (on the rows of the call
// before 448 / 427), 2500 of 32 against 8000 (153) 353 / 363, 300 of 64 against 40 000 790 / 789; on the rows of the call before, 12 000
// against 8000, d = 16 1121 / 1277, 32 1310 / 1404, 48 1517 / 1543, 64 1694 / 1639, 40 000 against 1000 d = 32 1384 / 1434, 64
// 1499 / 1513, 96 1727 / 1703.
size_t f32_logit_bytes(int64_t n_sel, int d, int V) {
  const double b = static_cast<double>(n_sel) * V * sizeof(double), most = d < 32 ? 33554432.0 : d < 64 ? 134217728.0 : 1073741824.0;
  return b <= most ? align_up(static_cast<size_t>(n_sel) * V * sizeof(double)) : 0;
}
// ... and, behind them, the statistics of parts of the rows that the update in few launches merges where it makes dz (one chunk of rows).
size_t f32_part_bytes(int64_t n_sel, int V) { return align_up(static_cast<size_t>(f32::part_plan(n_sel, V).splits) * n_sel * sizeof(f32::Stat)); }
bool f32_few_launches(int64_t n_sel, int d, int V, size_t room) {
  const size_t z = n_sel <= kF32ChunkRows ? f32_logit_bytes(n_sel, d, V) : 0;
  return z > 0 && chunk_bytes(n_sel, d, V, UMAS_F32) + z + f32_part_bytes(n_sel, V) <= room;
}
// The update with an entropy bonus keeps the logits of a chunk in float32 instead of computing them a second time where the
// workspace has room for chunks that are not small: the whole selection, or chunks whose dH tiles are whole ones (the same bits
// of dH as from larger workspaces).  0: it has not, the logits are computed twice.
// So they are for hidden sizes below kLogitWidth: a second product costs by the hidden size, the 10 bytes a logit that are stored and
// read more do not.  Update, computed twice / kept, 203, 700 and 3000 rows against 151 937: d = 256 211 / 220, 391 / 465, 1282 / 1622 us;
// 512 288 / 282, 578 / 613, 1985 / 2067; 640 355 / 336, 714 / 738, 2414 / 2459; 768 383 / 356, 765 / 763, 2610 / 2579; 896 452 / 386,
// 924 / 880, 3166 / 3011.
constexpr int kLogitWidth = 768;
// What the workspace is sized for.  A second chunk adds to dW, 0.3 to 0.5 ms at any size: in one and two chunks 8300 rows of 2048 14.15 and 14.43 ms,
// 10 590 (6 GiB) 17.77 and 18.16, 16 100 26.4 and 26.9, 24 000 39.4 and 39.7, 10 500 of 3584 28.9 and 29.3.  Beyond 6 GiB it is 2 % or less, which
// is not worth twice the memory.
constexpr size_t kLogitBytes = size_t{6} << 30;
int64_t logit_chunk_rows(int64_t n_sel, int d, int V, size_t room) {
  if (d < kLogitWidth) return 0;
  if (round_up(V, 256) / 256 > 8192) return 0;             // 32-bit offsets along a row of blocks
  if (dh_tiles(n_sel, d) < kDhSliceTiles) return logit_chunk_bytes(n_sel, d, V) + full_part_bytes(n_sel, n_sel, d, V) <= room ? n_sel : 0;
  const int64_t fit = std::min(static_cast<int64_t>(room / logit_chunk_bytes(256, d, V)) * 256, kMaxChunkRows);
  if (fit >= n_sel) return n_sel;
  if (fit == 0) return 0;
  const int64_t nchunk = (n_sel + fit - 1) / fit, mc = round_up((n_sel + nchunk - 1) / nchunk, 256);
  return dh_tiles(mc, d) >= kDhSliceTiles / 2 ? mc : 0;
}
size_t carve_ppo(Carver& c, PpoWs& w, int64_t n_sel, int d, int V, umas_dtype dt, int n_roles) {
  (void)d;                                      // the per-chunk buffers depend on d, the fixed part does not
  carve_score(c, w.score, n_sel, V, dt, true);
  const int64_t n_pad = round_up(n_sel > 0 ? n_sel : 1, Cfg::BN);
  w.g_c = c.take<float>(n_pad);
  w.a_c = c.take<float>(n_pad);
  w.kz_c = c.take<float>(n_pad);
  w.cref = w.sc = nullptr;
  w.rest = nullptr;
  if (dt == UMAS_F32) {
    w.rest = c.take<double>(n_pad);
  } else {
    w.cref = c.take<float>(n_pad);
    w.sc = c.take<float>(n_pad);
  }
  w.flags = c.take<int32_t>(static_cast<size_t>(cdiv(n_pad, kRowBlock)));
  w.blk_live = c.take<int32_t>(static_cast<size_t>(cdiv(n_pad, kRowBlock)));
  w.blk_cidx = c.take<int32_t>(static_cast<size_t>(cdiv(n_pad, kRowBlock)));
  w.blk_orig = c.take<int32_t>(static_cast<size_t>(cdiv(n_pad, kRowBlock)));
  w.live = c.take<LiveInfo>(1);
  w.blk_stats = c.take<double>(static_cast<size_t>(cdiv(n_pad, kRowBlock)) * (1 + n_roles) * kStat);
  w.chunk = c.base ? c.base + c.off : nullptr;
  w.fixed_bytes = c.off;
  return c.off;
}

// Four workgroups per compute unit, at most one wavefront per row: 203 rows of 3584 145 -> 29 us, 725 rows of 2048 88 ->
// 25 us, 39 000 rows (307 groups, three workgroups each) 203 -> 195 us; twice and four times as many are no faster.
dim3 onehot_grid(int64_t n_sel) {
  const unsigned groups = cdiv(n_sel, kOneHotRows);
  return dim3(groups, std::min(std::max(1024 / groups, 1u), static_cast<unsigned>(kOneHotRows / 4)));
}
template <int PPW, class... Args>
void launch_score_few_ppw(int ni, unsigned grid, hipStream_t st, Args... args) {
  if constexpr (PPW <= 4)
    if (ni > 2) { hipLaunchKernelGGL((k_score_few<4, PPW>), dim3(grid), dim3(kFewT), 0, st, args...); return; }
  if (ni <= 1) hipLaunchKernelGGL((k_score_few<1, PPW>), dim3(grid), dim3(kFewT), 0, st, args...);
  else hipLaunchKernelGGL((k_score_few<2, PPW>), dim3(grid), dim3(kFewT), 0, st, args...);
}
template <class... Args>
void launch_score_few(int ppw, Args... args) {
  switch (ppw) {
    case 1: return launch_score_few_ppw<1>(args...);
    case 2: return launch_score_few_ppw<2>(args...);
    case 3: return launch_score_few_ppw<3>(args...);
    case 4: return launch_score_few_ppw<4>(args...);
    case 5: return launch_score_few_ppw<5>(args...);
    case 6: return launch_score_few_ppw<6>(args...);
    case 7: return launch_score_few_ppw<7>(args...);
    default: return launch_score_few_ppw<8>(args...);
  }
}

// decided by the rows of the call, not of the chunk: a row's result does not depend on how the rows are chunked
template <class... Args>
void launch_finalize(int64_t rows, int64_t n_sel, hipStream_t st, Args... args) {
  if (n_sel < kFinSplitRows) hipLaunchKernelGGL(k_score_finalize<true>, dim3(cdiv(rows, 8)), dim3(256), 0, st, args...);
  else hipLaunchKernelGGL(k_score_finalize<false>, dim3(cdiv(rows, 32)), dim3(256), 0, st, args...);
}

// Forward scoring of the selected rows into compact arrays and/or scattered outputs.  float32: `room` holds statistics of
// parts of the vocabulary (no room: one workgroup per 32 rows walks all of it), rest_c goes with the compact arrays, z (may be
// NULL) takes the logits.
umas_status run_score(const void* H, const void* W, umas_dtype dt, int d, int V, const int32_t* ids,
                      const int32_t* rowsel, int64_t n_sel, const ScoreWs& w, void* room, size_t room_bytes, double* z, double* rest_c,
                      float* logp, float* lse, float* entropy, hipStream_t st) {
  if (n_sel == 0) return UMAS_OK;
  if (dt == UMAS_BF16) {
    int tiles_m = (V + Cfg::BM - 1) / Cfg::BM;
    const int tiles_n = static_cast<int>((n_sel + Cfg::BN - 1) / Cfg::BN);
    int64_t n_pad = round_up(n_sel, Cfg::BN);
    if (n_sel <= few_rows(d)) {
      // partials [workgroups][rows rounded to 16]: no more than the tiles' [V / 256][rows rounded to 256]
      const int ni = n_sel <= 16 ? 1 : n_sel <= 32 ? 2 : 4;
      n_pad = ni * 16;
      tiles_m = std::min(std::min(device_cus(), tiles_m * static_cast<int>(Cfg::BN / n_pad)), static_cast<int>(cdiv(V, 16)));
      launch_score_few(few_pieces(d), ni, tiles_m, st, static_cast<const uint16_t*>(W), static_cast<const uint16_t*>(H), d, V, rowsel,
                       static_cast<int>(n_sel), ids, w.partial, static_cast<int>(n_pad));
      UMAS_LAUNCHED("k_score_few");
    } else if (n_sel <= NarrowCfg::BN) {                     // ceil(V / 128) 128 <= ceil(V / 256) 256: the partials fit as well
      n_pad = NarrowCfg::BN;
      tiles_m = (V + NarrowCfg::BM - 1) / NarrowCfg::BM;
      hipLaunchKernelGGL(k_score_narrow, dim3(tile_grid<kGM, kGN>(tiles_m, 1, kGN, kTilesPerWg)), dim3(NarrowCfg::T), 0, st,
                         static_cast<const uint16_t*>(W), static_cast<const uint16_t*>(H), d, V, rowsel, n_sel, ids,
                         tiles_m, 1, kGN, w.partial, n_pad);
      UMAS_LAUNCHED("k_score_narrow");
    } else {
      const int panel = row_panel(tiles_n, d), halved = halved_tiles(tiles_m, tiles_n);
      hipLaunchKernelGGL(k_score_tiles, score_grid(tiles_m, tiles_n, panel, halved), dim3(Cfg::T), 0, st, static_cast<const uint16_t*>(W),
                         static_cast<const uint16_t*>(H), d, V, rowsel, n_sel, ids, tiles_m, tiles_n, panel, halved, w.partial, n_pad);
      UMAS_LAUNCHED("k_score_tiles");
    }
    launch_finalize(n_sel, n_sel, st, w.partial, tiles_m, n_pad, static_cast<int64_t>(0), n_sel, static_cast<const float*>(nullptr), rowsel, ids, V,
                    w.logp_c, w.lse_c, w.ent_c, logp, lse, entropy);
    UMAS_LAUNCHED("k_score_finalize");
  } else {
    return f32::score(static_cast<const float*>(W), static_cast<const float*>(H), d, V, rowsel, n_sel, ids, room, room_bytes,
                      f32::ScoreOut{z, rest_c, w.logp_c, w.lse_c, w.ent_c, logp, lse, entropy}, st);
  }
  return UMAS_OK;
}

}  // namespace
}  // namespace umas

using namespace umas;

extern "C" size_t umas_policy_logprobs_workspace_bytes(int64_t n_sel, int32_t d, int32_t V, umas_dtype dtype) {
  (void)d;
  if (n_sel < 0 || V < 1) return 0;
  Carver c(nullptr);
  ScoreWs w;
  const size_t b = carve_score(c, w, n_sel, V, dtype, false) + (dtype == UMAS_F32 ? align_up(f32::score_room(n_sel, V)) : 0);
  return b > 0 ? b : kAlign;
}

extern "C" umas_status umas_policy_logprobs(const void* H, const void* W, umas_dtype dtype, int64_t n_rows, int32_t d,
                                            int32_t V, const int32_t* ids, const int32_t* rowsel, int64_t n_sel,
                                            float* logp, float* lse, float* entropy, void* workspace,
                                            size_t workspace_bytes, void* hip_stream) {
  umas_status s = check_model_args(H, W, dtype, n_rows, d, V, ids, rowsel, n_sel);
  if (s != UMAS_OK) return s;
  UMAS_REQUIRE((logp && lse) || n_rows == 0, UMAS_EINVAL, "logp and lse must not be NULL");
  UMAS_REQUIRE(n_sel < (1LL << 31), UMAS_ESHAPE, "at most 2^31-1 selected rows");
  // float32 scores without any room as well
  s = check_ws(workspace, workspace_bytes, dtype == UMAS_F32 ? kAlign : umas_policy_logprobs_workspace_bytes(n_sel, d, V, dtype));
  if (s != UMAS_OK) return s;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  prof_mark(st);
  if (rowsel && n_rows > 0) {
    const size_t bytes = n_rows * sizeof(float);
    UMAS_HIP(clear_bytes(st, logp, bytes, lse, bytes, entropy, bytes));
  }
  Carver c(workspace);
  ScoreWs w;
  carve_score(c, w, n_sel, V, dtype, false);
  return run_score(H, W, dtype, d, V, ids, rowsel, n_sel, w, workspace, workspace_bytes, nullptr, nullptr, logp, lse, entropy, st);
}

// ------------------------------------------------------------------ scoring without any allocation
// The per-tile partials of the scoring pass live in a file-scope device array in place of a caller's workspace.
// Every GPU holds its own copy of the array at its own address, resolved once per device; host code only ever
// uses that resolved address.  Nothing in it has to start at zero: the tile kernel writes every partial that the
// merge kernel reads.
static __device__ __align__(256) unsigned char scratch[UMAS_STATIC_SCRATCH_BYTES];

namespace {
constexpr int kMaxDevices = 64;
std::mutex g_scratch_mutex;
void* g_scratch_ptr[kMaxDevices];   // per device: address of `scratch` there, NULL until first used

umas_status static_scratch(void** out) {
  int dev = -1;
  UMAS_HIP(hipGetDevice(&dev));
  UMAS_REQUIRE(dev >= 0 && dev < kMaxDevices, UMAS_ESHAPE, "device %d outside [0,%d)", dev, kMaxDevices);
  std::lock_guard<std::mutex> lock(g_scratch_mutex);
  if (!g_scratch_ptr[dev]) {
    void* p = nullptr;
    UMAS_HIP(hipGetSymbolAddress(&p, HIP_SYMBOL(scratch)));
    UMAS_REQUIRE(p, UMAS_EHIP, "hipGetSymbolAddress returned no address for the static scratch");
    g_scratch_ptr[dev] = p;
  }
  *out = g_scratch_ptr[dev];
  return UMAS_OK;
}
}  // namespace

extern "C" umas_status umas_policy_logprobs_static(const void* H, const void* W, umas_dtype dtype, int64_t n_rows,
                                                   int32_t d, int32_t V, const int32_t* ids, const int32_t* rowsel,
                                                   int64_t n_sel, float* logp, float* lse, float* entropy,
                                                   void* hip_stream) {
  umas_status s = check_model_args(H, W, dtype, n_rows, d, V, ids, rowsel, n_sel);
  if (s != UMAS_OK) return s;
  UMAS_REQUIRE((logp && lse) || n_rows == 0, UMAS_EINVAL, "logp and lse must not be NULL");
  UMAS_REQUIRE(n_sel < (1LL << 31), UMAS_ESHAPE, "at most 2^31-1 selected rows");
  const size_t need = dtype == UMAS_F32 ? 0 : umas_policy_logprobs_workspace_bytes(n_sel, d, V, dtype);   // float32 uses none
  UMAS_REQUIRE(need <= static_cast<size_t>(UMAS_STATIC_SCRATCH_BYTES), UMAS_EWORKSPACE,
               "%lld selected rows against a vocabulary of %d need %zu bytes of scratch, the static scratch holds %zu: "
               "score fewer rows per call or use umas_policy_logprobs with a workspace",
               static_cast<long long>(n_sel), V, need, static_cast<size_t>(UMAS_STATIC_SCRATCH_BYTES));
  void* ws = nullptr;
  s = static_scratch(&ws);
  if (s != UMAS_OK) return s;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  prof_mark(st);
  if (rowsel && n_rows > 0) {
    const size_t bytes = n_rows * sizeof(float);
    UMAS_HIP(clear_bytes(st, logp, bytes, lse, bytes, entropy, bytes));
  }
  Carver c(ws);
  ScoreWs w;
  carve_score(c, w, n_sel, V, dtype, false);
  return run_score(H, W, dtype, d, V, ids, rowsel, n_sel, w, nullptr, 0, nullptr, nullptr, logp, lse, entropy, st);
}

extern "C" size_t umas_ppo_loss_workspace_bytes_min(int64_t n_sel, int32_t d, int32_t V, umas_dtype dtype,
                                                    int32_t n_roles) {
  if (n_sel < 0 || d < 1 || V < 1 || n_roles < 0) return 0;
  Carver c(nullptr);
  PpoWs w;
  carve_ppo(c, w, n_sel, d, V, dtype, n_roles);
  const int64_t mc = n_sel < 256 ? (n_sel > 0 ? n_sel : 1) : 256;
  return c.off + chunk_bytes(mc, d, V, dtype);
}

namespace {
// The size at which an update runs in the fewest passes; `bonus`: with room for the logits that one with an entropy bonus keeps.
size_t full_ppo_bytes(int64_t n_sel, int d, int V, umas_dtype dtype, int n_roles, bool bonus) {
  if (n_sel < 0 || d < 1 || V < 1 || n_roles < 0) return 0;
  Carver c(nullptr);
  PpoWs w;
  carve_ppo(c, w, n_sel, d, V, dtype, n_roles);
  int64_t mc = n_sel > 0 ? n_sel : 1;
  const int64_t cap = dtype == UMAS_F32 ? kF32ChunkRows : kMaxChunkRows;
  if (mc > cap) {
    const int64_t nchunk = (mc + cap - 1) / cap;
    mc = round_up((mc + nchunk - 1) / nchunk, 256);
  }
  size_t chunk = chunk_bytes(mc, d, V, dtype);
  if (dtype == UMAS_F32) {                                                           // kept with any coefficient
    const size_t z = f32_logit_bytes(n_sel, d, V);
    return c.off + chunk + z + (z > 0 && n_sel <= kF32ChunkRows ? f32_part_bytes(n_sel, V) : 0);
  }
  const size_t parts = full_part_bytes(n_sel, mc, d, V);
  if (bonus) {
    // the logits of the whole selection, of half a chunk where they are many; no room that the call would not keep logits in
    const int64_t rows = mc >= n_sel && logit_chunk_bytes(mc, d, V) <= kLogitBytes ? mc : round_up((mc + 1) / 2, 256);
    const size_t with = std::max(chunk, logit_chunk_bytes(rows, d, V));
    if (logit_chunk_rows(n_sel, d, V, with + parts) > 0) chunk = with;
  }
  return c.off + chunk + parts;
}
}  // namespace

extern "C" size_t umas_ppo_loss_workspace_bytes(int64_t n_sel, int32_t d, int32_t V, umas_dtype dtype, int32_t n_roles) {
  return full_ppo_bytes(n_sel, d, V, dtype, n_roles, false);
}
extern "C" size_t umas_ppo_loss_workspace_bytes_entropy(int64_t n_sel, int32_t d, int32_t V, umas_dtype dtype, int32_t n_roles) {
  return full_ppo_bytes(n_sel, d, V, dtype, n_roles, true);
}

extern "C" umas_status umas_ppo_loss_fwd_bwd(const void* H, const void* W, umas_dtype dtype, int64_t n_rows, int32_t d,
                                             int32_t V, const int32_t* ids, const int32_t* rowsel, int64_t n_sel,
                                             const float* logp_old, const float* adv, const int32_t* tok_role,
                                             int32_t n_roles, float clip_eps, float entropy_coef, float dual_clip,
                                             int32_t accumulate_dW, int64_t norm_rows, const float* logp_ref,
                                             float kl_coef, umas_loss_stats* stats, float* logp_new, void* dH,
                                             float* dW, void* workspace, size_t workspace_bytes, void* hip_stream) {
  umas_status s = check_model_args(H, W, dtype, n_rows, d, V, ids, rowsel, n_sel);
  if (s != UMAS_OK) return s;
  UMAS_REQUIRE((adv && dH) || n_rows == 0, UMAS_EINVAL, "adv and dH must not be NULL");
  UMAS_REQUIRE(stats && dW, UMAS_EINVAL, "stats and dW must not be NULL");
  UMAS_REQUIRE(n_roles >= 0 && n_roles <= UMAS_MAX_ROLES, UMAS_ESHAPE, "n_roles=%d outside [0,%d]", n_roles, UMAS_MAX_ROLES);
  UMAS_REQUIRE(tok_role || n_roles == 0, UMAS_EINVAL, "tok_role is NULL but n_roles > 0");
  UMAS_REQUIRE(clip_eps > 0.f && clip_eps < 1.f, UMAS_EINVAL, "clip_eps=%g outside (0,1)", static_cast<double>(clip_eps));
  UMAS_REQUIRE(entropy_coef >= 0.f, UMAS_EINVAL, "entropy_coef=%g must not be negative", static_cast<double>(entropy_coef));
  UMAS_REQUIRE(dual_clip == 0.f || dual_clip > 1.f, UMAS_EINVAL, "dual_clip=%g must be 0 (off) or larger than 1",
               static_cast<double>(dual_clip));
  UMAS_REQUIRE(n_sel < (1LL << 31), UMAS_ESHAPE, "at most 2^31-1 selected rows");
  UMAS_REQUIRE(norm_rows == 0 || norm_rows >= n_sel, UMAS_EINVAL, "norm_rows=%lld must be 0 or at least n_sel=%lld",
               static_cast<long long>(norm_rows), static_cast<long long>(n_sel));
  UMAS_REQUIRE(kl_coef >= 0.f, UMAS_EINVAL, "kl_coef=%g must not be negative", static_cast<double>(kl_coef));
  UMAS_REQUIRE(kl_coef == 0.f || logp_ref || n_rows == 0, UMAS_EINVAL, "kl_coef > 0 needs logp_ref");
  s = check_ws(workspace, workspace_bytes, umas_ppo_loss_workspace_bytes_min(n_sel, d, V, dtype, n_roles));
  if (s != UMAS_OK) return s;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  prof_mark(st);
  const size_t esz = dtype == UMAS_BF16 ? 2 : 4;
  Carver c(workspace);
  PpoWs w;
  carve_ppo(c, w, n_sel, d, V, dtype, n_roles);

  if (dtype == UMAS_F32 && n_sel > 0 && f32_few_launches(n_sel, d, V, workspace_bytes - w.fixed_bytes)) {
    const int64_t norm = norm_rows > 0 ? norm_rows : n_sel;
    float* const dz = reinterpret_cast<float*>(w.chunk);
    const size_t z_at = chunk_bytes(n_sel, d, V, dtype), parts_at = z_at + f32_logit_bytes(n_sel, d, V);
    const f32::UpdateArgs U{static_cast<const float*>(W), static_cast<const float*>(H), d, n_sel, n_rows,
                            Surrogate{norm, rowsel, ids, V, logp_old, adv, tok_role, n_roles, clip_eps, dual_clip, logp_ref, kl_coef},
                            entropy_coef / static_cast<float>(norm), entropy_coef, norm_rows, w.score.logp_c, w.score.ent_c, logp_new,
                            reinterpret_cast<double*>(w.chunk + z_at), reinterpret_cast<f32::Stat*>(w.chunk + parts_at), dz,
                            static_cast<float*>(dH), dW, accumulate_dW ? 1 : 0, stats};
    return f32::update(U, st);
  }

  // Without an entropy bonus dz is a row factor times the softmax: the scoring pass keeps the numerators
  // and the logits are not computed a second time.
  const bool keep = dtype == UMAS_BF16 && entropy_coef == 0.f && n_sel > 0;
  // rows that are not selected, and (keeping path, see k_update_open) selected rows in blocks without any gradient,
  // are not visited by the backward
  if (!keep && rowsel && n_rows > 0) {
    UMAS_HIP(clear_bytes(st, logp_new, n_rows * sizeof(float), dH, static_cast<size_t>(n_rows) * d * esz));
  }
  if (!accumulate_dW && n_sel == 0) UMAS_HIP(clear_bytes(st, dW, static_cast<size_t>(V) * d * sizeof(float)));

  // chunks of selected rows sized to the workspace
  const size_t room = workspace_bytes - w.fixed_bytes;
  int64_t mc = n_sel > 0 ? n_sel : 1;
  const int64_t cap = dtype == UMAS_F32 ? kF32ChunkRows : kMaxChunkRows;
  if (mc > cap) mc = cap;
  if (mc > 256 && chunk_bytes(mc, d, V, dtype) > room)   // as many blocks of 256 rows as fit: their bytes are multiples of 256
    mc = std::max<int64_t>(static_cast<int64_t>(room / chunk_bytes(256, d, V, dtype)), 1) * 256;
  if (mc > 256) {   // balance the chunks
    const int64_t nchunk = (n_sel + mc - 1) / mc;
    const int64_t even = round_up((n_sel + nchunk - 1) / nchunk, 256);
    if (even < mc) mc = even;
  }
  UMAS_REQUIRE(chunk_bytes(mc < n_sel ? mc : (n_sel > 0 ? n_sel : 1), d, V, dtype) <= room, UMAS_EWORKSPACE,
               "workspace cannot hold one chunk of %lld rows", static_cast<long long>(mc));

  const int nblk = cdiv(n_sel > 0 ? n_sel : 1, kRowBlock);
  const size_t kPpoLds = (kRowBlock / kWave) * (1 + n_roles) * kStat * sizeof(double);
  const int64_t norm = norm_rows > 0 ? norm_rows : n_sel;   // rows the token mean is taken over
  const float k_ent = norm > 0 ? entropy_coef / static_cast<float>(norm) : 0.f;
  const Surrogate S{norm, rowsel, ids, V, logp_old, adv, tok_role, n_roles, clip_eps, dual_clip, logp_ref, kl_coef};
  const int64_t Vp = round_up(V, 256);
  const uint16_t* Wb = static_cast<const uint16_t*>(W);
  const uint16_t* Hb = static_cast<const uint16_t*>(H);

  // both gradient products of the chunk of `rows` rows from c0 on, and what the slices of dH leave; the partial sums lie
  // behind the chunk's operands or, once the scoring pass's own partials have been merged, in their place
  // (true: dW gets a launch of its own)
  auto dh_plan = [&](int64_t rows, size_t used, DhSlices* sl) {
    const size_t behind = room > used ? room - used : 0;
    const size_t front = static_cast<size_t>(reinterpret_cast<char*>(w.score.logp_c) - reinterpret_cast<char*>(w.score.partial));
    const GradPlan p = plan_gradients(n_sel, rows, d, V, slices_dh(n_sel, mc, d) ? std::max(behind, front) : 0);
    *sl = DhSlices{p.dh.slices, p.dh.voc_blks, behind > front ? reinterpret_cast<float*>(w.chunk + used) : reinterpret_cast<float*>(w.score.partial)};
    return p.dw_apart;
  };
  CloseArgs rest{};
  rest.H = Hb;
  rest.W = Wb;
  rest.d = d;
  rest.rowsel = rowsel;
  rest.n_sel = n_sel;
  rest.ids = ids;
  rest.g_c = w.g_c;
  rest.dW = dW;
  rest.n_stats = 1 + n_roles;
  rest.nblk = nblk;
  rest.n_roles = n_roles;
  rest.entropy_coef = entropy_coef;
  rest.norm_rows = norm_rows;
  rest.blk_stats = w.blk_stats;
  rest.S = S;
  rest.logp_c = w.score.logp_c;
  rest.ent_c = w.score.ent_c;
  rest.stats = stats;
  rest.info = w.live;
  rest.blk_orig = w.blk_orig;
  rest.dH = static_cast<uint16_t*>(dH);
  if (dtype == UMAS_BF16 && n_sel > 0) {
    const dim3 grid = onehot_grid(n_sel);
    rest.onehot_groups = grid.x;
    rest.onehot_parts = grid.y;
  }
  auto close = [&](const CloseArgs& C) -> umas_status {
    const unsigned grid = C.onehot_groups * C.onehot_parts + C.n_stats + C.reduce_rows * C.reduce_pieces;
    if (grid == 0) return UMAS_OK;
    hipLaunchKernelGGL(k_update_close, dim3(grid), dim3(256), 0, st, C);
    UMAS_LAUNCHED("k_update_close");
    return UMAS_OK;
  };
  auto gradients = [&](int64_t c0, int64_t rows, const DhSlices& sl, bool dw_apart, const uint16_t* op, int blk_pitch, const uint16_t* Hs, const float* sc) -> umas_status {
    const int64_t mcp = round_up(rows, 256);
    const int tiles_r = static_cast<int>(mcp / 256), tiles_v = static_cast<int>(Vp / 256), tiles_d = (d + 255) / 256;
    const unsigned grid = static_cast<unsigned>(round_up(device_cus(), 8));      // every XCD's sequence needs somebody
    hipLaunchKernelGGL(k_gemm_dh_dw, dim3(grid), dim3(Cfg::T), 0, st, op, blk_pitch, Vp, mcp, Wb, Hs, d, V, tiles_v,
                       tiles_d, sl, tiles_r, w.live, w.blk_orig, static_cast<uint16_t*>(dH), dW, (accumulate_dW || c0 > 0) ? 1 : 0,
                       rowsel, c0, rows, ids, w.g_c, sc);
    UMAS_LAUNCHED("k_gemm_dh_dw");
    if (dw_apart) {
      const int tiles_n = (d + ShortCfg::BN - 1) / ShortCfg::BN;
      hipLaunchKernelGGL(k_dw_short, dim3(static_cast<unsigned>(round_up(static_cast<int64_t>(tiles_v) * tiles_n, 8))), dim3(ShortCfg::T), 0, st, op, blk_pitch,
                         Vp, mcp, Hs, d, V, tiles_v, tiles_n, w.live, dW, (accumulate_dW || c0 > 0) ? 1 : 0);
      UMAS_LAUNCHED("k_dw_short");
    }
    CloseArgs C = rest;                                  // a chunk's slices are added up before the next one's are written
    if (c0 + rows < n_sel) C.onehot_groups = C.n_stats = 0;
    if (sl.n > 1) {
      C.reduce_rows = static_cast<unsigned>(mcp);
      C.reduce_pieces = cdiv(d, 1024);
      C.sl = sl;
      C.tiles_r = tiles_r;
      C.tiles_d = tiles_d;
      C.c0 = c0;
      C.rows = rows;
      C.sc = sc;
    }
    return close(C);
  };

  // With one the logits are kept instead where the workspace allows it.
  const int64_t mc_z = dtype == UMAS_BF16 && !keep && n_sel > 0 ? logit_chunk_rows(n_sel, d, V, room) : 0;
  if (mc_z > 0) mc = mc_z;
  auto ppo_rows = [&](int64_t c0, int64_t c1) -> umas_status {
    hipLaunchKernelGGL(k_ppo_rows, dim3(std::max(cdiv(c1 - c0, kRowBlock), 1u)), dim3(kRowBlock), kPpoLds, st, S, c0, c1, w.score.logp_c,
                       w.score.ent_c, k_ent, dtype == UMAS_BF16 ? 1 : 0, w.score.lse_c, w.g_c, w.a_c, w.kz_c, w.blk_stats);
    UMAS_LAUNCHED("k_ppo_rows");
    return UMAS_OK;
  };

  // float32: the logits lie behind the chunk's dz
  const size_t z_at = dtype == UMAS_F32 ? chunk_bytes(mc, d, V, dtype) : 0;
  double* const z_kept = dtype == UMAS_F32 && f32_logit_bytes(n_sel, d, V) > 0 && z_at + f32_logit_bytes(n_sel, d, V) <= room
                             ? reinterpret_cast<double*>(w.chunk + z_at) : nullptr;
  if (mc_z > 0) {
    // chunk by chunk, further down
  } else if (!keep) {
    // forward scoring and the surrogate
    s = run_score(H, W, dtype, d, V, ids, rowsel, n_sel, w.score, w.chunk, z_kept ? z_at : room, z_kept, w.rest, logp_new, nullptr, nullptr, st);
    if (s != UMAS_OK) return s;
    s = ppo_rows(0, n_sel);
    if (s != UMAS_OK) return s;
  } else {
    const int tiles_v = static_cast<int>(Vp / 256), tiles_d = (d + 255) / 256;
    auto live_args = [&](int64_t c0, int64_t rows, int slices, bool dw_apart) {
      return LiveArgs{static_cast<int>(c0 >> 8), static_cast<int>(round_up(rows, 256) / 256), rows, kl_coef != 0.f ? 1 : 0,   // a KL term gives every row a gradient
                      dw_apart ? 0 : tiles_v, tiles_d, Vp, slices, w.blk_live, w.blk_cidx, w.blk_orig, w.live};
    };
    OpenArgs O{Hb, Wb, d, V, rowsel, n_sel, ids, adv, nblk, w.blk_live, w.flags, w.cref, static_cast<uint32_t*>(dH),
               n_rows * static_cast<int64_t>(d) / 2, rowsel ? logp_new : nullptr, n_rows, 0, {}};
    if (mc >= n_sel && nblk <= kFewBlocks) {
      DhSlices sl;
      const bool dw_apart = dh_plan(n_sel, chunk_bytes(n_sel, d, V, dtype), &sl);
      O.nblk = O.pack = 1;
      O.live = live_args(0, n_sel, sl.n, dw_apart);
    }
    // (the statistics read the old log-probs and the advantages again once the new log-probs are written)
    auto apart = [&](const void* in) {
      const uintptr_t i = reinterpret_cast<uintptr_t>(in), o = reinterpret_cast<uintptr_t>(logp_new), bytes = static_cast<uintptr_t>(n_rows) * 4;
      return !in || !o || i + bytes <= o || o + bytes <= i;
    };
    const bool logp_new_apart = apart(logp_old) && apart(logp_ref) && apart(adv) && apart(tok_role) && apart(ids);
    // a wavefront per row up to 8192 workgroups; at least 1024 for the clearing
    hipLaunchKernelGGL(k_update_open, dim3(O.nblk + std::min<unsigned>(std::max<unsigned>(cdiv(n_sel, 4), 1024), 8192)), dim3(256), 0, st, O);
    UMAS_LAUNCHED("k_update_open");
    const bool narrow = n_sel <= NarrowCfg::BN;              // one chunk of one block
    const int64_t n_pad = round_up(n_sel, narrow ? NarrowCfg::BN : Cfg::BN);
    const int tiles_m = narrow ? static_cast<int>(Vp / NarrowCfg::BM) : tiles_v;   // of the scores: the partials are as large either way
    for (int64_t c0 = 0; c0 < n_sel; c0 += mc) {
      const int64_t rows = n_sel - c0 < mc ? n_sel - c0 : mc;
      const int64_t mcp = round_up(rows, 256);
      const int tiles_r = static_cast<int>(mcp / 256), panel = row_panel(tiles_r, d), halved = halved_tiles(tiles_v, tiles_r);
      uint16_t* E = reinterpret_cast<uint16_t*>(w.chunk);
      uint16_t* Hs = reinterpret_cast<uint16_t*>(w.chunk + align_up(static_cast<size_t>(mcp) * Vp * 2));
      DhSlices sl;
      const bool dw_apart = dh_plan(rows, chunk_bytes(rows, d, V, dtype), &sl);
      if (!O.pack) {
        hipLaunchKernelGGL(k_live_scan, dim3(1), dim3(512), 0, st, live_args(c0, rows, sl.n, dw_apart));
        UMAS_LAUNCHED("k_live_scan");
      }
      if (narrow)
        hipLaunchKernelGGL(k_score_keep_narrow, dim3(tile_grid<kGM, kGN>(tiles_m, 1, kGN, kTilesPerWg)), dim3(NarrowCfg::T), 0, st, Wb, Hb, d, V,
                           rowsel, rows, ids, tiles_m, w.score.partial, n_pad, w.cref, E, Vp, w.flags, w.blk_cidx);
      else
        hipLaunchKernelGGL(k_score_keep_tiles, score_grid(tiles_v, tiles_r, panel, halved), dim3(Cfg::T), 0, st, Wb, Hb, d, V, rowsel, c0, rows, ids,
                           tiles_v, tiles_r, panel, halved, w.score.partial, n_pad, w.cref, E, Vp, w.flags, w.blk_cidx);
      UMAS_LAUNCHED(narrow ? "k_score_keep_narrow" : "k_score_keep_tiles");
      const KeptRows K{Hb, d, V, E, tiles_v, w.cref, w.flags, w.blk_cidx, w.sc, Hs, mcp};
      if (O.pack && logp_new_apart) {
        const RowsArgs A{w.score.partial, tiles_m, n_pad, n_sel, S, w.score.logp_c, w.score.lse_c, w.score.ent_c, logp_new, w.g_c, w.a_c, w.kz_c, K};
        hipLaunchKernelGGL(k_rows_few, dim3(cdiv(n_sel, 8)), dim3(256), 0, st, A);
        UMAS_LAUNCHED("k_rows_few");
        rest.blk_stats = nullptr;
      } else {
        launch_finalize(rows, n_sel, st, w.score.partial, tiles_m, n_pad, c0, c0 + rows, w.cref, rowsel, ids, V, w.score.logp_c, w.score.lse_c,
                        w.score.ent_c, logp_new, static_cast<float*>(nullptr), static_cast<float*>(nullptr));
        UMAS_LAUNCHED("k_score_finalize");
        s = ppo_rows(c0, c0 + rows);
        if (s != UMAS_OK) return s;
        hipLaunchKernelGGL(k_keep_rows, dim3(cdiv(rows, 4)), dim3(256), 0, st, K, rowsel, c0, rows, ids, w.score.lse_c, w.a_c);
        UMAS_LAUNCHED("k_keep_rows");
      }
      // blocks of rows the scoring pass flagged (a logit far above the row's reference) get dz the long way
      hipLaunchKernelGGL(k_dz_flagged, dim3(kFlaggedGrid), dim3(Cfg::T), 0, st, Wb, Hb, d, V, rowsel, c0, rows, ids,
                         w.score.lse_c, w.a_c, w.kz_c, tiles_v, tiles_r, E, Vp, w.flags, w.blk_cidx);
      UMAS_LAUNCHED("k_dz_flagged");
      s = gradients(c0, rows, sl, dw_apart, E, 1, Hs, w.sc);
      if (s != UMAS_OK) return s;
    }
  }
  if (keep) return UMAS_OK;
  if (dtype == UMAS_F32 || n_sel == 0) {
    s = close(rest);                                     // only the statistics
    if (s != UMAS_OK || n_sel == 0) return s;
  }

  if (dtype == UMAS_F32) {
    float* dz = reinterpret_cast<float*>(w.chunk);
    for (int64_t c0 = 0; c0 < n_sel; c0 += mc) {
      const int64_t rows = n_sel - c0 < mc ? n_sel - c0 : mc;
      const float *Wf = static_cast<const float*>(W), *Hf = static_cast<const float*>(H);
      if (z_kept)
        hipLaunchKernelGGL(f32::k_dz_kept_f32, dim3(cdiv(V, 1024), static_cast<unsigned>(rows)), dim3(256), 0, st, z_kept, V, rowsel, c0, ids,
                           w.score.lse_c, w.rest, w.g_c, w.score.ent_c, w.kz_c, dz);
      else
        hipLaunchKernelGGL(f32::k_dz_f32, dim3(cdiv(V, f32::kVocBlock), cdiv(rows, f32::kTile)), dim3(f32::kWaves * kWave), 0, st, Wf, Hf, d, V,
                           rowsel, c0, rows, ids, w.score.lse_c, w.rest, w.g_c, w.score.ent_c, w.kz_c, dz);
      UMAS_LAUNCHED(z_kept ? "k_dz_kept_f32" : "k_dz_f32");
      f32::launch_gradients(f32::GradArgs{dz, Wf, Hf, d, V, rowsel, c0, static_cast<int>(rows), accumulate_dW || c0 > 0 ? 1 : 0,
                                          static_cast<float*>(dH), dW, 0, 0, 0}, f32::StatArgs{}, st);
      UMAS_LAUNCHED("k_dw_f32");                         // both products: one launch to a chunk
    }
    return UMAS_OK;
  }

  for (int64_t c0 = 0; c0 < n_sel; c0 += mc) {
    const int64_t rows = n_sel - c0 < mc ? n_sel - c0 : mc;
    const int64_t mcp = round_up(rows, 256);
    uint16_t* dZ = reinterpret_cast<uint16_t*>(w.chunk);
    const int tiles_v = static_cast<int>(Vp / 256), tiles_r = static_cast<int>(mcp / 256), tiles_d = (d + 255) / 256;
    const int blk_pitch = mc_z > 0 ? 2 : 1, panel = row_panel(tiles_r, d);
    if (mc_z > 0) {
      const int halved = halved_tiles(tiles_v, tiles_r);
      hipLaunchKernelGGL(k_score_logits, score_grid(tiles_v, tiles_r, panel, halved), dim3(Cfg::T), 0, st, Wb, Hb, d, V,
                         rowsel, c0, rows, ids, tiles_v, tiles_r, panel, halved, w.score.partial, round_up(n_sel, Cfg::BN),
                         reinterpret_cast<float*>(w.chunk), Vp);
      UMAS_LAUNCHED("k_score_logits");
      launch_finalize(rows, n_sel, st, w.score.partial, tiles_v, round_up(n_sel, Cfg::BN), c0, c0 + rows, static_cast<const float*>(nullptr), rowsel,
                      ids, V, w.score.logp_c, w.score.lse_c, w.score.ent_c, logp_new, static_cast<float*>(nullptr), static_cast<float*>(nullptr));
      UMAS_LAUNCHED("k_score_finalize");
      s = ppo_rows(c0, c0 + rows);
      if (s != UMAS_OK) return s;
      hipLaunchKernelGGL(k_dz_from_logits, dim3(static_cast<unsigned>(tiles_v * tiles_r)), dim3(kTurnWaves * kWave), 0, st,
                         reinterpret_cast<float*>(w.chunk), tiles_v, c0, rows, w.score.lse_c, w.a_c, w.kz_c);
      UMAS_LAUNCHED("k_dz_from_logits");
    } else {
      hipLaunchKernelGGL(k_dz_tiles, dim3(tile_grid<kGM, kGN>(tiles_v, tiles_r, panel, kTilesPerWg)), dim3(Cfg::T), 0, st, Wb, Hb, d, V, rowsel,
                         c0, rows, w.score.lse_c, w.a_c, w.kz_c, tiles_v, tiles_r, panel, dZ, Vp);
      UMAS_LAUNCHED("k_dz_tiles");
    }
    uint16_t* Hs = reinterpret_cast<uint16_t*>(w.chunk + align_up(static_cast<size_t>(mcp) * Vp * 2 * blk_pitch));
    hipLaunchKernelGGL(k_dz_rows, dim3(cdiv(rows, 4)), dim3(256), 0, st, Hb, d, V, rowsel, c0, rows, ids, dZ, static_cast<int64_t>(tiles_v),
                       blk_pitch, Hs, mcp);
    UMAS_LAUNCHED("k_dz_rows");
    // with an entropy bonus every row has a gradient: all blocks are live
    DhSlices sl;
    const bool dw_apart = dh_plan(rows, mc_z > 0 ? logit_chunk_bytes(rows, d, V) : chunk_bytes(rows, d, V, dtype), &sl);
    hipLaunchKernelGGL(k_live_scan, dim3(1), dim3(512), 0, st, LiveArgs{static_cast<int>(c0 >> 8), tiles_r, rows, 1, dw_apart ? 0 : tiles_v, tiles_d, Vp, sl.n,
                       w.blk_live, w.blk_cidx, w.blk_orig, w.live});
    UMAS_LAUNCHED("k_live_scan");
    s = gradients(c0, rows, sl, dw_apart, dZ, blk_pitch, Hs, nullptr);
    if (s != UMAS_OK) return s;
  }
  return UMAS_OK;
}
