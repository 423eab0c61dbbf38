// The logits of a head, Z = H W^T, in tiles on the matrix cores: what the calls that score, update or list share.  One workgroup's tile with the
// softmax statistics of its rows, what a pass may leave behind for a backward (numerators or logits), the merge of the tiles' statistics, and the
// host's side: checks of arguments, grids.
#pragma once

#include <math.h>

#include <algorithm>

#include "umas_common.h"
#include "umas_mfma.h"
#include "umas_plan.h"
#include "umas_surrogate.h"

namespace umas {
namespace {

using Cfg = TileCfg<256, 256, 2, 4>;   // 8 wavefronts, two per SIMD: one issues memory operations while the other feeds the matrix pipe
using Ring = Ring2Cfg<Cfg>;
constexpr int kLogitLds = Ring::LDS_BYTES;
constexpr int kGM = 4, kGN = 8;          // tile group resident on one XCD
constexpr int kTilesPerWg = 4;           // logit tiles a workgroup computes one after the other (short K: launch gaps and store drain overlap)
constexpr int kRowBlock = 256;
constexpr float kNegInf = -INFINITY;
constexpr float kMasked = -1e30f;        // stands for a logit that does not exist (vocabulary tail)

__device__ __forceinline__ uint16_t f2bf(float x) {
  return __builtin_bit_cast(uint16_t, static_cast<__bf16>(x));
}
// two floats rounded to bf16 in one word (first in the low half): one conversion instruction
__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}
__device__ __forceinline__ float bf2f(uint16_t b) { return __uint_as_float(static_cast<uint32_t>(b) << 16); }

// Online-softmax partial: m = max z, s = sum exp(z - m), t = sum exp(z - m) z.
struct Part {
  float m, s, t;
};
__device__ __forceinline__ Part part_merge(Part x, Part y) {
  if (x.m == kNegInf) return y;
  if (y.m == kNegInf) return x;
  const float M = fmaxf(x.m, y.m);
  const float ex = __expf(x.m - M), ey = __expf(y.m - M);
  return Part{M, fmaf(x.s, ex, y.s * ey), fmaf(x.t, ex, y.t * ey)};   // written out: the same rounding in every kernel
}

// ------------------------------------------------------------------ small helpers
__global__ void __launch_bounds__(256) k_clear(ClearArgs A) {
  clear_words(A, static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x, static_cast<int64_t>(gridDim.x) * blockDim.x);
}

// bytes are a multiple of 4 for every buffer cleared here
inline hipError_t clear_bytes(hipStream_t st, void* a, size_t bytes_a, void* b = nullptr, size_t bytes_b = 0, void* c = nullptr, size_t bytes_c = 0) {
  const ClearArgs A{{static_cast<uint32_t*>(a), static_cast<uint32_t*>(b), static_cast<uint32_t*>(c)},
                    {static_cast<int64_t>(bytes_a / 4), static_cast<int64_t>(bytes_b / 4), static_cast<int64_t>(bytes_c / 4)}};
  int64_t most = 0;
  for (int k = 0; k < 3; ++k) most = A.p[k] ? std::max(most, A.words[k]) : most;
  if (most == 0) return hipSuccess;
  hipLaunchKernelGGL(k_clear, dim3(static_cast<unsigned>(std::min<int64_t>(most / 256 + 1, 65536))), dim3(256), 0, st, A);
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess && g_prof_on) prof_kernel("k_clear", st);
  return e;
}

// Where every weight is read by one tile only (one column tile) and W is larger than the memory-side cache, it is read past it: 203
// rows of 3584 against 152 064, keeping 300 -> 270 us, 100 and 200 rows of 2048 against 151 936, scoring 153 -> 143 and 187 -> 182.
// A smaller W may still lie there from the call before (250 rows of 1024 against 30 001, 61 MB: 28 us, past the cache 31), and
// the better part of one that is a little larger: scoring 256 rows through the cache and past it on two cards, W of 257 MiB 102 and 114, 109 and
// 116 us (d = 2048), 87 and 96, 89 and 96 (4096), 272 MiB 108 and 116, 119 and 117, 288 MiB 115 and 117, 123 and 119, 312 MiB 117
// and 117, 125 and 120.  dH, which reads its other operand several times meanwhile, has its line at 256 MiB (update of 256 rows
// of 1024, 264 MiB: 370 and 343, 384 and 358).
constexpr int64_t kLogitsOnceBytes = int64_t{300} << 20, kDhOnceBytes = int64_t{256} << 20;
__device__ __forceinline__ bool beyond_cache(int d, int V, int64_t bytes) { return static_cast<int64_t>(V) * d * 2 > bytes; }

// Logit tile Z[v, n] = W[m0 + v, :] . H[row(n0 + n), :] for a 256x256 block of (vocabulary, selected rows),
// row(n) = rowsel[sel0 + n] or sel0 + n.  Rows past V and past n_lim are clamped to valid ones; the
// callers mask what comes out of them.
template <class C>
__device__ __forceinline__ void logit_tile(const uint16_t* __restrict__ W, const uint16_t* __restrict__ H, int d, int V,
                                           const int32_t* __restrict__ rowsel, int64_t sel0, int64_t n_lim, int m0,
                                           int64_t n0, bool w_once, uint16_t* lds, floatx4 (&acc)[C::MI][C::NI]) {
#pragma unroll
  for (int i = 0; i < C::MI; ++i)
#pragma unroll
    for (int j = 0; j < C::NI; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
  using R = Ring2Cfg<C>;
  const uint32_t kofs = ring2_kofs();
  uint32_t oa[R::NA], ob[R::NB];
#pragma unroll
  for (int i = 0; i < R::NA; ++i) oa[i] = (static_cast<uint32_t>(min(ring2_row<C>(i), V - 1 - m0)) * d + kofs) * 2u;
#pragma unroll
  for (int i = 0; i < R::NB; ++i) {
    const int64_t n = sel0 + min(n0 + ring2_row<C>(i), n_lim - 1);
    ob[i] = (static_cast<uint32_t>(rowsel ? rowsel[n] : n) * d + kofs) * 2u;   // host checks n_rows*d*2 < 2^32
  }
  const __amdgpu_buffer_rsrc_t ra = make_rsrc(W + static_cast<int64_t>(m0) * d), rb = make_rsrc(H);
  if (d % C::BK != 0) mfma_mainloop_ring2<C, true, kCached>(ra, oa, rb, ob, d, lds, acc);
  else if (w_once) mfma_mainloop_ring2<C, false, kStream>(ra, oa, rb, ob, d, lds, acc);
  else mfma_mainloop_ring2<C, false, kCached>(ra, oa, rb, ob, d, lds, acc);
}

// ------------------------------------------------------------------ bf16: logit tiles -> partials
// A = W (vocabulary rows on the M side, so one lane sees many vocabulary entries of one token),
// B = rows c0 .. c0 + mc - 1 of the selection.  partial[tile_m][n] = (m, s, t, taken logit or 0).
//
// The keeping variant serves the backward pass when the dense part of dz is a row factor times the softmax
// (no entropy bonus): it also writes E[n, v] = bf16(exp(z[n, v] - c_n)) to the chunk buffer [mcp, Vp], c_n a
// per-row reference known before the pass (the taken token's logit), so that dz = (a_n exp(c_n - lse_n)) E
// needs no second pass over the logits: the row factor is applied where dH is written and folded into the
// copy of H that dW reads.  A block of 256 rows in which some logit exceeds its reference by more than kKeepMaxGap
// (E could overflow) is flagged and gets its dz from the recomputing kernel instead.
constexpr float kKeepMaxGap = 50.f;
// The [rows, vocabulary] operand of the backward (E, or dz on the recomputing path) lies in blocks of 256 rows x 256
// vocabulary entries, 128 KB each, row-major inside, vocabulary blocks of one block row next to each other: what a
// gradient tile reads per K step is then one run of memory (32 KB of consecutive rows for dW, four steps per block
// for dH) instead of 256 or 64 pieces a row pitch of 300 KB apart.
constexpr int64_t kBlkElems = 256 * 256;
__host__ __device__ __forceinline__ int64_t blk_offset(int64_t row_blk, int64_t voc_blk, int64_t tiles_v) {
  return (row_blk * tiles_v + voc_blk) * kBlkElems;
}
template <class C>
struct Stage {                                                                  // every wavefront stages its block: WTN rows x WTM vocabulary entries
  static constexpr int kPitch = C::WTM * 2 + 16;                                // one staged row of bf16, 16-byte aligned
  static constexpr int kBytes = C::WM * C::WN * C::WTN * kPitch;
};
constexpr int kStagePitch = Stage<Cfg>::kPitch;
template <class C>
constexpr int kLogitPitch = C::WTM * 4 + 16;                                    // one staged row of logits: 128 (64) floats
static_assert(kLogitLds <= 160 * 1024, "LDS of one CU");

enum class Leave { kNothing, kNumerators, kLogits };   // what a scoring pass leaves behind for the backward
struct KeepArgs {
  const float* cref;   // [n_pad] reference per selected row, NaN for rows without a valid id
  uint16_t* E;         // [mcp, Vp]
  int64_t Vp;
  int32_t* flags;      // per block of 256 selected rows
  const int32_t* cidx; // per block of 256 selected rows: its place among the chunk's live blocks, -1 for a dead one
  float* Z;            // Leave::kLogits: the logits, in blocks of 256 x 256 floats in the place and order of the operand's blocks
};

template <Leave LEAVE, class C>
__device__ __forceinline__ void score_tile(const uint16_t* __restrict__ W, const uint16_t* __restrict__ H, int d, int V,
                                           const int32_t* __restrict__ rowsel, int64_t c0, int64_t mc,
                                           const int32_t* __restrict__ ids, int tile_m, int tile_n, bool w_once,
                                           float4* __restrict__ partial, int64_t n_pad, const KeepArgs& keep,
                                           uint16_t* lds) {
  constexpr bool KEEP = LEAVE == Leave::kNumerators;
  static_assert(256 % C::BM == 0 && 256 % C::BN == 0, "numerators are kept inside a block");
  constexpr int kPitch = Stage<C>::kPitch;
  constexpr int kLds = C::T == Cfg::T ? kLogitLds : Ring2Cfg<C>::LDS_BYTES;   // halves of a tile use the whole one's buffers
  static_assert(Ring2Cfg<C>::LDS_BYTES <= kLds, "the main loop's stages fit");
  static_assert((LEAVE == Leave::kNothing ? 0 : Stage<C>::kBytes) + (C::WM * C::BN * 3 + C::BN) * 4 <= kLds, "staging and the partials fit the tile buffers");
  static_assert(LEAVE != Leave::kLogits || 16 * kLogitPitch<C> <= C::WTN * kPitch, "sixteen rows of logits fit a wavefront's stage");
  const int m0 = tile_m * C::BM;
  const int64_t n0 = static_cast<int64_t>(tile_n) * C::BN;   // chunk-relative
  floatx4 acc[C::MI][C::NI];
  // (a tile that lies past V as a whole, the second half of a block that is kept, reads the last entry)
  logit_tile<C>(W, H, d, V, rowsel, c0, mc, min(m0, V - 1), n0, w_once, lds, acc);

  // epilogue: the tile buffers are free now.  A lane holds, for each of its NI columns (selected rows), the
  // vocabulary entries vbase + 16 i + r (i < MI, r < 4); the four lanes l, l + 16, l + 32, l + 48 share a column.
  float* s_part = reinterpret_cast<float*>(reinterpret_cast<char*>(lds) + (LEAVE == Leave::kNothing ? 0 : Stage<C>::kBytes));   // [WM][BN][3], behind the staging area
  float* s_zy = s_part + C::WM * C::BN * 3;               // [BN]
  // (the thread's own number instead kept what two kinds of tile derive from it in registers: logits of 203 rows of 3584 with 252 bytes of scratch a lane 327 us, now 277)
  const int tid = tile_thread(), lane = tid & 63, wave = tid >> 6;
  const int wm = wave / C::WN;
  char* stage = reinterpret_cast<char*>(lds) + wave * (LEAVE == Leave::kLogits ? 16 * kLogitPitch<C> : C::WTN * kPitch);
  if (threadIdx.x < C::BN) s_zy[threadIdx.x] = 0.f;
  __syncthreads();                                        // every wavefront has left the main loop's LDS reads
  const int vbase = m0 + wm * C::WTM + (lane >> 4) * 4;   // vocabulary id of element (i = 0, r = 0)
  const bool tail = m0 + C::BM > V;
  if (tail) {   // vocabulary ids past V: a large negative logit whose exponential is 0 and whose products stay finite
#pragma unroll
    for (int i = 0; i < C::MI; ++i)
#pragma unroll
      for (int j = 0; j < C::NI; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (vbase + i * 16 + r >= V) acc[i][j][r] = kMasked;
  }
  constexpr float kLog2e = 1.44269504088896341f;
  bool over = false;
  // a block of rows none of which has a gradient (all advantages 0) keeps nothing: the backward never looks at it
  const int64_t row_blk = (c0 + n0) >> 8;
  const int out_blk = KEEP ? keep.cidx[row_blk] : -1;
  const bool keeping = KEEP && out_blk >= 0;
#pragma unroll
  for (int j = 0; j < C::NI; ++j) {
    const int col = acc_col<C>(j);
    const int64_t n = n0 + col;
    // exponentials of this lane's entries of column j relative to m (log2 domain), their sum s and sum of e z; the
    // keeping variant stages them as bf16 in this wavefront's LDS region, stored in full lines below
    float m = kMasked, s = 0.f, t = 0.f;
    auto column = [&](float ref, auto premultiplied) {
      const float r2 = ref * kLog2e;
      s = 0.f;
      t = 0.f;
#pragma unroll
      for (int i = 0; i < C::MI; ++i) {
        float e[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float z = acc[i][j][r];
          // without a reference from outside: z - m first, exact 0 where a lane holds nothing but vocabulary tail
          e[r] = decltype(premultiplied)::value ? __builtin_amdgcn_exp2f(fmaf(z, kLog2e, -r2)) : __builtin_amdgcn_exp2f((z - ref) * kLog2e);
          s += e[r];
          t = fmaf(e[r], z, t);
        }
        if (keeping) {
          const uint32_t p01 = pack_bf16x2(e[0], e[1]), p23 = pack_bf16x2(e[2], e[3]);
          *reinterpret_cast<uint2*>(stage + (j * 16 + (lane & 15)) * kPitch + (i * 16 + (lane >> 4) * 4) * 2) =
              make_uint2(p01, p23);
        }
      }
    };
    auto lane_max = [&]() {
      float mx = kMasked;
#pragma unroll
      for (int i = 0; i < C::MI; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) mx = fmaxf(mx, acc[i][j][r]);
      return mx;
    };
    if (keeping) {
      // The keeping variant sums relative to the row's reference c_n instead of the lane's maximum (any reference
      // serves the merge as long as nothing overflows), so the exponentials it sums are the numerators it keeps,
      // and it does not look for the maximum first: a sum beyond 32 e^kKeepMaxGap (or not a number: rows without
      // a valid id have the reference NaN) shows afterwards that some logit may lie more than kKeepMaxGap above
      // c_n.  Only then is the column done again the long way, relative to the lane's maximum: a lane whose maximum
      // does lie that far above c_n flags the block (its dz is recomputed later); rows without a valid id flag
      // nothing, their row factor is 0.
      const float c = n < mc ? keep.cref[c0 + n] : 1e30f;   // rows past the chunk: every exponential is 0, E = 0
      m = c;
      column(c, std::true_type{});
      constexpr float kSumLimit = 1.6e23f;                   // 32 e^50 = 1.66e23
      if (!(s < kSumLimit)) {
        m = lane_max();
        const float gap = m - c;
        over |= gap > kKeepMaxGap;
        if (gap <= kKeepMaxGap) m = c;                       // many large terms, none too large: c serves after all
        else if (m == kMasked) m = 0.f;                     // nothing but vocabulary tail in this lane: exponentials 0 as well
        column(m, std::true_type{});
      }
    } else {
      m = lane_max();
      column(m, std::false_type{});
    }
    if (LEAVE == Leave::kLogits) {
      // sixteen rows of 128 (64) logits through the wavefront's part of LDS, so that a store covers 512 (256) bytes of two (four) rows
#pragma unroll
      for (int i = 0; i < C::MI; ++i)
        *reinterpret_cast<floatx4*>(stage + (lane & 15) * kLogitPitch<C> + (i * 16 + (lane >> 4) * 4) * 4) = acc[i][j];
      __builtin_amdgcn_wave_barrier();
      constexpr int kLanes = C::WTM / 4, kRows = kWave / kLanes;
      float* out = keep.Z + blk_offset(n0 >> 8, m0 >> 8, keep.Vp >> 8) + ((n0 & 255) + wave % C::WN * C::WTN + j * 16 + lane / kLanes) * 256 + (m0 & 255) +
                   wm * C::WTM + lane % kLanes * 4;
#pragma unroll
      for (int q = 0; q < 16 / kRows; ++q)
        if (n0 + wave % C::WN * C::WTN + j * 16 + q * kRows + lane / kLanes < mc)   // rows past the chunk: nobody reads them
          __builtin_nontemporal_store(*reinterpret_cast<const floatx4*>(stage + (q * kRows + lane / kLanes) * kLogitPitch<C> + lane % kLanes * 16),
                                      reinterpret_cast<floatx4*>(out + q * kRows * 256));
      __builtin_amdgcn_wave_barrier();
    }
    Part p{m, s, t};
#pragma unroll
    for (int o = 16; o < kWave; o <<= 1) {
      const Part q{__shfl_xor(p.m, o, kWave), __shfl_xor(p.s, o, kWave), __shfl_xor(p.t, o, kWave)};
      p = part_merge(p, q);
    }
    if (lane < 16) {
      float* dst = s_part + (wm * C::BN + col) * 3;
      dst[0] = p.m; dst[1] = p.s; dst[2] = p.t;
    }
    if (!KEEP && n < mc) {                                  // the keeping variant got the taken logits beforehand
      const int y = ids[rowsel ? rowsel[c0 + n] : c0 + n];
      const int rel = y - vbase;                           // offset from this lane's first element
      if (y >= 0 && y < V && rel >= 0 && rel < C::WTM && (rel & 12) == 0) {
        float zy = 0.f;
#pragma unroll
        for (int i = 0; i < C::MI; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (i * 16 + r == rel) zy = acc[i][j][r];
        s_zy[col] = zy;
      }
    }
  }
  if (keeping) {
    if (over) keep.flags[row_blk] = 1;
    // the staged block goes out 16 bytes per lane: one instruction covers 4 rows x 256 contiguous bytes (of 64 entries a row, 8 x 128)
    constexpr int kLanes = C::WTM / 8, kRows = kWave / kLanes;
    const int wn = wave % C::WN;
    uint16_t* out = keep.E + blk_offset(out_blk, m0 >> 8, keep.Vp >> 8) + ((n0 & 255) + wn * C::WTN) * 256 + (m0 & 255) + wm * C::WTM + lane % kLanes * 8;
#pragma unroll 8
    for (int i = 0; i < C::WTN / kRows; ++i) {
      const int row = i * kRows + lane / kLanes;
      const uint4 v = *reinterpret_cast<const uint4*>(stage + row * kPitch + lane % kLanes * 16);
      typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
      __builtin_nontemporal_store(u32x4{v.x, v.y, v.z, v.w}, reinterpret_cast<u32x4*>(out + row * 256));
    }
  }
  __syncthreads();
  if (threadIdx.x < C::BN) {
    const int col = threadIdx.x;
    Part p{kNegInf, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < C::WM; ++w) {
      const float* src = s_part + (w * C::BN + col) * 3;
      p = part_merge(p, Part{src[0], src[1], src[2]});
    }
    if (c0 + n0 + col < n_pad) partial[static_cast<int64_t>(tile_m) * n_pad + c0 + n0 + col] = make_float4(p.m, p.s, p.t, s_zy[col]);
  }
  __syncthreads();                              // the LDS is the next tile's again
}

// The tiles of a workgroup.  With few column tiles a workgroup has one tile, and the last round of compute units is often nearly empty: the tiles of
// one that is at most half full are cut into two of 128 rows of the selection.  594 tiles on 256 compute units, 256 rows: 2048 columns 190 -> 173 us, 3584
// 283 -> 270; 150 rows 188 -> 170 and 271 -> 262; the update of 203 rows of 3584 1037 -> 1022, with an entropy bonus 1056 -> 1026, 100 rows of 2048 609 ->
// 584.  (Up to 128 rows all tiles cut, whose other halves have no rows: 100 rows with a bonus 611, of 3584 957 -> 1036.)  Up to eight column tiles, beyond which
// a workgroup has several: 300, 1000 and 2000 rows of 1536 against 33 001 86.7 -> 76.6, 126.5 -> 114.9 and 204.9 -> 193.5, of 1024 against 100 001
// 130.1 -> 119.9, 217.8 -> 208.5 and 389.7 -> 382.4, of 2048 against 151 936 294.2 -> 276.9, 553.2 -> 547.4 and 1014 -> 1023, 900 of 3584 918 -> 900; where
// the last round is fuller nothing changes.
using HalfCfg = TileCfg<256, 128, 2, 4>;                 // the lanes of a row as in a whole tile: the same bits
using HalfNarrowCfg = TileCfg<128, 64, 2, 2>;            // of a NarrowCfg
// So is a tile whose rows end in its first half: 300 rows of 2048 against 151 936 265 -> 250 us, 600 371 -> 357, 4200 of 3584 3454 -> 3376, 262 of 1664 against 63 167 88 -> 81.
enum class HalfTile { kNone, kWhole, kHalf };
// The tile of a workgroup, `it` of its kTilesPerWg, of the `mc` rows; a half's number counts halves.
template <class Half>
__device__ __forceinline__ HalfTile half_tile(int tiles_m, int tiles_n, int panel, int halved, int it, int64_t mc, int* tile_m, int* tile_n) {
  if (halved > 0) {                               // the last `halved` tiles of every XCD
    const int per_xcd = (tiles_m * tiles_n + 7) / 8, xcd = static_cast<int>(blockIdx.x & 7), w = static_cast<int>(blockIdx.x >> 3), whole = per_xcd - halved;
    if (w >= whole) {
      const int in_xcd = whole + (w - whole) / 2, t = xcd * per_xcd + in_xcd;
      *tile_m = t / tiles_n;
      *tile_n = t % tiles_n * 2 + ((w - whole) & 1);
      return it == 0 && in_xcd < per_xcd && *tile_m < tiles_m && *tile_n * Half::BN < mc ? HalfTile::kHalf : HalfTile::kNone;
    }
  }
  if (!tile_coords<kGM, kGN>(tiles_m, tiles_n, panel, tile_m, tile_n, it, kTilesPerWg)) return HalfTile::kNone;
  if (*tile_n == 0 || mc - static_cast<int64_t>(*tile_n) * (2 * Half::BN) > Half::BN) return HalfTile::kWhole;   // (a single row tile reads W once: whole)
  *tile_n *= 2;
  return HalfTile::kHalf;
}
// ENDS: with halves where the rows end in the first half of a tile.  (A loop of its own, which costs whole tiles 0.8 %: 16 384 rows of 2048 7.82 -> 7.88 ms.)
template <Leave LEAVE, class C, bool ENDS = false>
__device__ __forceinline__ void score_tiles(const uint16_t* __restrict__ W, const uint16_t* __restrict__ H, int d, int V,
                                            const int32_t* __restrict__ rowsel, int64_t c0, int64_t mc,
                                            const int32_t* __restrict__ ids, int tiles_m, int tiles_n, int panel,
                                            float4* __restrict__ partial, int64_t n_pad, const KeepArgs& keep,
                                            uint16_t* lds, int halved = 0) {
  const bool w_once = tiles_n == 1 && beyond_cache(d, V, kLogitsOnceBytes);
  if constexpr (ENDS) {
    using Half = std::conditional_t<C::BN == HalfCfg::BN * 2, HalfCfg, HalfNarrowCfg>;
    for (int it = 0; it < kTilesPerWg; ++it) {
      int tile_m, tile_n;
      const HalfTile h = half_tile<Half>(tiles_m, tiles_n, panel, halved, it, mc, &tile_m, &tile_n);
      if (h == HalfTile::kNone) continue;
      if (h == HalfTile::kHalf) score_tile<LEAVE, Half>(W, H, d, V, rowsel, c0, mc, ids, tile_m, tile_n, false, partial, n_pad, keep, lds);
      else score_tile<LEAVE, C>(W, H, d, V, rowsel, c0, mc, ids, tile_m, tile_n, w_once, partial, n_pad, keep, lds);
    }
    return;
  }
  if constexpr (C::BM == 256 && C::BN == 256) {
    if (halved > 0) {                             // the last `halved` tiles of every XCD
      const int per_xcd = (tiles_m * tiles_n + 7) / 8, xcd = static_cast<int>(blockIdx.x & 7), w = static_cast<int>(blockIdx.x >> 3), whole = per_xcd - halved;
      if (w >= whole) {
        const int in_xcd = whole + (w - whole) / 2, t = xcd * per_xcd + in_xcd, tile_m = t / tiles_n, half = t % tiles_n * 2 + ((w - whole) & 1);
        if (in_xcd < per_xcd && tile_m < tiles_m && half * HalfCfg::BN < mc)
          score_tile<LEAVE, HalfCfg>(W, H, d, V, rowsel, c0, mc, ids, tile_m, half, false, partial, n_pad, keep, lds);
        return;
      }
    }
  }
  for (int it = 0; it < kTilesPerWg; ++it) {     // a workgroup walks the same place of kTilesPerWg consecutive tile groups
    int tile_m, tile_n;
    if (!tile_coords<kGM, kGN>(tiles_m, tiles_n, panel, &tile_m, &tile_n, it, kTilesPerWg)) continue;
    score_tile<LEAVE, C>(W, H, d, V, rowsel, c0, mc, ids, tile_m, tile_n, w_once, partial, n_pad, keep, lds);
  }
}

// Up to 128 selected rows: half-size tiles with a pipeline of their own, two workgroups to a compute unit, so that one
// fills its stages while the other multiplies (64 rows of 2048 / 3584 against 151 936: 156 / 215 us against 182 / 274 with
// the large tiles; 128x256 and 256x128 tiles 213 / 347 and 167 / 234).
using NarrowCfg = TileCfg<128, 128, 2, 2>;
constexpr int kNarrowLds = Ring2Cfg<NarrowCfg>::LDS_BYTES;

// ------------------------------------------------------------------ bf16: a few rows (see k_score_few)
constexpr int kFewWaves = 8, kFewT = kFewWaves * kWave;
inline int few_pieces(int d) { return static_cast<int>(cdiv(d, kFewWaves * 64)); }   // PPW
inline int few_rows(int d) { return few_pieces(d) <= 4 ? 64 : few_pieces(d) <= 8 ? 32 : 0; }   // what the registers hold

// Merge the per-tile partials of each selected row; compact results and optional scatter.  Eight lanes of a wavefront
// share a row (lane = 8 * part + row within the group of 8 rows, so a load covers whole 128-byte lines), four loads in
// flight each.  Where there are few rows the four wavefronts of the workgroup share the group's tiles as well (SPLIT):
// 24 rows of 594 tiles 41 -> 7 us, 16 100 rows 53 -> 36; with enough rows to fill the chip the extra merge only costs
// (39 000 rows, 373 MB: 82 us split, 69 not).
constexpr int64_t kFinSplitRows = 20000;
// Row n's parts merged; true in the thread that has the result (SPLIT: one of the first eight of the workgroup).
template <bool SPLIT>
__device__ __forceinline__ bool merge_parts(const float4* __restrict__ partial, int tiles_m, int64_t n_pad, int64_t n, bool live, Part& p, float& zy) {
  __shared__ float4 s_part[4][8];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  constexpr int kParts = SPLIT ? 32 : 8;
  p = Part{kNegInf, 0.f, 0.f};
  zy = 0.f;
  if (live) {
    for (int t0 = SPLIT ? threadIdx.x >> 3 : lane >> 3; t0 < tiles_m; t0 += 4 * kParts) {
      float4 q[4];
#pragma unroll
      for (int k = 0; k < 4; ++k)
        q[k] = t0 + k * kParts < tiles_m ? partial[static_cast<int64_t>(t0 + k * kParts) * n_pad + n] : make_float4(kNegInf, 0.f, 0.f, 0.f);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        p = part_merge(p, Part{q[k].x, q[k].y, q[k].z});
        zy += q[k].w;
      }
    }
  }
#pragma unroll
  for (int o = 8; o < kWave; o <<= 1) {
    const Part q{__shfl_xor(p.m, o, kWave), __shfl_xor(p.s, o, kWave), __shfl_xor(p.t, o, kWave)};
    p = part_merge(p, q);
    zy += __shfl_xor(zy, o, kWave);
  }
  if constexpr (SPLIT) {
    if (lane < 8) s_part[wave][lane] = make_float4(p.m, p.s, p.t, zy);
    __syncthreads();
    if (wave == 0) {
#pragma unroll
      for (int k = 1; k < 4; ++k) {
        const float4 q = s_part[k][lane & 7];
        p = part_merge(p, Part{q.x, q.y, q.z});
        zy += q.w;
      }
    }
  }
  return lane < 8 && live && (!SPLIT || wave == 0);
}
struct RowScore {
  float logp, lse, entropy;
};
__device__ __forceinline__ RowScore row_score(const Part& p, float zy, bool ok) {
  const float l = p.m + logf(p.s);
  return RowScore{ok ? zy - l : 0.f, l, ok ? l - p.t / p.s : 0.f};
}

__device__ __forceinline__ void bf16x8_to_f32(const uint4 v, float (&o)[8]) {
  o[0] = __uint_as_float(v.x << 16); o[1] = __uint_as_float(v.x & 0xffff0000u);
  o[2] = __uint_as_float(v.y << 16); o[3] = __uint_as_float(v.y & 0xffff0000u);
  o[4] = __uint_as_float(v.z << 16); o[5] = __uint_as_float(v.z & 0xffff0000u);
  o[6] = __uint_as_float(v.w << 16); o[7] = __uint_as_float(v.w & 0xffff0000u);
}

// ------------------------------------------------------------------ host side
constexpr int64_t kF32ChunkRows = 4096;
constexpr double kF32MaxWork = 137438953472.0;   // 2^37 multiply-adds per product
// A chunk of more rows is no faster: 73 728 rows of 2048 in one chunk 108.6 ms, in two 105.8; 122 880 of 3584 in one 326 ms, in two
// 320.7, in three 315; 163 840 in two 432, in three 427.
constexpr int64_t kMaxChunkRows = 1 << 16;

inline int64_t round_up(int64_t x, int64_t a) { return (x + a - 1) / a * a; }

inline umas_status check_model_args(const void* H, const void* W, umas_dtype dt, int64_t n_rows, int d, int V,
                             const int32_t* ids, const int32_t* rowsel, int64_t n_sel) {
  UMAS_REQUIRE(dt == UMAS_F32 || dt == UMAS_BF16, UMAS_EDTYPE, "dtype=%d is neither F32 nor BF16", static_cast<int>(dt));
  UMAS_REQUIRE(n_rows >= 0 && n_sel >= 0, UMAS_EINVAL, "negative row count");
  UMAS_REQUIRE(d >= 1 && V >= 1, UMAS_ESHAPE, "d=%d and V=%d must be positive", d, V);
  UMAS_REQUIRE(dt != UMAS_BF16 || d % 8 == 0, UMAS_ESHAPE, "bf16 needs d %% 8 == 0 (d=%d)", d);
  UMAS_REQUIRE(dt != UMAS_F32 || d <= 8192, UMAS_ESHAPE, "the float32 path supports d <= 8192 (d=%d)", d);
  // the float32 path sums in float64: small shapes only
  UMAS_REQUIRE(dt != UMAS_F32 || static_cast<double>(n_sel) * V * d <= kF32MaxWork, UMAS_ESHAPE,
               "the float32 path is for small shapes: n_sel * V * d = %.3g exceeds %.3g; use bf16",
               static_cast<double>(n_sel) * V * d, kF32MaxWork);
  UMAS_REQUIRE(dt != UMAS_BF16 || static_cast<uint64_t>(n_rows) * d * 2 < (1ull << 32), UMAS_ESHAPE,
               "bf16 H must be smaller than 4 GiB (32-bit buffer offsets): n_rows=%lld d=%d",
               static_cast<long long>(n_rows), d);
  UMAS_REQUIRE(dt != UMAS_BF16 || static_cast<uint64_t>(std::min(V, 256)) * d * 2 < (1ull << 32), UMAS_ESHAPE,
               "256 rows of a bf16 W must be smaller than 4 GiB (32-bit buffer offsets): V=%d d=%d", V, d);
  UMAS_REQUIRE(rowsel || n_sel == n_rows, UMAS_EINVAL, "rowsel is NULL but n_sel != n_rows");
  UMAS_REQUIRE(n_sel <= n_rows, UMAS_EINVAL, "n_sel=%lld exceeds n_rows=%lld", static_cast<long long>(n_sel),
               static_cast<long long>(n_rows));
  UMAS_REQUIRE((H && ids) || n_rows == 0, UMAS_EINVAL, "H and ids must not be NULL");
  UMAS_REQUIRE(W, UMAS_EINVAL, "W must not be NULL");
  UMAS_REQUIRE(reinterpret_cast<uintptr_t>(H) % 16 == 0 && reinterpret_cast<uintptr_t>(W) % 16 == 0, UMAS_EINVAL,
               "H and W must be 16-byte aligned");
  return UMAS_OK;
}

inline umas_status check_ws(void* ws, size_t have, size_t need) {
  UMAS_REQUIRE(ws && reinterpret_cast<uintptr_t>(ws) % kAlign == 0 && have >= need, UMAS_EWORKSPACE,
               "workspace must be 256-byte aligned and hold %zu bytes (got %zu)", need, have);
  return UMAS_OK;
}

inline int device_cus() {
  int dev = 0, n_cu = 0;
  if (hipGetDevice(&dev) != hipSuccess || hipDeviceGetAttribute(&n_cu, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n_cu < 1)
    n_cu = 64;
  return n_cu;
}

// Row tiles that the logit kernels work through together (see tile_coords): an XCD reads all rows of H once for every four
// vocabulary tiles, all XCDs at about the same time, so a panel that stays in the memory-side cache (256 MB) comes from HBM once
// instead of nineteen times.  40 960 rows of 3584 (293 MB), score: all rows 33.4 ms, panels of at most 40 / 64 / 96 / 128 / 160
// MiB 31.5 / 30.6 / 30.7 / 30.5 / 30.7; 24 576 rows kept 20.6 -> 19.3 ms; 40 960 rows of 2048 (168 MB) 18.2 either way.
constexpr int64_t kPanelBytes = int64_t{128} << 20;
inline int row_panel(int tiles_n, int d) {
  const int most = std::max(static_cast<int>(kPanelBytes / (static_cast<int64_t>(Cfg::BN) * d * 2)) / kGN * kGN, kGN);
  const int panels = (tiles_n + most - 1) / most;
  return ((tiles_n + panels - 1) / panels + kGN - 1) / kGN * kGN;
}

// Tiles of every XCD that are cut in two (see score_tiles): those of the last round of compute units where it is at most half full.
inline int halved_tiles(int tiles_m, int tiles_n, int per_cu = 1) {   // per_cu: workgroups to a compute unit
  if (tiles_n > kGN) return 0;
  const int per_xcd = static_cast<int>(cdiv(static_cast<size_t>(tiles_m) * tiles_n, 8)), round = std::max(device_cus() / 8, 1) * per_cu, rest = per_xcd % round;
  return rest * 2 <= round ? rest : 0;
}
inline dim3 score_grid(int tiles_m, int tiles_n, int panel, int halved) {
  return dim3(tile_grid<kGM, kGN>(tiles_m, tiles_n, panel, kTilesPerWg) + 8 * static_cast<unsigned>(halved));
}

}  // namespace
}  // namespace umas
