// The two gradient products behind the logits, dH = dZ W and dW = dZ^T H, over a bf16 operand [rows, vocabulary] that a scoring pass has left in
// blocks: which blocks there are and how the tiles are shared among the XCDs, the tiles, the sum of the slices of dH, and the sizes of the operand.
#pragma once

#include "umas_logits.h"

namespace umas {
namespace {

// ------------------------------------------------------------------ bf16: blocks of rows that have a gradient
// A selected row whose advantage is 0 has g = 0 and (without an entropy bonus or a KL term) no gradient at all; group-normalised
// outcome rewards make whole trajectory groups such rows.  The keeping pass therefore works on the chunk's live blocks
// of 256 selected rows only: E and the scaled copy of H hold them packed, dH has as many row tiles and dW as many K
// steps as there are, and everything that depends on their number is worked out on the device.
struct LiveInfo {
  int32_t n_live;        // live blocks of the chunk
  int32_t k_rows;        // rows of the packed operands that exist (the chunk's last block may be partly filled)
  XcdShares dw;          // dW tiles per XCD (see share_dw)
  int32_t next[8];       // per XCD: next place of its sequence of tiles, counted up by the workgroups of k_gemm_dh_dw
};
// Shares of the dW tiles per XCD for k_gemm_dh_dw: every XCD first works through its eighth of the dH tiles (contiguous
// ranges, slice after slice; a tile costs about Vp / slices of K), then dW tiles (k_len of K each) go to the XCDs so that all
// finish as evenly as possible.  Shares are whole groups where there are many: an XCD's workgroups that work on parts of two
// groups at a time read a third more through its L2 (39 000 rows of 2048: 6 % of the step).
constexpr int64_t kTileOverheadK = 768;   // what a tile costs besides its K steps (first loads, epilogue), as a length of K
__device__ __forceinline__ int share_unit(int tiles, int slices) { return slices == 1 && tiles >= 8 * kGM * kGN ? kGM * kGN : 1; }
__device__ __forceinline__ int dh_first(int tiles_dh, int slices, int xcd) {
  const int unit = share_unit(tiles_dh, slices), units = (tiles_dh + unit - 1) / unit;
  return min(static_cast<int>(static_cast<int64_t>(units) * xcd / 8) * unit, tiles_dh);
}
// K of the dW tiles: whole steps of 64 rows.  (With whole blocks of 256, and dH tiles that read and
// multiply the rows that are not there as well: both products of 30 / 100 rows of 3584 672 us, now 612 / 620; update of 300 / 550 rows of 2048 976 / 1327,
// now 890 / 1252.)
__device__ __forceinline__ int dw_k(int k_rows) { return (k_rows + 63) / 64 * 64; }
// Called by one wavefront; lane x of every eight works for XCD x (all eights do the same).  (One thread walking the eight XCDs took 20 us.)
__device__ void share_dw(int tiles_r, int tiles_v, int tiles_d, int64_t Vp, int slices, int64_t k_len, XcdShares* out) {
  const int x = threadIdx.x & 7;
  auto sum8 = [](int64_t v) {
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) v += static_cast<int64_t>(__shfl_xor(static_cast<long long>(v), o, kWave));
    return v;
  };
  const int tiles_dh = tiles_r * tiles_d * slices;
  const int64_t load = (dh_first(tiles_dh, slices, x + 1) - dh_first(tiles_dh, slices, x)) * (Vp / slices + kTileOverheadK);
  const int tiles_dw = tiles_v * tiles_d, unit = share_unit(tiles_dw, 1);
  const int64_t units = (tiles_dw + unit - 1) / unit;
  k_len *= unit;
  int64_t cnt;
  if (k_len <= 0 || units == 0) {                      // nothing to even out
    cnt = units / 8 + (x < units % 8 ? 1 : 0);
  } else {
    // the level up to which the XCDs would be filled if units could be cut: those that stand above it as they are take nothing ...
    // (a search for it among whole numbers took 23 rounds: k_live_scan 9.6 us, now 5.1)
    double level = 0.0;
    bool takes = true;
    for (int round = 0; round < 8; ++round) {
      level = static_cast<double>(units * k_len + sum8(takes ? load : 0)) / static_cast<double>(sum8(takes ? 1 : 0));
      const bool above = takes && static_cast<double>(load) >= level;
      if (!__any(above)) break;
      takes = takes && !above;
    }
    cnt = takes ? static_cast<int64_t>((level - static_cast<double>(load)) / static_cast<double>(k_len)) : 0;
    // ... and of the few units that are left every one goes where it is done first (or comes, by rounding, from where it would be last)
    for (int64_t left = units - sum8(cnt); left != 0; left -= left > 0 ? 1 : -1) {
      const int64_t end = left > 0 ? -(load + cnt * k_len) : cnt > 0 ? load + cnt * k_len : INT64_MIN;
      int64_t best = end;
#pragma unroll
      for (int o = 4; o > 0; o >>= 1) best = max(best, static_cast<int64_t>(__shfl_xor(static_cast<long long>(best), o, kWave)));
      if (x == __ffsll(static_cast<long long>(__ballot(end == best))) - 1) cnt += left > 0 ? 1 : -1;
    }
  }
  int first = static_cast<int>(cnt);                   // inclusive prefix sums: where the next XCD's units start
#pragma unroll
  for (int o = 1; o < 8; o <<= 1) {
    const int t = __shfl_up(first, o, kWave);
    if (x >= o) first += t;
  }
  if (threadIdx.x == 0) out->first[0] = 0;
  if (threadIdx.x < 8) out->first[x + 1] = static_cast<int>(min(static_cast<int64_t>(first) * unit, static_cast<int64_t>(tiles_dw)));
}
// Packs the live blocks of a chunk, blk0 its first block; one workgroup, thread t has block t and knows if it is live.
struct LiveArgs {
  int blk0, nblk;
  int64_t rows;
  int all_live, tiles_v, tiles_d;
  int64_t Vp;
  int slices;
  const int32_t* blk_live;
  int32_t *blk_cidx, *blk_orig;
  LiveInfo* info;
};
__device__ __forceinline__ void live_scan(const LiveArgs& A, int live) {
  __shared__ int smem[32];
  __shared__ int s_last_live;
  const int t = threadIdx.x;
  int total;
  const int pos = block_excl_scan<int>(live, smem, &total);
  if (t < A.nblk) {
    A.blk_cidx[A.blk0 + t] = live ? pos : -1;
    if (live) A.blk_orig[A.blk0 + pos] = t;
  }
  if (t == A.nblk - 1) s_last_live = live;
  __syncthreads();
  const int64_t last_rows = A.rows - static_cast<int64_t>(A.nblk - 1) * 256;   // rows of the chunk's last block
  const int k_rows = static_cast<int>(s_last_live ? static_cast<int64_t>(total - 1) * 256 + last_rows : static_cast<int64_t>(total) * 256);
  if (t == 0) {
    A.info->n_live = total;
    A.info->k_rows = k_rows;
  }
  if (t < 8) A.info->next[t] = 0;
  if (t < kWave) share_dw(total, A.tiles_v, A.tiles_d, A.Vp, A.slices, total > 0 ? dw_k(k_rows) + kTileOverheadK : 0, &A.info->dw);
}
// One launch per chunk (all blocks live with all_live).
__global__ void __launch_bounds__(512)
k_live_scan(LiveArgs A) {
  const int t = threadIdx.x;
  live_scan(A, t < A.nblk && (A.all_live || A.blk_live[A.blk0 + t]));
}

// ------------------------------------------------------------------ bf16: dz tiles into the chunk buffer
// For blocks of rows whose numerators do not serve, and with an entropy bonus for narrow heads and in a small workspace (16 100 rows of 2048 in 2 GB,
// chunks of 3300: 31.3 ms; chunks of logits of half that many rows would add to dW twice as often).  Same tile product as k_score_tiles; the epilogue forms the dense part of dz = g (onehot - softmax),
// -g exp(z - lse), plus the entropy bonus's term when its coefficient is not 0, and writes it as bf16 to
// dZ [mcp, Vp].  Rows past the chunk and vocabulary ids past V get 0.  The one-hot part g at v = y is a single term per row and is added in
// float32 where dH and dW are written, so that it never meets the bf16 rounding of the dense part.
// `fix` may change single entries before a row leaves: it gets a lane's staged row, the row's place in the selection (-1: none) and the row's first
// vocabulary entry.  ClearTaken leaves the taken token's entry at 0 (see k_ppo_rows); with LeaveRows that is left to who goes over the rows afterwards.
constexpr int kFlaggedGrid = 256;   // workgroups that look for flagged blocks
struct LeaveRows {};
struct ClearTaken {
  const int32_t* rowsel;
  const int32_t* ids;
  __device__ __forceinline__ void operator()(char* staged, int64_t n, int v0, int width) const {
    const int y = (n >= 0 ? ids[rowsel ? rowsel[n] : n] : -1) - v0;
    const uint16_t none = 0;
    if (y >= 0 && y < width) __builtin_memcpy(staged + y * 2, &none, 2);
  }
};
template <class Fix>
__device__ __forceinline__ void dz_tile(int tile_m, int tile_n, const uint16_t* __restrict__ W, const uint16_t* __restrict__ H,
                                        int d, int V, const int32_t* __restrict__ rowsel, int64_t c0, int64_t mc, const Fix& fix,
                                        const float* __restrict__ lse_c, const float* __restrict__ a_c,
                                        const float* __restrict__ kz_c, uint16_t* __restrict__ dZ, int64_t Vp, int out_blk,
                                        uint16_t* lds) {
  using C = Cfg;
  const int m0 = tile_m * C::BM;
  const int64_t n0 = static_cast<int64_t>(tile_n) * C::BN;   // chunk-relative
  floatx4 acc[C::MI][C::NI];
  logit_tile<C>(W, H, d, V, rowsel, c0, mc, m0, n0, false, lds, acc);

  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wm = wave / C::WN;
  const int vbase = m0 + wm * C::WTM + (lane >> 4) * 4;
  const bool tail = m0 + C::BM > V;
  // each wavefront stages its 64 (rows) x 128 (vocabulary) block; the 272-byte pitch keeps 16-byte alignment
  char* stage = reinterpret_cast<char*>(lds) + wave * (C::WTN * kStagePitch);
  __syncthreads();                              // every wavefront has left the main loop's LDS reads
  if (tail) {                                   // vocabulary ids past V: the exponential below is 0, the factor next to it finite
#pragma unroll
    for (int i = 0; i < C::MI; ++i)
#pragma unroll
      for (int j = 0; j < C::NI; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (vbase + i * 16 + r >= V) acc[i][j][r] = kMasked;
  }
#pragma unroll
  for (int j = 0; j < C::NI; ++j) {
    const int64_t n = n0 + acc_col<C>(j);
    // dz = p (a + kz z) with p = exp(z - lse), a = -g + k (entropy - lse), kz = k = entropy_coef / n_sel: the
    // dense part of g (onehot - p) plus the entropy bonus's k p (log p + entropy).  Rows past the chunk: p = 0.
    float l2 = 1e30f, a = 0.f, kz = 0.f;
    if (n < mc) {
      l2 = lse_c[c0 + n] * 1.44269504088896341f;
      a = a_c[c0 + n];
      kz = kz_c[c0 + n];
    }
#pragma unroll
    for (int i = 0; i < C::MI; ++i) {
      float dz[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float z = acc[i][j][r];
        dz[r] = __builtin_amdgcn_exp2f(fmaf(z, 1.44269504088896341f, -l2)) * fmaf(kz, z, a);
      }
      const uint32_t p01 = pack_bf16x2(dz[0], dz[1]), p23 = pack_bf16x2(dz[2], dz[3]);
      // staged in this wavefront's LDS region, stored in full lines below
      *reinterpret_cast<uint2*>(stage + (j * 16 + (lane & 15)) * kStagePitch + (i * 16 + (lane >> 4) * 4) * 2) =
          make_uint2(p01, p23);
    }
  }
  const int wn = wave % C::WN;
  if constexpr (!std::is_same<Fix, LeaveRows>::value) {   // a lane per staged row (every entry compared above: 60 bytes of scratch a lane, like this 20; with no block flagged 6.9 us and 6.55)
    static_assert(C::WTN == kWave, "a row a lane");
    __builtin_amdgcn_wave_barrier();
    const int64_t n = n0 + wn * C::WTN + lane;
    fix(stage + lane * kStagePitch, n < mc ? c0 + n : -1, m0 + wm * C::WTM, C::WTM);
    __builtin_amdgcn_wave_barrier();
  }
  // the staged block goes out 16 bytes per lane: one instruction covers 4 rows x 256 contiguous bytes
  uint16_t* out = dZ + blk_offset(out_blk, tile_m, Vp >> 8) + (wn * C::WTN) * 256 + wm * C::WTM + (lane & 15) * 8;
#pragma unroll 8
  for (int i = 0; i < C::WTN / 4; ++i) {
    const int row = i * 4 + (lane >> 4);
    const uint4 v = *reinterpret_cast<const uint4*>(stage + row * kStagePitch + (lane & 15) * 16);
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    __builtin_nontemporal_store(u32x4{v.x, v.y, v.z, v.w}, reinterpret_cast<u32x4*>(out + row * 256));
  }
  __syncthreads();                              // the LDS is the next tile's again
}

// ------------------------------------------------------------------ bf16: the two gradient products
// dH = dZ W: A = dZ [mcp, Vp] (or the kept numerators E) is K-contiguous (K = vocabulary), B = W [V, d] is K-major and is read as it lies.
//   dH[rowsel[c0 + m], j] = bf16(sc[m] C[m, j] + g[m] W[y[m], j]) for m < mc (sc: the keeping pass's row factor, else 1)
// dW = dZ^T H: K = rows of the chunk; A = dZ [mcp, Vp] and B = the selected rows of H, copied (and scaled), are both K-major.
//   dW[v, j] (+)= C[v, j]
// (kernel templates whose bodies use buffer resources do not get their host stubs emitted: plain kernels)
template <class C>
__device__ __forceinline__ void zero_acc(floatx4 (&acc)[C::MI][C::NI]) {
#pragma unroll
  for (int i = 0; i < C::MI; ++i)
#pragma unroll
    for (int j = 0; j < C::NI; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
}
// K-contiguous operand tile: block row `row_blk` of the blocked [rows, vocabulary] operand from vocabulary block `voc_blk` on, of which the
// first `rows` rows are wanted: a pass of loads behind them takes the lines of the first one again, which are on their way to this
// compute unit anyhow (the last row for all of them made one line hot: 203 rows of 2048 613 -> 650 us); K runs over the vocabulary, four steps of 64 per block
template <class C>
__device__ __forceinline__ KContig blocked_rows_tile(const uint16_t* X, int blk_pitch, int64_t tiles_v, int64_t row_blk, int voc_blk, int rows, int tid) {
  KContig c;
  c.rsrc = make_rsrc(X + blk_offset(row_blk, voc_blk, tiles_v) * blk_pitch);
  c.hi_bytes = static_cast<uint32_t>(kBlkElems * 2 * blk_pitch - 4 * 128);        // from the fourth step of a block to the next block
  const uint32_t kofs = ring2_kofs(tid);
#pragma unroll
  for (int i = 0; i < 4; ++i) c.off[i] = (static_cast<uint32_t>(ring2_row<C>(ring2_row<C>(i, 0) < rows ? i : 0, tid)) * 256u + kofs) * 2u;
  return c;
}

// A tile's accumulators go out as float32 rows, `ld` floats apart from `out` on (or are added to what is there); rows and cols
// of them exist, cols a multiple of 4.  A 16x16 block's registers cover 64 bytes of four rows each; stored like that, half a
// line at a time, they kept the dW tiles of short selections waiting (725 rows of 2048 against 151 936: both products 2.1
// ms, through LDS 1.3 ms).  Every wavefront turns its 128 x 64 block through its own part of LDS, 32 rows at a time, and
// stores 256 bytes of four rows.  In a tile that exists as a whole nothing depends on the row: what is there already is
// under way during the turn, and a piece's LDS reads and stores go out together (waiting for each of 32 pieces by itself:
// both products of 725 rows of 2048 that add to dW 1155 us, together 1020; 64 rows without adding 459 and 443).  With `past` what is there is read
// past the caches, which leaves them to the operands (see past_caches).  Such a piece is addressed by 32-bit offsets from the wavefront's first row; rows farther apart than
// kPieceLd take the way of the tiles that end early, with 64-bit addresses.
constexpr int kTurnBytes = 32 * 64 * 4;                              // 32 rows of 64 floats per wavefront
constexpr int64_t kPieceLd = int64_t{1} << 22;                       // floats
static_assert(((Cfg::WTM - 1) * kPieceLd + Cfg::WTN) * 4 < int64_t{1} << 31, "the last row of a wavefront's block is in reach");
static_assert(Cfg::WTN == 64 && Cfg::WM * Cfg::WN == 8 && 8 * kTurnBytes <= 2 * Cfg::BM * 128, "the turn fits two stages of an operand");
// 32 rows (blocks 2 h and 2 h + 1) of a wavefront's accumulators into its part of LDS, and four columns of four rows (4 i + lane /
// 16) back.  The 16-byte unit u of row r lies in unit u ^ 4 ((r >> 2) & 3): neither side meets a bank twice.
__device__ __forceinline__ void turn_in(const floatx4 (&acc)[Cfg::MI][Cfg::NI], int h, char* turn, int lane) {
#pragma unroll
  for (int bj = 0; bj < Cfg::NI; ++bj)
#pragma unroll
    for (int bi = 0; bi < 2; ++bi)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        *reinterpret_cast<float*>(turn + (bi * 16 + (lane >> 4) * 4 + r) * 256 + (((bj * 4 + ((lane >> 2) & 3)) ^ (4 * (lane >> 4))) * 16) + (lane & 3) * 4) =
            acc[h * 2 + bi][bj][r];
  __builtin_amdgcn_wave_barrier();
}
__device__ __forceinline__ floatx4 turn_out(const char* turn, int i, int lane) {
  return *reinterpret_cast<const floatx4*>(turn + (i * 4 + (lane >> 4)) * 256 + (((lane & 15) ^ (4 * (i & 3))) * 16));
}
// dW that is added to is read past the caches (two updates of which the second adds, 203 rows of 2048 1454 -> 1380 us, 300 1950 -> 1885, 725 rows four times 5.82 ->
// 5.73 ms) unless its rows start in the middle of 64 bytes: then every piece of a row shares lines with its neighbours, which read them once more.  Four updates of 200
// rows of 2048 against 115 915, first of all through the caches, past them: 2056 columns 1943.6 and 2199.1 us (both products), 3592 against 60 001 1777.9 and
// 2136.5, but 2064 1861.1 and 1930.8 in an update of 2966.7 and 2806.  A dW that the memory-side cache holds is read past the others all the same: eight of 367 rows
// of 1096 against 50 001 (209 MiB) 2461 us and 2383.
__device__ __forceinline__ bool past_caches(int d, int V) { return d % 16 == 0 || !beyond_cache(d, V, int64_t{128} << 20); }   // twice that in dW
// `turn` is the wavefront's own part of LDS
template <class C>
__device__ __forceinline__ void store_acc_f32(const floatx4 (&acc)[C::MI][C::NI], int tid, char* turn, float* out, int64_t ld, int64_t rows, int cols,
                                              int accumulate, bool past) {
  static_assert(C::WTM == Cfg::WTM && C::WTN == Cfg::WTN, "the turn is written for these");
  typedef float f32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));   // dW has the alignment of a float
  const int lane = tid & 63, wave = tid >> 6;
  const int r0 = wave / C::WN * C::WTM, c0 = wave % C::WN * C::WTN + (lane & 15) * 4;
  const bool whole = rows >= C::BM && cols >= C::BN && ld <= kPieceLd;   // the same for every thread
  float* const dst = out + (r0 + (lane >> 4)) * ld + c0;
  constexpr int kPieces = C::MI / 2;
  // Each case is a run of its own: with the branches inside, the waits cannot tell what is under way and are for everything, the stores of
  // the piece before included.
  auto pieces = [&](auto add, auto past) {
    constexpr bool kAdd = decltype(add)::value;
    constexpr int kRead = decltype(past)::value ? kStream : kCached;
    // (one offset a lane and one a piece: 32 addresses of 64 bits would be a quarter of the registers)
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    const int w_row = __builtin_amdgcn_readfirstlane(r0), w_col = __builtin_amdgcn_readfirstlane(wave) % C::WN * C::WTN;
    const __amdgpu_buffer_rsrc_t rsrc = make_rsrc(out + w_row * ld + w_col);
    const int at = static_cast<int>((lane >> 4) * ld + (lane & 15) * 4) * 4, step = static_cast<int>(ld) * 16;   // four rows
    floatx4 have[8];                                                 // what is there already, a piece ahead
    auto fetch = [&](int h) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        have[i] = __builtin_bit_cast(floatx4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, at, (h * 8 + i) * step, kRead));
    };
    if constexpr (kAdd) fetch(0);
#pragma unroll
    for (int h = 0; h < kPieces; ++h) {
      turn_in(acc, h, turn, lane);
      floatx4 x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = turn_out(turn, i, lane);
      if constexpr (kAdd) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] += have[i];
        if (h + 1 < kPieces) fetch(h + 1);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, x[i]), rsrc, at, (h * 8 + i) * step, kStream);
      }
      __builtin_amdgcn_wave_barrier();
    }
  };
  if (whole && accumulate && past) {
    pieces(std::true_type(), std::true_type());
  } else if (whole && accumulate) {
    pieces(std::true_type(), std::false_type());
  } else if (whole) {
    pieces(std::false_type(), std::false_type());
  } else {
#pragma unroll
    for (int h = 0; h < kPieces; ++h) {
      turn_in(acc, h, turn, lane);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const floatx4 x = turn_out(turn, i, lane);
        if (r0 + h * 32 + i * 4 + (lane >> 4) < rows && c0 < cols) {
          f32x4_a4* const at = reinterpret_cast<f32x4_a4*>(dst + (h * 32 + i * 4) * ld);
          *at = accumulate ? x + *at : x;
        }
      }
      __builtin_amdgcn_wave_barrier();
    }
  }
}
// More rows, whose products are longer than the stores, lose more by what the stores push out of the caches (455 rows of 2680 242 -> 252 us the pass).
__device__ __forceinline__ bool store_lines(int d, int rows) { return d % 64 == 0 || rows > 256; }
// The same into rows of bf16: eight columns of eight rows to a store, 128 bytes a row.  Sums are rounded once; what is added to was rounded by
// whoever wrote it.  The rows are 16-byte aligned.  `whole_lines`: stores past the caches, which is what pays where a piece of a row is lines of its own.  (Where rows start anywhere in a
// line, neighbours share one, and the caches put it together: both products of 31 rows of 2456 against 56 239 184 us, through the caches 120, dW of 200 of 3592 against 120 001
// 427 and 318; what they push out of the caches costs the next call's logits 30 to 45.)
template <class C>
__device__ __forceinline__ void store_acc_bf16(const floatx4 (&acc)[C::MI][C::NI], int tid, char* turn, uint16_t* out, int64_t ld, int64_t rows, int cols, int accumulate,
                                               bool whole_lines) {
  static_assert(C::WTM == Cfg::WTM && C::WTN == Cfg::WTN, "the turn is written for these");
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int w_row = wave / C::WN * C::WTM, c0 = wave % C::WN * C::WTN + (lane & 7) * 8;
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  // (a store's policy is part of the instruction)
  auto pieces = [&](auto stream) {
    constexpr int kWrite = decltype(stream)::value ? kStream : kCached;
#pragma unroll
    for (int h = 0; h < C::MI / 2; ++h) {
      turn_in(acc, h, turn, lane);
      const __amdgpu_buffer_rsrc_t rsrc = make_rsrc(out + (w_row + h * 32) * ld);   // 32 rows are in reach of 32 bits
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = i * 8 + (lane >> 3), unit = (lane & 7) * 2, turned = 4 * ((r >> 2) & 3);
        floatx4 lo = *reinterpret_cast<const floatx4*>(turn + r * 256 + (unit ^ turned) * 16);
        floatx4 hi = *reinterpret_cast<const floatx4*>(turn + r * 256 + ((unit + 1) ^ turned) * 16);
        if (w_row + h * 32 + r < rows && c0 < cols) {                // d is a multiple of 8: eight columns are all inside or all outside
          const int at = (r * static_cast<int>(ld) + c0) * 2;
          if (accumulate) {
            const u32x4 x = __builtin_amdgcn_raw_buffer_load_b128(rsrc, at, 0, kStream);
            lo += floatx4{__uint_as_float(x[0] << 16), __uint_as_float(x[0] & 0xffff0000u), __uint_as_float(x[1] << 16), __uint_as_float(x[1] & 0xffff0000u)};
            hi += floatx4{__uint_as_float(x[2] << 16), __uint_as_float(x[2] & 0xffff0000u), __uint_as_float(x[3] << 16), __uint_as_float(x[3] & 0xffff0000u)};
          }
          __builtin_amdgcn_raw_buffer_store_b128(u32x4{pack_bf16x2(lo[0], lo[1]), pack_bf16x2(lo[2], lo[3]), pack_bf16x2(hi[0], hi[1]), pack_bf16x2(hi[2], hi[3])}, rsrc, at, 0, kWrite);
        }
      }
      __builtin_amdgcn_wave_barrier();
    }
  };
  if (whole_lines) pieces(std::true_type());
  else pieces(std::false_type());
}
template <class C>
__device__ __forceinline__ void store_dw(const floatx4 (&acc)[C::MI][C::NI], int tid, char* turn, float* out, int64_t ld, int64_t rows, int cols, int accumulate, bool past, bool) {
  store_acc_f32<C>(acc, tid, turn, out, ld, rows, cols, accumulate, past);
}
template <class C>
__device__ __forceinline__ void store_dw(const floatx4 (&acc)[C::MI][C::NI], int tid, char* turn, uint16_t* out, int64_t ld, int64_t rows, int cols, int accumulate, bool, bool whole_lines) {
  store_acc_bf16<C>(acc, tid, turn, out, ld, rows, cols, accumulate, whole_lines);
}
typedef uint32_t u32x2_a2 __attribute__((ext_vector_type(2), aligned(2)));     // dH has the alignment of its entries
// What the sliced products leave behind: partial sums in blocks of 256 x 256 floats [slice][row tile][column tile].
struct DhSlices {
  int n;                // slices of the vocabulary (1: the tiles write dH themselves)
  int voc_blks;         // vocabulary blocks of 256 per slice (the last slice may have fewer)
  float* part;
};
// tile_m counts the chunk's live blocks of rows, of m_rows rows, nobody looks at those behind; orig_blk is the block's place in the chunk.
// ONE_HOT: the taken token's term is added in float32 here (g_c, ids), else it lies in the operand.
template <bool ONE_HOT>
__device__ __forceinline__ void dh_tile(int tile_m, int m_rows, int orig_blk, int tile_n, int slice, const DhSlices& sl, int tiles_r, int tiles_d,
                                        const uint16_t* __restrict__ dZ, int blk_pitch, int64_t Vp,
                                        const uint16_t* __restrict__ W, int d, int V, uint16_t* __restrict__ dH,
                                        const int32_t* __restrict__ rowsel, int64_t c0, int64_t rows,
                                        const int32_t* __restrict__ ids, const float* __restrict__ g_c,
                                        const float* __restrict__ sc, bool w_once, uint16_t* lds) {
  using C = Cfg;
  const int64_t m0 = static_cast<int64_t>(orig_blk) * C::BM;
  const int n0 = tile_n * C::BN;
  const int voc_blk = slice * sl.voc_blks, tiles_v = static_cast<int>(Vp >> 8);
  const int k_len = min(sl.voc_blks, tiles_v - voc_blk) * 256;       // a multiple of 256, at least 256
  int tid = cut_thread<C>(m_rows, d - n0);
  const KContig ca = blocked_rows_tile<C>(dZ, blk_pitch, tiles_v, tile_m, voc_blk, m_rows, tid);
  KMajor kb;
  kb.base = reinterpret_cast<const char*>(W + static_cast<int64_t>(voc_blk) * 256 * d + n0);
  kb.ld_bytes = static_cast<int64_t>(d) * 2;
  kb.hi_bytes = 0;
  kb.k_rows = V - voc_blk * 256;                                     // dz is zero for vocabulary ids past V
  kb.n_units = min(32, (d - n0) / 8);
  floatx4 acc[C::MI][C::NI];
  zero_acc<C>(acc);
  // the third LDS stage goes to W: every group of row tiles streams all of it (twice the bytes of the [rows, V] operand).  With one
  // row tile W is read once: past the caches where it is larger than they are, so that the operand, which every column tile
  // reads, stays there (both products of 203 rows of 3584 762 -> 707 us, of 60 rows of 2048 449 -> 384; with up to four row tiles
  // 725 rows that add to dW gain 1.7 %, 1000 rows lose 1 to 3).
  // Up to half a tile of rows or columns is multiplied by half of the wavefronts only, which halves the time of the matrix cores: every SIMD has one of either
  // half.  (With the same loop for all numbers of rows 203 and 725 rows take 0.4 % longer.)
  const bool cut = m_rows <= C::WTM || d - n0 <= C::BN / 2;
  if (cut && w_once) mfma_mainloop_mixed<C, false, true, 2, true, true>(ca, KMajor{}, KContig{}, kb, k_len, lds, acc, tid, m_rows, d - n0);
  else if (cut) mfma_mainloop_mixed<C, false, true, 2, false, true>(ca, KMajor{}, KContig{}, kb, k_len, lds, acc, tid, m_rows, d - n0);
  else if (w_once) mfma_mainloop_mixed<C, false, true, 2, true>(ca, KMajor{}, KContig{}, kb, k_len, lds, acc, tid);
  else mfma_mainloop_mixed<C, false, true, 2>(ca, KMajor{}, KContig{}, kb, k_len, lds, acc, tid);
  tid = cut_thread<C>(m_rows, d - n0);
  if (sl.n > 1) {
    float* out = sl.part + ((static_cast<int64_t>(slice) * tiles_r + tile_m) * tiles_d + tile_n) * (C::BM * C::BN);
    store_acc_f32<C>(acc, tid, reinterpret_cast<char*>(lds) + (tid >> 6) * kTurnBytes, out, C::BN, C::BM, C::BN, 0, false);
    return;
  }
  // dH rows leave like the float32 ones: 32 rows at a time through LDS, 128 bytes of four rows to a store, the row numbers,
  // factors and rows of W of a piece fetched together.  (One 2-byte entry after the other, each with its own chain of loads:
  // both products of 39 000 rows of 2048 37.43 ms, like this 37.16, 12 000 rows 11.48 and 11.37.)
  const int lane = tid & 63, wave = tid >> 6;
  char* turn = reinterpret_cast<char*>(lds) + wave * kTurnBytes;
  const int64_t r0 = m0 + wave / C::WN * C::WTM + (lane >> 4);
  const int j = n0 + wave % C::WN * C::WTN + (lane & 15) * 4, jw = min(j, d - 4);   // d is a multiple of 8: four columns are all inside or all outside
#pragma unroll
  for (int h = 0; h < C::MI / 2; ++h) {
    int64_t row[8];
    float g[8], f[8];
    uint2 w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t n = c0 + min(r0 + h * 32 + i * 4, rows - 1);
      row[i] = rowsel ? rowsel[n] : n;
      if constexpr (ONE_HOT) g[i] = g_c[n];
      f[i] = sc ? sc[n] : 1.f;
    }
    if constexpr (ONE_HOT) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {                                  // g = 0 for invalid ids
        const int64_t id = g[i] != 0.f ? ids[row[i]] : 0;
        w[i] = *reinterpret_cast<const uint2*>(W + id * d + jw);
      }
    }
    turn_in(acc, h, turn, lane);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      floatx4 v = turn_out(turn, i, lane);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        v[k] = sc ? f[i] * v[k] : v[k];
        if constexpr (ONE_HOT) {
          const uint32_t wk = k < 2 ? w[i].x : w[i].y;
          if (g[i] != 0.f) v[k] += g[i] * __uint_as_float(k & 1 ? wk & 0xffff0000u : wk << 16);
        }
      }
      if (r0 + h * 32 + i * 4 < rows && j < d)
        *reinterpret_cast<u32x2_a2*>(dH + row[i] * d + j) = u32x2_a2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
    }
    __builtin_amdgcn_wave_barrier();
  }
}
// Hs: the rows of H that go with the rows of dZ (scaled by the keeping pass), in column blocks [d / 256][mcp][256] so that a
// tile's k-rows are one run of memory
// k_len: rows of the packed [rows, V] operand, whole steps of 64 (0 when no block is live); rows: those that exist
// Out: float, or uint16_t for a dW of bf16
template <class Out>
__device__ __forceinline__ void dw_tile(int tile_m, int tile_n, const uint16_t* __restrict__ dZ, int blk_pitch, int64_t mcp, int64_t Vp,
                                        const uint16_t* __restrict__ Hs, int d, int V, int k_len, int rows, Out* __restrict__ dW,
                                        int accumulate, uint16_t* lds) {
  using C = Cfg;
  const int64_t m0 = static_cast<int64_t>(tile_m) * C::BM;
  const int n0 = tile_n * C::BN;
  KMajor ka;                                                         // blocked dZ: k = row of the chunk, entries = vocabulary
  ka.base = reinterpret_cast<const char*>(dZ + blk_offset(0, tile_m, Vp >> 8) * blk_pitch);
  ka.ld_bytes = 512;
  ka.hi_bytes = (Vp >> 8) * kBlkElems * 2 * blk_pitch - 256 * 512;               // from the last row of a block to the block below
  ka.k_rows = k_len;
  ka.n_units = 32;
  KMajor kb;                                                         // rows of H: k = row of the chunk, entries = hidden columns
  kb.base = reinterpret_cast<const char*>(Hs + static_cast<int64_t>(tile_n) * mcp * 256);
  kb.ld_bytes = 512;
  kb.hi_bytes = 0;
  kb.k_rows = rows;                                                  // dz is zero for rows past the chunk
  kb.n_units = min(32, (d - n0) / 8);
  floatx4 acc[C::MI][C::NI];
  zero_acc<C>(acc);
  int tid = cut_thread<C>(C::BM, d - n0);
  if (k_len > 0 && d - n0 <= C::BN / 2) mfma_mainloop_mixed<C, true, true, 1, false, true>(KContig{}, ka, KContig{}, kb, k_len, lds, acc, tid, C::BM, d - n0);
  else if (k_len > 0) mfma_mainloop_mixed<C, true, true, 1>(KContig{}, ka, KContig{}, kb, k_len, lds, acc, tid);
  tid = cut_thread<C>(C::BM, d - n0);
  store_dw<C>(acc, tid, reinterpret_cast<char*>(lds) + (tid >> 6) * kTurnBytes, dW + m0 * d + n0, d, V - m0, d - n0, accumulate, past_caches(d, V), store_lines(d, rows));   // d is a multiple of 8
}

// dW of at most 256 rows.  A tile of 256 x 256 that a compute unit works on alone is products, then stores, and the next tile's first loads wait for these
// stores (a wavefront's memory operations are counted in order): 203 rows of 3584 against 152 064 485 us, of which the products alone are 235 and the
// stores of 2.2 GB 396 (5.5 TB/s, as much as a kernel that only stores such tiles reaches).  Here tiles of 256 x 128 have two workgroups to
// a compute unit, so that one multiplies while the other stores, and a workgroup of its own each, which ends without waiting for its stores: 400
// to 430 us.  K is walked in steps of 32 rows through three LDS stages of 24 KB, loaded two steps ahead, the fragments half a step ahead (read when they are
// wanted: updates of 100 and 203 rows 1 % slower).  (Stored through the caches: 1075 us for
// the update in place of 972.)
using ShortCfg = TileCfg<256, 128, 2, 2>;
constexpr int kShortA = 32 * 512, kShortStage = kShortA + 32 * 256, kShortLds = 3 * kShortStage;
static_assert(2 * kShortLds <= 160 * 1024 && 3 * kTurnBytes <= kShortStage, "two workgroups to a compute unit; the turns of three wavefronts fit a stage");
constexpr int kShortGM = 4, kShortGN = 16;               // tiles that the 64 workgroups of an XCD work on together
template <class Out>
__device__ __forceinline__ void dw_short(const uint16_t* __restrict__ dZ, int blk_pitch, int64_t Vp, int64_t mcp, const uint16_t* __restrict__ Hs, int d, int V,
                                         int tiles_v, int tiles_n, const LiveInfo* __restrict__ info, Out* __restrict__ dW, int accumulate, char* lds) {
  using C = ShortCfg;
  const int total = tiles_v * tiles_n, per = (total + 7) / 8, t = static_cast<int>(blockIdx.x & 7) * per + static_cast<int>(blockIdx.x >> 3);
  if (static_cast<int>(blockIdx.x >> 3) >= per || t >= total) return;
  int tile_m, tile_n;
  tile_of_groups<kShortGM, kShortGN>(t, tiles_v, tiles_n, &tile_m, &tile_n);
  const int k_rows = info->k_rows, nsub = (k_rows + 31) / 32;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / C::WN, wn = wave % C::WN;
  const char* const a0 = reinterpret_cast<const char*>(dZ + blk_offset(0, tile_m, Vp >> 8) * blk_pitch);
  const int64_t blk_row = (Vp >> 8) * kBlkElems * 2 * blk_pitch;                                     // from a block of rows to the next
  const char* const b0 = reinterpret_cast<const char*>(Hs + (static_cast<int64_t>(tile_n >> 1) * mcp) * 256 + (tile_n & 1) * 128);
  // loads (K-major operands as in mfma_mainloop_mixed): one fills two k-rows of A, four of B
  const int ka = 2 * wave + (lane >> 5), kb = 4 * wave + (lane >> 4);                                // + 8 p; + 16 p
  const uint32_t ua = static_cast<uint32_t>((lane & 31) ^ (4 * (ka & 3))), ub = static_cast<uint32_t>((lane & 15) ^ (4 * (kb & 3)) ^ (2 * ((kb >> 3) & 1)));
  auto load = [&](int sub) {
    char* const st = lds + sub % 3 * kShortStage;
    const int k0 = sub * 32;
    const __amdgpu_buffer_rsrc_t ra = make_rsrc(a0 + (k0 >> 8) * blk_row + (k0 & 255) * 512), rb = make_rsrc(b0 + static_cast<int64_t>(k0) * 512);
#pragma unroll
    for (int p = 0; p < 4; ++p)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, reinterpret_cast<uint32_t*>(st + (8 * p + 2 * wave) * 512), 16,
                                               static_cast<uint32_t>(8 * p + ka) * 512u + (ua ^ (2u * (p & 1))) * 16u, 0, 0, kCached);
#pragma unroll
    for (int p = 0; p < 2; ++p)                            // dz is zero for rows that do not exist: the last one in their place
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, reinterpret_cast<uint32_t*>(st + kShortA + (16 * p + 4 * wave) * 256), 16,
                                               static_cast<uint32_t>(min(16 * p + kb, k_rows - 1 - k0)) * 512u + ub * 16u, 0, 0, kCached);
  };
  // fragments through the transposing reads
  const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char*)(lds)));
  const int tq = lane & 3, tj = (lane >> 2) & 3, tg = lane >> 4;
  uint32_t tra[C::MI], trb[C::NI];
#pragma unroll
  for (int i = 0; i < C::MI; ++i)
    tra[i] = lds0 + (tg * 8 + tj) * 512 + (tq & 1) * 8 + (((wm * (C::WTM / 8) + i * 2 + (tq >> 1)) ^ (4 * tj) ^ (2 * (tg & 1))) * 16);
#pragma unroll
  for (int j = 0; j < C::NI; ++j)
    trb[j] = lds0 + kShortA + (tg * 8 + tj) * 256 + (tq & 1) * 8 + (((wn * (C::WTN / 8) + j * 2 + (tq >> 1)) ^ (4 * tj) ^ (2 * (tg & 1))) * 16);
  typedef short short8v __attribute__((ext_vector_type(8)));
  constexpr int HA = C::MI / 2;
  bf16x8 af[2][HA], bfr[2][C::NI];
  auto read = [&](uint32_t addr, auto row_c) {
    short4v lo, hi;
    asm volatile("ds_read_b64_tr_b16 %0, %1" : "=v"(lo) : "v"(addr));
    asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(hi) : "v"(addr), "n"(4 * decltype(row_c)::value));
    const short8v v = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    return __builtin_bit_cast(bf16x8, v);
  };
  using RowA = std::integral_constant<int, 512>;
  using RowB = std::integral_constant<int, 256>;
  auto read_a = [&](int h, uint32_t st) {
#pragma unroll
    for (int i = 0; i < HA; ++i) af[h][i] = read(tra[h * HA + i] + st, RowA{});
  };
  auto read_b = [&](int buf, uint32_t st) {
#pragma unroll
    for (int j = 0; j < C::NI; ++j) bfr[buf][j] = read(trb[j] + st, RowB{});
  };
  auto wait_a = [&](int h) {
#pragma unroll
    for (int i = 0; i < HA; ++i) asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(af[h][i]));
  };
  auto wait_b = [&](int buf) {
#pragma unroll
    for (int j = 0; j < C::NI; ++j) asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(bfr[buf][j]));
  };
  floatx4 acc[C::MI][C::NI];
  zero_acc<C>(acc);
  auto mfmas = [&](int h, int buf) {
#pragma unroll
    for (int i = 0; i < HA; ++i)
#pragma unroll
      for (int jj = 0; jj < C::NI; ++jj) {
        const int j = i & 1 ? C::NI - 1 - jj : jj;
        acc[h * HA + i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(af[h][i], bfr[buf][j], acc[h * HA + i][j], 0, 0, 0);
      }
  };
  auto stage = [&](int sub) { return static_cast<uint32_t>(sub % 3 * kShortStage); };
  // One step: the second half of its A fragments is read under the products of the first, the next step's B and first half under those of the
  // second.  The barrier in between: the next step's loads have landed, and everybody has read this step's stage, which is loaded again.
  auto step = [&](int sub, auto buf_c) {
    constexpr int buf = decltype(buf_c)::value;
    wait_b(buf);
    wait_a(0);
    read_a(1, stage(sub));
    mfmas(0, buf);
    __builtin_amdgcn_sched_barrier(0);
    wait_a(1);
    if (sub + 1 < nsub) {
      if (sub + 2 < nsub) __builtin_amdgcn_s_waitcnt(0x0F70 | 6); else __builtin_amdgcn_s_waitcnt(0x0F70);
      __builtin_amdgcn_s_barrier();
      __builtin_amdgcn_sched_barrier(0);
      if (sub + 3 < nsub) load(sub + 3);
      read_b(buf ^ 1, stage(sub + 1));
      read_a(0, stage(sub + 1));
    }
    mfmas(1, buf);
    __builtin_amdgcn_sched_barrier(0);
  };
  if (nsub > 0) {
    load(0);
    if (nsub > 1) load(1);
    if (nsub > 2) load(2);
    if (nsub > 2) __builtin_amdgcn_s_waitcnt(0x0F70 | 12); else if (nsub > 1) __builtin_amdgcn_s_waitcnt(0x0F70 | 6); else __builtin_amdgcn_s_waitcnt(0x0F70);
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    read_b(0, 0);
    read_a(0, 0);
    for (int sub = 0; sub < nsub; sub += 2) {
      step(sub, std::integral_constant<int, 0>());
      if (sub + 1 < nsub) step(sub + 1, std::integral_constant<int, 1>());
    }
  }
  // the turns lie in the two stages that nobody reads any more and no load is under way to
  char* const turn = lds + (nsub + (wave == 3 ? 1 : 0)) % 3 * kShortStage + (wave == 3 ? 0 : wave) * kTurnBytes;
  const int64_t m0 = static_cast<int64_t>(tile_m) * C::BM;
  const int n0 = tile_n * C::BN;
  store_dw<C>(acc, tile_thread(), turn, dW + m0 * d + n0, d, V - m0, d - n0, accumulate, past_caches(d, V), store_lines(d, k_rows));
}
// Both products in one launch, in groups of 4 x 8 tiles that are worked on together on one XCD.  Every XCD owns a contiguous
// range of the dH tiles (slice after slice, so that its workgroups share a slice of both operands) and behind it the share
// of the dW tiles that evens out the sum (share_dw): dH tiles are long (K = vocabulary, or a slice of it) and few, on their
// own they leave a fifth of the last round idle; they go first and the many short dW tiles fill up.  (Sliced dH tiles and
// dW tiles taking turns instead: +-1 % at 725 rows, 8 % slower at 203.)
// One workgroup per compute unit stays for the whole launch and takes the next place of its XCD's sequence whenever it is done
// (the number of the next place is fetched a tile ahead): a workgroup per tile paid for its start at every tile, of which short
// selections have many short ones, and workgroups without a tile (groups cut off by the edge, places kept free because
// the shares are known on the device only) waited for a whole compute unit like the others.  A workgroup whose sequence is at
// its end goes on with the one that has most left.  203 rows of 3584 1316 -> 845 us, 64 rows of 2048 841 -> 455, 725 rows
// 1098 -> 930, 2000 rows of 3584 3.93 -> 3.52 ms, 39 000 rows of 2048 37.5 -> 36.5 ms.
template <bool ONE_HOT, class Out>
__device__ __forceinline__ void gemm_dh_dw(const uint16_t* __restrict__ dZ, int blk_pitch, int64_t Vp, int64_t mcp, const uint16_t* __restrict__ W,
                                           const uint16_t* __restrict__ Hs, int d, int V, int tiles_v,
                                           int tiles_d, DhSlices sl, int tiles_r, LiveInfo* __restrict__ info, const int32_t* __restrict__ blk_orig,
                                           uint16_t* __restrict__ dH, Out* __restrict__ dW, int accumulate, const int32_t* __restrict__ rowsel,
                                           int64_t c0, int64_t rows, const int32_t* __restrict__ ids, const float* __restrict__ g_c,
                                           const float* __restrict__ sc, uint16_t* lds) {
  const int n_live = info->n_live;                     // live blocks of rows: dH row tiles, dW K blocks
  const int k_rows = info->k_rows, tiles_mn = n_live * tiles_d, tiles_dh = tiles_mn * sl.n;
  // whose sequence of tiles the workgroup takes from, and the sequence: dH tiles, then dW tiles
  int xcd = static_cast<int>(blockIdx.x & 7), first_dh, n_dh, first_dw, n_all;
  auto sequence = [&]() {
    first_dh = dh_first(tiles_dh, sl.n, xcd);
    n_dh = dh_first(tiles_dh, sl.n, xcd + 1) - first_dh;
    first_dw = info->dw.first[xcd];
    n_all = n_dh + info->dw.first[xcd + 1] - first_dw;
  };
  sequence();
  volatile int* const word = reinterpret_cast<volatile int*>(lds);   // wavefront 0's own at the end of a tile
  int taken = threadIdx.x == 0 ? atomicAdd(&info->next[xcd], 1) : 0;
  for (;;) {
    if (threadIdx.x == 0) *word = taken;
    __syncthreads();
    int seq = __builtin_amdgcn_readfirstlane(*word);
    __syncthreads();
    while (seq >= n_all) {                               // the sequence is at its end: on with the one that has most left
      if (threadIdx.x < kWave) {
        const int x = threadIdx.x & 7;
        const int length = dh_first(tiles_dh, sl.n, x + 1) - dh_first(tiles_dh, sl.n, x) + info->dw.first[x + 1] - info->dw.first[x];
        const int left = length - __hip_atomic_load(&info->next[x], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        int most = left;
#pragma unroll
        for (int o = 4; o > 0; o >>= 1) most = max(most, __shfl_xor(most, o, kWave));
        if (most > 0) xcd = __ffsll(static_cast<long long>(__ballot(left == most))) - 1;
        if (threadIdx.x == 0) {
          word[0] = most > 0 ? atomicAdd(&info->next[xcd], 1) : -1;
          word[1] = xcd;
        }
      }
      __syncthreads();
      seq = __builtin_amdgcn_readfirstlane(word[0]);
      xcd = __builtin_amdgcn_readfirstlane(word[1]);
      __syncthreads();
      if (seq < 0) return;
      sequence();
    }
    if (threadIdx.x == 0) taken = atomicAdd(&info->next[xcd], 1);
    int tile_m, tile_n;
    if (seq < n_dh) {
      const int t = first_dh + seq, slice = t / tiles_mn;
      tile_of_groups<kGM, kGN>(t - slice * tiles_mn, n_live, tiles_d, &tile_m, &tile_n);
      dh_tile<ONE_HOT>(tile_m, min(k_rows - tile_m * 256, 256), blk_orig[(c0 >> 8) + tile_m], tile_n, slice, sl, tiles_r, tiles_d, dZ, blk_pitch, Vp, W, d, V, dH, rowsel, c0, rows, ids, g_c, sc, n_live == 1 && beyond_cache(d, V, kDhOnceBytes), lds);
    } else {
      tile_of_groups<kGM, kGN>(first_dw + seq - n_dh, tiles_v, tiles_d, &tile_m, &tile_n);
      dw_tile(tile_m, tile_n, dZ, blk_pitch, mcp, Vp, Hs, d, V, dw_k(k_rows), k_rows, dW, accumulate, lds);
    }
  }
}

// The slices' partial sums of dH added up in slice order, with what the tile epilogue does otherwise: row factor, one-hot
// part, bf16 row through the selection.  One workgroup per (row of the live blocks, 1024 columns), four columns a thread.
template <bool ONE_HOT>
__device__ __forceinline__ void
dh_reduce(int live_row, int piece, const DhSlices& sl, int tiles_r, int tiles_d, const uint16_t* __restrict__ W, int d, const LiveInfo* __restrict__ info,
          const int32_t* __restrict__ blk_orig, uint16_t* __restrict__ dH, const int32_t* __restrict__ rowsel, int64_t c0,
          int64_t rows, const int32_t* __restrict__ ids, const float* __restrict__ g_c, const float* __restrict__ sc) {
  const int tile_m = live_row >> 8, r = live_row & 255;
  if (tile_m >= info->n_live) return;
  const int64_t m = static_cast<int64_t>(blk_orig[(c0 >> 8) + tile_m]) * 256 + r;
  const int j = (piece * 256 + static_cast<int>(threadIdx.x)) * 4;
  if (m >= rows || j >= d) return;
  const float* src = sl.part + (static_cast<int64_t>(tile_m) * tiles_d + (j >> 8)) * 65536 + r * 256 + (j & 255);
  const int64_t stride = static_cast<int64_t>(tiles_r) * tiles_d * 65536;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int k0 = 0; k0 < sl.n; k0 += 8) {                             // eight slices in flight
    float4 v[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) v[q] = k0 + q < sl.n ? *reinterpret_cast<const float4*>(src + (k0 + q) * stride) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int q = 0; q < 8; ++q) { s.x += v[q].x; s.y += v[q].y; s.z += v[q].z; s.w += v[q].w; }
  }
  const int64_t row = rowsel ? rowsel[c0 + m] : c0 + m;
  const float f = sc ? sc[c0 + m] : 1.f, g = ONE_HOT ? g_c[c0 + m] : 0.f;
  s.x *= f; s.y *= f; s.z *= f; s.w *= f;
  if (ONE_HOT && g != 0.f) {                                                    // g = 0 for invalid ids
    const uint2 w = *reinterpret_cast<const uint2*>(W + static_cast<int64_t>(ids[row]) * d + j);
    s.x += g * __uint_as_float(w.x << 16); s.y += g * __uint_as_float(w.x & 0xffff0000u);
    s.z += g * __uint_as_float(w.y << 16); s.w += g * __uint_as_float(w.y & 0xffff0000u);
  }
  *reinterpret_cast<u32x2_a2*>(dH + row * d + j) = u32x2_a2{pack_bf16x2(s.x, s.y), pack_bf16x2(s.z, s.w)};
}

// ------------------------------------------------------------------ host side
// bytes one chunk of mc rows needs
inline size_t chunk_bytes(int64_t mc, int d, int V, umas_dtype dt) {
  if (dt == UMAS_F32) return align_up(static_cast<size_t>(mc) * V * sizeof(float));
  const int64_t Vp = round_up(V, 256), mcp = round_up(mc, 256);
  return align_up(static_cast<size_t>(mcp) * Vp * 2) + align_up(static_cast<size_t>(mcp) * round_up(d, 256) * 2);
}
// bytes one chunk of mc rows needs whose float32 logits are kept in place of the operand (entropy bonus)
inline size_t logit_chunk_bytes(int64_t mc, int d, int V) {
  return chunk_bytes(mc, d, V, UMAS_BF16) + static_cast<size_t>(round_up(mc, 256)) * round_up(V, 256) * 2;
}

// partial sums of as many slices as are wanted
inline size_t full_part_bytes(int64_t n_sel, int64_t chunk_rows, int d, int V) {
  if (!slices_dh(n_sel, chunk_rows, d)) return 0;
  const int tiles_r = static_cast<int>(cdiv(chunk_rows, 256)), tiles_d = (d + 255) / 256;
  return dh_part_bytes(plan_dh(tiles_r, tiles_d, (V + 255) / 256, SIZE_MAX), tiles_r, tiles_d);
}

}  // namespace
}  // namespace umas
