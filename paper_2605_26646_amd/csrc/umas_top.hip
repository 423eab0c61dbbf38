// The k largest logits of a head and its logsumexp, for selected rows.
//
// The logits of a row fall into groups, those that one lane of the product holds (32 of a tile of 256 x 256, 16 of a small one, a place of every block of 16 in
// a workgroup's part of the vocabulary with few rows).  The product leaves the groups' maxima, the tiles' sums of exponentials and the logits themselves,
// group by group.  Who is among the k largest lies in a group whose maximum is among the k largest maxima, so a row's selection reads the maxima,
// takes a bound that at least k of them reach, and then only the groups that reach it: k of thousands, give or take a few, whatever the logits are.
//
// A logit and its token make one 64-bit key whose order is that of the result: the logit's bits, turned so that they order as whole numbers, above the
// complement of the token.  A wavefront keeps the 64 largest keys it has seen, one to a lane in falling order, and takes only keys beyond its
// k-th: those collect in LDS until there are 64, are sorted (21 exchanges) and merged with what is there (7).
//
// What bounds it: up to 128 rows reading W (one row of 2048 against 151 936 104 us, 6.0 TB/s; 24 rows of 3584 against 152 064 200 us, 5.5 TB/s; 128 rows of 2048, by tiles that fetch W
// in pieces of 128 bytes, 160 us, 3.9 TB/s), then the product (8192 rows of 2048 with 64 places 3.72 ms, 1.37 PFLOP/s, of 3.84; 777 rows of 1544 against 50 001 174 us, whole rounds of
// tiles of 52 us, of 185).
#include <float.h>

#include "umas_f32.h"
#include "umas_few.h"
#include "umas_lanes.h"

namespace umas {
namespace {

// A logit may be any number, down to a type's lowest where a token is masked by it: entries that do not exist are -infinity here, whose exponential is 0, and
// references of sums start at the lowest number, so that no difference is of infinities.
constexpr float kLowest = -FLT_MAX;

typedef unsigned long long TopKey;                            // 0: nothing
__device__ __forceinline__ TopKey key_of(float z, int id) {   // z is a number above -infinity
  const uint32_t u = __float_as_uint(z + 0.f);               // one zero
  const uint32_t ord = u ^ (static_cast<uint32_t>(static_cast<int32_t>(u) >> 31) | 0x80000000u);
  return static_cast<TopKey>(ord) << 32 | (0xFFFFFFFFu - static_cast<uint32_t>(id));
}
__device__ __forceinline__ float logit_of(TopKey k) {
  const uint32_t ord = static_cast<uint32_t>(k >> 32);
  return k ? __uint_as_float(ord & 0x80000000u ? ord ^ 0x80000000u : ~ord) : -INFINITY;
}
__device__ __forceinline__ int token_of(TopKey k) { return k ? static_cast<int>(0xFFFFFFFFu - static_cast<uint32_t>(k)) : -1; }

struct WaveTop {
  TopKey list = 0;
  TopKey least = 0;                                          // keys up to it are not among the k largest (known from outside, or of the list)
  int waiting = 0;
  TopKey* buf;                                               // [128] in LDS, this wavefront's
  int k;
  __device__ __forceinline__ void take(TopKey x) {
    list = merged(list, sorted_desc(x));
    const TopKey kth = __shfl(list, k - 1, kWave);
    least = least > kth ? least : kth;
  }
  // one logit a lane
  __device__ __forceinline__ void offer(float z, int id, bool have) {
    const TopKey x = have && z > -INFINITY ? key_of(z, id) : 0;
    const bool in = x > least;
    const unsigned long long m = __ballot(in);
    if (!m) return;
    const int lane = threadIdx.x & 63;
    if (in) buf[waiting + __popcll(m & ((1ull << lane) - 1))] = x;
    waiting += __popcll(m);
    __builtin_amdgcn_wave_barrier();
    if (waiting < kWave) return;
    const TopKey y = buf[lane], rest = buf[kWave + lane];
    __builtin_amdgcn_wave_barrier();
    waiting -= kWave;
    if (lane < waiting) buf[lane] = rest;
    __builtin_amdgcn_wave_barrier();
    take(y);
  }
  __device__ __forceinline__ void finish() {
    if (!waiting) return;
    const int lane = threadIdx.x & 63;
    take(lane < waiting ? buf[lane] : 0);
    waiting = 0;
  }
};
constexpr int kSelectT = 256, kSelectWaves = kSelectT / kWave;
// The workgroup's lists into wavefront 0's.
__device__ __forceinline__ TopKey merge_waves(TopKey list, TopKey (*s_list)[kWave]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  __syncthreads();
  s_list[wave][lane] = list;
  __syncthreads();
  if (wave == 0)
#pragma unroll
    for (int w = 1; w < kSelectWaves; ++w) list = merged(list, s_list[w][lane]);
  return list;
}

// ------------------------------------------------------------------ bf16: logits in groups
// What a product leaves of its rows: per row and tile (of the vocabulary) G group maxima and a sum of exponentials relative to the largest of them, and the
// logits.  Entries that do not exist hold -infinity; a group of few rows without a number has kLowest for a maximum.
struct Groups {
  float* max;              // [rows][tiles][G]
  float* sum;              // [rows][tiles]
  float* z;                // [rows][tiles][G][E], of the kernel for few rows [rows][tiles][E][G]
  int tiles;
};
constexpr int kGroups = 8;                                   // of a tile: four lane groups, two wavefronts along the vocabulary
template <class C>
constexpr int kEntries = C::MI * 4;
template <class C, bool ALL>
__device__ __forceinline__ void top_tile(const uint16_t* __restrict__ W, const uint16_t* __restrict__ H, int d, int V, const int32_t* __restrict__ rowsel,
                                         int64_t c0, int64_t mc, int tile_m, int tile_n, bool w_once, const Groups& out, const float* __restrict__ bound,
                                         uint16_t* lds) {
  // a wavefront's part of LDS for sixteen rows on their way out: rows of its half of the tile, 16 bytes more to a group and to a row (banks)
  constexpr int kGroupPitch = kEntries<C> * 4 + 16, kRowPitch = 4 * kGroupPitch + 16, kStage = 16 * kRowPitch;
  static_assert(C::WM == 2 && C::BN * (kGroups + 2) * 4 + C::WM * C::WN * kStage <= Ring2Cfg<C>::LDS_BYTES, "maxima, sums and stages fit the tile buffers");
  const int m0 = tile_m * C::BM;
  const int64_t n0 = static_cast<int64_t>(tile_n) * C::BN;
  floatx4 acc[C::MI][C::NI];
  logit_tile<C>(W, H, d, V, rowsel, c0, mc, m0, n0, w_once, lds, acc);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave / C::WN, wn = wave % C::WN;
  float* const s_max = reinterpret_cast<float*>(lds);        // [BN][8]
  float* const s_sum = s_max + C::BN * kGroups;              // [2][BN]
  char* const stage = reinterpret_cast<char*>(s_sum + 2 * C::BN) + wave * kStage;
  __syncthreads();
  const int vbase = m0 + wm * C::WTM + (lane >> 4) * 4;
  if (m0 + C::BM > V) {
#pragma unroll
    for (int i = 0; i < C::MI; ++i)
#pragma unroll
      for (int j = 0; j < C::NI; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (vbase + i * 16 + r >= V) acc[i][j][r] = -INFINITY;
  }
  constexpr float kLog2e = 1.44269504088896341f;
  const int group = wm * 4 + (lane >> 4);
#pragma unroll
  for (int j = 0; j < C::NI; ++j) {
    const int col = wn * C::WTN + j * 16 + (lane & 15);
    float m = acc[0][j][0];
#pragma unroll
    for (int i = 0; i < C::MI; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) m = fmaxf(m, acc[i][j][r]);
    float most = fmaxf(m, kLowest);                          // of the column's four lanes
    most = fmaxf(most, __shfl_xor(most, 16, kWave));
    most = fmaxf(most, __shfl_xor(most, 32, kWave));
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < C::MI; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) s += __builtin_amdgcn_exp2f((acc[i][j][r] - most) * kLog2e);
    s += __shfl_xor(s, 16, kWave);
    s += __shfl_xor(s, 32, kWave);
    s_max[col * kGroups + group] = m;
    if (lane < 16) s_sum[wm * C::BN + col] = s;
    if constexpr (!ALL) {                                    // only groups that reach a bound that k logits are known to reach
      if (n0 + col < mc && m >= bound[n0 + col]) {
        floatx4* const z = reinterpret_cast<floatx4*>(out.z + (((n0 + col) * out.tiles + tile_m) * kGroups + group) * kEntries<C>);
#pragma unroll
        for (int i = 0; i < C::MI; ++i) z[i] = acc[i][j];
      }
    } else {
      char* const mine = stage + (lane & 15) * kRowPitch + (lane >> 4) * kGroupPitch;
#pragma unroll
      for (int i = 0; i < C::MI; ++i) *reinterpret_cast<floatx4*>(mine + i * 16) = acc[i][j];
      __builtin_amdgcn_wave_barrier();
      constexpr int kLanes = C::WTM / 4, kRows = kWave / kLanes, kPerGroup = kLanes / 4;   // lanes to a row, rows to a store, lanes to a group
      const int64_t r0 = n0 + wn * C::WTN + j * 16 + lane / kLanes;
      const int q = lane % kLanes;
#pragma unroll
      for (int i = 0; i < 16 / kRows; ++i)
        if (r0 + i * kRows < mc)
          *reinterpret_cast<floatx4*>(out.z + (((r0 + i * kRows) * out.tiles + tile_m) * kGroups + wm * 4) * kEntries<C> + q * 4) =
              *reinterpret_cast<const floatx4*>(stage + (i * kRows + lane / kLanes) * kRowPitch + q / kPerGroup * kGroupPitch + q % kPerGroup * 16);
      __builtin_amdgcn_wave_barrier();
    }
  }
  __syncthreads();
  if (threadIdx.x < C::BN && n0 + threadIdx.x < mc) {
    const int col = threadIdx.x;
    const floatx4 a = reinterpret_cast<const floatx4*>(s_max)[col * 2], b = reinterpret_cast<const floatx4*>(s_max)[col * 2 + 1];
    const float ma = fmaxf(fmaxf(fmaxf(a[0], a[1]), fmaxf(a[2], a[3])), kLowest), mb = fmaxf(fmaxf(fmaxf(b[0], b[1]), fmaxf(b[2], b[3])), kLowest);
    const float m = fmaxf(ma, mb);
    const int64_t at = (n0 + col) * out.tiles + tile_m;
    reinterpret_cast<floatx4*>(out.max)[at * 2] = a;
    reinterpret_cast<floatx4*>(out.max)[at * 2 + 1] = b;
    out.sum[at] = s_sum[col] * __expf(ma - m) + s_sum[C::BN + col] * __expf(mb - m);
  }
  __syncthreads();
}
template <class C, bool ALL>
__device__ __forceinline__ void top_tiles(const uint16_t* __restrict__ W, const uint16_t* __restrict__ H, int d, int V, const int32_t* __restrict__ rowsel,
                                          int64_t c0, int64_t mc, int first, int tiles_m, int tiles_n, int panel, const Groups& out,
                                          const float* __restrict__ bound, uint16_t* lds, int halved = 0) {
  const bool w_once = tiles_n == 1 && beyond_cache(d, V, kLogitsOnceBytes);
  for (int it = 0; it < kTilesPerWg; ++it) {
    int tile_m, tile_n;
    // halves as in score_tiles: of the last round 129 rows of 3584 291 -> 265 us, 1000 of 2048 554 -> 543, 777 of 1544 222 -> 215, else +- 1 %; at the end of the
    // rows 300 of 2048 319 -> 290, 600 of 3584 681 -> 645, 2100 of 2048 1188 -> 1120
    using Half = std::conditional_t<C::BN == HalfCfg::BN * 2, HalfCfg, HalfNarrowCfg>;
    const HalfTile h = half_tile<Half>(tiles_m, tiles_n, panel, halved, it, mc, &tile_m, &tile_n);
    if (h == HalfTile::kNone) continue;
    if (h == HalfTile::kHalf) top_tile<Half, ALL>(W, H, d, V, rowsel, c0, mc, first + tile_m, tile_n, false, out, bound, lds);
    else top_tile<C, ALL>(W, H, d, V, rowsel, c0, mc, first + tile_m, tile_n, w_once, out, bound, lds);
  }
}
__global__ void __launch_bounds__(Cfg::T)
k_top_tiles(const uint16_t* __restrict__ W, const uint16_t* __restrict__ H, int d, int V, const int32_t* __restrict__ rowsel, int64_t c0, int64_t mc,
            int tiles_m, int tiles_n, int panel, int halved, Groups out) {
  __shared__ __attribute__((aligned(16))) uint16_t lds[kLogitLds / 2];
  top_tiles<Cfg, true>(W, H, d, V, rowsel, c0, mc, 0, tiles_m, tiles_n, panel, out, nullptr, lds, halved);
}
__global__ void __launch_bounds__(Cfg::T)
k_top_tiles_bound(const uint16_t* __restrict__ W, const uint16_t* __restrict__ H, int d, int V, const int32_t* __restrict__ rowsel, int64_t c0, int64_t mc,
                  int first, int tiles_m, int tiles_n, int panel, int halved, Groups out, const float* __restrict__ bound) {
  __shared__ __attribute__((aligned(16))) uint16_t lds[kLogitLds / 2];
  top_tiles<Cfg, false>(W, H, d, V, rowsel, c0, mc, first, tiles_m, tiles_n, panel, out, bound, lds, halved);
}
__global__ void __launch_bounds__(NarrowCfg::T)
k_top_narrow(const uint16_t* __restrict__ W, const uint16_t* __restrict__ H, int d, int V, const int32_t* __restrict__ rowsel, int64_t c0, int64_t mc, int halved, Groups out) {
  __shared__ __attribute__((aligned(16))) uint16_t lds[kNarrowLds / 2];
  top_tiles<NarrowCfg, true>(W, H, d, V, rowsel, c0, mc, 0, out.tiles, 1, kGN, out, nullptr, lds, halved);
}

// A few rows (umas_few.h): a thread's place of every block of 16 entries of its workgroup's part of the vocabulary is a group.
constexpr int kFewGroups = 16;
template <int NI, int PPW>
__global__ void __launch_bounds__(kFewT)
k_top_few(const uint16_t* __restrict__ W, const uint16_t* __restrict__ H, int d, int V, const int32_t* __restrict__ rowsel, int n_sel, int per, Groups out) {
  few_logits<NI, PPW, false>(W, H, d, V, rowsel, n_sel, per, out.z, static_cast<int64_t>(out.tiles) * kFewGroups * per, [&](int n, int place, float m, float most, float sum, float) {
    const int64_t at = static_cast<int64_t>(n) * out.tiles + blockIdx.x;
    out.max[at * kFewGroups + place] = m;
    if (place == 0) out.sum[at] = sum;
  });
}

// ------------------------------------------------------------------ selection
// Where a group's entries lie in the vocabulary, and how many there are.
template <class C>
struct TileGroups {
  static constexpr int G = kGroups;
  __device__ __forceinline__ int entries() const { return kEntries<C>; }
  __device__ __forceinline__ int token(int tile, int g, int e) const { return tile * C::BM + (g >> 2) * C::WTM + (e >> 2) * 16 + (g & 3) * 4 + (e & 3); }
  __device__ __forceinline__ int64_t place(int tile, int g, int e) const { return (static_cast<int64_t>(tile) * G + g) * kEntries<C> + e; }
};
struct FewGroups {
  static constexpr int G = kFewGroups;
  int per;
  __device__ __forceinline__ int entries() const { return per; }
  __device__ __forceinline__ int token(int tile, int g, int e) const { return (tile * per + e) * 16 + g; }
  __device__ __forceinline__ int64_t place(int tile, int g, int e) const { return token(tile, g, e); }
};
struct TopOut {
  const int32_t* rowsel;
  int64_t c0;
  int k;
  int32_t* ids;
  float *logits, *lse;
};
__device__ __forceinline__ void write_top(const TopOut& O, int64_t row, TopKey list) {   // wavefront 0
  const int lane = threadIdx.x & 63;
  if (lane >= O.k) return;
  O.ids[row * O.k + lane] = token_of(list);
  O.logits[row * O.k + lane] = logit_of(list);
}
// A bound that at least k logits of a row reach: the threads of a workgroup take the maximum over the row's tiles in turn, and the k-th largest of these
// 256 numbers is it (k at most 64; with random logits 74 groups of thousands reach the 64th).  By itself, for what is left unwritten, 5 us for 777 rows, 10 for 4096.  `lm`, `ls`: the wavefront's part of the logsumexp.
template <int G>
__device__ __forceinline__ void load_maxima(const float* __restrict__ maxima, int t, float (&x)[G]) {
#pragma unroll
  for (int g = 0; g < G; g += 4) {
    const floatx4 v = *reinterpret_cast<const floatx4*>(maxima + static_cast<int64_t>(t) * G + g);
    x[g] = v[0]; x[g + 1] = v[1]; x[g + 2] = v[2]; x[g + 3] = v[3];
  }
}
template <int G>
__device__ __forceinline__ float row_bound(const float* __restrict__ maxima, const float* __restrict__ sums, int tiles, int k, float (*s_top)[kWave], float& lm, float& ls) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float x = -INFINITY;
  lm = kLowest;
  ls = 0.f;
  for (int t = threadIdx.x; t < tiles; t += kSelectT) {
    float g_max[G];
    load_maxima<G>(maxima, t, g_max);
    float tm = g_max[0];
#pragma unroll
    for (int g = 1; g < G; ++g) tm = fmaxf(tm, g_max[g]);
    x = fmaxf(x, tm);
    if (sums) {
      tm = fmaxf(tm, kLowest);
      const float s = sums[t], M = fmaxf(lm, tm);
      ls = ls * __expf(lm - M) + s * __expf(tm - M);
      lm = M;
    }
  }
  // fewer tiles than there may be places: the groups, dealt out (200 rows, 32 tiles, 64 places: 24 -> 11.5 us; 125 tiles 29 -> 31)
  if (tiles < kWave) {
    x = -INFINITY;
    for (int i = threadIdx.x; i < tiles * G; i += kSelectT) x = fmaxf(x, maxima[i]);
  }
  // the wavefront's 64 maxima, falling; then everybody merges the four lists
  x = sorted_desc(x);
  s_top[wave][lane] = x;
  __syncthreads();
  x = s_top[0][lane];
#pragma unroll
  for (int w = 1; w < kSelectWaves; ++w) x = merged(x, s_top[w][lane]);
  return __shfl(x, k - 1, kWave);
}
__global__ void __launch_bounds__(kSelectT)
k_top_bound(Groups A, int tiles, int k, float* __restrict__ bound) {   // of a row's first tiles
  __shared__ float s_top[kSelectWaves][kWave];
  float lm, ls;
  const int64_t m = blockIdx.x;
  const float b = row_bound<kGroups>(A.max + m * A.tiles * kGroups, nullptr, tiles, k, s_top, lm, ls);
  if (threadIdx.x == 0) bound[m] = b;
}
// A workgroup to a row: the groups that reach its bound are listed, and the wavefronts go through their entries.  The row's logsumexp comes from the tiles'
// sums on the way.  9 us for one row, a chain of reads and exchanges (through LDS one more); 8192 rows with 64 places 106 us.
// `written`: the bound below which k_top_tiles_bound left a group's logits unwritten (NULL: all are there).  The row's own can lie below it, as of few tiles it is one of groups
// and of many one of tiles, of which the large logits may share one; k logits reach either, so the larger of the two serves and only what was written is read.
constexpr int kAtOnce = 4;                                   // loads of entries under way
template <class Map>
__global__ void __launch_bounds__(kSelectT)
k_top_row(Groups A, Map map, int V, const float* __restrict__ written, TopOut O) {
  __shared__ TopKey s_buf[kSelectWaves][2 * kWave];
  __shared__ TopKey s_list[kSelectWaves][kWave];
  __shared__ float s_top[kSelectWaves][kWave], s_m[kSelectWaves], s_s[kSelectWaves];
  __shared__ int s_group[kSelectT * Map::G];
  __shared__ int s_n;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t m = blockIdx.x, n = O.c0 + m, row = O.rowsel ? O.rowsel[n] : n;
  const float* const maxima = A.max + m * A.tiles * Map::G;
  if (threadIdx.x == 0) s_n = 0;
  float lm, ls;
  float bound = row_bound<Map::G>(maxima, A.sum + m * A.tiles, A.tiles, O.k, s_top, lm, ls);
  if (written) bound = fmaxf(bound, written[m]);
  {
    const float M = wave_max(lm), sum = wave_sum(ls * __expf(lm - M));
    if (lane == 0) { s_m[wave] = M; s_s[wave] = sum; }
  }
  WaveTop top;
  top.buf = s_buf[wave];
  top.k = O.k;
  top.least = bound > -INFINITY ? key_of(bound, -1) : 0;     // below every logit of that size
  const int E = map.entries();
  const int side = E <= 16 ? 16 : E <= 32 ? 32 : 64, at_once = kWave / side;   // lanes to a group, groups to a load
  const int sub = lane / side, e0 = lane % side;
  const float* const z = A.z + m * A.tiles * Map::G * E;
  for (int t0 = 0; t0 < A.tiles; t0 += kSelectT) {
    const int t = t0 + threadIdx.x;
    if (t < A.tiles) {
      float g_max[Map::G];
      load_maxima<Map::G>(maxima, t, g_max);
#pragma unroll
      for (int g = 0; g < Map::G; ++g)
        if (g_max[g] >= bound && g_max[g] > -INFINITY) s_group[atomicAdd(&s_n, 1)] = t * Map::G + g;
    }
    __syncthreads();
    const int count = s_n;
    for (int i = wave * at_once; i < count; i += kSelectWaves * at_once * kAtOnce)
      for (int f = 0; f < E; f += side) {
        float v[kAtOnce];
        int id[kAtOnce];
#pragma unroll
        for (int b = 0; b < kAtOnce; ++b) {
          const int q = i + b * kSelectWaves * at_once + sub, e = f + e0, g = q < count ? s_group[q] : 0;
          id[b] = q < count && e < E ? map.token(g / Map::G, g % Map::G, e) : V;
          v[b] = id[b] < V ? z[map.place(g / Map::G, g % Map::G, e)] : 0.f;
        }
#pragma unroll
        for (int b = 0; b < kAtOnce; ++b) top.offer(v[b], id[b], id[b] < V);
      }
    __syncthreads();
    if (threadIdx.x == 0) s_n = 0;
    __syncthreads();
  }
  top.finish();
  const TopKey list = merge_waves(top.list, s_list);
  if (wave == 0) write_top(O, row, list);
  if (threadIdx.x != 0) return;
  float M = s_m[0], sum = s_s[0];
  for (int w = 1; w < kSelectWaves; ++w) {
    const float X = fmaxf(M, s_m[w]);
    sum = sum * __expf(M - X) + s_s[w] * __expf(s_m[w] - X);
    M = X;
  }
  O.lse[row] = M + logf(sum);
}

// float32: float64 logits [rows][V].  A workgroup goes over a part of a row's vocabulary, its wavefronts 256 entries at a time in turn: list[row][part] gets the 64
// largest keys.
__global__ void __launch_bounds__(kSelectT)
k_top_select(const double* __restrict__ Z, int V, int k, int parts, int per, TopKey* __restrict__ lists) {
  __shared__ TopKey s_buf[kSelectWaves][2 * kWave];
  __shared__ TopKey s_list[kSelectWaves][kWave];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t m = blockIdx.x;
  const int part = blockIdx.y, v0 = part * per, v1 = min(v0 + per, V);
  WaveTop top;
  top.buf = s_buf[wave];
  top.k = k;
  for (int b = v0 + wave * 256; b < v1; b += kSelectWaves * 256) {
    float z[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) z[q] = b + q * 64 + lane < v1 ? static_cast<float>(Z[m * V + b + q * 64 + lane]) : 0.f;
#pragma unroll
    for (int q = 0; q < 4; ++q) top.offer(z[q], b + q * 64 + lane, b + q * 64 + lane < v1);
  }
  top.finish();
  const TopKey all = merge_waves(top.list, s_list);
  if (wave == 0) lists[(m * parts + part) * kWave + lane] = all;
}
__global__ void __launch_bounds__(kSelectT)
k_top_merge(const TopKey* __restrict__ lists, int parts, TopOut O) {
  __shared__ TopKey s_list[kSelectWaves][kWave];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t m = blockIdx.x, n = O.c0 + m, row = O.rowsel ? O.rowsel[n] : n;
  TopKey list = 0;
  for (int p = wave; p < parts; p += kSelectWaves) list = merged(list, lists[(m * parts + p) * kWave + lane]);
  list = merge_waves(list, s_list);
  if (wave == 0) write_top(O, row, list);
}
// what the call defines on rows that are not selected
__global__ void __launch_bounds__(256)
k_top_clear(int32_t* __restrict__ ids, float* __restrict__ logits, float* __restrict__ lse, int64_t n_rows, int k) {
  const int64_t stride = static_cast<int64_t>(gridDim.x) * 256, i0 = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  for (int64_t i = i0; i < n_rows * k; i += stride) { ids[i] = -1; logits[i] = 0.f; }
  for (int64_t i = i0; i < n_rows; i += stride) lse[i] = 0.f;
}

// ------------------------------------------------------------------ host side
constexpr int64_t kTopChunkRows = 4096;
// workgroups to a row: as many as fill the chip, 256 entries to a wavefront at the least
constexpr int64_t kSelectLists = 2048;
int select_parts(int64_t rows, int V) { return static_cast<int>(std::min<int64_t>(std::max<int64_t>(kSelectLists / rows, 1), cdiv(V, kSelectWaves * 256))); }
struct TopWs {
  TopKey* lists;                                             // float32
  double* z64;
  char* room;                                                // ... for the scores' parts
  size_t room_bytes;
  Groups groups;                                             // bf16
  float* bound;
  size_t bytes;
};
// Tiles of the vocabulary whose logits are all kept: they give the bound that leaves most of the others unwritten.  With n entries in them a group of E = 32 among
// the others reaches the bound with a probability of about E k / n, and stores 16 bytes at a time, which costs about three times what the rows of whole tiles do:
// n^2 = 3 E k V; then whole rounds of compute units.  With the bound and all logits written: 8192 rows of 2048 against 151 936, 64 places 4.19 and 4.75 ms, 1000 rows, one place
// 543 and 617 us, 300 rows, 32 places 321 and 335, 777 rows of 1544 against 50 001 215 and 227, 2000 rows of 1024 against 32 000 160 and 170, 129 rows of 3584 265 and 282.
int first_tiles(int tiles, int tiles_n, int k) {
  const double n = sqrt(3.0 * kEntries<Cfg> * k * (static_cast<double>(tiles) * 256.0));
  const int round = static_cast<int>(cdiv(std::max(device_cus(), 1), tiles_n));
  const int first = static_cast<int>(round_up(static_cast<int64_t>(n / 256.0) + 1, round));
  return first * 2 > tiles ? tiles : first;
}
void carve(Carver& c, TopWs& w, int64_t rows, int d, int V, umas_dtype dt) {
  w = TopWs{};
  if (dt == UMAS_BF16) {
    // as many groups and entries as any of the kernels has: tiles of 256 or 128 entries, up to kFewMostTiles workgroups whose parts end unevenly
    const bool few = rows <= few_rows(d);
    const int64_t tiles = few ? kFewMostTiles : round_up(V, 256) / 128, groups = few ? int64_t{kFewMostTiles} * kFewGroups : tiles * kGroups;
    w.groups.max = c.take<float>(static_cast<size_t>(rows) * groups);
    w.groups.sum = c.take<float>(static_cast<size_t>(rows) * tiles);
    w.bound = c.take<float>(rows);
    w.groups.z = c.take<float>(few ? few_floats(rows, V) : static_cast<size_t>(rows) * round_up(V, 256));
  } else {
    w.lists = c.take<TopKey>(static_cast<size_t>(std::max(rows, kSelectLists)) * kWave);
    w.z64 = c.take<double>(static_cast<size_t>(rows) * V);
    w.room_bytes = align_up(f32::score_room(rows, V));
    w.room = c.take<char>(w.room_bytes);
  }
  w.bytes = c.off;
}
size_t top_bytes(int64_t n_sel, int64_t cap, int d, int V, umas_dtype dt) {
  Carver c(nullptr);
  TopWs w;
  carve(c, w, std::min(std::max<int64_t>(n_sel, 1), cap), d, V, dt);
  return w.bytes;
}

}  // namespace
}  // namespace umas

using namespace umas;

extern "C" size_t umas_top_logits_workspace_bytes_min(int64_t n_sel, int32_t d, int32_t V, int32_t k, umas_dtype dtype) {
  if (n_sel < 0 || d < 1 || V < 1 || k < 1 || k > UMAS_MAX_TOP) return 0;
  return top_bytes(n_sel, 256, d, V, dtype);
}
extern "C" size_t umas_top_logits_workspace_bytes(int64_t n_sel, int32_t d, int32_t V, int32_t k, umas_dtype dtype) {
  if (n_sel < 0 || d < 1 || V < 1 || k < 1 || k > UMAS_MAX_TOP) return 0;
  return top_bytes(n_sel, kTopChunkRows, d, V, dtype);
}

extern "C" umas_status umas_top_logits(const void* H, const void* W, umas_dtype dtype, int64_t n_rows, int32_t d, int32_t V, const int32_t* rowsel,
                                       int64_t n_sel, int32_t k, int32_t* top_ids, float* top_logits, float* lse, void* workspace,
                                       size_t workspace_bytes, void* hip_stream) {
  UMAS_REQUIRE(k >= 1 && k <= UMAS_MAX_TOP, UMAS_ESHAPE, "k=%d outside [1,%d]", k, UMAS_MAX_TOP);
  umas_status s = check_model_args(H, W, dtype, n_rows, d, V, top_ids, rowsel, n_sel);
  if (s != UMAS_OK) return s;
  UMAS_REQUIRE((top_logits && lse) || n_rows == 0, UMAS_EINVAL, "top_logits and lse must not be NULL");
  UMAS_REQUIRE(n_sel < (1LL << 31), UMAS_ESHAPE, "at most 2^31-1 selected rows");
  s = check_ws(workspace, workspace_bytes, umas_top_logits_workspace_bytes_min(n_sel, d, V, k, dtype));
  if (s != UMAS_OK) return s;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  prof_mark(st);
  if (rowsel && n_rows > 0) {
    hipLaunchKernelGGL(k_top_clear, dim3(static_cast<unsigned>(std::min<int64_t>(n_rows * k / 256 + 1, 4096))), dim3(256), 0, st, top_ids, top_logits, lse, n_rows, k);
    UMAS_LAUNCHED("k_top_clear");
  }
  if (n_sel == 0) return UMAS_OK;
  int64_t cap = std::min(n_sel, kTopChunkRows);
  while (cap > 256 && top_bytes(n_sel, cap, d, V, dtype) > workspace_bytes) cap = std::max<int64_t>(round_up(cap / 2, 256), 256);
  Carver c(workspace);
  TopWs w;
  carve(c, w, cap, d, V, dtype);
  for (int64_t c0 = 0; c0 < n_sel; c0 += cap) {
    const int64_t rows = std::min(cap, n_sel - c0);
    const TopOut O{rowsel, c0, k, top_ids, top_logits, lse};
    const dim3 grid(static_cast<unsigned>(rows));
    if (dtype == UMAS_BF16) {
      const uint16_t *Wb = static_cast<const uint16_t*>(W), *Hb = static_cast<const uint16_t*>(H);
      Groups A = w.groups;
      if (cap <= few_rows(d)) {                              // one chunk
        A.tiles = few_workgroups(V);
        const int per = few_per(V, A.tiles);
        with_few(d, rows, [&](auto ni, auto ppw) {
          hipLaunchKernelGGL((k_top_few<decltype(ni)::value, decltype(ppw)::value>), dim3(A.tiles), dim3(kFewT), 0, st, Wb, Hb, d, V, rowsel, static_cast<int>(rows), per, A);
        });
        UMAS_LAUNCHED("k_top_few");
        hipLaunchKernelGGL(k_top_row<FewGroups>, grid, dim3(kSelectT), 0, st, A, FewGroups{per}, V, nullptr, O);
      } else if (rows <= NarrowCfg::BN) {
        A.tiles = static_cast<int>(cdiv(V, NarrowCfg::BM));
        // (100 rows of 1024 against 32 000 23 -> 19 us, 70 of 3584 against 152 064 229 -> 223, 128 of 2048 169 -> 163, 121 of 3584 equal)
        const int halved = rows > HalfNarrowCfg::BN ? halved_tiles(A.tiles, 1, 2) : 0;
        hipLaunchKernelGGL(k_top_narrow, score_grid(A.tiles, 1, kGN, halved), dim3(NarrowCfg::T), 0, st, Wb, Hb, d, V, rowsel, c0, rows, halved, A);
        UMAS_LAUNCHED("k_top_narrow");
        hipLaunchKernelGGL(k_top_row<TileGroups<NarrowCfg>>, grid, dim3(kSelectT), 0, st, A, TileGroups<NarrowCfg>{}, V, nullptr, O);
      } else {
        A.tiles = static_cast<int>(cdiv(V, Cfg::BM));
        const int tiles_n = static_cast<int>(cdiv(rows, Cfg::BN)), panel = row_panel(tiles_n, d);
        const int first = first_tiles(A.tiles, tiles_n, k);
        const int halved = halved_tiles(first, tiles_n);
        hipLaunchKernelGGL(k_top_tiles, score_grid(first, tiles_n, panel, halved), dim3(Cfg::T), 0, st, Wb, Hb, d, V, rowsel, c0, rows, first, tiles_n, panel, halved, A);
        UMAS_LAUNCHED("k_top_tiles");
        if (first < A.tiles) {
          hipLaunchKernelGGL(k_top_bound, grid, dim3(kSelectT), 0, st, A, first, k, w.bound);
          UMAS_LAUNCHED("k_top_bound");
          const int rest = A.tiles - first, halved = halved_tiles(rest, tiles_n);
          hipLaunchKernelGGL(k_top_tiles_bound, score_grid(rest, tiles_n, panel, halved), dim3(Cfg::T), 0, st, Wb, Hb, d, V, rowsel, c0, rows, first, rest, tiles_n, panel,
                             halved, A, w.bound);
          UMAS_LAUNCHED("k_top_tiles_bound");
        }
        hipLaunchKernelGGL(k_top_row<TileGroups<Cfg>>, grid, dim3(kSelectT), 0, st, A, TileGroups<Cfg>{}, V, first < A.tiles ? w.bound : nullptr, O);
      }
      UMAS_LAUNCHED("k_top_row");
    } else {
      const int parts = select_parts(rows, V), per = static_cast<int>(round_up(cdiv(V, parts), 256));
      const float* Hf = static_cast<const float*>(H) + (rowsel ? 0 : c0 * d);
      s = f32::score(static_cast<const float*>(W), Hf, d, V, rowsel ? rowsel + c0 : nullptr, rows, nullptr, w.room, w.room_bytes,
                     f32::ScoreOut{w.z64, nullptr, nullptr, nullptr, nullptr, nullptr, rowsel ? lse : lse + c0, nullptr}, st);
      if (s != UMAS_OK) return s;
      hipLaunchKernelGGL(k_top_select, dim3(static_cast<unsigned>(rows), parts), dim3(kSelectT), 0, st, w.z64, V, k, parts, per, w.lists);
      UMAS_LAUNCHED("k_top_select");
      hipLaunchKernelGGL(k_top_merge, grid, dim3(kSelectT), 0, st, w.lists, parts, O);
      UMAS_LAUNCHED("k_top_merge");
    }
  }
  return UMAS_OK;
}
