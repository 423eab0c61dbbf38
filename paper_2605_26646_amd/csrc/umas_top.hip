// The k largest logits of a head and its logsumexp, for selected rows.
//
// A logit and its token make one 64-bit key whose order is that of the result: the logit's bits, turned so that they order as whole numbers, above the
// complement of the token.  A wavefront keeps the 64 largest keys it has seen, one to a lane in falling order, and looks only at logits that reach its
// k-th: those collect in LDS until there are 64, are sorted (21 exchanges) and merged with what is there (7).
#include "umas_f32.h"
#include "umas_logits.h"

namespace umas {
namespace {

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

__device__ __forceinline__ TopKey exchange(TopKey x, int j, bool larger) {
  const TopKey y = __shfl_xor(x, j, kWave);
  return (x > y) == larger ? x : y;
}
__device__ __forceinline__ TopKey sorted_desc(TopKey x) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int k = 2; k <= kWave; k <<= 1)
#pragma unroll
    for (int j = k >> 1; j > 0; j >>= 1) x = exchange(x, j, ((lane & j) == 0) == ((lane & k) == 0));
  return x;
}
// The 64 largest of two falling lists, falling.
__device__ __forceinline__ TopKey merged(TopKey x, TopKey y) {
  const int lane = threadIdx.x & 63;
  const TopKey r = __shfl(y, 63 - lane, kWave);
  x = x > r ? x : r;
#pragma unroll
  for (int j = kWave / 2; j > 0; j >>= 1) x = exchange(x, j, (lane & j) == 0);
  return x;
}
struct WaveTop {
  TopKey list = 0;
  float least = -INFINITY;                                   // logits below it are not among the k largest
  int waiting = 0;
  TopKey* buf;                                                // [128] in LDS, this wavefront's
  int k;
  __device__ __forceinline__ void take(TopKey x) {
    list = merged(list, sorted_desc(x));
    least = logit_of(__shfl(list, k - 1, kWave));
  }
  // one logit a lane
  __device__ __forceinline__ void offer(float z, int id, bool have) {
    const bool in = have && z >= least && z > -INFINITY;
    const unsigned long long m = __ballot(in);
    if (!m) return;
    const int lane = threadIdx.x & 63;
    if (in) buf[waiting + __popcll(m & ((1ull << lane) - 1))] = key_of(z, id);
    waiting += __popcll(m);
    __builtin_amdgcn_wave_barrier();
    if (waiting < kWave) return;
    const TopKey x = buf[lane], rest = buf[kWave + lane];
    __builtin_amdgcn_wave_barrier();
    waiting -= kWave;
    if (lane < waiting) buf[lane] = rest;
    __builtin_amdgcn_wave_barrier();
    take(x);
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

// ------------------------------------------------------------------ bf16: logit tiles that are kept, with (max, sum exp) of their rows
template <class C>
__device__ __forceinline__ void top_tile(const uint16_t* __restrict__ W, const uint16_t* __restrict__ H, int d, int V, const int32_t* __restrict__ rowsel,
                                         int64_t c0, int64_t mc, int tile_m, int tile_n, bool w_once, float2* __restrict__ partial, int64_t n_pad,
                                         float* __restrict__ Z, int64_t tiles_v, uint16_t* lds) {
  constexpr int kPitch = C::WTM * 4 + 16;                    // a staged row of logits
  constexpr int kStage = 16 * kPitch;                        // sixteen of them, a wavefront's
  static_assert(C::WM * C::WN * kStage + C::WM * C::BN * 8 <= Ring2Cfg<C>::LDS_BYTES, "staging and the partials fit the tile buffers");
  const int m0 = tile_m * C::BM;
  const int64_t n0 = static_cast<int64_t>(tile_n) * C::BN;
  floatx4 acc[C::MI][C::NI];
  logit_tile<C>(W, H, d, V, rowsel, c0, mc, m0, n0, w_once, lds, acc);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave / C::WN, wn = wave % C::WN;
  char* const stage = reinterpret_cast<char*>(lds) + wave * kStage;
  float2* const s_part = reinterpret_cast<float2*>(reinterpret_cast<char*>(lds) + C::WM * C::WN * kStage);
  __syncthreads();
  const int vbase = m0 + wm * C::WTM + (lane >> 4) * 4;
  if (m0 + C::BM > V) {
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
    const int col = wn * C::WTN + j * 16 + (lane & 15);
    float m = kMasked, s = 0.f;
#pragma unroll
    for (int i = 0; i < C::MI; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) m = fmaxf(m, acc[i][j][r]);
#pragma unroll
    for (int i = 0; i < C::MI; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) s += __builtin_amdgcn_exp2f((acc[i][j][r] - m) * 1.44269504088896341f);
#pragma unroll
    for (int o = 16; o < kWave; o <<= 1) {
      const float m2 = __shfl_xor(m, o, kWave), s2 = __shfl_xor(s, o, kWave), M = fmaxf(m, m2);
      s = s * __expf(m - M) + s2 * __expf(m2 - M);
      m = M;
    }
    if (lane < 16) s_part[wm * C::BN + col] = make_float2(m, s);
    // sixteen rows through the wavefront's part of LDS: a store covers whole lines
#pragma unroll
    for (int i = 0; i < C::MI; ++i) *reinterpret_cast<floatx4*>(stage + (lane & 15) * kPitch + (i * 16 + (lane >> 4) * 4) * 4) = acc[i][j];
    __builtin_amdgcn_wave_barrier();
    constexpr int kLanes = C::WTM / 4, kRows = kWave / kLanes;
    const int64_t r0 = n0 + wn * C::WTN + j * 16 + lane / kLanes;
    float* const out = Z + ((r0 >> 8) * tiles_v + (m0 >> 8)) * kBlkElems + (r0 & 255) * 256 + (m0 & 255) + wm * C::WTM + lane % kLanes * 4;
#pragma unroll
    for (int q = 0; q < 16 / kRows; ++q)
      if (r0 + q * kRows < mc) *reinterpret_cast<floatx4*>(out + q * kRows * 256) = *reinterpret_cast<const floatx4*>(stage + (q * kRows + lane / kLanes) * kPitch + lane % kLanes * 16);
    __builtin_amdgcn_wave_barrier();
  }
  __syncthreads();
  if (threadIdx.x < C::BN) {
    float2 p = s_part[threadIdx.x];
#pragma unroll
    for (int w = 1; w < C::WM; ++w) {
      const float2 q = s_part[w * C::BN + threadIdx.x];
      const float M = fmaxf(p.x, q.x);
      p = make_float2(M, p.y * __expf(p.x - M) + q.y * __expf(q.x - M));
    }
    partial[static_cast<int64_t>(tile_m) * n_pad + n0 + threadIdx.x] = p;
  }
  __syncthreads();
}
template <class C>
__device__ __forceinline__ void top_tiles(const uint16_t* __restrict__ W, const uint16_t* __restrict__ H, int d, int V, const int32_t* __restrict__ rowsel,
                                          int64_t c0, int64_t mc, int tiles_m, int tiles_n, int panel, float2* __restrict__ partial, int64_t n_pad,
                                          float* __restrict__ Z, int64_t tiles_v, uint16_t* lds) {
  const bool w_once = tiles_n == 1 && beyond_cache(d, V, kLogitsOnceBytes);
  for (int it = 0; it < kTilesPerWg; ++it) {
    int tile_m, tile_n;
    if (!tile_coords<kGM, kGN>(tiles_m, tiles_n, panel, &tile_m, &tile_n, it, kTilesPerWg)) continue;
    top_tile<C>(W, H, d, V, rowsel, c0, mc, tile_m, tile_n, w_once, partial, n_pad, Z, tiles_v, lds);
  }
}
__global__ void __launch_bounds__(Cfg::T)
k_top_tiles(const uint16_t* __restrict__ W, const uint16_t* __restrict__ H, int d, int V, const int32_t* __restrict__ rowsel, int64_t c0, int64_t mc,
            int tiles_m, int tiles_n, int panel, float2* __restrict__ partial, int64_t n_pad, float* __restrict__ Z, int64_t tiles_v) {
  __shared__ __attribute__((aligned(16))) uint16_t lds[kLogitLds / 2];
  top_tiles<Cfg>(W, H, d, V, rowsel, c0, mc, tiles_m, tiles_n, panel, partial, n_pad, Z, tiles_v, lds);
}
__global__ void __launch_bounds__(NarrowCfg::T)
k_top_narrow(const uint16_t* __restrict__ W, const uint16_t* __restrict__ H, int d, int V, const int32_t* __restrict__ rowsel, int64_t c0, int64_t mc,
             int tiles_m, float2* __restrict__ partial, int64_t n_pad, float* __restrict__ Z, int64_t tiles_v) {
  __shared__ __attribute__((aligned(16))) uint16_t lds[kNarrowLds / 2];
  top_tiles<NarrowCfg>(W, H, d, V, rowsel, c0, mc, tiles_m, 1, kGN, partial, n_pad, Z, tiles_v, lds);
}

// ------------------------------------------------------------------ selection
// Logits of row m (of the chunk), four next to each other from v on; those past V are not looked at.
struct Blocked {                                             // float32 in blocks of 256 x 256
  const float* Z;
  int64_t tiles_v;
  __device__ __forceinline__ float4 load(int64_t m, int v, int) const {
    return *reinterpret_cast<const float4*>(Z + ((m >> 8) * tiles_v + (v >> 8)) * kBlkElems + (m & 255) * 256 + (v & 255));
  }
};
struct Doubles {                                             // float64 [rows][V]
  const double* Z;
  __device__ __forceinline__ float4 load(int64_t m, int v, int V) const {
    const double* p = Z + m * V + v;
    return make_float4(static_cast<float>(p[0]), v + 1 < V ? static_cast<float>(p[1]) : 0.f, v + 2 < V ? static_cast<float>(p[2]) : 0.f,
                       v + 3 < V ? static_cast<float>(p[3]) : 0.f);
  }
};
// A workgroup goes over a part of a row's vocabulary, its wavefronts 256 entries at a time in turn: list[row][part] gets the 64 largest keys.
template <class Logits>
__global__ void __launch_bounds__(kSelectT)
k_top_select(Logits L, int V, int k, int parts, int per, TopKey* __restrict__ lists) {
  __shared__ TopKey s_buf[kSelectWaves][2 * kWave];
  __shared__ TopKey s_list[kSelectWaves][kWave];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t m = blockIdx.x;
  const int part = blockIdx.y, v0 = part * per, v1 = min(v0 + per, V);
  WaveTop top;
  top.buf = s_buf[wave];
  top.k = k;
  for (int b = v0 + wave * 256; b < v1; b += kSelectWaves * 256) {
    const int v = b + lane * 4;
    const float4 z = v < v1 ? L.load(m, v, V) : make_float4(0.f, 0.f, 0.f, 0.f);
    top.offer(z.x, v, v < v1);
    top.offer(z.y, v + 1, v + 1 < v1);
    top.offer(z.z, v + 2, v + 2 < v1);
    top.offer(z.w, v + 3, v + 3 < v1);
  }
  top.finish();
  const TopKey all = merge_waves(top.list, s_list);
  if (wave == 0) lists[(m * parts + part) * kWave + lane] = all;
}
// A workgroup merges a row's lists and, where there are parts of its softmax, its logsumexp; writes the results.
struct TopOut {
  const int32_t* rowsel;
  int64_t c0;
  int k;
  int32_t* ids;
  float *logits, *lse;
};
__global__ void __launch_bounds__(kSelectT)
k_top_merge(const TopKey* __restrict__ lists, int parts, const float2* __restrict__ partial, int tiles_m, int64_t n_pad, TopOut O) {
  __shared__ TopKey s_list[kSelectWaves][kWave];
  __shared__ float s_m[kSelectWaves], s_s[kSelectWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t m = blockIdx.x, n = O.c0 + m, row = O.rowsel ? O.rowsel[n] : n;
  TopKey list = 0;
  for (int p = wave; p < parts; p += kSelectWaves) list = merged(list, lists[(m * parts + p) * kWave + lane]);
  list = merge_waves(list, s_list);
  if (wave == 0 && lane < O.k) {
    O.ids[row * O.k + lane] = token_of(list);
    O.logits[row * O.k + lane] = logit_of(list);
  }
  if (!partial) return;
  float mx = -INFINITY, s = 0.f;
  for (int t = threadIdx.x; t < tiles_m; t += kSelectT) {
    const float2 p = partial[static_cast<int64_t>(t) * n_pad + m];
    const float M = fmaxf(mx, p.x);
    s = s * __expf(mx - M) + p.y * __expf(p.x - M);
    mx = M;
  }
  const float M = wave_max(mx);
  s = wave_sum(mx == -INFINITY ? 0.f : s * __expf(mx - M));
  if (lane == 0) { s_m[wave] = M; s_s[wave] = s; }
  __syncthreads();
  if (threadIdx.x != 0) return;
  float a = s_m[0], b = s_s[0];
  for (int w = 1; w < kSelectWaves; ++w) {
    if (s_m[w] == -INFINITY) continue;
    const float X = fmaxf(a, s_m[w]);
    b = b * __expf(a - X) + s_s[w] * __expf(s_m[w] - X);
    a = X;
  }
  O.lse[row] = a + logf(b);
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
  TopKey* lists;
  float2* partial;
  void* z;
  char* room;                                                // float32: for the scores' parts
  size_t bytes, room_bytes;
};
void carve(Carver& c, TopWs& w, int64_t rows, int V, umas_dtype dt) {
  const int64_t pad = round_up(rows, 256), Vp = round_up(V, 256);
  w = TopWs{};
  w.lists = c.take<TopKey>(static_cast<size_t>(std::max(rows, kSelectLists)) * kWave);
  if (dt == UMAS_BF16) {
    w.partial = c.take<float2>(static_cast<size_t>(Vp / 128) * pad);
    w.z = c.take<float>(static_cast<size_t>(pad) * Vp);
  } else {
    w.z = c.take<double>(static_cast<size_t>(rows) * V);
    w.room_bytes = align_up(f32::score_room(rows, V));
    w.room = c.take<char>(w.room_bytes);
  }
  w.bytes = c.off;
}
size_t top_bytes(int64_t n_sel, int64_t cap, int V, umas_dtype dt) {
  Carver c(nullptr);
  TopWs w;
  carve(c, w, std::min(std::max<int64_t>(n_sel, 1), cap), V, dt);
  return w.bytes;
}

}  // namespace
}  // namespace umas

using namespace umas;

extern "C" size_t umas_top_logits_workspace_bytes_min(int64_t n_sel, int32_t d, int32_t V, int32_t k, umas_dtype dtype) {
  if (n_sel < 0 || d < 1 || V < 1 || k < 1 || k > UMAS_MAX_TOP) return 0;
  return top_bytes(n_sel, 256, V, dtype);
}
extern "C" size_t umas_top_logits_workspace_bytes(int64_t n_sel, int32_t d, int32_t V, int32_t k, umas_dtype dtype) {
  if (n_sel < 0 || d < 1 || V < 1 || k < 1 || k > UMAS_MAX_TOP) return 0;
  return top_bytes(n_sel, kTopChunkRows, V, dtype);
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
  while (cap > 256 && top_bytes(n_sel, cap, V, dtype) > workspace_bytes) cap = std::max<int64_t>(round_up(cap / 2, 256), 256);
  Carver c(workspace);
  TopWs w;
  carve(c, w, cap, V, dtype);
  for (int64_t c0 = 0; c0 < n_sel; c0 += cap) {
    const int64_t rows = std::min(cap, n_sel - c0), tiles_v = round_up(V, 256) / 256;
    int tiles_m = static_cast<int>(tiles_v);
    int64_t n_pad = round_up(rows, 256);
    const int parts = select_parts(rows, V), per = static_cast<int>(round_up(cdiv(V, parts), 256));
    const dim3 select(static_cast<unsigned>(rows), parts);
    if (dtype == UMAS_BF16) {
      const uint16_t *Wb = static_cast<const uint16_t*>(W), *Hb = static_cast<const uint16_t*>(H);
      float* const Z = static_cast<float*>(w.z);
      if (rows <= NarrowCfg::BN) {
        tiles_m = (V + NarrowCfg::BM - 1) / NarrowCfg::BM;
        n_pad = NarrowCfg::BN;
        hipLaunchKernelGGL(k_top_narrow, dim3(tile_grid<kGM, kGN>(tiles_m, 1, kGN, kTilesPerWg)), dim3(NarrowCfg::T), 0, st, Wb, Hb, d, V, rowsel, c0, rows, tiles_m,
                           w.partial, n_pad, Z, tiles_v);
        UMAS_LAUNCHED("k_top_narrow");
      } else {
        const int tiles_n = static_cast<int>(n_pad / 256), panel = row_panel(tiles_n, d);
        hipLaunchKernelGGL(k_top_tiles, score_grid(tiles_m, tiles_n, panel, 0), dim3(Cfg::T), 0, st, Wb, Hb, d, V, rowsel, c0, rows, tiles_m, tiles_n, panel,
                           w.partial, n_pad, Z, tiles_v);
        UMAS_LAUNCHED("k_top_tiles");
      }
      hipLaunchKernelGGL(k_top_select<Blocked>, select, dim3(kSelectT), 0, st, Blocked{Z, tiles_v}, V, k, parts, per, w.lists);
    } else {
      const float* Hf = static_cast<const float*>(H) + (rowsel ? 0 : c0 * d);
      double* const Z = static_cast<double*>(w.z);
      s = f32::score(static_cast<const float*>(W), Hf, d, V, rowsel ? rowsel + c0 : nullptr, rows, nullptr, w.room, w.room_bytes,
                     f32::ScoreOut{Z, nullptr, nullptr, nullptr, nullptr, nullptr, rowsel ? lse : lse + c0, nullptr}, st);
      if (s != UMAS_OK) return s;
      hipLaunchKernelGGL(k_top_select<Doubles>, select, dim3(kSelectT), 0, st, Doubles{Z}, V, k, parts, per, w.lists);
    }
    UMAS_LAUNCHED("k_top_select");
    hipLaunchKernelGGL(k_top_merge, dim3(static_cast<unsigned>(rows)), dim3(kSelectT), 0, st, w.lists, parts, dtype == UMAS_BF16 ? w.partial : nullptr, tiles_m, n_pad,
                       TopOut{rowsel, c0, k, top_ids, top_logits, lse});
    UMAS_LAUNCHED("k_top_merge");
  }
  return UMAS_OK;
}
