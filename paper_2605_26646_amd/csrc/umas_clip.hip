// The global norm of a list of gradients, and clipping: N = sqrt(sum g^2), c = min(1, max_norm / N), g <- c g.
//
// The arrays are cut into chunks, the chunks dealt to the workgroups in equal runs.  Squares are summed in float64 (a float32 square overflows from 1.8e19 on; a fused
// multiply-add of float64 costs what one of float32 does, and memory is what bounds the pass), in an order that depends on the sizes alone.  The scaling pass
// goes through the chunks from the last one back: what the norm's pass read last still lies in the memory-side cache, and what it reads and writes itself goes past the caches, so that the
// rest stays there (into other arrays, 170 MB 106 -> 84 us, 0.5 GB 311 -> 265, 1.6 GB 923 -> 888; 42 MB 26).  The norm alone of 1.6 GB takes 292 us, 5.5 TB/s; of 42 MB, which
// lie in that cache, 15 us, of 2 MB 7.2: two launches.
#include <algorithm>
#include <new>
#include <type_traits>

#include "umas_logits.h"

namespace umas {
namespace {

constexpr int kCT = 256;
constexpr int kChunk = 8192;                                 // elements
// Workgroups at most; every one of the second launch sums what those of the first left.  With 512, 1024 and 2048 the norm of 42 MB takes 13.8, 15 and 19 us, of 170 MB 42, 38 and 40, of
// 1.6 GB 330, 293 and 295.
constexpr int kClipGrid = 1024;
constexpr int kTable = 96;                                   // arrays that travel with a launch
// 16 bytes of an array that starts at any multiple of its element's size
typedef uint32_t u32x4u __attribute__((ext_vector_type(4), aligned(2)));

struct ClipEntry {
  const void* in;
  void* out;
  int64_t n;
  uint32_t first;                                            // chunk
  int32_t bf16;
};
struct ClipTable {
  ClipEntry e[kTable];
};
struct ClipPart {
  double sum;
  int64_t not_finite;
};
__global__ void __launch_bounds__(kTable)
k_clip_table(ClipTable t, int n, ClipEntry* __restrict__ to) {
  if (static_cast<int>(threadIdx.x) < n) to[threadIdx.x] = t.e[threadIdx.x];
}
__device__ __forceinline__ int entry_of(const ClipEntry* __restrict__ e, int n, uint32_t chunk) {   // the last one that starts at or before it
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (e[mid].first <= chunk) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}
template <typename E>
__device__ __forceinline__ float value_of(E x) {
  if constexpr (std::is_same<E, uint16_t>::value) return __uint_as_float(static_cast<uint32_t>(x) << 16);
  else return x;
}
template <typename E>
__device__ __forceinline__ void unpacked(const u32x4u& v, float (&x)[16 / sizeof(E)]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(E) == 2) {
      x[2 * i] = __uint_as_float(v[i] << 16);
      x[2 * i + 1] = __uint_as_float(v[i] & 0xFFFF0000u);
    } else {
      x[i] = __uint_as_float(v[i]);
    }
  }
}
__device__ __forceinline__ void take(float x, double& sum, int& bad) {
  sum = fma(static_cast<double>(x), static_cast<double>(x), sum);
  bad += (__float_as_uint(x) & 0x7F800000u) == 0x7F800000u;
}
template <typename E>
__device__ __forceinline__ void square_chunk(const E* __restrict__ p, int64_t n, double& sum, int& bad) {   // up to kChunk elements
  constexpr int N = 16 / sizeof(E), kAt = kChunk / N / kCT;
  if (n >= kChunk) {
    u32x4u v[kAt];
#pragma unroll
    for (int k = 0; k < kAt; ++k) v[k] = *reinterpret_cast<const u32x4u*>(p + (k * kCT + threadIdx.x) * N);
#pragma unroll
    for (int k = 0; k < kAt; ++k) {
      float x[N];
      unpacked<E>(v[k], x);
#pragma unroll
      for (int i = 0; i < N; ++i) take(x[i], sum, bad);
    }
    return;
  }
  const int whole = static_cast<int>(n) / N;
  for (int i = threadIdx.x; i < whole; i += kCT) {
    float x[N];
    unpacked<E>(*reinterpret_cast<const u32x4u*>(p + i * N), x);
#pragma unroll
    for (int j = 0; j < N; ++j) take(x[j], sum, bad);
  }
  const int at = whole * N + threadIdx.x;
  if (at < n) take(value_of(p[at]), sum, bad);
}
template <class Table>
struct ClipArgs {
  Table table;
  int n;
  uint32_t chunks;
  double max_norm;
  ClipPart* part;
  umas_clip_stats* stats;
  __device__ __forceinline__ const ClipEntry* entries() const {
    if constexpr (std::is_pointer<Table>::value) return table;
    else return table.e;
  }
};
template <class Table>
__global__ void __launch_bounds__(kCT)
k_clip_norm(const ClipArgs<Table> A) {
  __shared__ double s_sum[kCT / kWave];
  __shared__ int s_bad[kCT / kWave];
  const ClipEntry* const e = A.entries();
  const uint32_t c0 = static_cast<uint32_t>(static_cast<uint64_t>(A.chunks) * blockIdx.x / gridDim.x), c1 = static_cast<uint32_t>(static_cast<uint64_t>(A.chunks) * (blockIdx.x + 1) / gridDim.x);
  double sum = 0.0;
  int64_t all_bad = 0;
  int at = c0 < c1 ? entry_of(e, A.n, c0) : 0;
  for (uint32_t c = c0; c < c1; ++c) {
    while (at + 1 < A.n && e[at + 1].first <= c) ++at;
    const int64_t off = static_cast<int64_t>(c - e[at].first) * kChunk, rest = e[at].n - off;
    int bad = 0;
    if (e[at].bf16) square_chunk(static_cast<const uint16_t*>(e[at].in) + off, rest, sum, bad);
    else square_chunk(static_cast<const float*>(e[at].in) + off, rest, sum, bad);
    all_bad += bad;
  }
  sum = wave_sum(sum);
  const int bad = wave_sum(static_cast<int>(all_bad));
  if ((threadIdx.x & 63) == 0) { s_sum[threadIdx.x >> 6] = sum; s_bad[threadIdx.x >> 6] = bad; }
  __syncthreads();
  if (threadIdx.x != 0) return;
  int64_t b = 0;
  sum = 0.0;
  for (int w = 0; w < kCT / kWave; ++w) { sum += s_sum[w]; b += s_bad[w]; }
  A.part[blockIdx.x] = ClipPart{sum, b};
}
// c, in float64 where float32 has few bits for it or none (a norm of 1e38 and more, a max_norm of 1e-30)
template <typename C>
struct Factor {
  C c;
  __device__ __forceinline__ float operator()(float x) const { return static_cast<float>(x * c); }
};
template <typename E, class Times>
__device__ __forceinline__ void scale_chunk(const E* p, E* o, int64_t n, Times times) {   // p may be o
  constexpr int N = 16 / sizeof(E);
  const int whole = static_cast<int>(n < kChunk ? n : kChunk) / N;
  for (int i = threadIdx.x; i < whole; i += kCT) {
    float x[N];
    unpacked<E>(__builtin_nontemporal_load(reinterpret_cast<const u32x4u*>(p + i * N)), x);
    u32x4u v;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (sizeof(E) == 2) v[j] = pack_bf16x2(times(x[2 * j]), times(x[2 * j + 1]));
      else v[j] = __float_as_uint(times(x[j]));
    }
    __builtin_nontemporal_store(v, reinterpret_cast<u32x4u*>(o + i * N));
  }
  if (n >= kChunk) return;
  const int at = whole * N + threadIdx.x;
  if (at < n) {
    const float x = times(value_of(p[at]));
    if constexpr (std::is_same<E, uint16_t>::value) o[at] = f2bf(x);
    else o[at] = x;
  }
}
template <class Table>
__global__ void __launch_bounds__(kCT)
k_clip_scale(const ClipArgs<Table> A, int parts) {
  __shared__ double s_sum[kCT / kWave];
  __shared__ int64_t s_bad[kCT / kWave];
  double sum = 0.0;
  int64_t bad = 0;
  for (int p = threadIdx.x; p < parts; p += kCT) { sum += A.part[p].sum; bad += A.part[p].not_finite; }
  sum = wave_sum(sum);
  bad = wave_sum(bad);
  if ((threadIdx.x & 63) == 0) { s_sum[threadIdx.x >> 6] = sum; s_bad[threadIdx.x >> 6] = bad; }
  __syncthreads();
  sum = 0.0;
  bad = 0;
  for (int w = 0; w < kCT / kWave; ++w) { sum += s_sum[w]; bad += s_bad[w]; }
  const double norm = sqrt(sum);
  // a norm that is no finite number scales nothing: the comparison is false for one that is none
  const double exact = norm > A.max_norm && norm < INFINITY ? A.max_norm / norm : 1.0;
  const float c = static_cast<float>(exact);
  if (blockIdx.x == 0 && threadIdx.x == 0) *A.stats = umas_clip_stats{static_cast<float>(norm), c, bad};
  const ClipEntry* const e = A.entries();
  const unsigned wg = gridDim.x - 1 - blockIdx.x;            // from the end
  const uint32_t c0 = static_cast<uint32_t>(static_cast<uint64_t>(A.chunks) * wg / gridDim.x), c1 = static_cast<uint32_t>(static_cast<uint64_t>(A.chunks) * (wg + 1) / gridDim.x);
  int at = c0 < c1 ? entry_of(e, A.n, c1 - 1) : 0;
  for (uint32_t k = c1; k > c0; --k) {
    while (e[at].first > k - 1) --at;
    if (c == 1.f && e[at].in == e[at].out) continue;         // as it is
    const int64_t off = static_cast<int64_t>(k - 1 - e[at].first) * kChunk, rest = e[at].n - off;
    auto scale = [&](auto times) {
      if (e[at].bf16) scale_chunk(static_cast<const uint16_t*>(e[at].in) + off, static_cast<uint16_t*>(e[at].out) + off, rest, times);
      else scale_chunk(static_cast<const float*>(e[at].in) + off, static_cast<float*>(e[at].out) + off, rest, times);
    };
    if (exact < 0x1p-100) scale(Factor<double>{exact});
    else scale(Factor<float>{c});
  }
}

// ------------------------------------------------------------------ host side
// What is written may overlap nothing else of the list but its own input, and that as a whole: the order of reads and writes is open.
struct Span {
  uintptr_t a, b;
  int32_t entry;
  bool out;
  bool operator<(const Span& o) const { return a != o.a ? a < o.a : b < o.b; }
};
umas_status check_spans(const umas_gradient* g, int32_t n) {
  Span* const s = new (std::nothrow) Span[2 * static_cast<size_t>(n)];
  UMAS_REQUIRE(s, UMAS_EINVAL, "no host memory for a list of %d gradients", n);
  size_t m = 0;
  for (int32_t i = 0; i < n; ++i) {
    if (g[i].n == 0) continue;
    const size_t bytes = static_cast<size_t>(g[i].n) * (g[i].dtype == UMAS_BF16 ? 2 : 4);
    const uintptr_t in = reinterpret_cast<uintptr_t>(g[i].grad), out = reinterpret_cast<uintptr_t>(g[i].out);
    s[m++] = Span{out, out + bytes, i, true};
    if (in != out) s[m++] = Span{in, in + bytes, i, false};
  }
  std::sort(s, s + m);
  // the furthest ends so far of what is written and of what is read
  int32_t bad = -1;
  uintptr_t end_out = 0, end_in = 0;
  for (size_t k = 0; k < m && bad < 0; ++k) {
    if (s[k].a < end_out || (s[k].out && s[k].a < end_in)) bad = s[k].entry;
    (s[k].out ? end_out : end_in) = std::max(s[k].out ? end_out : end_in, s[k].b);
  }
  delete[] s;
  UMAS_REQUIRE(bad < 0, UMAS_EINVAL, "gradient %d overlaps an output of the list", bad);
  return UMAS_OK;
}
struct ClipWs {
  ClipPart* part;
  ClipEntry* table;
  size_t bytes;
};
void carve(Carver& c, ClipWs& w, int32_t n) {
  w.part = c.take<ClipPart>(kClipGrid);
  w.table = n > kTable ? c.take<ClipEntry>(n) : nullptr;
  w.bytes = c.off;
}
template <class Table>
umas_status launch(const ClipArgs<Table>& A, hipStream_t st) {
  const unsigned grid = std::max<unsigned>(std::min<unsigned>(A.chunks, kClipGrid), 1);
  hipLaunchKernelGGL(k_clip_norm<Table>, dim3(grid), dim3(kCT), 0, st, A);
  UMAS_LAUNCHED("k_clip_norm");
  hipLaunchKernelGGL(k_clip_scale<Table>, dim3(grid), dim3(kCT), 0, st, A, static_cast<int>(grid));
  UMAS_LAUNCHED("k_clip_scale");
  return UMAS_OK;
}

}  // namespace
}  // namespace umas

using namespace umas;

extern "C" size_t umas_clip_workspace_bytes(int32_t n) {
  if (n < 0) return 0;
  Carver c(nullptr);
  ClipWs w;
  carve(c, w, n);
  return w.bytes;
}

extern "C" umas_status umas_clip_gradients(const umas_gradient* gradients, int32_t n, double max_norm, umas_clip_stats* stats, void* workspace,
                                           size_t workspace_bytes, void* hip_stream) {
  UMAS_REQUIRE(n >= 0, UMAS_EINVAL, "negative count of gradients");
  UMAS_REQUIRE(gradients || n == 0, UMAS_EINVAL, "gradients must not be NULL");
  UMAS_REQUIRE(max_norm > 0.0, UMAS_EINVAL, "max_norm must be positive");
  UMAS_REQUIRE(stats && reinterpret_cast<uintptr_t>(stats) % 8 == 0, UMAS_EINVAL, "stats must not be NULL, and 8-byte aligned");
  uint64_t chunks = 0;
  for (int32_t i = 0; i < n; ++i) {
    const umas_gradient& g = gradients[i];
    UMAS_REQUIRE(g.dtype == UMAS_F32 || g.dtype == UMAS_BF16, UMAS_EDTYPE, "gradient %d: dtype=%d is neither F32 nor BF16", i, g.dtype);
    UMAS_REQUIRE(g.n >= 0 && g.n < (int64_t{1} << 44), UMAS_EINVAL, "gradient %d: n=%lld", i, static_cast<long long>(g.n));
    UMAS_REQUIRE((g.grad && g.out) || g.n == 0, UMAS_EINVAL, "gradient %d: grad and out must not be NULL", i);
    const size_t size = g.dtype == UMAS_BF16 ? 2 : 4;
    UMAS_REQUIRE(reinterpret_cast<uintptr_t>(g.grad) % size == 0 && reinterpret_cast<uintptr_t>(g.out) % size == 0, UMAS_EINVAL,
                 "gradient %d: grad and out must be aligned to their type", i);
    chunks += static_cast<uint64_t>(g.n + kChunk - 1) / kChunk;
  }
  UMAS_REQUIRE(chunks < (1ull << 31), UMAS_ESHAPE, "the gradients hold too many numbers");
  umas_status s = check_spans(gradients, n);
  if (s != UMAS_OK) return s;
  s = check_ws(workspace, workspace_bytes, umas_clip_workspace_bytes(n));
  if (s != UMAS_OK) return s;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  prof_mark(st);
  Carver c(workspace);
  ClipWs w;
  carve(c, w, n);
  ClipArgs<ClipTable> A{};
  uint32_t first = 0;
  int32_t count = 0, in_table = 0;
  auto put = [&](ClipEntry* e, const umas_gradient& g) {
    *e = ClipEntry{g.grad, g.out, g.n, first, g.dtype == UMAS_BF16};
    first += static_cast<uint32_t>((g.n + kChunk - 1) / kChunk);
  };
  for (int32_t i = 0; i < n; ++i) {
    if (gradients[i].n == 0) continue;
    if (count == kTable) {                                   // more than travel with a launch: by way of the workspace
      hipLaunchKernelGGL(k_clip_table, dim3(1), dim3(kTable), 0, st, A.table, count, w.table + in_table);
      UMAS_LAUNCHED("k_clip_table");
      in_table += count;
      count = 0;
    }
    put(&A.table.e[count++], gradients[i]);
  }
  A.max_norm = max_norm;
  A.part = w.part;
  A.stats = stats;
  A.chunks = static_cast<uint32_t>(chunks);
  A.n = in_table + count;
  if (in_table == 0) return launch(A, st);
  hipLaunchKernelGGL(k_clip_table, dim3(1), dim3(kTable), 0, st, A.table, count, w.table + in_table);
  UMAS_LAUNCHED("k_clip_table");
  return launch(ClipArgs<const ClipEntry*>{w.table, A.n, A.chunks, max_norm, w.part, stats}, st);
}
