// Global L2 norm of a list of gradients, the factor that clips them to it, and the scaling by that factor.
//     norm = |s| sqrt(sum G^2),  scale = s min(1, max_norm / (norm + 1e-6)),  finite = every entry is finite
// Two launches: partial sums of squares per workgroup, then their sum and the square root.  Squares are formed and added
// in 64 bits: no fp32 or bf16 entry overflows or underflows there, so the sum is finite exactly if every entry is (4
// instructions per element, a third of what a read at 6.6 TB/s leaves time for).  Bound by HBM: norm of 405M bf16 gradients
// 123 us (6.6 TB/s), scaling of 151M bf16 93 us (6.5 TB/s).  A scaling by 1 moves nothing, but starts its workgroups all the
// same: 22 us for 202M bf16 gradients, 330 for 3.2 billion.
#include "adamw.hpp"
#include "tensor_list.hpp"

namespace galore {
namespace {

constexpr int kNormThreads = 512;   // 151M bf16 gradients: 49.8 us; 256 threads 52, 1024 52
// Workgroups of a list: 2048, or, where the work of each would be short, fewer than the 1024 that the chip holds at once, so
// that there is no second round (33M bf16 elements: 43.6 us with 2048, 37.7 with 960; 151M: 49.9 and 50.5).
constexpr int kPartialTarget = 2048, kOneRound = 960;
constexpr int64_t kOneRoundElements = (int64_t)1 << 26;
// What follows a norm (AdamW, the scaling) reads the same gradients again and finds a part of them in the 256 MiB cache if
// they were loaded through it, which the norm itself pays for: norm and AdamW of 25 MB of gradients 53.4 us (loads past the
// caches 56.1), 240 MB 433 (457), 400 MB 734 (772), 800 MB 1505 (1532), 1600 MB 3046 (3054); the norm alone 76 (67) at 400 MB,
// 138 (122) at 800.  The limit serves the pair, and lets go where the norm would pay for little: at 400 MB the pair gains 4
// times what a norm alone loses (38 us and 9), at 800 MB less than twice (27 and 16).
constexpr int64_t kCachedBytes = (int64_t)512 << 20;
constexpr int kScaleThreads = 128;
// Of a tensor, per workgroup: two 16-byte accesses of every thread (151M bf16 / 200M fp32: 94 / 243 us; one access 113 / 287,
// four 98 / 252; two with 256 threads 95 / 250, with 512 96 / 253).
constexpr int kScaleBytes = 2 * 16 * kScaleThreads;

__device__ __forceinline__ double workgroup_sum(double x) {
  __shared__ double waves[kNormThreads / 64];
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = x;
  __syncthreads();
  double all = 0.0;
#pragma unroll
  for (int i = 0; i < kNormThreads / 64; ++i) all += waves[i];
  return all;
}

template <class T, bool CACHED> __device__ __forceinline__ double squares(const GradTensor& p, int64_t first, int64_t n) {
  constexpr int N = 16 / sizeof(T);
  constexpr int kPiece = 1 << 19;   // offsets that RowWalk takes
  const T* G = static_cast<const T*>(p.G);
  double sum[N] = {};
  const auto add = [&](const ListF32<N>& g) {
#pragma unroll
    for (int e = 0; e < N; ++e) sum[e] = __builtin_fma((double)g[e], (double)g[e], sum[e]);
  };
  if (p.ld == p.cols) {
    constexpr int kStep = kNormThreads * N;
    G += first;
    int64_t o = (int64_t)threadIdx.x * N;
    for (; o + kStep + N <= n; o += 2 * kStep) {   // two requests at a time
      const ListF32<N> a = list_load<N, CACHED>(G + o), b = list_load<N, CACHED>(G + o + kStep);
      add(a);
      add(b);
    }
    for (; o < n; o += kStep) add(row_load<N, CACHED>(G + o, 0, 0, RowWalk::Place::in_run(0), n - o < N ? (int)(n - o) : N));
  } else {
    for (int64_t base = 0; base < n; base += kPiece) {
      const RowWalk walk(first + base, p.cols);
      const int len = n - base < kPiece ? (int)(n - base) : kPiece;
      for (int o = threadIdx.x * N; o < len; o += kNormThreads * N) {
        add(row_load<N, CACHED>(G, p.ld, p.cols, walk.at(o), len - o));
      }
    }
  }
  double all = 0.0;
#pragma unroll
  for (int e = 0; e < N; ++e) all += sum[e];
  return all;
}

template <bool CACHED> __global__ __launch_bounds__(kNormThreads) void grad_squares_kernel(const GradGroup grp, double* partials) {
  const int i = tensor_of_block(grp.begin, grp.count, blockIdx.x);
  const GradTensor& p = grp.t[i];
  const int64_t span = (int64_t)grp.span * 1024, first = (blockIdx.x - grp.begin[i]) * span, rest = p.count - first;
  const int64_t n = rest < span ? rest : span;
  const double x = workgroup_sum(grp.bf16[i] ? squares<__bf16, CACHED>(p, first, n) : squares<float, CACHED>(p, first, n));
  if (threadIdx.x == 0) partials[blockIdx.x] = x;
}

__global__ __launch_bounds__(kNormThreads) void grad_stats_kernel(const double* partials, int count, float grad_scale, float max_norm, GradStats* stats) {
  double x = 0.0;
  for (int base = threadIdx.x; base < count; base += 4 * kNormThreads) {   // four requests at a time
    double y[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = base + j * kNormThreads < count ? partials[base + j * kNormThreads] : 0.0;
    x += (y[0] + y[1]) + (y[2] + y[3]);
  }
  x = workgroup_sum(x);
  if (threadIdx.x == 0) {
    const bool finite = x <= 1.7976931348623157e308;   // false for NaN
    const double norm = __builtin_fabs((double)grad_scale) * __builtin_sqrt(x);
    double clip = max_norm / (norm + 1e-6);
    if (!(clip < 1.0)) clip = 1.0;
    stats->norm = (float)norm;
    stats->scale = finite ? (float)(grad_scale * clip) : 0.f;
    stats->finite = finite ? 1.f : 0.f;
    stats->reserved = 0.f;
  }
}

template <class T> __device__ __forceinline__ void scale_span(const GradTensor& p, float c, bool zero, int64_t first) {
  constexpr int N = 16 / sizeof(T), kElements = kScaleBytes / (int)sizeof(T), kStep = kScaleThreads * N;
  const int64_t rest = p.count - first;
  const int n = rest < kElements ? (int)rest : kElements;
  T* G = static_cast<T*>(p.G);
  if (p.ld == p.cols && n == kElements) {
    G += first + threadIdx.x * N;
    ListF32<N> a = 0.f, b = 0.f;
    if (!zero) {
      a = list_load<N>(G); b = list_load<N>(G + kStep);
      a *= c; b *= c;
    }
    list_store<N>(G, a);
    list_store<N>(G + kStep, b);
    return;
  }
  const RowWalk walk(first, p.cols);
  for (int o = threadIdx.x * N; o < n; o += kStep) {
    const RowWalk::Place at = walk.at(o);
    ListF32<N> g = 0.f;
    if (!zero) g = row_load<N>(G, p.ld, p.cols, at, n - o) * c;
    row_store<N>(G, p.ld, p.cols, at, n - o, g);
  }
}

__global__ __launch_bounds__(kScaleThreads) void scale_grads_kernel(const GradGroup grp, const GradStats* stats) {
  const bool zero = stats->finite != 1.f;
  const float c = stats->scale;
  if (!zero && c == 1.f) return;
  const int block = grp.block0 + (int)blockIdx.x;
  const int i = tensor_of_block(grp.begin, grp.count, block);
  const GradTensor& p = grp.t[i];
  const int64_t span = block - grp.begin[i];
  if (grp.bf16[i]) scale_span<__bf16>(p, c, zero, span * (kScaleBytes / 2));
  else scale_span<float>(p, c, zero, span * (kScaleBytes / 4));
}

// Workgroups of a list; elements(i): those of tensor i that one takes.  -1: too many.
template <class F> int64_t lay_out(GradGroup& g, F elements) {
  int64_t blocks = 0;
  for (int i = 0; i < g.count; ++i) {
    g.begin[i] = (int32_t)blocks;
    blocks += (g.t[i].count + elements(i) - 1) / elements(i);
    if (blocks > INT32_MAX) return -1;
  }
  return blocks;
}

}  // namespace

size_t grad_norm_partials(int32_t count) { return (size_t)kPartialTarget + (size_t)count; }

hipError_t launch_grad_norm(GradGroup* lists, int n_lists, float grad_scale, float max_norm, GradStats* stats, double* partials, hipStream_t stream) {
  int64_t total = 0, bytes = 0;
  for (int l = 0; l < n_lists; ++l)
    for (int i = 0; i < lists[l].count; ++i) {
      total += lists[l].t[i].count;
      bytes += lists[l].t[i].count * (lists[l].bf16[i] ? 2 : 4);
    }
  const auto kernel = bytes <= kCachedBytes ? grad_squares_kernel<true> : grad_squares_kernel<false>;
  // sum over tensors of ceil(count / elements) <= total / elements + tensors <= kPartialTarget + tensors
  const int64_t target = (int64_t)(total <= kOneRoundElements ? kOneRound : kPartialTarget) * 1024;
  int64_t span = (total + target - 1) / target;
  span = span < 4 ? 4 : span;
  if (span > INT32_MAX) return hipErrorInvalidValue;
  int64_t done = 0;
  for (int l = 0; l < n_lists; ++l) {
    const int64_t blocks = lay_out(lists[l], [&](int) { return span * 1024; });
    if (blocks < 0) return hipErrorInvalidValue;
    lists[l].span = (int32_t)span;
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(kNormThreads), 0, stream, lists[l], partials + done);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    done += blocks;
  }
  hipLaunchKernelGGL(grad_stats_kernel, dim3(1), dim3(kNormThreads), 0, stream, partials, (int)done, grad_scale, max_norm, stats);
  return hipGetLastError();
}

hipError_t launch_scale_grads(GradGroup& g, const GradStats* stats, hipStream_t stream) {
  if (g.count > kGradTensors) return hipErrorInvalidValue;
  const int64_t blocks = lay_out(g, [&](int i) { return (int64_t)kScaleBytes / (g.bf16[i] ? 2 : 4); });
  if (blocks < 0) return hipErrorInvalidValue;
  for (int64_t b = 0; b < blocks; b += kMaxBlocks) {
    g.block0 = (int32_t)b;
    const int64_t grid = blocks - b < kMaxBlocks ? blocks - b : kMaxBlocks;
    hipLaunchKernelGGL(scale_grads_kernel, dim3((unsigned)grid), dim3(kScaleThreads), 0, stream, g, stats);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace galore
