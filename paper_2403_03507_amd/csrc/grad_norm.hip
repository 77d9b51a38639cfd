// Global L2 norm of a list of gradients, the factor that clips them to it, and the scaling by that factor.
//     norm = |s| sqrt(sum G^2),  scale = s min(1, max_norm / (norm + 1e-6)),  finite = every entry is finite
// Two launches: partial sums of squares per workgroup, then their sum and the square root.  Squares are formed and added
// in 64 bits: no fp32 or bf16 entry overflows or underflows there, so the sum is finite exactly if every entry is.
#include "adamw.hpp"
#include "tensor_list.hpp"

namespace galore {
namespace {

constexpr int kThreads = 256;
constexpr int kPartialTarget = 2048;   // workgroups of a large list

__device__ __forceinline__ double workgroup_sum(double x) {
  __shared__ double waves[kThreads / 64];
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = x;
  __syncthreads();
  return (waves[0] + waves[1]) + (waves[2] + waves[3]);
}

template <class T> __device__ __forceinline__ double squares(const GradTensor& p, int64_t first, int64_t n) {
  constexpr int N = 16 / sizeof(T);
  constexpr int kPiece = 1 << 19;   // offsets that RowWalk takes
  const T* G = static_cast<const T*>(p.G);
  double sum[N] = {};
  const auto add = [&](const T* x) {
    const ListF32<N> g = list_load<N>(x);
#pragma unroll
    for (int e = 0; e < N; ++e) sum[e] = __builtin_fma((double)g[e], (double)g[e], sum[e]);
  };
  const auto one = [&](T x) { sum[0] = __builtin_fma((double)(float)x, (double)(float)x, sum[0]); };
  if (p.ld == p.cols) {
    G += first;
    for (int64_t o = (int64_t)threadIdx.x * N; o < n; o += kThreads * N) {
      if (o + N <= n) add(G + o);
      else for (int64_t e = o; e < n; ++e) one(G[e]);
    }
  } else {
    for (int64_t base = 0; base < n; base += kPiece) {
      const RowWalk walk(first + base, p.cols, p.ld);
      const int len = n - base < kPiece ? (int)(n - base) : kPiece;
      for (int o = threadIdx.x * N; o < len; o += kThreads * N) {
        uint32_t left;
        const int64_t a = walk.at(o, left);
        if (o + N <= len && left >= N) add(G + a);
        else for (int e = o; e < o + N && e < len; ++e) one(G[walk.at(e, left)]);
      }
    }
  }
  double all = 0.0;
#pragma unroll
  for (int e = 0; e < N; ++e) all += sum[e];
  return all;
}

__global__ __launch_bounds__(kThreads) void grad_squares_kernel(const GradGroup grp, double* partials) {
  const int i = tensor_of_block(grp.begin, grp.count, blockIdx.x);
  const GradTensor& p = grp.t[i];
  const int64_t span = (int64_t)grp.span * 1024, first = (blockIdx.x - grp.begin[i]) * span, rest = p.count - first;
  const int64_t n = rest < span ? rest : span;
  const double x = workgroup_sum(grp.bf16[i] ? squares<__bf16>(p, first, n) : squares<float>(p, first, n));
  if (threadIdx.x == 0) partials[blockIdx.x] = x;
}

__global__ __launch_bounds__(kThreads) void grad_stats_kernel(const double* partials, int count, float grad_scale, float max_norm, GradStats* stats) {
  double x = 0.0;
  for (int i = threadIdx.x; i < count; i += kThreads) x += partials[i];
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

template <class T> __device__ __forceinline__ void scale_span(const GradTensor& p, float c, bool zero, int64_t first, int n) {
  constexpr int N = 16 / sizeof(T);
  T* G = static_cast<T*>(p.G);
  const bool dense = p.ld == p.cols;
  const RowWalk walk(first, p.cols, p.ld);
  if (dense) G += first;
  for (int o = threadIdx.x * N; o < n; o += kThreads * N) {
    uint32_t left = N;
    const int64_t a = dense ? o : walk.at(o, left);
    if (o + N <= n && left >= N) {
      ListF32<N> g = 0.f;
      if (!zero) g = list_load<N>(G + a) * c;
      list_store<N>(G + a, g);
    } else {
      for (int e = o; e < o + N && e < n; ++e) {
        const int64_t ae = dense ? e : walk.at(e, left);
        G[ae] = zero ? (T)0.f : (T)((float)G[ae] * c);
      }
    }
  }
}

__global__ __launch_bounds__(kThreads) void scale_grads_kernel(const GradGroup grp, const GradStats* stats) {
  const bool zero = stats->finite != 1.f;
  const float c = stats->scale;
  if (!zero && c == 1.f) return;
  const int i = tensor_of_block(grp.begin, grp.count, blockIdx.x);
  const GradTensor& p = grp.t[i];
  const int64_t span = (int64_t)grp.span * 1024, first = (blockIdx.x - grp.begin[i]) * span, rest = p.count - first;
  const int n = (int)(rest < span ? rest : span);
  if (grp.bf16[i]) scale_span<__bf16>(p, c, zero, first, n);
  else scale_span<float>(p, c, zero, first, n);
}

// Workgroups of a list at `span` * 1024 elements each.
int64_t lay_out(GradGroup& g, int64_t span) {
  int64_t blocks = 0;
  for (int i = 0; i < g.count; ++i) {
    g.begin[i] = (int32_t)blocks;
    blocks += (g.t[i].count + span * 1024 - 1) / (span * 1024);
    if (blocks > kMaxBlocks) return 0;
  }
  g.span = (int32_t)span;
  return blocks;
}

}  // namespace

size_t grad_norm_partials(int32_t count) { return (size_t)kPartialTarget + (size_t)count; }

hipError_t launch_grad_norm(GradGroup* lists, int n_lists, float grad_scale, float max_norm, GradStats* stats, double* partials, hipStream_t stream) {
  int64_t total = 0;
  for (int l = 0; l < n_lists; ++l)
    for (int i = 0; i < lists[l].count; ++i) total += lists[l].t[i].count;
  // sum over tensors of ceil(count / span) <= total / span + tensors <= kPartialTarget + tensors
  int64_t span = (total + (int64_t)kPartialTarget * 1024 - 1) / ((int64_t)kPartialTarget * 1024);
  span = span < 4 ? 4 : span;
  if (span > INT32_MAX) return hipErrorInvalidValue;
  int64_t done = 0;
  for (int l = 0; l < n_lists; ++l) {
    const int64_t blocks = lay_out(lists[l], span);
    if (blocks == 0) return hipErrorInvalidValue;
    hipLaunchKernelGGL(grad_squares_kernel, dim3((unsigned)blocks), dim3(kThreads), 0, stream, lists[l], partials + done);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    done += blocks;
  }
  hipLaunchKernelGGL(grad_stats_kernel, dim3(1), dim3(kThreads), 0, stream, partials, (int)done, grad_scale, max_norm, stats);
  return hipGetLastError();
}

hipError_t launch_scale_grads(GradGroup& g, const GradStats* stats, hipStream_t stream) {
  if (g.count <= 0) return hipSuccess;
  if (g.count > kGradTensors) return hipErrorInvalidValue;
  int64_t span = 4, blocks;
  while ((blocks = lay_out(g, span)) == 0) {
    span *= 2;
    if (span > 512) return hipErrorInvalidValue;   // offsets within a span stay under 2^20
  }
  hipLaunchKernelGGL(scale_grads_kernel, dim3((unsigned)blocks), dim3(kThreads), 0, stream, g, stats);
  return hipGetLastError();
}

}  // namespace galore
