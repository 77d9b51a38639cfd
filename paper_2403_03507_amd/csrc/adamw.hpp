// AdamW over a list of tensors (adamw.hip) and the norm and scaling of a list of gradients (grad_norm.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "common.hpp"

namespace galore {

// What galore_grad_norm leaves on the device and the calls after it read.
struct GradStats {
  float norm, scale, finite, reserved;
};

// Step count, learning rate and bias corrections on the device (galore_adamw_clock).
struct AdamWClock {
  int64_t t;
  float lr, inv_c1, inv_c2, reserved;
};
hipError_t launch_adamw_tick(AdamWClock* clock, float beta1, float beta2, const GradStats* stats, hipStream_t stream);

// A kernel's arguments stay under 4 KiB: so many tensors per launch.
constexpr int kAdamWTensors = 56, kAdamWRuns = 89;
constexpr int kAdamWQ8Tensors = 44, kAdamWQ8Runs = 66;
constexpr int kGradTensors = 128;

struct AdamWTensor {
  void* W;
  const void* G;
  float* M;
  float* V;
  float* master;   // NULL: W is its own master
  int64_t count;   // rows * cols
  int32_t cols, ldw, ldg;
  float decay;     // weight decay
};

struct AdamWQ8Tensor {
  void* W;
  const void* G;
  uint8_t* Mc;
  uint8_t* Vc;
  float* Ms;
  float* Vs;
  float* master;
  int64_t count;
  int32_t cols, ldw, ldg;
  float decay;
};

// A tensor without a master copy and without gaps between its rows, of fewer than 2^31 elements: what most lists hold.  The
// shorter description saves launches of long lists (65 norm weights of 4096: one instead of two, 9.2 us a call instead of 11.6;
// 279 matrices and vectors with 8-bit moments: five instead of seven, 82.6 instead of 92.7).
struct AdamWRun {
  void* W;
  const void* G;
  float* M;
  float* V;
  int32_t count;
  float decay;
};
struct AdamWQ8Run {
  void* W;
  const void* G;
  uint8_t* Mc;
  uint8_t* Vc;
  float* Ms;
  float* Vs;
  int32_t count;
  float decay;
};

struct AdamWCall {
  const GradStats* stats;  // NULL: gradients as they are
  const AdamWClock* clock; // NULL: lr and the corrections below
  float beta1, beta2, eps, lr;
  float inv_c1, inv_c2;    // 1 / (1 - beta^k)
  int32_t count;
  int32_t block0;          // first workgroup of the launch in the list
};

template <class Tensor, int N> struct AdamWList {
  AdamWCall call;
  int32_t begin[N];        // first workgroup of a tensor in the launch
  uint8_t types[N];        // bit 0: W is bf16, bit 1: G is bf16
  Tensor t[N];
};
typedef AdamWList<AdamWTensor, kAdamWTensors> AdamWGroup;
typedef AdamWList<AdamWRun, kAdamWRuns> AdamWRunGroup;
typedef AdamWList<AdamWQ8Tensor, kAdamWQ8Tensors> AdamWQ8Group;
typedef AdamWList<AdamWQ8Run, kAdamWQ8Runs> AdamWQ8RunGroup;
static_assert(sizeof(AdamWGroup) <= 4096 && sizeof(AdamWRunGroup) <= 4096, "kernel arguments");
static_assert(sizeof(AdamWQ8Group) <= 4096 && sizeof(AdamWQ8RunGroup) <= 4096, "kernel arguments");

// The host fills everything but begin and block0.
hipError_t launch_adamw(AdamWGroup& g, hipStream_t stream);
hipError_t launch_adamw(AdamWRunGroup& g, hipStream_t stream);
hipError_t launch_adamw(AdamWQ8Group& g, hipStream_t stream);
hipError_t launch_adamw(AdamWQ8RunGroup& g, hipStream_t stream);

struct GradTensor {
  void* G;
  int64_t count;
  int32_t cols, ld;
};

struct GradGroup {
  int32_t count;
  int32_t span;            // norm: 1024s of elements per workgroup
  int32_t block0;          // scaling: first workgroup of the launch in the list
  int32_t begin[kGradTensors];
  uint8_t bf16[kGradTensors];
  GradTensor t[kGradTensors];
};
static_assert(sizeof(GradGroup) <= 4000, "kernel arguments");

// Partial sums of squares, one per workgroup: an upper bound for a list of `count` tensors.
size_t grad_norm_partials(int32_t count);
// lists: the whole list in groups of kGradTensors.  partials: grad_norm_partials(count) doubles.
hipError_t launch_grad_norm(GradGroup* lists, int n_lists, float grad_scale, float max_norm, GradStats* stats, double* partials, hipStream_t stream);
hipError_t launch_scale_grads(GradGroup& g, const GradStats* stats, hipStream_t stream);

}  // namespace galore
