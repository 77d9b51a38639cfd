// AdamW over a list of tensors, the global norm of a list of gradients and their scaling, behind the C ABI: validation
// of the whole list, then as few launches as the kernels' argument space allows.  No context, nothing allocated.
#include "adamw.hpp"
#include "api_internal.hpp"

#include <cmath>
#include <type_traits>
#include <vector>

using namespace galore;
using namespace galore::api;

static_assert(sizeof(galore_grad_stats) == sizeof(GradStats) && sizeof(galore_adamw_clock) == sizeof(AdamWClock) &&
                  offsetof(galore_adamw_clock, lr) == offsetof(AdamWClock, lr),
              "the device's view of the ABI's structs");

namespace {

constexpr int64_t kBlock = 256;   // elements under one scale of the 8-bit moments

// No two of the addresses that a call writes may be the same (the same tensor twice in a list, one buffer for two states).
// A table with open addressing: a call on a small list costs the host more than the GPU (67 tensors: 6 us in all; 16 with the
// addresses sorted).
class Addresses {
 public:
  explicit Addresses(size_t most) {
    size_t n = 16;
    while (n < 2 * most) n *= 2;
    slots_.assign(n, nullptr);
  }
  bool add(const void* p) {   // false: already there
    const void*& slot = find(p);
    if (slot) return false;
    slot = p;
    return true;
  }
  bool has(const void* p) { return find(p) != nullptr; }

 private:
  const void*& find(const void* p) {   // p's slot, or the free one where it belongs
    size_t h = (size_t)((reinterpret_cast<uintptr_t>(p) >> 2) * 0x9E3779B97F4A7C15ull >> 20);
    for (;; ++h) {
      const void*& slot = slots_[h & (slots_.size() - 1)];
      if (!slot || slot == p) return slot;
    }
  }
  std::vector<const void*> slots_;   // no tensor starts at NULL
};

galore_status fail_twice(const char* what, int i) {
  return fail(nullptr, GALORE_ERR_INVALID_ARG, "%s[%d] starts at the same address as a tensor that the call writes", what, i);
}

galore_status check_stats(const galore_grad_stats* stats) {
  if (reinterpret_cast<uintptr_t>(stats) & 15) return fail(nullptr, GALORE_ERR_ALIGN, "stats must be 16-byte aligned");
  return GALORE_OK;
}

galore_status check_clock(const galore_adamw_clock* clock) {
  if (reinterpret_cast<uintptr_t>(clock) & 7) return fail(nullptr, GALORE_ERR_ALIGN, "clock must be 8-byte aligned");
  return GALORE_OK;
}

galore_status check_betas(float beta1, float beta2) {
  if (!(beta1 >= 0.f && beta1 < 1.f) || !(beta2 >= 0.f && beta2 < 1.f)) return fail(nullptr, GALORE_ERR_INVALID_ARG, "betas must lie in [0, 1)");
  return GALORE_OK;
}

// fp32 or U8 state of W's shape, dense and aligned
galore_status check_moment(const galore_tensor& t, const char* what, int i, const galore_tensor& W, int32_t dtype) {
  galore_status s = check_matrix(nullptr, t, what, i, true, true);
  if (s) return s;
  if (t.dtype != dtype) return fail(nullptr, GALORE_ERR_DTYPE, "%s[%d] has the wrong dtype", what, i);
  if (t.rows != W.rows || t.cols != W.cols || t.ld != t.cols) return fail(nullptr, GALORE_ERR_STATE, "%s[%d] must be dense with W's shape", what, i);
  if (reinterpret_cast<uintptr_t>(t.data) & 15) return fail(nullptr, GALORE_ERR_ALIGN, "%s[%d] must be 16-byte aligned", what, i);
  return GALORE_OK;
}

galore_status check_scales(const galore_tensor& t, const char* what, int i, int64_t blocks) {
  galore_status s = check_matrix(nullptr, t, what, i, true);
  if (s) return s;
  if (t.dtype != GALORE_F32) return fail(nullptr, GALORE_ERR_DTYPE, "%s[%d] must be fp32", what, i);
  if (t.rows * t.cols != blocks || t.ld != t.cols)
    return fail(nullptr, GALORE_ERR_STATE, "%s[%d] must hold %lld scales, dense", what, i, (long long)blocks);
  if (reinterpret_cast<uintptr_t>(t.data) & 3) return fail(nullptr, GALORE_ERR_ALIGN, "%s[%d] must be 4-byte aligned", what, i);
  return GALORE_OK;
}

galore_status check_element_alignment(const galore_tensor& t, const char* what, int i) {
  if (reinterpret_cast<uintptr_t>(t.data) % (t.dtype == GALORE_F32 ? 4 : 2))
    return fail(nullptr, GALORE_ERR_ALIGN, "%s[%d] must be aligned to its elements", what, i);
  return GALORE_OK;
}

// A matrix of one row, or with rows that follow each other, is one run of elements.
int32_t run_ld(const galore_tensor& t) { return (int32_t)(t.rows == 1 ? t.cols : t.ld); }

galore_status fill_grads(const galore_tensor* G, int32_t count, std::vector<GradGroup>& lists) {
  if (count < 0) return fail(nullptr, GALORE_ERR_INVALID_ARG, "count %d < 0", count);
  if (count > 0 && !G) return fail(nullptr, GALORE_ERR_INVALID_ARG, "G is NULL");
  lists.resize(((size_t)count + kGradTensors - 1) / kGradTensors);
  for (int32_t i = 0; i < count; ++i) {
    galore_status s = check_matrix(nullptr, G[i], "G", i, true);
    if (s || (s = check_element_alignment(G[i], "G", i))) return s;
    GradGroup& g = lists[(size_t)i / kGradTensors];
    const int j = g.count++;
    g.bf16[j] = G[i].dtype == GALORE_BF16;
    g.t[j].G = G[i].data;
    g.t[j].count = G[i].rows * G[i].cols;
    g.t[j].cols = (int32_t)G[i].cols;
    g.t[j].ld = run_ld(G[i]);
  }
  return GALORE_OK;
}

}  // namespace

extern "C" {

galore_status galore_adamw(const galore_tensor* W, const galore_tensor* G, const galore_adamw_state* S, int32_t count, float beta1,
                           float beta2, float eps, float lr, int64_t k, const galore_adamw_clock* clock, const galore_grad_stats* stats,
                           void* hip_stream) try {
  if (count < 0) return fail(nullptr, GALORE_ERR_INVALID_ARG, "count %d < 0", count);
  if (count > 0 && (!W || !G || !S)) return fail(nullptr, GALORE_ERR_INVALID_ARG, "W / G / S is NULL");
  galore_status s;
  if ((s = check_betas(beta1, beta2)) || (s = check_stats(stats)) || (s = check_clock(clock))) return s;
  if (!(eps >= 0.f)) return fail(nullptr, GALORE_ERR_INVALID_ARG, "eps out of range");
  if (!clock) {
    if (!std::isfinite(lr)) return fail(nullptr, GALORE_ERR_INVALID_ARG, "lr is not finite");
    if (k < 1) return fail(nullptr, GALORE_ERR_INVALID_ARG, "k must be >= 1");
  }
  Addresses written((size_t)count * 6);
  for (int32_t i = 0; i < count; ++i) {
    const galore_adamw_state& st = S[i];
    if ((s = check_matrix(nullptr, W[i], "W", i, true)) || (s = check_matrix(nullptr, G[i], "G", i, true)) ||
        (s = check_element_alignment(W[i], "W", i)) || (s = check_element_alignment(G[i], "G", i)))
      return s;
    if (G[i].rows != W[i].rows || G[i].cols != W[i].cols) return fail(nullptr, GALORE_ERR_SHAPE, "G[%d] must have W's shape", i);
    if (!(st.weight_decay >= 0.f) || !std::isfinite(st.weight_decay)) return fail(nullptr, GALORE_ERR_INVALID_ARG, "weight_decay of tensor %d out of range", i);
    const bool q8 = st.m.dtype == GALORE_U8;
    if ((s = check_moment(st.m, "m", i, W[i], q8 ? GALORE_U8 : GALORE_F32)) || (s = check_moment(st.v, "v", i, W[i], q8 ? GALORE_U8 : GALORE_F32)))
      return s;
    if (q8) {
      const int64_t blocks = (W[i].rows * W[i].cols + kBlock - 1) / kBlock;
      if ((s = check_scales(st.m_scale, "m_scale", i, blocks)) || (s = check_scales(st.v_scale, "v_scale", i, blocks))) return s;
      if (!written.add(st.m_scale.data)) return fail_twice("m_scale", i);
      if (!written.add(st.v_scale.data)) return fail_twice("v_scale", i);
    }
    if (st.master.data) {
      if (W[i].dtype != GALORE_BF16) return fail(nullptr, GALORE_ERR_DTYPE, "master copies belong to bf16 weights (tensor %d)", i);
      if ((s = check_moment(st.master, "master", i, W[i], GALORE_F32))) return s;
      if (!written.add(st.master.data)) return fail_twice("master", i);
    }
    if (!written.add(W[i].data)) return fail_twice("W", i);
    if (!written.add(st.m.data)) return fail_twice("m", i);
    if (!written.add(st.v.data)) return fail_twice("v", i);
  }
  for (int32_t i = 0; i < count; ++i)
    if (written.has(G[i].data)) return fail_twice("G", i);

  AdamWCall call{};
  call.stats = reinterpret_cast<const GradStats*>(stats);
  call.clock = reinterpret_cast<const AdamWClock*>(clock);
  call.beta1 = beta1; call.beta2 = beta2; call.eps = eps;
  if (!clock) {
    call.lr = lr;
    call.inv_c1 = (float)(1.0 / (1.0 - std::pow((double)beta1, (double)k)));
    call.inv_c2 = (float)(1.0 / (1.0 - std::pow((double)beta2, (double)k)));
  }
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  hipError_t e = hipSuccess;
  // Tensors of one state format share launches; the short descriptions if they suit all of them.
  const auto is_q8 = [&](int32_t i) { return S[i].m.dtype == GALORE_U8; };
  const auto fill = [&](auto& t, int32_t i) {
    t.W = W[i].data; t.G = G[i].data;
    t.decay = S[i].weight_decay;
    if constexpr (std::is_same<decltype(t.count), int64_t>::value) {
      t.master = static_cast<float*>(S[i].master.data);
      t.cols = (int32_t)W[i].cols; t.ldw = run_ld(W[i]); t.ldg = run_ld(G[i]);
    }
    t.count = static_cast<decltype(t.count)>(W[i].rows * W[i].cols);
  };
  const auto fill_f32 = [&](auto& t, int32_t i) {
    fill(t, i);
    t.M = static_cast<float*>(S[i].m.data); t.V = static_cast<float*>(S[i].v.data);
  };
  const auto fill_q8 = [&](auto& t, int32_t i) {
    fill(t, i);
    t.Mc = static_cast<uint8_t*>(S[i].m.data); t.Vc = static_cast<uint8_t*>(S[i].v.data);
    t.Ms = static_cast<float*>(S[i].m_scale.data); t.Vs = static_cast<float*>(S[i].v_scale.data);
  };
  const auto launch = [&](auto group, bool q8, const auto& fill_one) -> hipError_t {
    constexpr int kMost = (int)(sizeof(group.t) / sizeof(group.t[0]));
    group.call = call;
    for (int32_t i = 0; i < count; ++i) {
      if (is_q8(i) != q8) continue;
      const int j = group.call.count++;
      group.types[j] = (uint8_t)((W[i].dtype == GALORE_BF16 ? 1 : 0) | (G[i].dtype == GALORE_BF16 ? 2 : 0));
      fill_one(group.t[j], i);
      if (group.call.count == kMost) {
        const hipError_t e = launch_adamw(group, stream);
        if (e != hipSuccess) return e;
        group.call.count = 0;
      }
    }
    return launch_adamw(group, stream);
  };
  int32_t tensors[2] = {0, 0}, runs[2] = {0, 0};   // by format
  for (int32_t i = 0; i < count; ++i) {
    ++tensors[is_q8(i)];
    runs[is_q8(i)] += !S[i].master.data && run_ld(W[i]) == W[i].cols && run_ld(G[i]) == G[i].cols && W[i].rows * W[i].cols <= INT32_MAX;
  }
  if (tensors[0]) e = runs[0] == tensors[0] ? launch(AdamWRunGroup{}, false, fill_f32) : launch(AdamWGroup{}, false, fill_f32);
  if (e == hipSuccess && tensors[1]) e = runs[1] == tensors[1] ? launch(AdamWQ8RunGroup{}, true, fill_q8) : launch(AdamWQ8Group{}, true, fill_q8);
  return e == hipSuccess ? GALORE_OK : hip_fail(nullptr, e, "AdamW launch");
} catch (...) {
  return fail(nullptr, GALORE_ERR_INVALID_ARG, "out of host memory");
}

galore_status galore_adamw_tick(galore_adamw_clock* clock, float beta1, float beta2, const galore_grad_stats* stats, void* hip_stream) {
  if (!clock) return fail(nullptr, GALORE_ERR_INVALID_ARG, "clock is NULL");
  galore_status s;
  if ((s = check_betas(beta1, beta2)) || (s = check_stats(stats)) || (s = check_clock(clock))) return s;
  const hipError_t e = launch_adamw_tick(reinterpret_cast<AdamWClock*>(clock), beta1, beta2, reinterpret_cast<const GradStats*>(stats),
                                         static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? GALORE_OK : hip_fail(nullptr, e, "AdamW tick launch");
}

galore_status galore_grad_norm_workspace_bytes(int32_t count, size_t* out_bytes) {
  if (count < 0 || !out_bytes) return fail(nullptr, GALORE_ERR_INVALID_ARG, "count < 0 or out_bytes is NULL");
  *out_bytes = align_up(grad_norm_partials(count) * sizeof(double));
  return GALORE_OK;
}

galore_status galore_grad_norm(const galore_tensor* G, int32_t count, float grad_scale, float max_norm, galore_grad_stats* stats,
                               void* workspace, size_t workspace_bytes, void* hip_stream) try {
  if (!stats) return fail(nullptr, GALORE_ERR_INVALID_ARG, "stats is NULL");
  if (!std::isfinite(grad_scale)) return fail(nullptr, GALORE_ERR_INVALID_ARG, "grad_scale is not finite");
  if (!(max_norm > 0.f)) return fail(nullptr, GALORE_ERR_INVALID_ARG, "max_norm must be > 0 (infinity: no clipping)");
  galore_status s = check_stats(stats);
  if (s) return s;
  std::vector<GradGroup> lists;
  if ((s = fill_grads(G, count, lists))) return s;
  if (!workspace) return fail(nullptr, GALORE_ERR_WORKSPACE, "workspace is NULL");
  if (reinterpret_cast<uintptr_t>(workspace) % kAlign != 0) return fail(nullptr, GALORE_ERR_ALIGN, "workspace must be 256-byte aligned");
  const size_t need = grad_norm_partials(count) * sizeof(double);
  if (workspace_bytes < need) return fail(nullptr, GALORE_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", workspace_bytes, need);
  const hipError_t e = launch_grad_norm(lists.data(), (int)lists.size(), grad_scale, max_norm, reinterpret_cast<GradStats*>(stats),
                                        static_cast<double*>(workspace), static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? GALORE_OK : hip_fail(nullptr, e, "gradient norm launch");
} catch (...) {
  return fail(nullptr, GALORE_ERR_INVALID_ARG, "out of host memory");
}

galore_status galore_scale_grads(const galore_tensor* G, int32_t count, const galore_grad_stats* stats, void* hip_stream) try {
  if (!stats) return fail(nullptr, GALORE_ERR_INVALID_ARG, "stats is NULL");
  galore_status s = check_stats(stats);
  if (s) return s;
  std::vector<GradGroup> lists;
  if ((s = fill_grads(G, count, lists))) return s;
  Addresses written((size_t)count);
  for (int32_t i = 0; i < count; ++i)
    if (!written.add(G[i].data)) return fail_twice("G", i);
  hipError_t e = hipSuccess;
  for (size_t l = 0; l < lists.size() && e == hipSuccess; ++l)
    e = launch_scale_grads(lists[l], reinterpret_cast<const GradStats*>(stats), static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? GALORE_OK : hip_fail(nullptr, e, "gradient scaling launch");
} catch (...) {
  return fail(nullptr, GALORE_ERR_INVALID_ARG, "out of host memory");
}

}  // extern "C"
