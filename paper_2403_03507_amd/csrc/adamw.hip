// AdamW (decoupled weight decay) over a list of tensors, one launch for up to 56 of them (44 with 8-bit moments): the
// step of the parameters that GaLore leaves alone.  Per element, with g = scale * G (scale: the clip factor of
// galore_grad_norm, or 1):
//     m = b1 m + (1-b1) g ;  v = b2 v + (1-b2) g^2 ;  n = (m / (1-b1^k)) / (sqrt(v / (1-b2^k)) + eps)
//     W = (1 - lr wd) W - lr n
// evaluated in fp32; W is rounded once, to its own type (with a master copy the fp32 master takes the update and W is its
// rounding).  Moments: fp32 (adam_entry.hpp: the expression of the low-rank kernels) or the 8-bit block-wise codes of
// adam_q8.hip, with blocks of 256 consecutive elements of the whole tensor.
#include "adamw.hpp"

#include "adam_entry.hpp"
#include "tensor_list.hpp"

namespace galore {
namespace {

constexpr int kThreads = 256;

struct Scalars {
  float scale, beta1, beta2, eps, lr, inv_c1, inv_c2, keep;
};

__device__ __forceinline__ float apply(float w, float n, const Scalars& s) { return __builtin_fmaf(-s.lr, n, s.keep * w); }

// ---- fp32 moments ----------------------------------------------------------------------------------

template <class TW, class TG, bool MASTER>
__device__ __forceinline__ void adamw_span(const AdamWTensor& p, const Scalars& s, int64_t first, int n) {
  typedef ListF32<4> f4;
  float* __restrict__ M = p.M + first;
  float* __restrict__ V = p.V + first;
  float* __restrict__ X = MASTER ? p.master + first : nullptr;
  TW* __restrict__ W = static_cast<TW*>(p.W);
  const TG* __restrict__ G = static_cast<const TG*>(p.G);
  const auto step4 = [&](f4 g, f4& m, f4& v, f4& w) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float me = m[e], ve = v[e];
      const float ne = adam_entry(s.scale * g[e], me, ve, s.beta1, s.beta2, s.eps, s.inv_c1, s.inv_c2);
      m[e] = me; v[e] = ve;
      w[e] = apply(w[e], ne, s);
    }
  };
  const auto one = [&](int o, int64_t aw, int64_t ag) {
    float m = M[o], v = V[o];
    const float ne = adam_entry(s.scale * (float)G[ag], m, v, s.beta1, s.beta2, s.eps, s.inv_c1, s.inv_c2);
    M[o] = m; V[o] = v;
    const float w = apply(MASTER ? X[o] : (float)W[aw], ne, s);
    if (MASTER) X[o] = w;
    W[aw] = (TW)w;
  };
  const bool dense = p.ldw == p.cols && p.ldg == p.cols;
  if (dense) {
    W += first; G += first;
    for (int o = threadIdx.x * 4; o < n; o += kThreads * 4) {
      if (o + 4 <= n) {
        const f4 g = list_load<4>(G + o);
        f4 m = list_load<4>(M + o), v = list_load<4>(V + o);
        f4 w = MASTER ? list_load<4>(X + o) : list_load<4>(W + o);
        step4(g, m, v, w);
        list_store<4>(M + o, m);
        list_store<4>(V + o, v);
        if (MASTER) list_store<4>(X + o, w);
        list_store<4>(W + o, w);
      } else {
        for (int e = o; e < n; ++e) one(e, e, e);
      }
    }
    return;
  }
  const RowWalk walk_w(first, p.cols, p.ldw), walk_g(first, p.cols, p.ldg);
  for (int o = threadIdx.x * 4; o < n; o += kThreads * 4) {
    uint32_t left;
    const int64_t aw = walk_w.at(o, left), ag = walk_g.at(o, left);
    if (o + 4 <= n && left >= 4) {
      const f4 g = list_load<4>(G + ag);
      f4 m = list_load<4>(M + o), v = list_load<4>(V + o);
      f4 w = MASTER ? list_load<4>(X + o) : list_load<4>(W + aw);
      step4(g, m, v, w);
      list_store<4>(M + o, m);
      list_store<4>(V + o, v);
      if (MASTER) list_store<4>(X + o, w);
      list_store<4>(W + aw, w);
    } else {
      for (int e = o; e < o + 4 && e < n; ++e) one(e, walk_w.at(e, left), walk_g.at(e, left));
    }
  }
}

__global__ __launch_bounds__(kThreads) void adamw_list_kernel(const AdamWGroup grp) {
  Scalars s{1.f, grp.call.beta1, grp.call.beta2, grp.call.eps, grp.call.lr, grp.call.inv_c1, grp.call.inv_c2, 1.f};
  if (grp.call.stats) {
    if (grp.call.stats->finite != 1.f) return;  // the whole step is left out
    s.scale = grp.call.stats->scale;
  }
  const int i = tensor_of_block(grp.begin, grp.call.count, blockIdx.x);
  const AdamWTensor& p = grp.t[i];
  s.keep = p.keep;
  const int64_t first = (int64_t)(blockIdx.x - grp.begin[i]) * grp.call.span, rest = p.count - first;
  const int n = rest < grp.call.span ? (int)rest : grp.call.span;
  const bool master = p.master != nullptr;
  switch (grp.types[i]) {
    case 0: adamw_span<float, float, false>(p, s, first, n); break;
    case 2: adamw_span<float, __bf16, false>(p, s, first, n); break;
    case 1:
      if (master) adamw_span<__bf16, float, true>(p, s, first, n);
      else adamw_span<__bf16, float, false>(p, s, first, n);
      break;
    default:
      if (master) adamw_span<__bf16, __bf16, true>(p, s, first, n);
      else adamw_span<__bf16, __bf16, false>(p, s, first, n);
  }
}

// ---- 8-bit moments -----------------------------------------------------------------------------------

typedef float q_f32x2 __attribute__((ext_vector_type(2)));

// Maximum over the 32 lanes that hold one block, every lane gets it; NaN if one of them is NaN.
__device__ __forceinline__ float block_max(float x) {
  auto dpp = [](float v, auto ctrl) {
    const int b = __builtin_bit_cast(int, v);
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(b, b, decltype(ctrl)::value, 0xF, 0xF, false));
  };
  using std::integral_constant;
  x = __builtin_elementwise_maximum(x, dpp(x, integral_constant<int, 0xB1>{}));    // quad_perm [1,0,3,2]
  x = __builtin_elementwise_maximum(x, dpp(x, integral_constant<int, 0x4E>{}));    // quad_perm [2,3,0,1]
  x = __builtin_elementwise_maximum(x, dpp(x, integral_constant<int, 0x141>{}));   // row_half_mirror
  x = __builtin_elementwise_maximum(x, dpp(x, integral_constant<int, 0x140>{}));   // row_mirror
  const int y = __builtin_amdgcn_ds_swizzle(__builtin_bit_cast(int, x), 0x401F);   // the lane 16 away
  return __builtin_elementwise_maximum(x, __builtin_bit_cast(float, y));
}

// First-moment codes are OCP e4m3 numbers, 256 times the magnitude: the hardware's conversions decode and encode them
// (round to nearest even, subnormals included).
__device__ __forceinline__ void decode_m4(uint32_t c, float scale, float* m) {
  const q_f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(c, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(c, true);
  m[0] = a[0] * 0x1p-8f * scale; m[1] = a[1] * 0x1p-8f * scale;
  m[2] = b[0] * 0x1p-8f * scale; m[3] = b[1] * 0x1p-8f * scale;
}
__device__ __forceinline__ uint32_t encode_m4(const float* m, float inverse) {
  float y[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = __builtin_amdgcn_fmed3f(m[e] * inverse, -1.f, 1.f) * 256.f;
  int c = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], c, true);
}
// Second-moment codes (5 exponent bits from 2^-30, 3 mantissa bits, no sign) are the bits of an fp32 number from bit 20
// on, 2^96 too small; its subnormals are the codes' own.
__device__ __forceinline__ void decode_v4(uint32_t c, float scale, float* v) {
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = __builtin_bit_cast(float, ((c >> (8 * e)) & 0xFFu) << 20) * 0x1p96f * scale;
}
__device__ __forceinline__ uint32_t encode_v4(const float* v, float inverse) {
  uint32_t out = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float y = fminf(v[e] * inverse, 1.f);
    const uint32_t bits = __builtin_bit_cast(uint32_t, y);
    // nearest, ties to even, in 3 mantissa bits; below 2^-30 in steps of 2^-33, which an addition to 2^-10 rounds to
    const uint32_t normal = ((bits + 0x7FFFFu + ((bits >> 20) & 1u)) >> 20) - (96u << 3);
    const uint32_t small = __builtin_bit_cast(uint32_t, y + 0x1p-10f) & 0xFu;
    out |= (y >= 0x1p-30f ? normal : small) << (8 * e);
  }
  return out;
}

template <class TW, class TG, bool MASTER>
__device__ __forceinline__ void adamw_q8_span(const AdamWQ8Tensor& p, const Scalars& s, int64_t first, int n) {
#pragma clang fp contract(off)
  typedef ListF32<8> f8;
  uint8_t* __restrict__ Mc = p.Mc + first;
  uint8_t* __restrict__ Vc = p.Vc + first;
  float* __restrict__ Ms = p.Ms + (first >> 8);
  float* __restrict__ Vs = p.Vs + (first >> 8);
  float* __restrict__ X = MASTER ? p.master + first : nullptr;
  TW* __restrict__ W = static_cast<TW*>(p.W);
  const TG* __restrict__ G = static_cast<const TG*>(p.G);
  const bool dense = p.ldw == p.cols && p.ldg == p.cols;
  const RowWalk walk_w(first, p.cols, p.ldw), walk_g(first, p.cols, p.ldg);
  if (dense) { W += first; G += first; }
  const float omb1 = 1.f - s.beta1, omb2 = 1.f - s.beta2;
  const int in_block = (threadIdx.x & 31) * 8;
  for (int b = threadIdx.x >> 5; b * 256 < n; b += kThreads / 32) {  // the 32 lanes of a block stay together
    const int o = b * 256 + in_block;
    uint32_t left_w = 8, left_g = 8;
    const int64_t aw = dense ? o : walk_w.at(o, left_w), ag = dense ? o : walk_g.at(o, left_g);
    const bool whole = o + 8 <= n && left_w >= 8 && left_g >= 8;
    uint2 cm{0, 0}, cv{0, 0};
    f8 g = 0.f, w = 0.f;
    if (whole) {
      g = list_load<8>(G + ag);
      cm = *reinterpret_cast<const uint2*>(Mc + o);
      cv = *reinterpret_cast<const uint2*>(Vc + o);
      w = MASTER ? list_load<8>(X + o) : list_load<8>(W + aw);
    } else {
      uint32_t lm[2] = {0, 0}, lv[2] = {0, 0};
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (o + e < n) {
          uint32_t left;
          g[e] = (float)G[dense ? o + e : walk_g.at(o + e, left)];
          w[e] = MASTER ? X[o + e] : (float)W[dense ? o + e : walk_w.at(o + e, left)];
          lm[e >> 2] |= (uint32_t)Mc[o + e] << (8 * (e & 3));
          lv[e >> 2] |= (uint32_t)Vc[o + e] << (8 * (e & 3));
        }
      }
      cm = uint2{lm[0], lm[1]}; cv = uint2{lv[0], lv[1]};
    }
    const float sm = Ms[b], sv = Vs[b];
    float m[8], v[8];
    decode_m4(cm.x, sm, m); decode_m4(cm.y, sm, m + 4);
    decode_v4(cv.x, sv, v); decode_v4(cv.y, sv, v + 4);
    float amax = 0.f, vmax = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float ge = s.scale * g[e];
      const float gm = omb1 * ge;
      m[e] = __builtin_fmaf(s.beta1, m[e], gm);
      float gv = omb2 * ge;
      gv = gv * ge;
      v[e] = __builtin_fmaf(s.beta2, v[e], gv);
      const float den = __builtin_sqrtf(v[e] * s.inv_c2) + s.eps;
      w[e] = apply(w[e], (m[e] * s.inv_c1) / den, s);
      amax = __builtin_elementwise_maximum(amax, __builtin_fabsf(m[e]));
      vmax = __builtin_elementwise_maximum(vmax, v[e]);
    }
    amax = block_max(amax);
    vmax = block_max(vmax);
    const float inv_m = amax != 0.f ? 1.f / amax : 0.f, inv_v = vmax != 0.f ? 1.f / vmax : 0.f;
    cm = uint2{encode_m4(m, inv_m), encode_m4(m + 4, inv_m)};
    cv = uint2{encode_v4(v, inv_v), encode_v4(v + 4, inv_v)};
    if (in_block == 0) { Ms[b] = amax; Vs[b] = vmax; }
    if (whole) {
      *reinterpret_cast<uint2*>(Mc + o) = cm;
      *reinterpret_cast<uint2*>(Vc + o) = cv;
      if (MASTER) list_store<8>(X + o, w);
      list_store<8>(W + aw, w);
    } else {
      const uint32_t lm[2] = {cm.x, cm.y}, lv[2] = {cv.x, cv.y};
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (o + e < n) {
          uint32_t left;
          Mc[o + e] = (uint8_t)(lm[e >> 2] >> (8 * (e & 3)));
          Vc[o + e] = (uint8_t)(lv[e >> 2] >> (8 * (e & 3)));
          if (MASTER) X[o + e] = w[e];
          W[dense ? o + e : walk_w.at(o + e, left)] = (TW)w[e];
        }
      }
    }
  }
}

__global__ __launch_bounds__(kThreads) void adamw_q8_list_kernel(const AdamWQ8Group grp) {
  Scalars s{1.f, grp.call.beta1, grp.call.beta2, grp.call.eps, grp.call.lr, grp.call.inv_c1, grp.call.inv_c2, 1.f};
  if (grp.call.stats) {
    if (grp.call.stats->finite != 1.f) return;
    s.scale = grp.call.stats->scale;
  }
  const int i = tensor_of_block(grp.begin, grp.call.count, blockIdx.x);
  const AdamWQ8Tensor& p = grp.t[i];
  s.keep = p.keep;
  const int64_t first = (int64_t)(blockIdx.x - grp.begin[i]) * grp.call.span, rest = p.count - first;
  const int n = rest < grp.call.span ? (int)rest : grp.call.span;
  const bool master = p.master != nullptr;
  switch (grp.types[i]) {
    case 0: adamw_q8_span<float, float, false>(p, s, first, n); break;
    case 2: adamw_q8_span<float, __bf16, false>(p, s, first, n); break;
    case 1:
      if (master) adamw_q8_span<__bf16, float, true>(p, s, first, n);
      else adamw_q8_span<__bf16, float, false>(p, s, first, n);
      break;
    default:
      if (master) adamw_q8_span<__bf16, __bf16, true>(p, s, first, n);
      else adamw_q8_span<__bf16, __bf16, false>(p, s, first, n);
  }
}

// Elements per workgroup for a list, and the first workgroup of every tensor; returns the number of workgroups, 0 if the
// list does not fit one launch.
template <class Group> int64_t lay_out(Group& g) {
  int64_t total = 0;
  for (int i = 0; i < g.call.count; ++i) total += g.t[i].count;
  int64_t span = 2048;
  int64_t blocks;
  for (;; span *= 2) {
    blocks = 0;
    for (int i = 0; i < g.call.count; ++i) {
      g.begin[i] = (int32_t)blocks;
      blocks += (g.t[i].count + span - 1) / span;
      if (blocks > kMaxBlocks) break;
    }
    if (blocks <= kMaxBlocks && (total <= (int64_t)1 << 22 || span >= 8192)) break;
    if (span >= (int64_t)1 << 19) return 0;
  }
  g.call.span = (int32_t)span;
  return blocks;
}

}  // namespace

hipError_t launch_adamw(AdamWGroup& g, hipStream_t stream) {
  if (g.call.count <= 0) return hipSuccess;
  if (g.call.count > kAdamWTensors) return hipErrorInvalidValue;
  const int64_t blocks = lay_out(g);
  if (blocks == 0) return hipErrorInvalidValue;
  hipLaunchKernelGGL(adamw_list_kernel, dim3((unsigned)blocks), dim3(kThreads), 0, stream, g);
  return hipGetLastError();
}

hipError_t launch_adamw_q8(AdamWQ8Group& g, hipStream_t stream) {
  if (g.call.count <= 0) return hipSuccess;
  if (g.call.count > kAdamWQ8Tensors) return hipErrorInvalidValue;
  const int64_t blocks = lay_out(g);
  if (blocks == 0) return hipErrorInvalidValue;
  hipLaunchKernelGGL(adamw_q8_list_kernel, dim3((unsigned)blocks), dim3(kThreads), 0, stream, g);
  return hipGetLastError();
}

}  // namespace galore
