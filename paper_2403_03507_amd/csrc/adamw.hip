// AdamW (decoupled weight decay) over a list of tensors, one launch for up to 89 of them (66 with 8-bit moments): the step
// of the parameters that GaLore leaves alone.  Per element, with g = scale * G (scale: the clip factor of
// galore_grad_norm, or 1):
//     m = b1 m + (1-b1) g ;  v = b2 v + (1-b2) g^2 ;  n = (m / (1-b1^k)) / (sqrt(v / (1-b2^k)) + eps)
//     W = (1 - lr wd) W - lr n
// evaluated in fp32; W is rounded once, to its own type (with a master copy the fp32 master takes the update and W is its
// rounding).  Moments: fp32 (adam_entry.hpp: the expression of the low-rank kernels) or the 8-bit block-wise codes of
// adam_q8.hip, with blocks of 256 consecutive elements of the whole tensor.
#include "adamw.hpp"

#include <type_traits>

#include "adam_entry.hpp"
#include "tensor_list.hpp"

namespace galore {
namespace {

// A stream that is bound by HBM: what counts is that neighbours in memory are in flight together.  So a thread takes one
// group of elements and is done (262M bf16 weights, fp32 moments: workgroups of 256 over 8192 elements 1062 us, over 2048
// 1029, over 1024 948, of 128 over 512 934, of 512 over 2048 985; two groups a thread 981).
constexpr int kThreads = 128;
constexpr int kSpan = 512;      // elements per workgroup: one group of 4 per thread
constexpr int kSpanQ8 = 1024;   // 8 per thread

struct Scalars {
  float scale, beta1, beta2, eps, lr, inv_c1, inv_c2, keep;
};

// What the tensors of a call have in common; false: the step is left out.
__device__ __forceinline__ bool scalars(const AdamWCall& c, Scalars& s) {
  s = Scalars{1.f, c.beta1, c.beta2, c.eps, c.lr, c.inv_c1, c.inv_c2, 1.f};
  if (c.clock) { s.lr = c.clock->lr; s.inv_c1 = c.clock->inv_c1; s.inv_c2 = c.clock->inv_c2; }
  if (!c.stats) return true;
  s.scale = c.stats->scale;
  return c.stats->finite == 1.f;
}

// What the short descriptions leave out.
template <class Tensor> __device__ __forceinline__ float* master_of(const Tensor& p) {
  if constexpr (std::is_same<decltype(p.count), int64_t>::value) return p.master;
  else return nullptr;
}
struct Lengths {
  int32_t cols, ldw, ldg;   // a row's length, and from one to the next in W and G
  __device__ __forceinline__ bool run() const { return ldw == cols && ldg == cols; }
};
template <class Tensor> __device__ __forceinline__ Lengths lengths_of(const Tensor& p) {
  if constexpr (std::is_same<decltype(p.count), int64_t>::value) return Lengths{p.cols, p.ldw, p.ldg};
  else return Lengths{INT32_MAX, INT32_MAX, INT32_MAX};   // one row
}

__device__ __forceinline__ float apply(float w, float n, const Scalars& s) { return __builtin_fmaf(-s.lr, n, s.keep * w); }

// ---- fp32 moments ----------------------------------------------------------------------------------
// 22 bytes per bf16 element, 28 with fp32 or master weights, each moved once and past the caches; bound by HBM: 262M bf16
// weights 908 us (6.36 TB/s), 101M with master copies 442 (6.37), 30M fp32 131 (6.39).  Arithmetic (48 instructions per
// element, IEEE square root and division among them) takes a third of that.

template <class TW, class TG, bool MASTER, class Tensor>
__device__ __forceinline__ void adamw_span(const Tensor& p, const Scalars& s, int64_t first, int n) {
  const int o = threadIdx.x * 4, have = n - o;
  if (have <= 0) return;
  float* M = p.M + first;
  float* V = p.V + first;
  float* X = MASTER ? master_of(p) + first : nullptr;
  TW* W = static_cast<TW*>(p.W);
  const TG* G = static_cast<const TG*>(p.G);
  const Lengths len = lengths_of(p);
  const RowWalk::Place run = RowWalk::Place::in_run(o);
  RowWalk::Place at = run;
  if (len.run()) { W += first; G += first; }
  else at = RowWalk(first, len.cols).at(o);
  ListF32<4> g = row_load<4>(G, len.ldg, len.cols, at, have), m = row_load<4>(M, 0, 0, run, have), v = row_load<4>(V, 0, 0, run, have);
  ListF32<4> w = MASTER ? row_load<4>(X, 0, 0, run, have) : row_load<4>(W, len.ldw, len.cols, at, have);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float me = m[e], ve = v[e];
    const float ne = adam_entry(s.scale * g[e], me, ve, s.beta1, s.beta2, s.eps, s.inv_c1, s.inv_c2);
    m[e] = me; v[e] = ve;
    w[e] = apply(w[e], ne, s);
  }
  row_store<4>(M, 0, 0, run, have, m);
  row_store<4>(V, 0, 0, run, have, v);
  if (MASTER) row_store<4>(X, 0, 0, run, have, w);
  row_store<4>(W, len.ldw, len.cols, at, have, w);
}

template <class List> __global__ __launch_bounds__(kThreads) void adamw_list_kernel(const List grp) {
  Scalars s;
  if (!scalars(grp.call, s)) return;
  const int block = grp.call.block0 + span_of_block();
  const int i = tensor_of_block(grp.begin, grp.call.count, block);
  const auto& p = grp.t[i];
  s.keep = __builtin_fmaf(-s.lr, p.decay, 1.f);
  const int64_t first = (int64_t)(block - grp.begin[i]) * kSpan, rest = p.count - first;
  const int n = rest < kSpan ? (int)rest : kSpan;
  const bool master = master_of(p) != nullptr;
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
// Half a wavefront owns a block of 256 elements, 8 to a lane.  With 10 bytes to move per bf16 element the arithmetic counts
// as much as the traffic: 64 additions or the like per element would take as long as the bytes do.  So first-moment codes
// go through the hardware's e4m3 conversions, second-moment codes are cut from fp32 bits, and the square root and the
// reciprocal of the update are the hardware's approximations of one unit in the last place (exact ones: 202M bf16 elements
// 388 us instead of 331).  Measured: 202M bf16 weights 326 us (6.2 TB/s), 60M fp32 154 (6.3).

typedef float q_f32x2 __attribute__((ext_vector_type(2)));
typedef short q_s16x2 __attribute__((ext_vector_type(2)));
constexpr int kBlock = 256, kLanes = 32;

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
  x = __builtin_elementwise_maximum(x, dpp(x, integral_constant<int, 0x140>{}));   // row_mirror: each row of 16 holds its maximum
  const int y = __builtin_amdgcn_ds_swizzle(__builtin_bit_cast(int, x), 0x401F);   // the lane 16 away, of the same 32
  return __builtin_elementwise_maximum(x, __builtin_bit_cast(float, y));
}

// First-moment codes are OCP e4m3 numbers, 256 times the magnitude: the hardware's conversions decode and encode them
// (round to nearest even, subnormals included) and take the factor 2^-8 along.
__device__ __forceinline__ void decode_m4(uint32_t c, float scale, float* m) {
  const q_f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c, 0x1p-8f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c, 0x1p-8f, true);
  m[0] = a[0] * scale; m[1] = a[1] * scale; m[2] = b[0] * scale; m[3] = b[1] * scale;
}
__device__ __forceinline__ uint32_t encode_m4(const float* m, float inverse) {
  q_s16x2 c{0, 0};
  c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, m[0] * inverse, m[1] * inverse, 0x1p-8f, false);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, m[2] * inverse, m[3] * inverse, 0x1p-8f, true);
  return __builtin_bit_cast(uint32_t, c);
}
// Second-moment codes (5 exponent bits from 2^-30, 3 mantissa bits, no sign) are the bits of an fp32 number from bit 20
// on, 2^96 too small; its subnormals are the codes' own.
__device__ __forceinline__ void decode_v4(uint32_t c, float scale, float* v) {
  const float k = 0x1p96f * scale;
  if (scale < 0x1p31f) {  // k is finite: one exact factor
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = __builtin_bit_cast(float, ((c >> (8 * e)) & 0xFFu) << 20) * k;
  } else {                // NaN comes here as well
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = __builtin_bit_cast(float, ((c >> (8 * e)) & 0xFFu) << 20) * 0x1p96f * scale;
  }
}
__device__ __forceinline__ uint32_t encode_v4(const float* v, float inverse) {
  uint32_t out = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float y = v[e] * inverse;   // at most 1 and an ulp, which rounds to 1
    const uint32_t bits = __builtin_bit_cast(uint32_t, y);
    // nearest, ties to even, in 3 mantissa bits; below 2^-30 in steps of 2^-33, which an addition to 2^-10 rounds to
    const uint32_t normal = ((bits + 0x7FFFFu + ((bits >> 20) & 1u)) >> 20) - (96u << 3);
    const uint32_t small = __builtin_bit_cast(uint32_t, y + 0x1p-10f) & 0xFu;
    out |= (y >= 0x1p-30f ? normal : small) << (8 * e);
  }
  return out;
}

// The step of one lane's 8 elements: g, w, and the codes of the block with scales sm, sv, in and out.
__device__ __forceinline__ void step_q8(const ListF32<8>& g, ListF32<8>& w, uint32_t (&cm)[2], uint32_t (&cv)[2], float& sm, float& sv,
                                        const Scalars& s) {
#pragma clang fp contract(off)
  const float omb1 = 1.f - s.beta1, omb2 = 1.f - s.beta2, rate = -s.lr * s.inv_c1;
  float m[8], v[8];
  decode_m4(cm[0], sm, m); decode_m4(cm[1], sm, m + 4);
  decode_v4(cv[0], sv, v); decode_v4(cv[1], sv, v + 4);
  float amax = 0.f, vmax = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float ge = s.scale * g[e];
    const float gm = omb1 * ge;
    m[e] = __builtin_fmaf(s.beta1, m[e], gm);
    float gv = omb2 * ge;
    gv = gv * ge;
    v[e] = __builtin_fmaf(s.beta2, v[e], gv);
    // the approximations take no subnormal numbers: 1.1e-19 is the smallest square root (and 0 / 0 at eps = 0 is 0).  The
    // maximum keeps NaN: a block whose scale overflowed decodes to it, and a number in its place would be a step of m / eps
    const float den = __builtin_amdgcn_sqrtf(__builtin_elementwise_maximum(v[e] * s.inv_c2, 0x1p-126f)) + s.eps;
    w[e] = __builtin_fmaf(rate, m[e] * __builtin_amdgcn_rcpf(den), s.keep * w[e]);
    amax = __builtin_elementwise_maximum(amax, __builtin_fabsf(m[e]));
    vmax = __builtin_elementwise_maximum(vmax, v[e]);
  }
  sm = amax = block_max(amax);
  sv = vmax = block_max(vmax);
  float inv_m = amax != 0.f ? 1.f / amax : 0.f, inv_v = vmax != 0.f ? 1.f / vmax : 0.f;
  // a scale below 2^-128 has no finite reciprocal: every entry but zero takes the largest code
  if (inv_m > 0x1.fffffep127f) {
#pragma unroll
    for (int e = 0; e < 8; ++e) m[e] = m[e] == 0.f ? 0.f : __builtin_copysignf(1.f, m[e]);
    inv_m = 1.f;
  }
  if (inv_v > 0x1.fffffep127f) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = v[e] == 0.f ? 0.f : 1.f;
    inv_v = 1.f;
  }
  cm[0] = encode_m4(m, inv_m); cm[1] = encode_m4(m + 4, inv_m);
  cv[0] = encode_v4(v, inv_v); cv[1] = encode_v4(v + 4, inv_v);
}

// One lane's share of a block: where its 8 elements are and what it needs to reach them.
struct LaneQ8 {
  int64_t first;       // the span's first element in the tensor
  int at0, at1;        // the lane's two groups of 4 in the span
  int n0, n1;          // how many of them the tensor has
  bool simple;         // a whole block of a tensor without gaps between its rows
};

template <class TW, class TG, bool MASTER, bool ROW, class Tensor>
__device__ __forceinline__ void load_q8(const Tensor& p, const LaneQ8& l, ListF32<8>& g, ListF32<8>& w) {
  typedef typename std::conditional<MASTER, float, TW>::type TX;
  const TX* X = MASTER ? reinterpret_cast<const TX*>(master_of(p)) : static_cast<const TX*>(p.W);
  const TG* G = static_cast<const TG*>(p.G);
  ListF32<4> g0, g1, w0, w1;
  if (l.simple) {
    X += l.first; G += l.first;
    if (ROW) {
      g = list_load<8>(G + l.at0);
      w = list_load<8>(X + l.at0);
      return;
    }
    g0 = list_load<4>(G + l.at0); g1 = list_load<4>(G + l.at1);
    w0 = list_load<4>(X + l.at0); w1 = list_load<4>(X + l.at1);
  } else {
    const Lengths len = lengths_of(p);
    const RowWalk walk(l.first, len.cols);
    const RowWalk::Place p0 = walk.at(l.at0);
    if (ROW && l.n0 >= 8 && p0.left >= 8) {
      g = list_load<8>(G + p0.offset(len.ldg));
      w = list_load<8>(X + p0.offset(len.ldw));
      return;
    }
    const RowWalk::Place p1 = walk.at(l.at1);
    const int32_t ldx = MASTER ? len.cols : len.ldw;
    g0 = row_load<4>(G, len.ldg, len.cols, p0, l.n0); g1 = row_load<4>(G, len.ldg, len.cols, p1, l.n1);
    w0 = row_load<4>(X, ldx, len.cols, p0, l.n0); w1 = row_load<4>(X, ldx, len.cols, p1, l.n1);
  }
  g = __builtin_shufflevector(g0, g1, 0, 1, 2, 3, 4, 5, 6, 7);
  w = __builtin_shufflevector(w0, w1, 0, 1, 2, 3, 4, 5, 6, 7);
}

template <class TW, bool MASTER, bool ROW, class Tensor>
__device__ __forceinline__ void store_q8(const Tensor& p, const LaneQ8& l, const ListF32<8>& w) {
  TW* W = static_cast<TW*>(p.W);
  const ListF32<4> w0 = __builtin_shufflevector(w, w, 0, 1, 2, 3), w1 = __builtin_shufflevector(w, w, 4, 5, 6, 7);
  if (l.simple) {
    W += l.first;
    if (MASTER) {
      float* X = master_of(p) + l.first;
      list_store<4>(X + l.at0, w0);
      list_store<4>(X + l.at1, w1);
    }
    if (ROW) {
      list_store<8>(W + l.at0, w);
    } else {
      list_store<4>(W + l.at0, w0);
      list_store<4>(W + l.at1, w1);
    }
    return;
  }
  const Lengths len = lengths_of(p);
  const RowWalk walk(l.first, len.cols);
  const RowWalk::Place p0 = walk.at(l.at0);
  if (ROW && l.n0 >= 8 && p0.left >= 8) {
    list_store<8>(W + p0.offset(len.ldw), w);
    return;
  }
  const RowWalk::Place p1 = walk.at(l.at1);
  if (MASTER) {
    row_store<4>(master_of(p), len.cols, len.cols, p0, l.n0, w0);
    row_store<4>(master_of(p), len.cols, len.cols, p1, l.n1, w1);
  }
  row_store<4>(W, len.ldw, len.cols, p0, l.n0, w0);
  row_store<4>(W, len.ldw, len.cols, p1, l.n1, w1);
}

typedef uint32_t q_u32x2 __attribute__((ext_vector_type(2)));

// The codes of a lane's two groups; those of a tensor lie without gaps, so only the tensor's end is not whole.
__device__ __forceinline__ uint32_t load_code4(const uint8_t* p, int n) {
  if (n >= 4) return __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(p));
  uint32_t c = 0;
#pragma unroll
  for (int e = 0; e < 3; ++e)
    if (e < n) c |= (uint32_t)p[e] << (8 * e);
  return c;
}
__device__ __forceinline__ void store_code4(uint8_t* p, int n, uint32_t c) {
  if (n >= 4) { __builtin_nontemporal_store(c, reinterpret_cast<uint32_t*>(p)); return; }
#pragma unroll
  for (int e = 0; e < 3; ++e)
    if (e < n) p[e] = (uint8_t)(c >> (8 * e));
}
__device__ __forceinline__ void load_codes(const uint8_t* p, const LaneQ8& l, bool row, uint32_t (&c)[2]) {
  if (row && l.n1 >= 4) {
    const q_u32x2 x = __builtin_nontemporal_load(reinterpret_cast<const q_u32x2*>(p + l.at0));
    c[0] = x[0]; c[1] = x[1];
  } else {
    c[0] = load_code4(p + l.at0, l.n0);
    c[1] = load_code4(p + l.at1, l.n1);
  }
}
__device__ __forceinline__ void store_codes(uint8_t* p, const LaneQ8& l, bool row, const uint32_t (&c)[2]) {
  if (row && l.n1 >= 4) {
    __builtin_nontemporal_store(q_u32x2{c[0], c[1]}, reinterpret_cast<q_u32x2*>(p + l.at0));
  } else {
    store_code4(p + l.at0, l.n0, c[0]);
    store_code4(p + l.at1, l.n1, c[1]);
  }
}

template <class List> __global__ __launch_bounds__(kThreads) void adamw_q8_list_kernel(const List grp) {
  Scalars s;
  if (!scalars(grp.call, s)) return;
  const int block = grp.call.block0 + span_of_block();
  const int i = tensor_of_block(grp.begin, grp.call.count, block);
  const auto& p = grp.t[i];
  s.keep = __builtin_fmaf(-s.lr, p.decay, 1.f);
  const int64_t first = (int64_t)(block - grp.begin[i]) * kSpanQ8, rest = p.count - first;
  const int n = rest < kSpanQ8 ? (int)rest : kSpanQ8;
  const int types = grp.types[i] + (master_of(p) ? 4 : 0);
  const int b = threadIdx.x / kLanes, base = b * kBlock, len = n - base;
  if (len <= 0) return;   // the 32 lanes of a block stay together
  // A lane's elements: 4 and the 4 that are 128 further on, so that the 16-byte accesses of fp32 lanes follow each other
  // (60M fp32 elements: 178 us with 8 in a row, 154).  Where weight and gradient are bf16 16 bytes hold 8 in a row: one
  // place in the row instead of two to find where rows lie apart (32.8M elements: 66 us, and 76 with two groups of 4).
  const bool row = types == 3;
  const int lane = threadIdx.x % kLanes, at0 = base + (row ? lane * 8 : lane * 4), at1 = row ? at0 + 4 : at0 + kBlock / 2;
  const LaneQ8 l{first, at0, at1, n - at0, n - at1, lengths_of(p).run() && len >= kBlock};
  uint8_t* const Mc = p.Mc + first;
  uint8_t* const Vc = p.Vc + first;
  float* const Ms = p.Ms + (first >> 8);
  float* const Vs = p.Vs + (first >> 8);
  uint32_t cm[2], cv[2];
  load_codes(Mc, l, row, cm);
  load_codes(Vc, l, row, cv);
  float sm = Ms[b], sv = Vs[b];
  ListF32<8> g, w;
  switch (types) {
    case 0: load_q8<float, float, false, false>(p, l, g, w); break;
    case 1: load_q8<__bf16, float, false, false>(p, l, g, w); break;
    case 2: load_q8<float, __bf16, false, false>(p, l, g, w); break;
    case 3: load_q8<__bf16, __bf16, false, true>(p, l, g, w); break;
    case 5: load_q8<__bf16, float, true, false>(p, l, g, w); break;
    default: load_q8<__bf16, __bf16, true, false>(p, l, g, w);
  }
  step_q8(g, w, cm, cv, sm, sv, s);
  if (lane == 0) { Ms[b] = sm; Vs[b] = sv; }
  store_codes(Mc, l, row, cm);
  store_codes(Vc, l, row, cv);
  switch (types) {
    case 0: case 2: store_q8<float, false, false>(p, l, w); break;
    case 1: store_q8<__bf16, false, false>(p, l, w); break;
    case 3: store_q8<__bf16, false, true>(p, l, w); break;
    default: store_q8<__bf16, true, false>(p, l, w);
  }
}

// One thread: the corrections of a step are two powers in 64 bits, which the threads of the step itself would each repeat.
__global__ void adamw_tick_kernel(AdamWClock* clock, double beta1, double beta2, const GradStats* stats) {
  if (stats && stats->finite != 1.f) return;
  const int64_t t = ++clock->t;
  clock->inv_c1 = (float)(1.0 / (1.0 - pow(beta1, (double)t)));
  clock->inv_c2 = (float)(1.0 / (1.0 - pow(beta2, (double)t)));
}

// Spans of the list's tensors and the launches over them: one, unless a launch cannot have so many workgroups.
template <class Tensor, int N>
hipError_t launch_spans(AdamWList<Tensor, N>& g, int64_t span, void (*kernel)(AdamWList<Tensor, N>), hipStream_t stream) {
  if (g.call.count > N) return hipErrorInvalidValue;
  int64_t blocks = 0;
  for (int i = 0; i < g.call.count; ++i) {
    g.begin[i] = (int32_t)blocks;
    blocks += ((int64_t)g.t[i].count + span - 1) / span;
    if (blocks > INT32_MAX) return hipErrorInvalidValue;
  }
  for (int64_t b = 0; b < blocks; b += kMaxBlocks) {
    g.call.block0 = (int32_t)b;
    const int64_t grid = blocks - b < kMaxBlocks ? blocks - b : kMaxBlocks;
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(kThreads), 0, stream, g);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_adamw_tick(AdamWClock* clock, float beta1, float beta2, const GradStats* stats, hipStream_t stream) {
  hipLaunchKernelGGL(adamw_tick_kernel, dim3(1), dim3(1), 0, stream, clock, (double)beta1, (double)beta2, stats);
  return hipGetLastError();
}

hipError_t launch_adamw(AdamWGroup& g, hipStream_t stream) { return launch_spans(g, kSpan, adamw_list_kernel<AdamWGroup>, stream); }
hipError_t launch_adamw(AdamWRunGroup& g, hipStream_t stream) { return launch_spans(g, kSpan, adamw_list_kernel<AdamWRunGroup>, stream); }
hipError_t launch_adamw(AdamWQ8Group& g, hipStream_t stream) { return launch_spans(g, kSpanQ8, adamw_q8_list_kernel<AdamWQ8Group>, stream); }
hipError_t launch_adamw(AdamWQ8RunGroup& g, hipStream_t stream) { return launch_spans(g, kSpanQ8, adamw_q8_list_kernel<AdamWQ8RunGroup>, stream); }

}  // namespace galore
