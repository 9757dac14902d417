// layer_device.hpp -- device code shared by the layer operators' kernels:
// element types, the counter-based generator, activations and the epilogue of
// a product.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "layers.hpp"

namespace ar {

using bf16 = __bf16;
using f16 = _Float16;

template <typename T> constexpr Elem elem_of();
template <> constexpr Elem elem_of<float>() { return kF32; }
template <> constexpr Elem elem_of<f16>() { return kF16; }
template <> constexpr Elem elem_of<bf16>() { return kBF16; }


// V elements that start on any element, as floats.
template <int V, typename T>
__device__ __forceinline__ void load_group(float (&x)[V], const T* p) {
  typedef T U __attribute__((ext_vector_type(V), aligned(sizeof(T))));
  const U u = *reinterpret_cast<const U*>(p);
#pragma unroll
  for (int i = 0; i < V; ++i) x[i] = float(u[i]);
}
// Rounded to nearest, ties to even, where T is narrower.
template <int V, typename T>
__device__ __forceinline__ void store_group(T* p, const float (&x)[V]) {
  typedef T U __attribute__((ext_vector_type(V), aligned(sizeof(T))));
  U u;
#pragma unroll
  for (int i = 0; i < V; ++i) u[i] = T(x[i]);
  *reinterpret_cast<U*>(p) = u;
}
// Where a row of V elements at least ends within a group, its last V elements
// are loaded, `back` before the group's own, and moved down to their places; 0
// follows.  So a row of any length is loaded as wide as any other, and the one
// group costs a few moves (element by element, the last group of 1001 columns
// held up its workgroup for several times the latency of memory).
template <int V>
__device__ __forceinline__ void move_down(float (&x)[V], int back) {
  if (back == 0) return;
#pragma unroll
  for (int step = V / 2; step > 0; step /= 2)
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = back & step ? (i + step < V ? x[i + step] : 0.0f) : x[i];
}
// The elements of a group that lie in the row, all but `back` < V.
template <int V, typename T>
__device__ __forceinline__ void store_most(T* p, const float (&x)[V], int back) {
  if (back == 0) {
    store_group<V>(p, x);
  } else {
    float y[V];
#pragma unroll
    for (int i = 0; i < V; ++i) y[i] = x[i];
#pragma unroll
    for (int step = V / 2; step > 0; step /= 2) {
      if ((V - back) & step) {
        if (step == 4) store_group<4>(p, {y[0], y[1], y[2 % V], y[3 % V]});
        if (step == 2) store_group<2>(p, {y[0], y[1]});
        if (step == 1) store_group<1>(p, {y[0]});
        p += step;
#pragma unroll
        for (int i = 0; i + step < V; ++i) y[i] = y[i + step];
      }
    }
  }
}
// The first `have` < V of V elements, of rows shorter than V; the rest 0.
template <int V, typename T>
__device__ __forceinline__ void load_tail(float (&x)[V], const T* p, int have) {
#pragma unroll
  for (int i = 0; i < V - 1; ++i) x[i] = i < have ? float(p[i]) : 0.0f;
  x[V - 1] = 0.0f;
}
template <int V, typename T>
__device__ __forceinline__ void store_tail(T* p, const float (&x)[V], int have) {
#pragma unroll
  for (int i = 0; i < V - 1; ++i)
    if (i < have) p[i] = T(x[i]);
}

// a ^ b ^ c in one instruction (truth table 0x96).
__device__ __forceinline__ uint32_t xor3(uint32_t a, uint32_t b, uint32_t c) {
  return uint32_t(__builtin_amdgcn_bitop3_b32(int(a), int(b), int(c), 0x96));
}

// The counter-based generator on four 32-bit words with seven rounds (J. K.
// Salmon et al., "Parallel random numbers: as easy as 1, 2, 3", 2011): the
// fewest rounds that pass the whole of that paper's tests (ten is its cautious
// choice).  A round is two 32 x 32 -> 64 bit products, a quarter of the rate of
// other instructions, and two three-way exclusive ors: about 280 cycles of a
// wave for 256 words.
__device__ __forceinline__ uint4 counter_words(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0,
                                               uint32_t k1) {
#pragma unroll
  for (int r = 0; r < 7; ++r) {
    const uint64_t a = uint64_t(0xD2511F53u) * c0, b = uint64_t(0xCD9E8D57u) * c2;
    c0 = xor3(uint32_t(b >> 32), c1, k0);
    c1 = uint32_t(b);
    c2 = xor3(uint32_t(a >> 32), c3, k1);
    c3 = uint32_t(a);
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return make_uint4(c0, c1, c2, c3);
}

// drop() of V (4 or 8) consecutive elements of one row, the first at a column
// that is a multiple of 4.  A dropped element is 0 whatever it held.
template <int V>
__device__ __forceinline__ void drop_some(float (&x)[V], const DropArgs& d, uint64_t row, uint32_t col) {
  if (d.none) {
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = 0.0f;
    return;
  }
#pragma unroll
  for (int q = 0; q < V / 4; ++q) {
    const uint4 w = counter_words((col >> 2) + q, uint32_t(row), uint32_t(row >> 32), d.site, d.k0, d.k1);
    x[4 * q + 0] = w.x <= d.last ? x[4 * q + 0] * d.scale : 0.0f;
    x[4 * q + 1] = w.y <= d.last ? x[4 * q + 1] * d.scale : 0.0f;
    x[4 * q + 2] = w.z <= d.last ? x[4 * q + 2] * d.scale : 0.0f;
    x[4 * q + 3] = w.w <= d.last ? x[4 * q + 3] * d.scale : 0.0f;
  }
}

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.69314718055994531f;
constexpr float kHalfLog2e = 0.72134752044448170f;
constexpr float kHalfLog2eRest = 9.62981517e-09f;  // what the former lacks
constexpr float kInvSqrt2Pi = 0.39894228040143268f;
constexpr float kGeluTanh2 = 1.5957691216057308f;      // 2 sqrt(2 / pi)
constexpr float kGeluCubic = 0.044715f;

// 1 / (1 + 2^u).
__device__ __forceinline__ float logistic2(float u) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(u));
}

// exp(-z^2 / 2), and the normal distribution's tail beyond |z|: t P(t) exp(-z^2 / 2)
// with t = 1 / (1 + c |z|) and polynomials P fitted to erfcx for the least relative
// error: small where the tail is, unlike 1 + erf.  x is |z|, 64 at most; from there
// on, and for NaN, both are 0.
//   FINE, for operands of 32 bits: degree 8, 7e-8, and the exponent's rounding, which
//   would grow with z^2 to 1e-5 of the tail, is carried along (lost).  With an exp2
//   and a reciprocal of one unit in the last place the tail is off by 12 * 2^-24
//   of itself at most (7 * 2^-24 is the most seen in 4e5 places from 0 to 12.5).
//   Otherwise: degree 5, fitted where the tail is large for the least error itself:
//   off by 3.4e-7, and by 6e-5 of itself, at most, an eighth of fp16's rounding.  With
//   the longer form 8192 x 4096 x 4096 bf16 with a bias and z kept takes 231 us for
//   209, the pass that makes dz of 8192 x 16384 124 for 105; with both forms in one
//   kernel, for results of either type, 219.
template <bool FINE>
__device__ __forceinline__ float normal_tail(float z, float& x, float& gauss) {
  x = __builtin_fminf(__builtin_fabsf(z), 64.0f);
  const float h = x * x, u = -kHalfLog2e * h;
  gauss = __builtin_amdgcn_exp2f(u);
  if constexpr (FINE) {
    float lost = __builtin_fmaf(-kHalfLog2e, h, -u);
    lost = __builtin_fmaf(-kHalfLog2eRest, h, lost);
    lost = __builtin_fmaf(-kHalfLog2e, __builtin_fmaf(x, x, -h), lost);
    gauss = __builtin_fmaf(gauss * kLn2, lost, gauss);
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.2775f, x, 1.0f));
    float p = __builtin_fmaf(0.0266462043f, t, -0.10478624f);
    p = __builtin_fmaf(p, t, 0.115219638f);
    p = __builtin_fmaf(p, t, -0.0238516629f);
    p = __builtin_fmaf(p, t, 0.081743136f);
    p = __builtin_fmaf(p, t, 0.0809703395f);
    p = __builtin_fmaf(p, t, 0.102675281f);
    p = __builtin_fmaf(p, t, 0.110676117f);
    p = __builtin_fmaf(p, t, 0.110707216f);
    return p * t * gauss;
  } else {
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.2925f, x, 1.0f));
    float p = __builtin_fmaf(-0.0872766301f, t, 0.271199584f);
    p = __builtin_fmaf(p, t, -0.0777925625f);
    p = __builtin_fmaf(p, t, 0.172719866f);
    p = __builtin_fmaf(p, t, 0.103415728f);
    p = __builtin_fmaf(p, t, 0.117734119f);
    return p * t * gauss;
  }
}

__device__ __forceinline__ float act_relu(float z) { return z > 0.0f ? z : (z != z ? z : 0.0f); }
// max(z, 0) - |z| tail(|z|); the product with 0 keeps NaN and -inf * 0.
template <bool FINE>
__device__ __forceinline__ float act_gelu(float z) {
  float x, gauss;
  const float q = normal_tail<FINE>(z, x, gauss);
  return __builtin_fmaf(-x, q, z > 0.0f ? z : z * 0.0f);
}
// (1 + tanh(u)) / 2 is the logistic function of 2 u.
__device__ __forceinline__ float act_gelu_tanh(float z) {
  return z * logistic2(z * __builtin_fmaf(-kLog2e * kGeluTanh2 * kGeluCubic * z, z, -kLog2e * kGeluTanh2));
}
__device__ __forceinline__ float act_silu(float z) { return z * logistic2(-kLog2e * z); }

template <bool FINE>
__device__ __forceinline__ float slope_gelu(float z) {
  float x, gauss;
  const float q = normal_tail<FINE>(z, x, gauss);
  return __builtin_fmaf(z * kInvSqrt2Pi, gauss, z > 0.0f ? 1.0f - q : q);
}
__device__ __forceinline__ float slope_gelu_tanh(float z) {
  // far out g or 1 - g is 0, which must not meet an infinite square
  const float t = __builtin_fminf(z * z, 1e8f);
  const float g = logistic2(z * __builtin_fmaf(-kLog2e * kGeluTanh2 * kGeluCubic, t, -kLog2e * kGeluTanh2));
  return __builtin_fmaf(z * g * (1.0f - g), __builtin_fmaf(3.0f * kGeluCubic * kGeluTanh2, t, kGeluTanh2), g);
}
__device__ __forceinline__ float slope_silu(float z) {
  const float g = logistic2(-kLog2e * z);
  return g * __builtin_fmaf(z, 1.0f - g, 1.0f);
}

// v = act(v), of Q rows and a product of operands of type T: one branch for all, so
// that the rows' long operations overlap.
template <int V, int Q, typename F>
__device__ __forceinline__ void each(float (&v)[Q][V], F&& f) {
#pragma unroll
  for (int q = 0; q < Q; ++q)
#pragma unroll
    for (int i = 0; i < V; ++i) v[q][i] = f(v[q][i]);
}
template <typename T, int V, int Q>
__device__ __forceinline__ void activate(float (&v)[Q][V], int act) {
  switch (act) {
    case kActRelu: each(v, act_relu); break;
    case kActGelu: each(v, act_gelu<sizeof(T) == 4>); break;
    case kActGeluTanh: each(v, act_gelu_tanh); break;
    case kActSilu: each(v, act_silu); break;
    default: break;
  }
}

// v[i] *= act'(z[i]), for products of operands of type T
template <typename T, int V>
__device__ __forceinline__ void times_slope(float (&v)[V], const float (&z)[V], int act) {
  switch (act) {
    case kActRelu:
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] *= z[i] > 0.0f ? 1.0f : 0.0f;
      break;
    case kActGelu:
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] *= slope_gelu<sizeof(T) == 4>(z[i]);
      break;
    case kActGeluTanh:
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] *= slope_gelu_tanh(z[i]);
      break;
    case kActSilu:
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] *= slope_silu(z[i]);
      break;
    default: break;
  }
}

// The bias of V columns from n on, `back` of them behind the row's end (zeros
// without one, or where the row is shorter than V or ends before n).
template <typename T, int V>
__device__ __forceinline__ void load_bias(float (&b)[V], const Epilogue& e, int32_t n, int back = 0) {
  if (!e.bias || e.N - n < V - back || e.N < V) {
#pragma unroll
    for (int i = 0; i < V; ++i) b[i] = 0.0f;
    return;
  }
  if (e.bias_f32) load_group<V>(b, static_cast<const float*>(e.bias) + n - back);
  else load_group<V>(b, static_cast<const T*>(e.bias) + n - back);
  move_down<V>(b, back);
}

// V columns of a residual, as they lie in memory: 2 V bytes, and of 32-bit
// ones the other 2 V.
template <int V>
struct Residual {
  typedef uint32_t Half __attribute__((ext_vector_type(V / 2), aligned(2)));
  uint32_t __attribute__((ext_vector_type(V / 2))) first, second;
};

// The residuals of V columns from n on, all within the row, of Q rows from m on
// `step` apart; of rows past the last one, that one's.  The first halves of all
// are loaded without a branch between them, so that they go out together.
template <typename T, int V, int Q>
__device__ __forceinline__ void load_residuals(Residual<V> (&r)[Q], const Epilogue& e, int32_t m, int32_t step, int32_t n) {
  using Half = typename Residual<V>::Half;
  if (!e.res) return;
  const int shift = e.y_f32 ? 2 : 1;
  const char* p[Q];
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    const int32_t row = m + q * step < e.M ? m + q * step : e.M - 1;
    p[q] = static_cast<const char*>(e.res) + ((int64_t(row) * e.ldr + n) << shift);
    r[q].first = *reinterpret_cast<const Half*>(p[q]);
  }
  if (sizeof(T) == 4 || e.y_f32) {
#pragma unroll
    for (int q = 0; q < Q; ++q) r[q].second = *reinterpret_cast<const Half*>(p[q] + 2 * V);
  }
}

// v += the residuals, which were loaded `back` columns early
template <typename T, int V, int Q>
__device__ __forceinline__ void add_residuals(float (&v)[Q][V], const Residual<V> (&r)[Q], const Epilogue& e, int back) {
  if (!e.res) return;
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    float x[V];
    if (sizeof(T) == 4 || e.y_f32) {
#pragma unroll
      for (int i = 0; i < V / 2; ++i) {
        x[i] = __builtin_bit_cast(float, uint32_t(r[q].first[i]));
        x[V / 2 + i] = __builtin_bit_cast(float, uint32_t(r[q].second[i]));
      }
    } else if constexpr (sizeof(T) == 2) {
      typedef T P __attribute__((ext_vector_type(2)));
#pragma unroll
      for (int i = 0; i < V / 2; ++i) {
        const P p = __builtin_bit_cast(P, uint32_t(r[q].first[i]));
        x[2 * i] = float(p[0]);
        x[2 * i + 1] = float(p[1]);
      }
    }
    move_down<V>(x, back);
#pragma unroll
    for (int i = 0; i < V; ++i) v[q][i] += x[i];
  }
}

// The epilogue of V (4 or 8) columns from n on (a multiple of V), the last
// `back` of them behind the row's end, of Q rows from m on `step` apart; v holds
// the product's sums.  Rows past the last one are worked on and not stored.
// BIAS, STAGES: whether there may be a bias; a kept z, an activation, dropout.
template <typename T, int V, int Q, bool BIAS = true, bool STAGES = true>
__device__ __forceinline__ void emit(float (&v)[Q][V], const float (&b)[V], const Residual<V> (&r)[Q], const Epilogue& e,
                                     int32_t m, int32_t step, int32_t n, int back = 0) {
  auto store = [&](auto* to, int64_t ld) {
#pragma unroll
    for (int q = 0; q < Q; ++q)
      if (m + q * step < e.M) store_most<V>(to + int64_t(m + q * step) * ld + n, v[q], back);
  };
  if constexpr (BIAS) {
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
      for (int i = 0; i < V; ++i) v[q][i] += b[i];
  }
  if constexpr (STAGES) {
    if (e.z) store(static_cast<T*>(e.z), e.ldz);
    activate<T>(v, e.act);
    if (e.drop.on) {
#pragma unroll
      for (int q = 0; q < Q; ++q) drop_some<V>(v[q], e.drop, e.drop.row0 + uint32_t(m + q * step), uint32_t(n));
    }
  }
  add_residuals<T, V, Q>(v, r, e, back);
  if (e.y_f32) store(static_cast<float*>(e.y), e.ldy);
  else store(static_cast<T*>(e.y), e.ldy);
}

// The same for the `have` < V columns of a row's end, of Q rows from m on `step`
// apart, whose sums sum(q, i) gives, where the rows are shorter than V or only
// few are left; all loads of the Q rows go out before the first is used.
template <typename T, int V, int Q, bool BIAS = true, bool STAGES = true, typename F>
__device__ __forceinline__ void emit_tail(F&& sum, const Epilogue& e, int32_t m, int32_t step, int32_t n, int have) {
  float b[V], r[Q][V];
#pragma unroll
  for (int i = 0; i < V; ++i) b[i] = 0.0f;
  if (BIAS && e.bias) {
    if (e.bias_f32) load_tail<V>(b, static_cast<const float*>(e.bias) + n, have);
    else load_tail<V>(b, static_cast<const T*>(e.bias) + n, have);
  }
  if (e.res) {
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const int64_t at = int64_t(m + q * step < e.M ? m + q * step : e.M - 1) * e.ldr + n;
      if (e.y_f32) load_tail<V>(r[q], static_cast<const float*>(e.res) + at, have);
      else load_tail<V>(r[q], static_cast<const T*>(e.res) + at, have);
    }
  }
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    const int32_t row = m + q * step;
    if (row >= e.M) break;
    float w[1][V];
    float(&v)[V] = w[0];
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = i < have ? sum(q, i) + b[i] : 0.0f;
    if constexpr (STAGES) {
      if (e.z) store_tail<V>(static_cast<T*>(e.z) + int64_t(row) * e.ldz + n, v, have);
      activate<T>(w, e.act);
      if (e.drop.on) drop_some<V>(v, e.drop, e.drop.row0 + uint32_t(row), uint32_t(n));
    }
    if (e.res) {
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] += r[q][i];
    }
    if (e.y_f32) store_tail<V>(static_cast<float*>(e.y) + int64_t(row) * e.ldy + n, v, have);
    else store_tail<V>(static_cast<T*>(e.y) + int64_t(row) * e.ldy + n, v, have);
  }
}

}  // namespace ar
