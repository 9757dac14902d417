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


// The first `have` (all V where have >= V) of V elements as floats; the rest 0.
template <int V, typename T>
__device__ __forceinline__ void load_some(float (&x)[V], const T* p, int have) {
  if (have >= V) {
    typedef T U __attribute__((ext_vector_type(V), aligned(sizeof(T))));
    const U u = *reinterpret_cast<const U*>(p);
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = float(u[i]);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = i < have ? float(p[i]) : 0.0f;
  }
}

// Rounded to nearest, ties to even, where T is narrower.
template <int V, typename T>
__device__ __forceinline__ void store_some(T* p, const float (&x)[V], int have) {
  if (have >= V) {
    typedef T U __attribute__((ext_vector_type(V), aligned(sizeof(T))));
    U u;
#pragma unroll
    for (int i = 0; i < V; ++i) u[i] = T(x[i]);
    *reinterpret_cast<U*>(p) = u;
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < have) p[i] = T(x[i]);
  }
}

// The counter-based generator on four 32-bit words with seven rounds (J. K.
// Salmon et al., "Parallel random numbers: as easy as 1, 2, 3", 2011): the
// fewest rounds that pass the whole of that paper's tests (ten is its cautious
// choice).  A round is two 32 x 32 -> 64 bit products.
__device__ __forceinline__ uint4 counter_words(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0,
                                               uint32_t k1) {
#pragma unroll
  for (int r = 0; r < 7; ++r) {
    const uint64_t a = uint64_t(0xD2511F53u) * c0, b = uint64_t(0xCD9E8D57u) * c2;
    c0 = uint32_t(b >> 32) ^ c1 ^ k0;
    c1 = uint32_t(b);
    c2 = uint32_t(a >> 32) ^ c3 ^ k1;
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

// drop() of one element.
__device__ __forceinline__ float drop_one(float x, const DropArgs& d, uint64_t row, uint32_t col) {
  if (d.none) return 0.0f;
  const uint4 w = counter_words(col >> 2, uint32_t(row), uint32_t(row >> 32), d.site, d.k0, d.k1);
  const uint32_t word = col & 2 ? (col & 1 ? w.w : w.z) : (col & 1 ? w.y : w.x);
  return word <= d.last ? x * d.scale : 0.0f;
}

constexpr float kSqrtHalf = 0.70710678118654752f;
constexpr float kInvSqrt2Pi = 0.39894228040143268f;
constexpr float kGeluTanh2 = 1.5957691216057308f;      // 2 sqrt(2 / pi)
constexpr float kGeluCubic = 0.044715f;

__device__ __forceinline__ float logistic(float u) { return __builtin_amdgcn_rcpf(1.0f + __expf(-u)); }

// (1 + tanh(u)) / 2 is the logistic function of 2 u.
__device__ __forceinline__ float act_value(float z, int act) {
  switch (act) {
    case kActRelu: return z > 0.0f ? z : (z != z ? z : 0.0f);
    case kActGelu: return 0.5f * z * (1.0f + erff(z * kSqrtHalf));
    case kActGeluTanh: return z * logistic(kGeluTanh2 * z * __builtin_fmaf(kGeluCubic * z, z, 1.0f));
    case kActSilu: return z * logistic(z);
    default: return z;
  }
}

__device__ __forceinline__ float act_slope(float z, int act) {
  switch (act) {
    case kActRelu: return z > 0.0f ? 1.0f : 0.0f;
    case kActGelu: return 0.5f * (1.0f + erff(z * kSqrtHalf)) + z * kInvSqrt2Pi * __expf(-0.5f * z * z);
    case kActGeluTanh: {
      const float t = z * z;
      const float g = logistic(kGeluTanh2 * z * __builtin_fmaf(kGeluCubic, t, 1.0f));
      return __builtin_fmaf(z * g * (1.0f - g), kGeluTanh2 * __builtin_fmaf(3.0f * kGeluCubic, t, 1.0f), g);
    }
    case kActSilu: {
      const float g = logistic(z);
      return g * __builtin_fmaf(z, 1.0f - g, 1.0f);
    }
    default: return 1.0f;
  }
}

// The bias of V columns from n on (zeros without one, or where the row ends
// before the last).
template <typename T, int V>
__device__ __forceinline__ void load_bias(float (&b)[V], const Epilogue& e, int32_t n) {
  if (!e.bias || e.N - n < V) {
#pragma unroll
    for (int i = 0; i < V; ++i) b[i] = 0.0f;
  } else if (e.bias_f32) {
    load_some<V>(b, static_cast<const float*>(e.bias) + n, V);
  } else {
    load_some<V>(b, static_cast<const T*>(e.bias) + n, V);
  }
}

// The residual of V columns from n on, all within the row, of row m (zeros
// without one).
template <typename T, int V>
__device__ __forceinline__ void load_residual(float (&r)[V], const Epilogue& e, int32_t m, int32_t n) {
  if (!e.res) {
#pragma unroll
    for (int i = 0; i < V; ++i) r[i] = 0.0f;
  } else if (e.y_f32) {
    load_some<V>(r, static_cast<const float*>(e.res) + int64_t(m) * e.ldr + n, V);
  } else {
    load_some<V>(r, static_cast<const T*>(e.res) + int64_t(m) * e.ldr + n, V);
  }
}

// The epilogue of V (4 or 8) columns from n on (a multiple of V), all within
// the row, of row m; v holds the product's sums.
template <typename T, int V>
__device__ __forceinline__ void emit(float (&v)[V], const float (&b)[V], const float (&r)[V], const Epilogue& e,
                                     int32_t m, int32_t n) {
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] += b[i];
  if (e.z) store_some<V>(static_cast<T*>(e.z) + int64_t(m) * e.ldz + n, v, V);
  if (e.act != kActNone) {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = act_value(v[i], e.act);
  }
  if (e.drop.on) drop_some<V>(v, e.drop, e.drop.row0 + uint32_t(m), uint32_t(n));
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] += r[i];
  if (e.y_f32) store_some<V>(static_cast<float*>(e.y) + int64_t(m) * e.ldy + n, v, V);
  else store_some<V>(static_cast<T*>(e.y) + int64_t(m) * e.ldy + n, v, V);
}

// The same for one element, where a row ends inside a group of columns.
template <typename T>
__device__ __forceinline__ void emit_one(float v, const Epilogue& e, int32_t m, int32_t n) {
  if (e.bias) v += e.bias_f32 ? static_cast<const float*>(e.bias)[n] : float(static_cast<const T*>(e.bias)[n]);
  if (e.z) static_cast<T*>(e.z)[int64_t(m) * e.ldz + n] = T(v);
  v = act_value(v, e.act);
  if (e.drop.on) v = drop_one(v, e.drop, e.drop.row0 + uint32_t(m), uint32_t(n));
  const int64_t ry = int64_t(m) * e.ldr + n, yy = int64_t(m) * e.ldy + n;
  if (e.y_f32) {
    if (e.res) v += static_cast<const float*>(e.res)[ry];
    static_cast<float*>(e.y)[yy] = v;
  } else {
    if (e.res) v += float(static_cast<const T*>(e.res)[ry]);
    static_cast<T*>(e.y)[yy] = T(v);
  }
}

}  // namespace ar
