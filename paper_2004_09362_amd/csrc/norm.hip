// norm.hip -- layer norm and its gradient.
//
// y = (x - mean) rstd w + b over each row; with h = (x - mean) rstd and
// g = dy w, dx = res + rstd (g - mean(g) - h mean(g h)), dw = sum of dy h and
// db = sum of dy over the rows.  All in 32 bits, rounded once when stored.
//
// Bound by memory: each element is read once and written once.  A row lies in
// the registers of a team of lanes (one or two groups of 8 columns a lane, 16
// bytes of halves each), from which its mean, then its variance about that mean,
// and then its results are taken: no cancellation, no second reading.  A lane keeps
// its columns from row to row, so w, b and the sums of the weight's gradient stay
// with it, and the next row is on its way while one is worked on.  Teams of up to a
// wave sum by exchanges of registers; larger ones meet once a sum, in LDS.
// Forward, 8192 x 8192 bf16 50.2 us (5.3 TB/s; a copy 46), 8192 x 4096 fp32 to bf16
// 38.3 (35); gradient with a residual 110 (4.9 TB/s), 65536 x 1024 108.
// Two rows on their way instead of one: 67.4 for 65.6 us then; a wave to each row of
// 4096 (64 columns a lane) with w and b in LDS: 74.5 for 60.8, 43.6 for 42.3.
#include <algorithm>
#include <type_traits>

#include "layer_device.hpp"
#include "training.hpp"

namespace ar {

namespace {

constexpr int kMaxThreads = 1024;

// V elements as they lie in memory, at any element's address.
template <typename T, int V>
struct Raw {
  typedef T U __attribute__((ext_vector_type(V), aligned(sizeof(T))));
  typedef T W __attribute__((ext_vector_type(V)));
  W w;
  __device__ __forceinline__ void load(const T* p) { w = *reinterpret_cast<const U*>(p); }
  // as floats, moved down by `back` with zeros after them
  __device__ __forceinline__ void get(float (&x)[V], int back) const {
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = float(w[i]);
    if constexpr (V > 1) move_down<V>(x, back);
  }
};
template <typename T>
struct Raw<T, 1> {
  T w;
  __device__ __forceinline__ void load(const T* p) { w = *p; }
  __device__ __forceinline__ void get(float (&x)[1], int) const { x[0] = float(w); }
};

template <int V, typename T>
__device__ __forceinline__ void store_row(T* p, const float (&x)[V], int back) {
  if constexpr (V == 1) *p = T(x[0]);
  else store_most<V>(p, x, back);
}

// Parameters of V columns, of any type.
template <int V>
__device__ __forceinline__ void load_params(float (&v)[V], const void* p, int32_t e, int64_t col, int back) {
  auto of = [&](auto* t) {
    Raw<std::remove_cv_t<std::remove_pointer_t<decltype(t)>>, V> r;
    r.load(t + col - back);
    r.get(v, back);
  };
  if (e == kF32) of(static_cast<const float*>(p));
  else if (e == kF16) of(static_cast<const f16*>(p));
  else of(static_cast<const bf16*>(p));
}

// v of a lane's partner: within 16 lanes the one at a distance of 1 or 2, or the
// mirrored one of 8 or 16, whose sums so far are those of the other half.
template <int CONTROL>
__device__ __forceinline__ float partner(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CONTROL, 0xf, 0xf, true));
}
// The sum over 16 lanes, over 32, over the wave, without LDS: halves are exchanged
// in the registers.
__device__ __forceinline__ float sum16(float v) {
  v += partner<0xb1>(v);
  v += partner<0x4e>(v);
  v += partner<0x141>(v);
  return v + partner<0x140>(v);
}
__device__ __forceinline__ float add_halves32(float v) {
  const uint32_t u = __builtin_bit_cast(uint32_t, v);
  const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const uint32_t x = r[0], y = r[1];
  return __builtin_bit_cast(float, x) + __builtin_bit_cast(float, y);
}
__device__ __forceinline__ float add_halves64(float v) {
  const uint32_t u = __builtin_bit_cast(uint32_t, v);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  const uint32_t x = r[0], y = r[1];
  return __builtin_bit_cast(float, x) + __builtin_bit_cast(float, y);
}

// The sum over a team's lanes, for each of K values at once, in all of its lanes.
// SMALL: a team is a part of a wave, or one.  Forward, 8192 x 8192 bf16: with
// exchanges through LDS and a loop over the waves' sums 65.6 us, so 61.0.
template <int K, bool SMALL>
struct TeamSum {
  float (*lds)[16][K];  // [2][16 waves]
  int lanes, waves, turn, mine;

  __device__ __forceinline__ void init(float (*buffer)[16][K], int lanes_) {
    lds = buffer;
    lanes = lanes_;
    waves = lanes >> 6;
    turn = 0;
    if (SMALL) return;
    // the wave of the team whose sum this lane takes, or none
    const int of = int(threadIdx.x & 15);
    mine = of < waves ? (int(threadIdx.x >> 6) & ~(waves - 1)) + of : -1;
  }
  __device__ __forceinline__ void operator()(float (&v)[K]) {
    if constexpr (SMALL) {  // of 8 lanes or more
#pragma unroll
      for (int k = 0; k < K; ++k) {
        v[k] += partner<0xb1>(v[k]);
        v[k] += partner<0x4e>(v[k]);
        v[k] += partner<0x141>(v[k]);
        if (lanes > 8) v[k] += partner<0x140>(v[k]);
        if (lanes > 16) v[k] = add_halves32(v[k]);
        if (lanes > 32) v[k] = add_halves64(v[k]);
      }
    } else {
#pragma unroll
      for (int k = 0; k < K; ++k) v[k] = add_halves64(add_halves32(sum16(v[k])));
      if (waves == 1) return;
      // the buffer was read two meetings ago
      if ((threadIdx.x & 63) == 0) {
#pragma unroll
        for (int k = 0; k < K; ++k) lds[turn][threadIdx.x >> 6][k] = v[k];
      }
      __syncthreads();
#pragma unroll
      for (int k = 0; k < K; ++k) v[k] = sum16(mine >= 0 ? lds[turn][mine][k] : 0.0f);
      turn ^= 1;
    }
  }
};

// Element i of a row, whose start is the same for a wave: one register of a lane.
template <typename T>
__device__ __forceinline__ T* element(T* row, uint32_t i) {
  using C = std::conditional_t<std::is_const_v<T>, const char, char>;
  return reinterpret_cast<T*>(reinterpret_cast<C*>(row) + uint64_t(i * uint32_t(sizeof(T))));
}

// Which of the workgroup's teams a thread is in; teams of more than a wave are
// known to be the same for it, and so are their rows' addresses.
template <bool SMALL>
__device__ __forceinline__ int team_of(int lanes) {
  const int team = int(threadIdx.x) / lanes;
  if constexpr (SMALL) return team;
  else return __builtin_amdgcn_readfirstlane(team);
}

// The columns of a lane: group q is columns col(q) on, of which V - back(q) are
// there; it is loaded from column from(q) on.  WHOLE: rows of whole groups, which
// take fewer instructions (8192 x 8192 bf16 58.9 us for 60.8).
template <int V, int R, bool WHOLE>
struct Columns {
  uint32_t first, apart;
  int32_t missing[R];  // of group q, V where it is not there
  __device__ __forceinline__ void init(int t, int lanes, int64_t cols) {
    first = uint32_t(t) * V;
    apart = uint32_t(lanes) * V;
#pragma unroll
    for (int q = 0; q < R; ++q) {
      const int have = int(cols) - int(col(q));
      missing[q] = have >= V ? 0 : have > 0 ? V - have : V;
    }
  }
  __device__ __forceinline__ uint32_t col(int q) const { return first + uint32_t(q) * apart; }
  __device__ __forceinline__ bool there(int q) const { return missing[q] < V; }
  __device__ __forceinline__ int back(int q) const { return WHOLE ? 0 : missing[q]; }
  __device__ __forceinline__ uint32_t from(int q) const { return col(q) - uint32_t(back(q)); }
  __device__ __forceinline__ bool there(int q, int i) const { return WHOLE || i < V - missing[q]; }
};

// Teams of `lanes` lanes take rows in turn, the next one on its way.
template <typename X, typename Y, int V, int R, bool WHOLE>
__global__ __launch_bounds__(kMaxThreads) void norm_kernel(NormCall c, int32_t lanes) {
  __shared__ float buffer[2][16][1];
  const int t = int(threadIdx.x) & (lanes - 1), team = team_of<R == 1>(lanes), teams = int(blockDim.x) / lanes;
  const int64_t step = int64_t(gridDim.x) * teams;
  Columns<V, R, WHOLE> at;
  at.init(t, lanes, c.cols);
  TeamSum<1, R == 1> sum;
  sum.init(buffer, lanes);
  const float inv = 1.0f / float(c.cols);
  float w[R][V], b[R][V];
  Raw<X, V> raw[R];
  auto fetch = [&](int64_t r) {
    if (r >= c.rows) return;
    const X* const p = static_cast<const X*>(c.x) + r * c.ldx;
#pragma unroll
    for (int q = 0; q < R; ++q)
      if (at.there(q)) raw[q].load(element(p, at.from(q)));
  };
  // the workgroup's teams go round together, as they meet
  int64_t first = int64_t(blockIdx.x) * teams;
  fetch(first + team);
#pragma unroll
  for (int q = 0; q < R; ++q) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      w[q][i] = 1.0f;
      b[q][i] = 0.0f;
    }
    if (at.there(q) && c.w) load_params<V>(w[q], c.w, c.we, at.col(q), at.back(q));
    if (at.there(q) && c.b) load_params<V>(b[q], c.b, c.be, at.col(q), at.back(q));
  }
  for (; first < c.rows; first += step) {
    const int64_t row = first + team;
    const bool mine = row < c.rows;
    float v[R][V], s[1] = {0.0f};
#pragma unroll
    for (int q = 0; q < R; ++q) {
#pragma unroll
      for (int i = 0; i < V; ++i) v[q][i] = 0.0f;
      if (at.there(q) && mine) raw[q].get(v[q], at.back(q));
#pragma unroll
      for (int i = 0; i < V; ++i) s[0] += v[q][i];
    }
    fetch(row + step);
    sum(s);
    const float mean = s[0] / float(c.cols);
    s[0] = 0.0f;
#pragma unroll
    for (int q = 0; q < R; ++q) {
      if (!at.there(q)) continue;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        v[q][i] -= mean;
        s[0] = at.there(q, i) ? __builtin_fmaf(v[q][i], v[q][i], s[0]) : s[0];
      }
    }
    sum(s);
    const float rstd = 1.0f / sqrtf(__builtin_fmaf(s[0], inv, c.eps));
    if (!mine) continue;
    if (c.stats && t == 0) {
      c.stats[row * c.lds] = mean;
      c.stats[row * c.lds + 1] = rstd;
    }
    Y* const p = static_cast<Y*>(c.y) + row * c.ldy;
#pragma unroll
    for (int q = 0; q < R; ++q) {
      if (!at.there(q)) continue;
#pragma unroll
      for (int i = 0; i < V; ++i) v[q][i] = __builtin_fmaf(v[q][i] * rstd, w[q][i], b[q][i]);
      store_row<V>(element(p, at.col(q)), v[q], at.back(q));
    }
  }
}

// A long row's groups of 8 columns in turn, by a whole workgroup; f(values,
// first column, columns that are there).
template <typename X, typename F>
__device__ __forceinline__ void along(const X* p, int64_t cols, F&& f) {
  for (int64_t col = int64_t(threadIdx.x) * 8; col < cols; col += int64_t(blockDim.x) * 8) {
    const int have = cols - col < 8 ? int(cols - col) : 8;
    float v[8];
    if (have == 8) load_group<8>(v, p + col);
    else load_tail<8>(v, p + col, have);
    f(v, col, have);
  }
}
template <int V, typename T>
__device__ __forceinline__ void store_part(T* p, const float (&x)[V], int have) {
  if (have == V) store_group<V>(p, x);
  else store_tail<V>(p, x, have);
}
// Parameters of up to 8 columns; 0 where there are none.
__device__ __forceinline__ void params_part(float (&v)[8], const void* p, int32_t e, int64_t col, int have) {
  auto of = [&](auto* t) {
    if (have == 8) load_group<8>(v, t + col);
    else load_tail<8>(v, t + col, have);
  };
  if (e == kF32) of(static_cast<const float*>(p));
  else if (e == kF16) of(static_cast<const f16*>(p));
  else of(static_cast<const bf16*>(p));
}

// Rows longer than a team holds, three times over from the caches.
template <typename X, typename Y>
__global__ __launch_bounds__(kMaxThreads) void norm_wide_kernel(NormCall c) {
  __shared__ float buffer[2][16][1];
  TeamSum<1, false> sum;
  sum.init(buffer, int(blockDim.x));
  const float inv = 1.0f / float(c.cols);
  for (int64_t row = blockIdx.x; row < c.rows; row += gridDim.x) {
    const X* const x = static_cast<const X*>(c.x) + row * c.ldx;
    Y* const y = static_cast<Y*>(c.y) + row * c.ldy;
    float s[1] = {0.0f};
    along(x, c.cols, [&](float (&v)[8], int64_t, int) {
#pragma unroll
      for (int i = 0; i < 8; ++i) s[0] += v[i];
    });
    sum(s);
    const float mean = s[0] / float(c.cols);
    s[0] = 0.0f;
    along(x, c.cols, [&](float (&v)[8], int64_t, int have) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float d = v[i] - mean;
        s[0] += i < have ? d * d : 0.0f;
      }
    });
    sum(s);
    const float rstd = 1.0f / sqrtf(s[0] * inv + c.eps);
    if (c.stats && threadIdx.x == 0) {
      c.stats[row * c.lds] = mean;
      c.stats[row * c.lds + 1] = rstd;
    }
    along(x, c.cols, [&](float (&v)[8], int64_t col, int have) {
      float w[8] = {1, 1, 1, 1, 1, 1, 1, 1}, b[8] = {0, 0, 0, 0, 0, 0, 0, 0};
      if (c.w) params_part(w, c.w, c.we, col, have);
      if (c.b) params_part(b, c.b, c.be, col, have);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = (v[i] - mean) * rstd * w[i] + b[i];
      store_part<8>(y + col, v, have);
    });
  }
}

// The gradient: as norm_kernel, with the sums of dy h and dy kept by the lanes
// over their rows, then over the workgroup's teams through LDS, in their order.
// w lies in LDS, in 32 bits; the sums take its place at the end.
template <typename X, typename D, int V, int R, bool WHOLE>
__global__ __launch_bounds__(kMaxThreads) void norm_grad_kernel(NormGradCall c, int32_t lanes) {
  __shared__ float buffer[2][16][2];
  extern __shared__ __attribute__((aligned(16))) float shared[];  // lanes R V of w; a team's lanes V for the sums
  const int t = int(threadIdx.x) & (lanes - 1), team = team_of<R == 1>(lanes), teams = int(blockDim.x) / lanes;
  const int64_t step = int64_t(gridDim.x) * teams;
  int64_t row = int64_t(blockIdx.x) * teams + team;
  Columns<V, R, WHOLE> at;
  at.init(t, lanes, c.cols);
  TeamSum<2, R == 1> sum;
  sum.init(buffer, lanes);
  const float inv = 1.0f / float(c.cols);
  float dw[R][V], db[R][V], mean = 0.0f, rstd = 0.0f;
  Raw<X, V> rx[R], rr[sizeof(X) == 2 && sizeof(D) == 2 ? R : 1];
  Raw<D, V> rd[R];
  auto fetch = [&](int64_t r) {
    if (r >= c.rows) return;
    const X* const p = static_cast<const X*>(c.x) + r * c.ldx;
    const D* const d = static_cast<const D*>(c.dy) + r * c.lddy;
    mean = c.stats[r * c.lds];
    rstd = c.stats[r * c.lds + 1];
#pragma unroll
    for (int q = 0; q < R; ++q) {
      if (at.there(q)) {
        rx[q].load(element(p, at.from(q)));
        rd[q].load(element(d, at.from(q)));
      }
    }
  };
  // of 32 bits it would not fit the registers: each group when it is added
  constexpr bool kAhead = sizeof(X) == 2 && sizeof(D) == 2;
  auto residual = [&](int q, int64_t r) {
    rr[kAhead ? q : 0].load(element(static_cast<const X*>(c.res) + r * c.ldr, at.from(q)));
  };
  auto fetch_residual = [&](int64_t r) {
    if (!kAhead || !c.res || r >= c.rows) return;
#pragma unroll
    for (int q = 0; q < R; ++q)
      if (at.there(q)) residual(q, r);
  };
  fetch(row);
  fetch_residual(row);
#pragma unroll
  for (int q = 0; q < R; ++q) {
    float w[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      w[i] = 1.0f;
      dw[q][i] = db[q][i] = 0.0f;
    }
    if (team == 0 && c.w && at.there(q)) load_params<V>(w, c.w, c.we, at.col(q), at.back(q));
    if (team == 0) {
#pragma unroll
      for (int i = 0; i < V; ++i) shared[at.col(q) + i] = w[i];
    }
  }
  __syncthreads();
  for (int64_t first = row - team; first < c.rows; first += step, row += step) {
    float h[R][V], g[R][V], s[2] = {0.0f, 0.0f};
    const bool mine = row < c.rows;
    const float scale = rstd;
#pragma unroll
    for (int q = 0; q < R; ++q) {
#pragma unroll
      for (int i = 0; i < V; ++i) h[q][i] = g[q][i] = 0.0f;
      if (!mine || !at.there(q)) continue;
      rx[q].get(h[q], at.back(q));
      rd[q].get(g[q], at.back(q));
#pragma unroll
      for (int i = 0; i < V; ++i) {
        h[q][i] = at.there(q, i) ? (h[q][i] - mean) * scale : 0.0f;
        dw[q][i] = __builtin_fmaf(g[q][i], h[q][i], dw[q][i]);
        db[q][i] += g[q][i];
        g[q][i] *= shared[at.col(q) + i];
        s[0] += g[q][i];
        s[1] = __builtin_fmaf(g[q][i], h[q][i], s[1]);
      }
      __builtin_amdgcn_sched_barrier(0);  // a group's temporaries at a time, here and below: 128 registers hold no more
    }
    fetch(row + step);
    if (!c.dx) continue;  // the same for all
    __builtin_amdgcn_sched_barrier(0);
    sum(s);
    __builtin_amdgcn_sched_barrier(0);
    if (!mine) continue;
    const float g0 = s[0] * inv, g1 = s[1] * inv;
    X* const p = static_cast<X*>(c.dx) + row * c.lddx;
#pragma unroll
    for (int q = 0; q < R; ++q) {
      if (!at.there(q)) continue;
      float r[V];
#pragma unroll
      for (int i = 0; i < V; ++i) g[q][i] = scale * __builtin_fmaf(h[q][i], -g1, g[q][i] - g0);
      if (c.res) {
        if (!kAhead) residual(q, row);
        rr[kAhead ? q : 0].get(r, at.back(q));
#pragma unroll
        for (int i = 0; i < V; ++i) g[q][i] += r[i];
      }
      store_row<V>(element(p, at.col(q)), g[q], at.back(q));
      __builtin_amdgcn_sched_barrier(0);
    }
    fetch_residual(row + step);
  }
  if (!c.parts) return;
  float* const parts = c.parts + int64_t(blockIdx.x) * 2 * c.cols;
  if (teams == 1) {
#pragma unroll
    for (int q = 0; q < R; ++q) {
      if (!at.there(q)) continue;
      store_row<V>(parts + at.col(q), dw[q], at.back(q));
      store_row<V>(parts + c.cols + at.col(q), db[q], at.back(q));
    }
    return;
  }
  const int width = lanes * V;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
#pragma unroll
    for (int q = 0; q < R; ++q) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < V; ++i) shared[team * width + t * V + i] = which ? db[q][i] : dw[q][i];
      __syncthreads();
      for (int n = int(threadIdx.x); n < width && q * width + n < c.cols; n += int(blockDim.x)) {
        float v = 0.0f;
        for (int s = 0; s < teams; ++s) v += shared[s * width + n];
        parts[which * c.cols + q * width + n] = v;
      }
    }
  }
}

// dx of rows longer than a team holds.
template <typename X, typename D>
__global__ __launch_bounds__(kMaxThreads) void norm_grad_wide_kernel(NormGradCall c) {
  __shared__ float buffer[2][16][2];
  TeamSum<2, false> sum;
  sum.init(buffer, int(blockDim.x));
  const float inv = 1.0f / float(c.cols);
  for (int64_t row = blockIdx.x; row < c.rows; row += gridDim.x) {
    const X* const x = static_cast<const X*>(c.x) + row * c.ldx;
    const D* const dy = static_cast<const D*>(c.dy) + row * c.lddy;
    X* const dx = static_cast<X*>(c.dx) + row * c.lddx;
    const float mean = c.stats[row * c.lds], rstd = c.stats[row * c.lds + 1];
    // f(g, h, first column, columns that are there)
    auto each = [&](auto&& f) {
      along(x, c.cols, [&](float (&h)[8], int64_t col, int have) {
        float g[8], w[8] = {1, 1, 1, 1, 1, 1, 1, 1};
        if (have == 8) load_group<8>(g, dy + col);
        else load_tail<8>(g, dy + col, have);
        if (c.w) params_part(w, c.w, c.we, col, have);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          h[i] = i < have ? (h[i] - mean) * rstd : 0.0f;
          g[i] = i < have ? g[i] * w[i] : 0.0f;
        }
        f(g, h, col, have);
      });
    };
    float s[2] = {0.0f, 0.0f};
    each([&](float (&g)[8], float (&h)[8], int64_t, int) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        s[0] += g[i];
        s[1] += g[i] * h[i];
      }
    });
    sum(s);
    const float g0 = s[0] * inv, g1 = s[1] * inv;
    each([&](float (&g)[8], float (&h)[8], int64_t col, int have) {
      float r[8] = {0, 0, 0, 0, 0, 0, 0, 0};
      if (c.res) {
        const X* const p = static_cast<const X*>(c.res) + row * c.ldr + col;
        if (have == 8) load_group<8>(r, p);
        else load_tail<8>(r, p, have);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) g[i] = r[i] + rstd * (g[i] - g0 - h[i] * g1);
      store_part<8>(dx + col, g, have);
    });
  }
}

// The sums of dy h and dy of long rows: 256 threads take 2048 columns of the
// rows of one block, which are rows block, block + blocks, ...
template <typename X, typename D>
__global__ __launch_bounds__(256) void norm_sums_kernel(NormGradCall c) {
  const int64_t col = (int64_t(blockIdx.x) * 256 + threadIdx.x) * 8;
  if (col >= c.cols) return;
  const int have = c.cols - col < 8 ? int(c.cols - col) : 8;
  float dw[8] = {0, 0, 0, 0, 0, 0, 0, 0}, db[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  for (int64_t row = blockIdx.y; row < c.rows; row += gridDim.y) {
    const X* const x = static_cast<const X*>(c.x) + row * c.ldx + col;
    const D* const dy = static_cast<const D*>(c.dy) + row * c.lddy + col;
    float h[8], g[8];
    if (have == 8) {
      load_group<8>(h, x);
      load_group<8>(g, dy);
    } else {
      load_tail<8>(h, x, have);
      load_tail<8>(g, dy, have);
    }
    const float mean = c.stats[row * c.lds], rstd = c.stats[row * c.lds + 1];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      dw[i] += g[i] * ((h[i] - mean) * rstd);
      db[i] += g[i];
    }
  }
  float* const parts = c.parts + int64_t(blockIdx.y) * 2 * c.cols + col;
  store_part<8>(parts, dw, have);
  store_part<8>(parts + c.cols, db, have);
}

// 16 columns a workgroup, 16 threads to each column's blocks; blockIdx.y: dw, db.
__global__ __launch_bounds__(256) void norm_join_kernel(NormJoinCall c) {
  __shared__ float part[16][17];
  void* const out = blockIdx.y ? c.db : c.dw;
  if (!out) return;
  const int ct = threadIdx.x & 15, rt = threadIdx.x >> 4;
  for (int64_t n0 = int64_t(blockIdx.x) * 16; n0 < c.cols; n0 += int64_t(gridDim.x) * 16) {
    const int64_t n = n0 + ct;
    float s = 0.0f;
    if (n < c.cols) {
      const float* const p = c.parts + blockIdx.y * c.cols + n;
#pragma unroll 16
      for (int32_t k = rt; k < c.blocks; k += 16) s += p[int64_t(k) * 2 * c.cols];
    }
    __syncthreads();
    part[rt][ct] = s;
    __syncthreads();
    if (rt != 0 || n >= c.cols) continue;
    auto finish = [&](auto* to) {
      float v = c.accumulate ? float(to[n]) : 0.0f;
#pragma unroll
      for (int r = 0; r < 16; ++r) v += part[r][ct];
      to[n] = std::remove_pointer_t<decltype(to)>(v);
    };
    const int32_t e = blockIdx.y ? c.dbe : c.dwe;
    if (e == kF32) finish(static_cast<float*>(out));
    else if (e == kF16) finish(static_cast<f16*>(out));
    else finish(static_cast<bf16*>(out));
  }
}

constexpr int64_t kCus = 256;

template <typename X, typename Y>
int launch_norm_of(const NormCall& c, hipStream_t st) {
  const RowTeams k = row_teams(c.cols);
  if (k.wide) {
    const dim3 grid(uint32_t(c.rows < 8 * kCus ? c.rows : 8 * kCus));
    norm_wide_kernel<X, Y><<<grid, dim3(kMaxThreads), 0, st>>>(c);
    return int(hipGetLastError());
  }
  const int threads = k.lanes > 256 ? k.lanes : 256;
  // as many workgroups as their registers let in at once: one more on some units
  // runs its rows by itself at the end (8192 x 8192 bf16 58.8 us for 50.2)
  const int waves = k.per == 1 ? 32 : sizeof(X) == 4 ? 20 : 24;
  const int64_t teams = threads / k.lanes, need = (c.rows + teams - 1) / teams, most = kCus * std::max(1, waves * 64 / threads);
  const dim3 grid(uint32_t(need < most ? need : most));
  const bool whole = c.cols % 8 == 0;
  if (k.V == 1) norm_kernel<X, Y, 1, 1, true><<<grid, dim3(threads), 0, st>>>(c, k.lanes);
  else if (k.per == 1 && whole) norm_kernel<X, Y, 8, 1, true><<<grid, dim3(threads), 0, st>>>(c, k.lanes);
  else if (k.per == 1) norm_kernel<X, Y, 8, 1, false><<<grid, dim3(threads), 0, st>>>(c, k.lanes);
  else if (whole) norm_kernel<X, Y, 8, 2, true><<<grid, dim3(threads), 0, st>>>(c, k.lanes);
  else norm_kernel<X, Y, 8, 2, false><<<grid, dim3(threads), 0, st>>>(c, k.lanes);
  return int(hipGetLastError());
}

template <typename X>
int launch_norm_x(const NormCall& c, int32_t ye, hipStream_t st) {
  switch (ye) {
    case kF32: return launch_norm_of<X, float>(c, st);
    case kF16: return launch_norm_of<X, f16>(c, st);
    case kBF16: return launch_norm_of<X, bf16>(c, st);
  }
  return int(hipErrorInvalidValue);
}

// Threads of a gradient's workgroup: teams enough for its rows.
int grad_threads(const RowTeams& k, int64_t rows) {
  int threads = k.lanes > 64 ? k.lanes : 64;
  while (threads < kMaxThreads && rows > kCus * (threads / k.lanes)) threads *= 2;
  return threads;
}

template <typename X, typename D>
int launch_norm_grad_of(const NormGradCall& c, hipStream_t st) {
  const RowTeams k = row_teams(c.cols);
  if (k.wide) {
    if (c.parts) {  // first: dx may be dy
      const dim3 grid(uint32_t((c.cols + 2047) / 2048), uint32_t(c.blocks));
      norm_sums_kernel<X, D><<<grid, dim3(256), 0, st>>>(c);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return int(e);
    }
    if (c.dx) {
      const dim3 grid(uint32_t(c.rows < 8 * kCus ? c.rows : 8 * kCus));
      norm_grad_wide_kernel<X, D><<<grid, dim3(kMaxThreads), 0, st>>>(c);
    }
    return int(hipGetLastError());
  }
  const int threads = grad_threads(k, c.rows);
  const dim3 grid(uint32_t(c.blocks)), block{uint32_t(threads)};
  const int lds = k.V * std::max(k.lanes * k.per, threads) * int(sizeof(float));
  const bool whole = c.cols % 8 == 0;
  if (k.V == 1) norm_grad_kernel<X, D, 1, 1, true><<<grid, block, lds, st>>>(c, k.lanes);
  else if (k.per == 1 && whole) norm_grad_kernel<X, D, 8, 1, true><<<grid, block, lds, st>>>(c, k.lanes);
  else if (k.per == 1) norm_grad_kernel<X, D, 8, 1, false><<<grid, block, lds, st>>>(c, k.lanes);
  else if (whole) norm_grad_kernel<X, D, 8, 2, true><<<grid, block, lds, st>>>(c, k.lanes);
  else norm_grad_kernel<X, D, 8, 2, false><<<grid, block, lds, st>>>(c, k.lanes);
  return int(hipGetLastError());
}

template <typename X>
int launch_norm_grad_x(const NormGradCall& c, int32_t dye, hipStream_t st) {
  switch (dye) {
    case kF32: return launch_norm_grad_of<X, float>(c, st);
    case kF16: return launch_norm_grad_of<X, f16>(c, st);
    case kBF16: return launch_norm_grad_of<X, bf16>(c, st);
  }
  return int(hipErrorInvalidValue);
}

}  // namespace

RowTeams row_teams(int64_t cols) {
  if (cols > kTeamColumns) return {8, kMaxThreads, 0, 1};
  RowTeams k{cols < 8 ? 1 : 8, 8, 1, 0};
  while (int64_t(k.lanes) * k.per * k.V < cols) {
    // one group a lane in a part of a wave, then two
    if (k.lanes < 64 || k.per == 2) k.lanes *= 2;
    else k.per = 2;
  }
  return k;
}

int32_t norm_grad_blocks(int64_t rows, int64_t cols) {
  const RowTeams k = row_teams(cols);
  if (k.wide) {
    const int64_t across = (cols + 2047) / 2048, most = across < 4 * kCus ? 4 * kCus / across : 1;
    return int32_t(rows < most ? rows : most);
  }
  const int64_t teams = grad_threads(k, rows) / k.lanes, need = (rows + teams - 1) / teams;
  return int32_t(need < kCus ? need : kCus);
}

int launch_norm(const NormCall& c, int32_t xe, int32_t ye, void* stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  switch (xe) {
    case kF32: return launch_norm_x<float>(c, ye, st);
    case kF16: return launch_norm_x<f16>(c, ye, st);
    case kBF16: return launch_norm_x<bf16>(c, ye, st);
  }
  return int(hipErrorInvalidValue);
}

int launch_norm_grad(const NormGradCall& c, int32_t xe, int32_t dye, void* stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  switch (xe) {
    case kF32: return launch_norm_grad_x<float>(c, dye, st);
    case kF16: return launch_norm_grad_x<f16>(c, dye, st);
    case kBF16: return launch_norm_grad_x<bf16>(c, dye, st);
  }
  return int(hipErrorInvalidValue);
}

int launch_norm_join(const NormJoinCall& c, void* stream) {
  const int64_t need = (c.cols + 15) / 16, most = int64_t(1) << 20;
  const dim3 grid(uint32_t(need < most ? need : most), 2);
  norm_join_kernel<<<grid, dim3(256), 0, static_cast<hipStream_t>(stream)>>>(c);
  return int(hipGetLastError());
}

}  // namespace ar
