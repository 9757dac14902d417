// orthogonal.hip -- the orthogonalised update of a weight by Newton-Schulz
// products: with X = x / (|x| + eps) (Frobenius norm) and m the shorter side,
//   A = X X^T,  X <- a X + (b A + c A^2) X     each step,
// an odd polynomial of X's singular values, which sends them to about 1.
//
// Precision.  The gain of small singular values (a^steps, 485 for five steps of
// 3.4445) multiplies whatever is added to X in their directions, so X itself is
// held in two halves, 22 bits, and both enter a X.  The products may take rounded
// operands all the same: with E the rounding of X's high half, (Q + E_Q)(X + E)
// is off by E_Q X, which lies in X's row space, and by Q E, which lies in its
// column space, and neither grows with the gain.  So one product of high halves
// serves results in bfloat16: off by 2e-4 to 2.5e-3 of the result before its
// rounding of 1.7e-3, of low and of full rank, as long as the roundings even out.
// They do not where entries are equal: a block of ones rounds all of X, A and Q the
// same way, and each step's slope adds that up, to 2.6e-2 at worst (four blocks of
// 318 x 544; sparse rows and equal singular values 4e-3).  Three products (high high,
// high low, low high) serve the others, to about what 32-bit arithmetic gives.  The
// diagonal of Q, a quarter of the roundings' effect, stays in 32 bits beside it.
// Halves are stored times 2^13 (Q: 2^12), so that values far below a matrix' norm
// keep their bits; the entry point admits only coefficients that keep |X| below
// 2.5 and |Q| below 15.
//
// Bound by the matrix units, and by X's own traffic between their tiles, where
// matrices are large (4096 x 16384 bf16: 270 to 310, 88 and 500 us for a step's
// products, 4420 to 4700 in all; 2700 at the best rate of a large product), by the
// latency of three launches a step where they are small (4096 x 1024: 15.6, 7.9 and
// 19 us, 220 in all).
#include <hip/hip_runtime.h>

#include <type_traits>

#include "gemm.hpp"
#include "training.hpp"

namespace ar {

namespace {

constexpr int kThreads = 256;

// ---- from x to X and from X to y ----

// The sum over a workgroup of 256, in all of its threads.
__device__ __forceinline__ double block_sum(double v, double (&lds)[4]) {
#pragma unroll
  for (int m = 1; m < 64; m *= 2) v += __shfl_xor(v, m);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  return lds[0] + lds[1] + lds[2] + lds[3];
}

// 8 columns of a row, of which `have` are there: the others 0.
template <typename T>
__device__ __forceinline__ void load_some(float (&v)[8], const T* p, int64_t have) {
  if (have >= 8) load_group<8>(v, p);
  else load_tail<8>(v, p, have > 0 ? int(have) : 0);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void ortho_norm_kernel(OrthoShape s, OrthoOuter x, double* sums) {
  __shared__ double lds[4];
  const T* const p = static_cast<const T*>(x.data) + int64_t(blockIdx.y) * x.stride;
  const int64_t groups = (s.cols + 7) / 8, step = int64_t(gridDim.x) * kThreads;
  const int64_t dr = step / groups, dg = step % groups;
  int64_t id = int64_t(blockIdx.x) * kThreads + threadIdx.x, row = id / groups, g = id % groups;
  double sum = 0.0;
  constexpr int kAhead = 4;  // groups on their way together
  while (row < s.rows) {
    float v[kAhead][8];
#pragma unroll
    for (int q = 0; q < kAhead; ++q) {
      load_some(v[q], p + (row < s.rows ? row * x.ld + g * 8 : 0), row < s.rows ? s.cols - g * 8 : 0);
      row += dr;
      g += dg;
      if (g >= groups) {
        g -= groups;
        ++row;
      }
    }
#pragma unroll
    for (int q = 0; q < kAhead; ++q)
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += double(v[q][i]) * double(v[q][i]);
  }
  sum = block_sum(sum, lds);
  if (threadIdx.x == 0) sums[int64_t(blockIdx.y) * gridDim.x + blockIdx.x] = sum;
}

typedef f16 f16x8 __attribute__((ext_vector_type(8)));

// Eight values as their high and low halves.
__device__ __forceinline__ void split8(const float (&v)[8], f16x8& high, f16x8& low) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    high[i] = f16(v[i]);
    low[i] = f16(v[i] - float(high[i]));
  }
}

// 64 x 64 values of X a workgroup, a thread two groups of 8; turned ones through LDS.
template <typename T>
__global__ __launch_bounds__(kThreads) void ortho_load_kernel(OrthoShape s, OrthoOuter x, const double* sums, double eps,
                                                              f16* planes) {
  __shared__ double lds[4];
  __shared__ float turn[64][65];
  const double* const mine = sums + int64_t(blockIdx.z) * s.blocks;
  double part = 0.0;
  for (int32_t i = threadIdx.x; i < s.blocks; i += kThreads) part += mine[i];
  const double norm = sqrt(block_sum(part, lds));
  const double factor = double(kOrthoScaleX) / (norm + eps);
  const T* const p = static_cast<const T*>(x.data) + int64_t(blockIdx.z) * x.stride;
  const int64_t plane = s.mp * s.np, m0 = int64_t(blockIdx.y) * 64, n0 = int64_t(blockIdx.x) * 64;
  f16* const out = planes + int64_t(blockIdx.z) * 2 * plane;
  const int r = int(threadIdx.x) >> 3, c = (int(threadIdx.x) & 7) * 8;
  if (s.turned) {
#pragma unroll
    for (int h = 0; h < 64; h += 32) {
      const int64_t row = n0 + r + h, col = m0 + c;
      float v[8];
      load_some(v, p + (row < s.rows ? row * x.ld : 0) + (col < s.cols ? col : 0), row < s.rows ? s.cols - col : 0);
#pragma unroll
      for (int i = 0; i < 8; ++i) turn[r + h][c + i] = v[i];
    }
    __syncthreads();
  }
#pragma unroll
  for (int h = 0; h < 64; h += 32) {
    const int64_t row = m0 + r + h, col = n0 + c;
    float v[8];
    if (s.turned) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = turn[c + i][r + h];
    } else {
      load_some(v, p + (row < s.rows ? row * x.ld : 0) + (col < s.cols ? col : 0), row < s.rows ? s.cols - col : 0);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = float(double(v[i]) * factor);
    f16x8 high, low;
    split8(v, high, low);
    *reinterpret_cast<f16x8*>(out + row * s.np + col) = high;
    *reinterpret_cast<f16x8*>(out + plane + row * s.np + col) = low;
  }
}

// ---- the products ----

// Where steps first, first + STRIDE, first + 2 STRIDE and so on of a tile lie.  The
// steps of a pair of planes follow those of the pair before: low high, high low,
// high high (the last are added to sums of their own size).
template <int PLANES, int STRIDE>
struct InPlanes {
  int32_t first, each;           // each: the steps of a pair of planes
  int64_t low_left, low_right;   // bytes from an operand's high plane to its low one
  template <typename Op>
  __device__ __forceinline__ const char* at(const Op& op, int32_t t) const {
    int32_t u = first + t * STRIDE;
    if constexpr (PLANES == 1) return op.base + u * op.step();
    const int32_t pair = u >= 2 * each ? 2 : u >= each ? 1 : 0;
    u -= pair * each;
    // which pair takes an operand's low plane: the left one's first, the right one's second
    const bool low = op.kRight ? pair == 1 : pair == 0;
    return op.base + (low ? (op.kRight ? low_right : low_left) : 0) + u * op.step();
  }
  template <typename Op>
  __device__ __forceinline__ void move(const char*& p, const Op& op, int32_t t, int32_t whole) const {
    if constexpr (PLANES == 1) p += t < whole ? STRIDE * op.step() : 0;
    else if (t < whole) p = at(op, t);
  }
};
template <typename Op, bool RIGHT>
struct Side : Op {
  static constexpr bool kRight = RIGHT;
};

// Tile `t` of a symmetric result's tiles on and below the diagonal, by rows.
__device__ __forceinline__ void below_diagonal(uint32_t t, uint32_t& m, uint32_t& n) {
  m = uint32_t((sqrtf(8.0f * float(t) + 1.0f) - 1.0f) * 0.5f);
  while (m * (m + 1) / 2 > t) --m;
  while ((m + 1) * (m + 2) / 2 <= t) ++m;
  n = t - m * (m + 1) / 2;
}

template <int KIND>
struct TileAt {
  uint32_t matrix, m, n;
  __device__ __forceinline__ TileAt(const OrthoProduct& g, uint32_t tile) {
    matrix = tile / uint32_t(g.tiles);
    const uint32_t t = tile - matrix * uint32_t(g.tiles);
    if constexpr (KIND == kOrthoApply) {
      // groups of 8 rows of tiles, as in tile_of
      const uint32_t tm = uint32_t(g.tiles_m), tn = uint32_t(g.tiles_n), group = t / (8 * tn), first = group * 8;
      const uint32_t h = tm - first < 8 ? tm - first : 8, in = t - group * 8 * tn;
      m = first + in % h;
      n = in / h;
    } else {
      below_diagonal(t, m, n);
    }
  }
};

// Of eight lanes r = 0 to 7 (of 8 consecutive ones), lane r gets the r-th half of
// each: 8 x 8 halves turned, first within pairs of lanes, then pairs of halves.
__device__ __forceinline__ f16x8 turn8(const f16x8& v) {
  typedef uint32_t U4 __attribute__((ext_vector_type(4)));
  U4 d = __builtin_bit_cast(U4, v);
  const int lane = int(threadIdx.x);
  auto other = [](uint32_t x, auto how) {
    constexpr int m = decltype(how)::value;
    if constexpr (m == 4) return uint32_t(__builtin_amdgcn_ds_swizzle(int(x), 0x101f));
    else return uint32_t(__builtin_amdgcn_mov_dpp(int(x), m == 1 ? 0xb1 : 0x4e, 0xf, 0xf, true));
  };
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const uint32_t o = other(d[q], std::integral_constant<int, 1>{});
    d[q] = lane & 1 ? o >> 16 | (d[q] & 0xffff0000u) : (d[q] & 0xffffu) | o << 16;
  }
#pragma unroll
  for (int q = 0; q < 4; q += 2) {
    const uint32_t o = other(lane & 2 ? d[q] : d[q + 1], std::integral_constant<int, 2>{});
    d[q] = lane & 2 ? o : d[q];
    d[q + 1] = lane & 2 ? d[q + 1] : o;
  }
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const uint32_t o = other(lane & 4 ? d[q] : d[q + 2], std::integral_constant<int, 4>{});
    d[q] = lane & 4 ? o : d[q];
    d[q + 2] = lane & 4 ? d[q + 2] : o;
  }
  return __builtin_bit_cast(f16x8, d);
}

// What becomes of 8 sums of row m, columns n on.  Y: the type of y, for the last
// step's product, which writes y.
template <int KIND, int PLANES, typename Y>
struct Finish {
  static constexpr bool kLast = !std::is_void_v<Y>;
  static constexpr bool kLow = PLANES == 2 || KIND == kOrthoApply;  // whether old and out have low halves
  const OrthoProduct& g;
  f16* out;
  const f16* old;
  float* diag;
  int64_t outer;  // the matrix' place in x and y
  bool mirror;    // a tile below the diagonal: its transpose is written too

  __device__ __forceinline__ Finish(const OrthoProduct& g_, const TileAt<KIND>& at) : g(g_) {
    out = static_cast<f16*>(g.out) + int64_t(at.matrix) * g.batch_out;
    old = static_cast<const f16*>(g.old) + int64_t(at.matrix) * g.batch_out;
    diag = g.diag + int64_t(at.matrix) * g.M;
    outer = at.matrix;
    mirror = KIND != kOrthoApply && at.m != at.n;
  }

  // The values there, which may be on their way while the sums are made.
  struct Old {
    f16x8 high, low;
  };
  __device__ __forceinline__ Old fetch(int32_t m, int32_t n) const {
    Old o;
    if constexpr (KIND != kOrthoGram) {
      const int64_t at = int64_t(m) * g.ld_out + n;
      o.high = *reinterpret_cast<const f16x8*>(old + at);
      if constexpr (kLow) o.low = *reinterpret_cast<const f16x8*>(old + g.plane_out + at);
    }
    return o;
  }

  // y's elements of X's row m, columns n on, or where x is turned of its column.
  __device__ __forceinline__ void last(f16x8 high, f16x8 low, int32_t m, int32_t n) const {
    using T = std::conditional_t<kLast, Y, float>;
    int64_t row = m, col = n;
    if (g.turned) {
      high = turn8(high);
      low = turn8(low);
      row = n + int(threadIdx.x & 7);
      col = m & ~7;
    }
    if (row >= g.rows || col >= g.cols) return;
    const int64_t have = g.cols - col;
    float v[8], w[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (g.residual.data)
      load_some(w, static_cast<const T*>(g.residual.data) + outer * g.residual.stride + row * g.residual.ld + col, have);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = w[i] + g.scale * ((float(high[i]) + float(low[i])) * (1.0f / kOrthoScaleX));
    T* const to = const_cast<T*>(static_cast<const T*>(g.y.data)) + outer * g.y.stride + row * g.y.ld + col;
    if (have >= 8) store_group<8>(to, v);
    else store_tail<8>(to, v, int(have));
  }

  __device__ __forceinline__ void operator()(float (&v)[8], const Old& o, int32_t m, int32_t n) const {
    if constexpr (KIND == kOrthoGram) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] *= kOrthoScaleA / (kOrthoScaleX * kOrthoScaleX);
    } else if constexpr (KIND == kOrthoSquare) {
      // of A as the products take it: rounded once
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float x = PLANES == 2 ? float(o.high[i]) + float(o.low[i]) : float(o.high[i]);
        v[i] = g.b * (x * (kOrthoScaleQ / kOrthoScaleA)) + g.c * (v[i] * (kOrthoScaleQ / (kOrthoScaleA * kOrthoScaleA)));
        if (m == n + i) {
          diag[m] = v[i] * (1.0f / kOrthoScaleQ);
          v[i] = 0.0f;
        }
      }
    } else {
      const float d = diag[m];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float x = float(o.high[i]) + float(o.low[i]);
        // the diagonal multiplies what the products took
        v[i] = g.a * x + (d * (PLANES == 2 ? x : float(o.high[i])) + v[i] * (1.0f / kOrthoScaleQ));
      }
    }
    f16x8 high, low;
    split8(v, high, low);
    if constexpr (kLast) {
      last(high, low, m, n);
    } else {
      f16* const to = out + int64_t(m) * g.ld_out + n;
      *reinterpret_cast<f16x8*>(to) = high;
      if constexpr (kLow) *reinterpret_cast<f16x8*>(to + g.plane_out) = low;
      if (KIND != kOrthoApply && mirror) {
        f16* const turned = out + int64_t(n + int(threadIdx.x & 7)) * g.ld_out + (m & ~7);
        *reinterpret_cast<f16x8*>(turned) = turn8(high);
        if constexpr (kLow) *reinterpret_cast<f16x8*>(turned + g.plane_out) = turn8(low);
      }
    }
  }
};

// The place of a part's eight sums: unit u of thread `tid`.
__device__ __forceinline__ float* part_at(float* slot, int u, int tid) { return slot + (u * kThreads + tid) * 8; }

template <int KIND, int PLANES, typename Y, int MT, int NT>
__global__ __launch_bounds__(kThreads, MT * NT <= 16 ? 2 : 1) void ortho_product_kernel(OrthoProduct g) {
  constexpr bool BK = KIND != kOrthoApply;
  constexpr int TM = 2 * MT * 16, TN = 2 * NT * 16, kPairs = NT / 2;
  constexpr bool kPinned = MT * NT == 64, kSplits = ortho_splits(KIND, PLANES, TM);
  __shared__ __attribute__((aligned(1024))) char lds[ring_bytes(TM)];
  using OpA = Side<Operand<f16, true, false, TM, kThreads>, false>;
  using OpB = Side<Operand<f16, BK, true, TN, kThreads>, true>;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / 2, wn = wave % 2;
  Fragments<f16, true, false, TM> ra;
  Fragments<f16, BK, true, TN> rb;
  ra.init(wm * MT * 16, lane);
  rb.init(wn * NT * 16, lane);
  // each XCD takes a contiguous range of shares
  const uint32_t W = gridDim.x, xcd = blockIdx.x & 7, per = W >> 3, more = W & 7;
  const uint32_t w = xcd * per + (xcd < more ? xcd : more) + (blockIdx.x >> 3);
  const int64_t all = int64_t(g.batch) * g.tiles * g.steps, begin = int64_t(w) * g.share;
  const int64_t end = begin + g.share < all ? begin + g.share : all;
  for (int64_t at = begin; at < end;) {
    const uint32_t tile = uint32_t(at / g.steps);
    const int32_t k0 = int32_t(at - int64_t(tile) * g.steps);
    const int32_t whole = end - at < g.steps - k0 ? int32_t(end - at) : g.steps - k0;
    __builtin_assume(whole > 0);
    const TileAt<KIND> place(g, tile);
    const int32_t m0 = int32_t(place.m) * TM, n0 = int32_t(place.n) * TN;
    OpA a;
    OpB b;
    a.init(static_cast<const f16*>(g.left) + int64_t(place.matrix) * g.batch_left, g.ld_left, m0, 0, g.M, g.K, tid);
    b.init(static_cast<const f16*>(g.right) + int64_t(place.matrix) * g.batch_right, g.ld_right, n0, 0, g.N, g.K, tid);
    const InPlanes<PLANES, 1> where{k0, g.K / OpA::kInner, g.plane_left * 2, g.plane_right * 2};
    const Finish<KIND, PLANES, Y> finish(g, place);
    const int32_t m = m0 + wm * MT * 16 + (lane & 15), n = n0 + wn * NT * 16 + 8 * (lane >> 4);
    f32x4v acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j) acc[i][j] = f32x4v{0.0f, 0.0f, 0.0f, 0.0f};
    i32x4v fa[2][MT], fb[2][NT];
    multiply_ring<f16, MT, NT, 2>(acc, a, b, ra, rb, fa, fb, lds, wave, whole, where);
    if constexpr (kPinned) mma_done(acc[MT - 1], acc[MT - 2], acc[MT - 3]);
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): the loads to LDS that nobody waits for
    const bool swap = !BK && (lane & 16);
    auto units = [&](auto&& f) {
      unrolled([&](auto index) {
        constexpr int i = decltype(index)::value / kPairs, j = decltype(index)::value % kPairs;
        f32x4v x, y;
        if constexpr (kPinned) {
          x = unpinned(acc[i][2 * j]);
          y = unpinned(acc[i][2 * j + 1]);
        } else {
          x = acc[i][2 * j];
          y = acc[i][2 * j + 1];
        }
        float v[8];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          v[k] = swap ? y[k] : x[k];
          v[4 + k] = swap ? x[k] : y[k];
        }
        f(i, j, v);
        __builtin_amdgcn_sched_barrier(0);
      }, std::make_integer_sequence<int, MT * kPairs>{});
    };
    if (!kSplits || whole == g.steps) {
      // the values there of some units are on their way while others are finished
      constexpr int kUnits = MT * kPairs, kAhead = KIND == kOrthoGram ? 0 : 8;
      typename Finish<KIND, PLANES, Y>::Old old[kAhead + 1];
      auto fetch = [&](int u) { old[u % (kAhead + 1)] = finish.fetch(m + u / kPairs * 16, n + u % kPairs * 32); };
      if constexpr (kAhead > 0) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) fetch(u);
        __builtin_amdgcn_sched_barrier(0);
      }
      units([&](int i, int j, float (&v)[8]) {
        const int u = i * kPairs + j;
        if (kAhead > 0 && u + kAhead < kUnits) fetch(u + kAhead);
        finish(v, old[u % (kAhead + 1)], m + 16 * i, n + 32 * j);
      });
    } else {
      float* const slot = g.parts + (int64_t(w) * 2 + (at != begin)) * (TM * TN);
      units([&](int i, int j, float (&v)[8]) { store_group<8>(part_at(slot, i * kPairs + j, tid), v); });
    }
    at += whole;
    if (at < end) {  // all have read the last tile; the stores are not among the loads that are counted next
      __builtin_amdgcn_s_waitcnt(0x0f70);
      __syncthreads();
    }
  }
}

// The tiles whose steps several workgroups took: one unit of a tile a workgroup,
// the parts summed in the order of the inner length.
template <int KIND, int PLANES, int MT, int NT>
__global__ __launch_bounds__(kThreads) void ortho_join_kernel(OrthoProduct g) {
  using Y = void;  // the last product of all is not split
  constexpr int TM = 2 * MT * 16, TN = 2 * NT * 16, kPairs = NT / 2, kUnits = MT * kPairs;
  const uint32_t tile = blockIdx.x / kUnits;
  const int u = int(blockIdx.x - tile * kUnits), i = u / kPairs, j = u % kPairs;
  const int64_t from = int64_t(tile) * g.steps, to = from + g.steps;
  const int64_t w0 = from / g.share, w1 = (to - 1) / g.share;
  if (w0 == w1) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wm = wave / 2, wn = wave % 2;
  const TileAt<KIND> place(g, tile);
  const Finish<KIND, PLANES, Y> finish(g, place);
  const int32_t m = int32_t(place.m) * TM + wm * MT * 16 + (lane & 15) + 16 * i;
  const int32_t n = int32_t(place.n) * TN + wn * NT * 16 + 8 * (lane >> 4) + 32 * j;
  const auto old = finish.fetch(m, n);
  float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll 4
  for (int64_t w = w0; w <= w1; ++w) {
    // the tile is its workgroup's first, or else its last
    float* const slot = g.parts + (w * 2 + (w * g.share < from)) * (TM * TN);
    float p[8];
    load_group<8>(p, part_at(slot, u, tid));
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] += p[k];
  }
  finish(v, old, m, n);
}

// Tiles of 64 x 64, for products with few of them: the steps are dealt out in turn
// to a workgroup's four waves, each with its own operands in LDS and the whole
// tile's sums in its registers, which meet in LDS in the order of the waves.
constexpr int kSmallShare = ring_bytes(64);  // of LDS, for a wave
// The LDS, all of a compute unit's, is asked for at the launch: a size that the
// compiler knows lets it take 512 registers, in half of which it puts the sums and
// moves them out and back in the loop (one tile of 128 steps 24.2 us, and 17.8
// without).  Hence the bound of two workgroups, which never are there.
template <int KIND, int PLANES, typename Y>
__global__ __launch_bounds__(kThreads, 2) void ortho_small_kernel(OrthoProduct g) {
  constexpr bool BK = KIND != kOrthoApply;
  constexpr int TILE = 64, kPairs = 2, kUnits = 8, kShare = kSmallShare;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  using OpA = Side<Operand<f16, true, false, TILE, 64>, false>;
  using OpB = Side<Operand<f16, BK, true, TILE, 64>, true>;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  Fragments<f16, true, false, TILE> ra;
  Fragments<f16, BK, true, TILE> rb;
  ra.init(0, lane);
  rb.init(0, lane);
  const uint32_t W = gridDim.x, xcd = blockIdx.x & 7, per = W >> 3, more = W & 7;
  const TileAt<KIND> place(g, xcd * per + (xcd < more ? xcd : more) + (blockIdx.x >> 3));
  const int32_t m0 = int32_t(place.m) * TILE, n0 = int32_t(place.n) * TILE;
  OpA a;
  OpB b;
  a.init(static_cast<const f16*>(g.left) + int64_t(place.matrix) * g.batch_left, g.ld_left, m0, 0, g.M, g.K, lane);
  b.init(static_cast<const f16*>(g.right) + int64_t(place.matrix) * g.batch_right, g.ld_right, n0, 0, g.N, g.K, lane);
  const int32_t whole = (g.steps - wave + 3) / 4;
  const InPlanes<PLANES, 4> where{wave, g.K / OpA::kInner, g.plane_left * 2, g.plane_right * 2};
  // a wave finishes two of the tile's units
  const Finish<KIND, PLANES, Y> finish(g, place);
  typename Finish<KIND, PLANES, Y>::Old old[kUnits / 4];
  int32_t m[kUnits / 4], n[kUnits / 4];
#pragma unroll
  for (int q = 0; q < kUnits / 4; ++q) {
    const int u = wave * (kUnits / 4) + q;
    m[q] = m0 + 16 * (u / kPairs) + (lane & 15);
    n[q] = n0 + 32 * (u % kPairs) + 8 * (lane >> 4);
    old[q] = finish.fetch(m[q], n[q]);
  }
  f32x4v acc[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = f32x4v{0.0f, 0.0f, 0.0f, 0.0f};
  char* const own = lds + wave * kShare;
  if (whole > 0) {
    i32x4v fa[2][4], fb[2][4];
    multiply_ring<f16, 4, 4, 2, true>(acc, a, b, ra, rb, fa, fb, own, 0, whole, where);
  }
  wait_own<0>();  // the loads that nobody reads have arrived before anything else is written there
  const bool swap = !BK && (lane & 16);
  auto unit_at = [&](char* share, int u) { return reinterpret_cast<float*>(share) + (u * 64 + lane) * 8; };
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    const f32x4v x = acc[u / kPairs][u % kPairs * 2], y = acc[u / kPairs][u % kPairs * 2 + 1];
    float v[8];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      v[k] = swap ? y[k] : x[k];
      v[4 + k] = swap ? x[k] : y[k];
    }
    store_group<8>(unit_at(own, u), v);
  }
  __syncthreads();
#pragma unroll
  for (int q = 0; q < kUnits / 4; ++q) {
    const int u = wave * (kUnits / 4) + q;
    float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      float p[8];
      load_group<8>(p, unit_at(lds + s * kShare, u));
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] += p[k];
    }
    finish(v, old[q], m[q], n[q]);
  }
}

template <int KIND, int PLANES, typename Y, int MT, int NT>
int launch_product_of(const OrthoProduct& g, hipStream_t st) {
  constexpr bool kSplits = ortho_splits(KIND, PLANES, 32 * MT);
  const bool split = g.share % g.steps != 0;
  if (split && !kSplits) return int(hipErrorInvalidValue);
  ortho_product_kernel<KIND, PLANES, Y, MT, NT><<<dim3(uint32_t(g.workgroups)), dim3(kThreads), 0, st>>>(g);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !split) return int(e);
  if constexpr (kSplits) {
    const uint32_t units = uint32_t(g.batch) * uint32_t(g.tiles) * uint32_t(MT * NT / 2);
    ortho_join_kernel<KIND, PLANES, MT, NT><<<dim3(units), dim3(kThreads), 0, st>>>(g);
  }
  return int(hipGetLastError());
}

template <int KIND, int PLANES, typename Y = void>
int launch_product_kind(const OrthoProduct& g, int32_t tile, hipStream_t st) {
  switch (tile) {
    case 256: return launch_product_of<KIND, PLANES, Y, 8, 8>(g, st);
    case 128: return launch_product_of<KIND, PLANES, Y, 4, 4>(g, st);
    case 64:
      if (g.share != g.steps) return int(hipErrorInvalidValue);
      ortho_small_kernel<KIND, PLANES, Y><<<dim3(uint32_t(g.workgroups)), dim3(kThreads), 4 * kSmallShare, st>>>(g);
      return int(hipGetLastError());
  }
  return int(hipErrorInvalidValue);
}

template <typename F>
int with_type(int32_t elem, F&& f) {
  switch (elem) {
    case kF32: f(float()); break;
    case kF16: f(f16()); break;
    case kBF16: f(bf16()); break;
    default: return int(hipErrorInvalidValue);
  }
  return int(hipGetLastError());
}

dim3 grid64(const OrthoShape& s) { return dim3(uint32_t(s.np / 64), uint32_t(s.mp / 64), uint32_t(s.batch)); }

}  // namespace

int launch_ortho_norm(const OrthoShape& s, const OrthoOuter& x, double* sums, void* stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  return with_type(x.elem, [&](auto t) {
    ortho_norm_kernel<decltype(t)><<<dim3(uint32_t(s.blocks), uint32_t(s.batch)), dim3(kThreads), 0, st>>>(s, x, sums);
  });
}

int launch_ortho_load(const OrthoShape& s, const OrthoOuter& x, const double* sums, double eps, void* planes, void* stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  return with_type(x.elem, [&](auto t) {
    ortho_load_kernel<decltype(t)><<<grid64(s), dim3(kThreads), 0, st>>>(s, x, sums, eps, static_cast<f16*>(planes));
  });
}

int launch_ortho_product(const OrthoProduct& g, int32_t kind, int32_t planes, int32_t tile, void* stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  const bool one = planes == 1;
  if (kind == kOrthoGram) return one ? launch_product_kind<kOrthoGram, 1>(g, tile, st) : launch_product_kind<kOrthoGram, 2>(g, tile, st);
  if (kind == kOrthoSquare) return one ? launch_product_kind<kOrthoSquare, 1>(g, tile, st) : launch_product_kind<kOrthoSquare, 2>(g, tile, st);
  if (kind != kOrthoApply) return int(hipErrorInvalidValue);
  if (!g.y.data) return one ? launch_product_kind<kOrthoApply, 1>(g, tile, st) : launch_product_kind<kOrthoApply, 2>(g, tile, st);
  if (one) return launch_product_kind<kOrthoApply, 1, bf16>(g, tile, st);  // only towards bfloat16
  switch (g.y.elem) {
    case kF32: return launch_product_kind<kOrthoApply, 2, float>(g, tile, st);
    case kF16: return launch_product_kind<kOrthoApply, 2, f16>(g, tile, st);
    case kBF16: return launch_product_kind<kOrthoApply, 2, bf16>(g, tile, st);
  }
  return int(hipErrorInvalidValue);
}

}  // namespace ar
