// gemm_few.hip -- the linear layer's product for few rows (a token of each of
// some sequences): v[m][n] = sum_k x[m][k] w[n][k], M <= 64.
//
// Bound by reading w once.  A workgroup of 8 or 16 waves takes 16 NW rows of w
// and deals the inner length out over its waves (and over workgroups, g.splits,
// where N is small): one token through 4096 x 4096 bf16 takes 8.0 us, 4.2 TB/s
// with the launch.  w goes from memory straight to the registers that the
// matrix instructions read, 16 bytes a lane, a batch ahead of the products.  x
// comes from the caches: every lane group reads the rows it multiplies.  The
// waves' sums are added in LDS in the order of the waves, so the result does
// not depend on timing.  Rows may start on any element.
#include "gemm.hpp"

namespace ar {

template <typename T, int MT, int NW, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void gemm_few_kernel(GemmArgs g) {
  constexpr int NT = 1, kWaves = WAVES, kGroups = kWaves / NW, kElems = 16 / int(sizeof(T)), kStep = 4 * kElems, kBatch = WAVES == 8 ? 8 : MT >= 4 ? 2 : 4;
  __shared__ f32x4v sums[kGroups][MT * NW][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i = lane & 15, p = lane >> 4;
  const int part = wave / NW, column = wave % NW;  // of the inner length, and of the columns
  const int32_t n0 = int32_t(blockIdx.x) * 16 * NW;
  const int32_t K = g.K, k0 = int32_t(blockIdx.y) * g.k_split;
  const int32_t klen = K - k0 < g.k_split ? K - k0 : g.k_split;
  // batches of steps for each wave; the last of all may reach past the row
  const int32_t batches = (klen + kStep * kBatch - 1) / (kStep * kBatch), full = klen / (kStep * kBatch);
  const int32_t per = (batches + kGroups - 1) / kGroups;
  const int32_t b0 = part * per, b1 = b0 + per < full ? b0 + per : full;

  const T* xr[MT];
  const T* wr[NT];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const int32_t m = 16 * t + i;
    xr[t] = static_cast<const T*>(g.a) + int64_t(m < g.e.M ? m : g.e.M - 1) * g.lda;
  }
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int32_t n = n0 + 16 * (column * NT + t) + i;
    wr[t] = static_cast<const T*>(g.b) + int64_t(n < g.e.N ? n : g.e.N - 1) * g.ldb;
  }
  const int32_t kl = k0 + p * kElems;

  f32x4v acc[MT][NT];
#pragma unroll
  for (int a = 0; a < MT; ++a)
#pragma unroll
    for (int b = 0; b < NT; ++b) acc[a][b] = f32x4v{0.0f, 0.0f, 0.0f, 0.0f};
  // a batch of both operands is on its way while one is multiplied
  i32x4v ws[2][NT][kBatch], xs[2][MT][kBatch];
  auto fetch = [&](int set, int32_t batch) {
    const int32_t k = kl + batch * (kBatch * kStep);
#pragma unroll
    for (int q = 0; q < kBatch; ++q) {
#pragma unroll
      for (int t = 0; t < NT; ++t) ws[set][t][q] = load_whole<T>(wr[t] + k + q * kStep);
#pragma unroll
      for (int t = 0; t < MT; ++t) xs[set][t][q] = load_whole<T>(xr[t] + k + q * kStep);
    }
  };
  auto multiply = [&](int set) {
#pragma unroll
    for (int q = 0; q < kBatch; ++q)
#pragma unroll
      for (int a = 0; a < MT; ++a)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[a][t] = mma<T>(ws[set][t][q], xs[set][a][q], acc[a][t]);
  };
  // Workgroups start at different batches, so that they do not all ask for the
  // same part of every row, which may lie a power of two apart, at a time.
  const int32_t mine = b1 - b0, turn = mine > 0 ? int32_t(blockIdx.x % uint32_t(mine)) : 0;
  auto at = [&](int32_t b) { return b0 + (b + turn < mine ? b + turn : b + turn - mine); };
  if (mine > 0) fetch(0, at(0));
  int32_t b = 0;
  for (; b + 2 < mine; b += 2) {
    fetch(1, at(b + 1));
    multiply(0);
    fetch(0, at(b + 2));
    multiply(1);
  }
  if (b + 1 < mine) fetch(1, at(b + 1));
  if (b < mine) multiply(0);
  if (b + 1 < mine) multiply(1);
  if (batches > full && part == full / per) {  // what is left of the row
#pragma unroll 1
    for (int32_t k = kl + full * (kBatch * kStep); k - p * kElems < k0 + klen; k += kStep) {
      i32x4v w[NT], x[MT];
      const int32_t have = k0 + klen - k;
      if (K >= kElems) {
#pragma unroll
        for (int t = 0; t < NT; ++t) w[t] = load_end(wr[t] + k, have);
#pragma unroll
        for (int t = 0; t < MT; ++t) x[t] = load_end(xr[t] + k, have);
#pragma unroll
        for (int t = 0; t < NT; ++t) w[t] = end_chunk<T>(w[t], have);
#pragma unroll
        for (int t = 0; t < MT; ++t) x[t] = end_chunk<T>(x[t], have);
      } else {
#pragma unroll
        for (int t = 0; t < NT; ++t) w[t] = short_chunk(wr[t] + k, have);
#pragma unroll
        for (int t = 0; t < MT; ++t) x[t] = short_chunk(xr[t] + k, have);
      }
#pragma unroll
      for (int a = 0; a < MT; ++a)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[a][t] = mma<T>(w[t], x[a], acc[a][t]);
    }
  }

#pragma unroll
  for (int a = 0; a < MT; ++a) sums[part][a * NW + column][lane] = acc[a][0];
  __syncthreads();
  for (int s = tid; s < MT * NW * 64; s += kWaves * 64) {
    const int tile = s >> 6, l = s & 63;
    const int32_t m = 16 * (tile / NW) + (l & 15), n = n0 + 16 * (tile % NW) + 4 * (l >> 4);
    if (m >= g.e.M || n >= g.e.N) continue;
    f32x4v v = sums[0][tile][l];
#pragma unroll
    for (int w = 1; w < kGroups; ++w) v += sums[w][tile][l];
    if (g.splits > 1) {
      *reinterpret_cast<f32x4v*>(g.part + (int64_t(blockIdx.y) * g.e.M + m) * g.ldp + n) = v;
    } else if (g.e.N - n < 4) {
      emit_tail<T, 4, 1>([&](int, int c) { return v[c]; }, g.e, m, 1, n, g.e.N - n);
    } else {
      float x[1][4] = {{v[0], v[1], v[2], v[3]}}, bias[4];
      Residual<4> res[1];
      load_bias<T, 4>(bias, g.e, n);
      load_residuals<T, 4, 1>(res, g.e, m, 1, n);
      emit<T, 4, 1>(x, bias, res, g.e, m, 1, n);
    }
  }
}

// Both operands through LDS, for rows on 16-byte boundaries: a workgroup takes
// TM rows and 64 columns, and a ring of tiles (128 bytes of inner length each)
// is on its way asynchronously, up to 144 KB, so that w streams at the rate of
// memory whatever the products wait for.  Every row of x is read once for 64
// columns; in the kernel above, whose waves read it for 16, that traffic out
// of the L2s bounds M > 16.  24 rows through 16384 x 4096 bf16 take 27.8 us, 4.9
// TB/s.
template <typename T, int TM>
__global__ __launch_bounds__(256) void gemm_stream_kernel(GemmArgs g) {
  constexpr int kThreads = 256, kCols = 64, MT = TM / 16;
  using OpA = Operand<T, true, false, TM, kThreads>;
  using OpB = Operand<T, true, false, kCols, kThreads>;
  constexpr int kTile = OpA::kBytes + OpB::kBytes, kRing = 147456 / kTile < 12 ? 147456 / kTile : 12;
  constexpr int kLoads = OpA::kSlots + OpB::kSlots, kInner = OpA::kInner;
  __shared__ __attribute__((aligned(1024))) char lds[kRing * kTile];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int32_t n0 = int32_t(blockIdx.x) * kCols, k0 = int32_t(blockIdx.y) * g.k_split;
  const int32_t klen = g.K - k0 < g.k_split ? g.K - k0 : g.k_split;
  const int32_t tiles = (klen + kInner - 1) / kInner, whole = klen / kInner;
  OpA a;
  OpB b;
  a.init(static_cast<const T*>(g.a), g.lda, 0, k0, g.e.M, g.K, tid);
  b.init(static_cast<const T*>(g.b), g.ldb, n0, k0, g.e.N, g.K, tid);
  Fragments<T, true, false, TM> ra;
  Fragments<T, true, false, kCols> rb;
  ra.init(0, lane);
  rb.init(wave * 16, lane);
  f32x4v acc[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) acc[i] = f32x4v{0.0f, 0.0f, 0.0f, 0.0f};

  const uint32_t lds0 = lds_offset(lds);
  // Workgroups start at different tiles, so that they do not all ask for the
  // same 128 bytes of every row, which may lie a power of two apart, at a time
  // (w of 16384 x 4096 bf16: 27 us against 31), while x stays in the L2s.
  const bool apart = int64_t(g.e.M) * g.K * int64_t(sizeof(T)) <= (int64_t(2) << 20);
  const int32_t turn = apart && whole > 0 ? int32_t((blockIdx.x * 5u + blockIdx.y) % uint32_t(whole)) : 0;
  auto start = [&](int32_t t, uint32_t at) {
    const int32_t k = t + turn < whole ? t + turn : t + turn - whole;
    const char* pa = settled(a.at(k));
    const char* pb = settled(b.at(k));
#pragma unroll
    for (int x = 0; x < kLoads; ++x) {
      if (x < OpB::kSlots) b.aim(x, lds0 + at + OpA::kBytes, wave);
      else a.aim(x - OpB::kSlots, lds0 + at, wave);
      asm volatile("s_nop 0");
      if (x < OpB::kSlots) b.issue(pb, x);
      else a.issue(pa, x - OpB::kSlots);
    }
  };
  auto multiply = [&](uint32_t at) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const i32x4v fb = rb.read(lds + at + OpA::kBytes, 0, s);
#pragma unroll
      for (int i = 0; i < MT; ++i) acc[i] = mma<T>(fb, ra.read(lds + at, i, s), acc[i]);
    }
  };
  auto after = [](uint32_t at) { return at == (kRing - 1) * kTile ? 0 : at + kTile; };
  // tile t lies at place t mod kRing; the one after the ring's last is loaded
  // to where tile t - 1 lay, once every wave has read that
  uint32_t at = 0, free = (kRing - 1) * kTile;
#pragma unroll 1
  for (int32_t t = 0; t < kRing - 1 && t < whole; ++t) start(t, uint32_t(t) * kTile);
  int32_t t = 0;
  for (; t + kRing - 1 < whole; ++t) {
    wait_all<(kRing - 2) * kLoads>();
    start(t + kRing - 1, free);
    multiply(at);
    free = at;
    at = after(at);
  }
  for (; t < tiles; ++t) {
    if (t == whole) {  // the last tile, not whole: through registers, to a place that nothing is read from
      wait_all<0>();
      a.copy(t, klen - int64_t(t) * kInner, lds + at, tid);
      b.copy(t, klen - int64_t(t) * kInner, lds + at + OpA::kBytes, tid);
    }
    wait_all<0>();
    multiply(at);
    at = after(at);
  }

  // lane (i, p): columns 4 p to 4 p + 3 of the wave's 16, row 16 t + i
  const int32_t n = n0 + 16 * wave + 4 * (lane >> 4);
  float bias[4];
  load_bias<T, 4>(bias, g.e, n);
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int32_t m = 16 * i + (lane & 15);
    if (m >= g.e.M || n >= g.e.N) continue;
    if (g.splits > 1) {
      *reinterpret_cast<f32x4v*>(g.part + (int64_t(blockIdx.y) * g.e.M + m) * g.ldp + n) = acc[i];
    } else if (g.e.N - n < 4) {
      emit_tail<T, 4, 1>([&](int, int c) { return acc[i][c]; }, g.e, m, 1, n, g.e.N - n);
    } else {
      float x[1][4] = {{acc[i][0], acc[i][1], acc[i][2], acc[i][3]}};
      Residual<4> res[1];
      load_residuals<T, 4, 1>(res, g.e, m, 1, n);
      emit<T, 4, 1>(x, bias, res, g.e, m, 1, n);
    }
  }
}

namespace {

template <typename T, int MT>
int launch_few(const GemmArgs& g, hipStream_t st) {
  // One, two or four tiles of 16 columns a workgroup, so that two rounds of
  // workgroups become one.  w of 4096 / 6144 / 8192 / 12288 / 16384 / 32768 rows of 1024
  // halves, M = 24, us in a graph: one 5.6 / 9.7 / 9.9 / 14.2 / 18.5 / 35.1, two 7.6 / 7.8 /
  // 7.9 / 14.0 / 14.9 / 27.7, four 12.1 / 12.5 / 12.3 / 12.6 / 13.4 / 24.9; of 512 floats 5.9 /
  // 10.1 / 10.5 / 15.1 / 19.2 / 35.9, 8.0 / 8.2 / 8.5 / 15.0 / 15.6 / 28.9 and 12.7 / 12.9 / 13.1 /
  // 13.2 / 13.4 / 25.3; at 4096 inner indices (6144 columns) one and two are even.
  const int32_t tiles = (g.e.N + 15) / 16, nw = tiles >= 4 * 256 ? 4 : tiles >= 2 * 256 ? 2 : 1;
  const dim3 grid(uint32_t((tiles + nw - 1) / nw), uint32_t(g.splits));
  if constexpr (MT == 1) {
    // up to 8 KB of a row: eight waves that each ask for all of theirs at once.
    // w of 4096 rows of 2 / 4 / 8 / 12 / 16 KB, M = 1, us in a graph: bf16 4.3 / 6.3 /
    // 9.1 / 12.4 / 16.7 and with sixteen 4.6 / 6.3 / 9.8 / 12.5 / 17.1; fp32 4.6 / 6.6 /
    // 10.7 / 13.2 / 17.7 and 4.7 / 6.7 / 10.2 / 12.7 / 17.8; M = 16 within 2%, at 16 KB
    // 21.7 and 22.8.  At 32 KB of bf16 36.8 and 30.7.
    if (nw == 1 && int64_t(g.K) * int64_t(sizeof(T)) <= 8192) {
      gemm_few_kernel<T, 1, 1, 8><<<grid, dim3(512), 0, st>>>(g);
      return int(hipGetLastError());
    }
  }
  if (nw == 4) gemm_few_kernel<T, MT, 4, 16><<<grid, dim3(1024), 0, st>>>(g);
  else if (nw == 2) gemm_few_kernel<T, MT, 2, 16><<<grid, dim3(1024), 0, st>>>(g);
  else gemm_few_kernel<T, MT, 1, 16><<<grid, dim3(1024), 0, st>>>(g);
  return int(hipGetLastError());
}

template <typename T>
int launch_few_of(const GemmArgs& g, hipStream_t st) {
  if (g.e.M <= 16) return launch_few<T, 1>(g, st);
  if (g.e.M <= 32) return launch_few<T, 2>(g, st);
  return launch_few<T, 4>(g, st);
}

}  // namespace

int launch_gemm_few(const GemmArgs& g, int32_t elem, void* stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (g.e.M < 1 || g.e.M > kFewMaxRows) return int(hipErrorInvalidValue);
  switch (elem) {
    case kF32: return launch_few_of<float>(g, st);
    case kF16: return launch_few_of<f16>(g, st);
    case kBF16: return launch_few_of<bf16>(g, st);
  }
  return int(hipErrorInvalidValue);
}

namespace {

template <typename T>
int launch_stream_of(const GemmArgs& g, hipStream_t st) {
  const dim3 grid(uint32_t((g.e.N + 63) / 64), uint32_t(g.splits));
  if (g.e.M <= 32) gemm_stream_kernel<T, 32><<<grid, dim3(256), 0, st>>>(g);
  else gemm_stream_kernel<T, 64><<<grid, dim3(256), 0, st>>>(g);
  return int(hipGetLastError());
}

}  // namespace

int launch_gemm_stream(const GemmArgs& g, int32_t elem, void* stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (g.e.M < 1 || g.e.M > kFewMaxRows) return int(hipErrorInvalidValue);
  switch (elem) {
    case kF32: return launch_stream_of<float>(g, st);
    case kF16: return launch_stream_of<f16>(g, st);
    case kBF16: return launch_stream_of<bf16>(g, st);
  }
  return int(hipErrorInvalidValue);
}

}  // namespace ar
