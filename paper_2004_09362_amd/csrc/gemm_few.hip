// gemm_few.hip -- the linear layer's product for few rows (a token of each of
// some sequences): v[m][n] = sum_k x[m][k] w[n][k], M <= 64.
//
// Bound by reading w once.  A workgroup of eight waves takes 16 NT rows of w
// and deals the inner length out over its waves (and over workgroups, g.splits,
// where N is small); w goes from memory straight to the registers that the
// matrix instructions read, 16 bytes a lane, a batch ahead of the products.  x
// comes from the caches: every lane group reads the rows it multiplies.  The
// waves' sums are added in LDS in the order of the waves, so the result does
// not depend on timing.  Rows may start on any element.
#include "gemm.hpp"

namespace ar {

template <typename T, int MT, int NT>
__global__ __launch_bounds__(512) void gemm_few_kernel(GemmArgs g) {
  constexpr int kWaves = 8, kElems = 16 / int(sizeof(T)), kStep = 4 * kElems, kBatch = MT * NT >= 4 ? 2 : MT * NT == 2 ? 4 : 8;
  __shared__ f32x4v sums[kWaves][MT * NT][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, i = lane & 15, p = lane >> 4;
  const int32_t n0 = int32_t(blockIdx.x) * 16 * NT;
  const int32_t K = g.K, k0 = int32_t(blockIdx.y) * g.k_split;
  const int32_t klen = K - k0 < g.k_split ? K - k0 : g.k_split;
  // whole batches of steps for each wave
  const int32_t steps = (klen + kStep - 1) / kStep;
  const int32_t batches = (steps + kBatch - 1) / kBatch, per = (batches + kWaves - 1) / kWaves;
  const int32_t b0 = wave * per, b1 = b0 + per < batches ? b0 + per : batches;

  const T* xr[MT];
  const T* wr[NT];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const int32_t m = 16 * t + i;
    xr[t] = static_cast<const T*>(g.a) + int64_t(m < g.e.M ? m : g.e.M - 1) * g.lda;
  }
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int32_t n = n0 + 16 * t + i;
    wr[t] = static_cast<const T*>(g.b) + int64_t(n < g.e.N ? n : g.e.N - 1) * g.ldb;
  }
  auto read = [&](const T* row, int32_t batch, int q) {
    const int32_t k = k0 + (batch * kBatch + q) * kStep + p * kElems;
    return load_chunk(row + k, k0 + klen - k);
  };

  f32x4v acc[MT][NT];
#pragma unroll
  for (int a = 0; a < MT; ++a)
#pragma unroll
    for (int b = 0; b < NT; ++b) acc[a][b] = f32x4v{0.0f, 0.0f, 0.0f, 0.0f};
  // a batch of both operands is on its way while one is multiplied
  i32x4v ws[2][NT][kBatch], xs[2][MT][kBatch];
  auto fetch = [&](int set, int32_t batch) {
#pragma unroll
    for (int q = 0; q < kBatch; ++q) {
#pragma unroll
      for (int t = 0; t < NT; ++t) ws[set][t][q] = read(wr[t], batch, q);
#pragma unroll
      for (int t = 0; t < MT; ++t) xs[set][t][q] = read(xr[t], batch, q);
    }
  };
  if (b0 < b1) fetch(0, b0);
  for (int32_t b = b0; b < b1; b += 2) {
#pragma unroll
    for (int set = 0; set < 2; ++set) {
      if (b + set >= b1) break;
      if (b + set + 1 < b1) fetch(1 - set, b + set + 1);
#pragma unroll
      for (int q = 0; q < kBatch; ++q)
#pragma unroll
        for (int a = 0; a < MT; ++a)
#pragma unroll
          for (int t = 0; t < NT; ++t) acc[a][t] = mma<T>(ws[set][t][q], xs[set][a][q], acc[a][t]);
    }
  }

#pragma unroll
  for (int a = 0; a < MT; ++a)
#pragma unroll
    for (int t = 0; t < NT; ++t) sums[wave][a * NT + t][lane] = acc[a][t];
  __syncthreads();
  for (int s = tid; s < MT * NT * 64; s += 512) {
    const int tile = s >> 6, l = s & 63;
    const int32_t m = 16 * (tile / NT) + (l & 15), n = n0 + 16 * (tile % NT) + 4 * (l >> 4);
    if (m >= g.e.M || n >= g.e.N) continue;
    f32x4v v = sums[0][tile][l];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) v += sums[w][tile][l];
    if (g.splits > 1) {
      *reinterpret_cast<f32x4v*>(g.part + (int64_t(blockIdx.y) * g.e.M + m) * g.ldp + n) = v;
    } else if (g.e.N - n < 4) {
#pragma unroll
      for (int c = 0; c < 3; ++c)
        if (n + c < g.e.N) emit_one<T>(v[c], g.e, m, n + c);
    } else {
      float x[4] = {v[0], v[1], v[2], v[3]}, bias[4];
      Residual<4> res[1];
      load_bias<T, 4>(bias, g.e, n);
      load_residuals<T, 4, 1>(res, g.e, m, 1, n);
      emit<T, 4>(x, bias, res[0], g.e, m, n);
    }
  }
}

namespace {

template <typename T, int MT>
int launch_few(const GemmArgs& g, hipStream_t st) {
  // two tiles of 16 columns a workgroup where that still fills the chip
  const bool two = g.e.N >= 16 * 2 * 512;
  const dim3 grid(uint32_t((g.e.N + (two ? 31 : 15)) / (two ? 32 : 16)), uint32_t(g.splits));
  if (two) gemm_few_kernel<T, MT, 2><<<grid, dim3(512), 0, st>>>(g);
  else gemm_few_kernel<T, MT, 1><<<grid, dim3(512), 0, st>>>(g);
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

}  // namespace ar
