// rowwise.hip -- the layer operators that read and write each element once:
// dropout, the gradient through an activation and dropout with its column
// sums, and the joins of split products and of sums.
//
// All are bound by memory.  A thread takes 8 consecutive columns of a row (16
// bytes of halves), at any alignment; 8 columns are two counters of the
// generator.
#include "device_common.hpp"
#include "layer_device.hpp"

namespace ar {

namespace {

constexpr int kThreads = 256;

// A thread's group of 8 columns: groups are numbered through the rows, so that
// no thread is left over at the end of a row of any length.  8192 x 8192 fp32 to
// bf16 onto a residual 93 us (5.7 TB/s), 30011 x 4099 fp16 88 us (5.6 TB/s).  A launch takes
// rows from row0 on, with fewer than 2^32 groups.
template <typename X, typename Y>
__global__ __launch_bounds__(kThreads) void dropout_kernel(DropCall c, FastDiv groups, int64_t row0, uint32_t count) {
  const uint32_t id = blockIdx.x * kThreads + threadIdx.x;
  if (id >= count) return;
  const uint32_t down = fdiv(id, groups), col = (id - down * groups.d) * 8;
  const int64_t row = row0 + down;
  const X* const x = static_cast<const X*>(c.x) + row * c.ldx + col;
  const Y* const res = static_cast<const Y*>(c.res) + row * c.ldr + col;
  Y* const y = static_cast<Y*>(c.y) + row * c.ldy + col;
  const int have = c.cols - col < 8 ? int(c.cols - col) : 8;
  float v[8], r[8];
  if (c.cols >= 8) {
    const int back = 8 - have;
    load_group<8>(v, x - back);
    if (c.res) load_group<8>(r, res - back);
    move_down<8>(v, back);
    if (c.drop.on) drop_some<8>(v, c.drop, c.drop.row0 + uint64_t(row), col);
    if (c.res) {
      move_down<8>(r, back);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] += r[i];
    }
    store_most<8>(y, v, back);
  } else {
    load_tail<8>(v, x, have);
    load_tail<8>(r, res, c.res ? have : 0);
    if (c.drop.on) drop_some<8>(v, c.drop, c.drop.row0 + uint64_t(row), col);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += r[i];
    store_tail<8>(y, v, have);
  }
}

// A workgroup takes 256 columns (32 threads of 8) of one chunk of rows, 8
// rows at a time, four of these together so that enough loads are in flight;
// the sums of its 8 row threads meet in LDS in their order.  8192 x 16384 bf16
// through an activation 146 us (5.5 TB/s).
template <typename D, typename Z>
__global__ __launch_bounds__(kThreads) void slope_kernel(SlopeCall c) {
  constexpr int kRows = 4;
  __shared__ float part[8][32][9];
  const int ct = threadIdx.x & 31, rt = threadIdx.x >> 5;
  const int64_t col = (int64_t(blockIdx.x) * 32 + ct) * 8;
  const int have = c.N - col < 8 ? int(c.N - col > 0 ? c.N - col : 0) : 8;
  const int64_t r0 = int64_t(blockIdx.y) * c.rows_per;
  const int64_t r1 = r0 + c.rows_per < c.M ? r0 + c.rows_per : c.M;
  float s[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  const D* const dy = static_cast<const D*>(c.dy) + col;
  const Z* const z = static_cast<const Z*>(c.z) + col;
  Z* const dz = static_cast<Z*>(c.dz) + col;
  if (have > 0 && c.N >= 8) {
    const int back = 8 - have;
    for (int64_t row0 = r0 + rt; row0 < r1; row0 += 8 * kRows) {
      float v[kRows][8], t[kRows][8];
#pragma unroll
      for (int q = 0; q < kRows; ++q)  // of rows past the chunk's last, that one's
        load_group<8>(v[q], dy + (row0 + 8 * q < r1 ? row0 + 8 * q : r1 - 1) * c.lddy - back);
      if (c.z) {
#pragma unroll
        for (int q = 0; q < kRows; ++q)
          load_group<8>(t[q], z + (row0 + 8 * q < r1 ? row0 + 8 * q : r1 - 1) * c.ldz - back);
      }
#pragma unroll
      for (int q = 0; q < kRows; ++q) {
        const int64_t row = row0 + 8 * q;
        if (row >= r1) break;
        move_down<8>(v[q], back);
        if (c.z) move_down<8>(t[q], back);
        if (c.drop.on) drop_some<8>(v[q], c.drop, c.drop.row0 + uint64_t(row), uint32_t(col));
        if (c.z) times_slope<Z, 8>(v[q], t[q], c.act);
#pragma unroll
        for (int i = 0; i < 8; ++i) s[i] += v[q][i];
        if (c.dz) store_group<8>(dz + row * c.lddz, v[q]);  // its rows have whole groups
      }
    }
  } else if (have > 0) {
    for (int64_t row = r0 + rt; row < r1; row += 8) {
      float v[8], t[8];
      load_tail<8>(v, dy + row * c.lddy, have);
      load_tail<8>(t, z + row * c.ldz, c.z ? have : 0);
      if (c.drop.on) drop_some<8>(v, c.drop, c.drop.row0 + uint64_t(row), uint32_t(col));
      if (c.z) times_slope<Z, 8>(v, t, c.act);
#pragma unroll
      for (int i = 0; i < 8; ++i) s[i] += i < have ? v[i] : 0.0f;
      if (c.dz) store_tail<8>(dz + row * c.lddz, v, have);
    }
  }
  if (!c.sums) return;
#pragma unroll
  for (int i = 0; i < 8; ++i) part[rt][ct][i] = s[i];
  __syncthreads();
  const int64_t out = int64_t(blockIdx.x) * 256 + threadIdx.x;
  if (out < c.N) {
    float t = 0.0f;
#pragma unroll
    for (int r = 0; r < 8; ++r) t += part[r][threadIdx.x >> 3][threadIdx.x & 7];
    c.sums[int64_t(blockIdx.y) * c.N + out] = t;
  }
}

// 16 columns a workgroup, 16 threads to each column's chunks.
template <typename T>
__device__ __forceinline__ void column_sums(const SumsCall& c, uint32_t block, float (&part)[16][17]) {
  const int ct = threadIdx.x & 15, rt = threadIdx.x >> 4;
  const int64_t n = int64_t(block) * 16 + ct;
  float s = 0.0f;
  if (n < c.N) {
#pragma unroll 8
    for (int32_t k = rt; k < c.chunks; k += 16) s += c.sums[int64_t(k) * c.ld + n];
  }
  part[rt][ct] = s;
  __syncthreads();
  if (rt == 0 && n < c.N) {
    T* const db = static_cast<T*>(c.db);
    float t = c.accumulate ? float(db[n]) : 0.0f;
#pragma unroll
    for (int r = 0; r < 16; ++r) t += part[r][ct];
    db[n] = T(t);
  }
}

// A thread joins 8 columns of a row, in the order of the parts; groups are
// numbered through the rows.  4 parts of 1024 x 1024 and the sums of 1024 columns
// 5.9 us.
template <typename T>
__device__ __forceinline__ void join(const GemmArgs& g, const FastDiv& groups, uint32_t id) {
  const uint32_t m = fdiv(id, groups), n = (id - m * groups.d) * 8;
  if (m >= uint32_t(g.e.M)) return;
  const float* part = g.part + int64_t(m) * g.ldp + n;
  const int64_t step = int64_t(g.e.M) * g.ldp;
  float w[1][8] = {{0, 0, 0, 0, 0, 0, 0, 0}}, bias[8];
  float(&v)[8] = w[0];
  Residual<8> res[1];
  const int have = g.e.N - int32_t(n), back = have < 8 ? 8 - have : 0;
  load_bias<T, 8>(bias, g.e, int32_t(n), back);
  if (g.e.N >= 8) load_residuals<T, 8, 1>(res, g.e, int32_t(m), 1, int32_t(n) - back);
#pragma unroll 4
  for (int32_t s = 0; s < g.splits; ++s) {
    const float4* p = reinterpret_cast<const float4*>(part + s * step);
    const float4 a = p[0], b = p[1];
    v[0] += a.x; v[1] += a.y; v[2] += a.z; v[3] += a.w;
    v[4] += b.x; v[5] += b.y; v[6] += b.z; v[7] += b.w;
  }
  // ldp is a multiple of 8: whole groups lie there
  if (g.e.N >= 8) emit<T, 8, 1>(w, bias, res, g.e, int32_t(m), 1, int32_t(n), back);
  else emit_tail<T, 8, 1>([&](int, int i) { return v[i]; }, g.e, int32_t(m), 1, int32_t(n), have);
}

// Workgroups: those of g, of h, and of the column sums.
template <typename T>
__global__ __launch_bounds__(kThreads) void gemm_join_kernel(GemmArgs g, GemmArgs h, FastDiv gdiv, FastDiv hdiv,
                                                             uint32_t gblocks, uint32_t hblocks, SumsCall c) {
  __shared__ float part[16][17];
  if (blockIdx.x < gblocks) {
    join<T>(g, gdiv, blockIdx.x * kThreads + threadIdx.x);
  } else if (blockIdx.x < gblocks + hblocks) {
    join<T>(h, hdiv, (blockIdx.x - gblocks) * kThreads + threadIdx.x);
  } else {
    const uint32_t block = blockIdx.x - gblocks - hblocks;
    if (c.elem == kF32) column_sums<float>(c, block, part);
    else if (c.elem == kF16) column_sums<f16>(c, block, part);
    else column_sums<bf16>(c, block, part);
  }
}

template <typename X>
int launch_dropout_x(const DropCall& c, int32_t ye, hipStream_t st) {
  const int64_t groups = (c.cols + 7) / 8, most = (int64_t(1) << 31) / groups;  // groups <= 2^27
  const FastDiv div = make_fastdiv(uint32_t(groups));
  for (int64_t row0 = 0; row0 < c.rows; row0 += most) {
    const int64_t rows = c.rows - row0 < most ? c.rows - row0 : most;
    const uint32_t count = uint32_t(rows * groups);
    const dim3 grid((count + kThreads - 1) / kThreads);
    switch (ye) {
      case kF32: dropout_kernel<X, float><<<grid, dim3(kThreads), 0, st>>>(c, div, row0, count); break;
      case kF16: dropout_kernel<X, f16><<<grid, dim3(kThreads), 0, st>>>(c, div, row0, count); break;
      case kBF16: dropout_kernel<X, bf16><<<grid, dim3(kThreads), 0, st>>>(c, div, row0, count); break;
      default: return int(hipErrorInvalidValue);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return int(e);
  }
  return int(hipSuccess);
}

template <typename Z>
int launch_slope_z(const SlopeCall& c, int32_t dye, hipStream_t st) {
  const dim3 grid(uint32_t((c.N + 255) / 256), uint32_t(c.chunks));
  if (dye == elem_of<Z>()) slope_kernel<Z, Z><<<grid, dim3(kThreads), 0, st>>>(c);
  else if (dye == kF32) slope_kernel<float, Z><<<grid, dim3(kThreads), 0, st>>>(c);
  else return int(hipErrorInvalidValue);
  return int(hipGetLastError());
}

}  // namespace

int launch_dropout(const DropCall& c, int32_t xe, int32_t ye, void* stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  switch (xe) {
    case kF32: return launch_dropout_x<float>(c, ye, st);
    case kF16: return launch_dropout_x<f16>(c, ye, st);
    case kBF16: return launch_dropout_x<bf16>(c, ye, st);
  }
  return int(hipErrorInvalidValue);
}

int launch_slope(const SlopeCall& c, int32_t dye, int32_t ze, void* stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  switch (ze) {
    case kF32: return launch_slope_z<float>(c, dye, st);
    case kF16: return launch_slope_z<f16>(c, dye, st);
    case kBF16: return launch_slope_z<bf16>(c, dye, st);
  }
  return int(hipErrorInvalidValue);
}

int launch_join(const GemmArgs& g, const GemmArgs& h, const SumsCall& c, int32_t elem, void* stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  FastDiv div[2];
  uint32_t blocks[2];
  const GemmArgs* const both[2] = {&g, &h};
  for (int i = 0; i < 2; ++i) {
    const int64_t groups = (int64_t(both[i]->e.N) + 7) / 8, threads = both[i]->splits > 1 ? groups * both[i]->e.M : 0;
    if (threads > (int64_t(1) << 30)) return int(hipErrorInvalidValue);  // products this large are not split
    div[i] = make_fastdiv(uint32_t(groups > 0 ? groups : 1));
    blocks[i] = uint32_t((threads + kThreads - 1) / kThreads);
  }
  // a launch takes so many columns that it has fewer than 2^32 threads
  constexpr int64_t kMost = int64_t(1) << 26;
  const int64_t size = c.elem == kF32 ? 4 : 2;
  SumsCall s = c;
  for (int64_t n0 = 0; n0 == 0 || n0 < c.N; n0 += kMost, blocks[0] = blocks[1] = 0) {
    if (c.sums) {
      s.sums = c.sums + n0;
      s.db = static_cast<char*>(c.db) + n0 * size;
      s.N = c.N - n0 < kMost ? c.N - n0 : kMost;
    }
    const uint32_t all = blocks[0] + blocks[1] + (c.sums ? uint32_t((s.N + 15) / 16) : 0);
    if (all == 0) return int(hipSuccess);
    const dim3 grid(all), block(kThreads);
    switch (elem) {
      case kF32: gemm_join_kernel<float><<<grid, block, 0, st>>>(g, h, div[0], div[1], blocks[0], blocks[1], s); break;
      case kF16: gemm_join_kernel<f16><<<grid, block, 0, st>>>(g, h, div[0], div[1], blocks[0], blocks[1], s); break;
      case kBF16: gemm_join_kernel<bf16><<<grid, block, 0, st>>>(g, h, div[0], div[1], blocks[0], blocks[1], s); break;
      default: return int(hipErrorInvalidValue);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return int(e);
  }
  return int(hipSuccess);
}

}  // namespace ar
