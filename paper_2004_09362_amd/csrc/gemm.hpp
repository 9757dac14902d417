// gemm.hpp -- the tiled matrix product of the linear layer and its gradient,
// with the epilogue in its registers.  Instantiated per element type in
// gemm_f32.hip, gemm_f16.hip and gemm_bf16.hip.
//
// v[m][n] = sum_k a(m, k) b(n, k), sums in 32 bits.  A workgroup of WM x WN
// waves computes a tile of TM x TN, each wave (16 MT) x (16 NT) of it in
// 16 x 16 matrix instructions.  The instructions take b's rows as their first
// operand and a's as their second, so that a lane's sums are consecutive
// columns n of one row m and leave in 16-byte pieces.
//
// Bound by the matrix units on large products: a 256 x 256 tile (a wave: 128 x
// 128, whose 256 sums a lane fill half of the register file) reads 64 KB of LDS'
// 128 bytes a cycle for 1024 cycles of products each step.  Measured, bf16:
// 8192 x 16384 x 4096 785 us (1400 TFLOP/s), its input gradient 751 us, 4096^3
// 94 us; a step of one tile 0.96 us, 0.43 us of it the products' own at full
// clock, and up to 1.4 us where the chip lowers its clock for its power.
// Around a tile's steps lie 4000 cycles until its first loads are there, and
// the epilogue, which nothing hides: one tile takes a compute unit's LDS.
// Smaller products take 128 x 128 tiles, two to a unit, which hide each other's
// but read LDS twice as much for each product.  fp32: 2048 x 4096 x 1024 124 us
// (138 TFLOP/s; the unit's rate is 157).
//
// Inner lengths of 128 bytes at a time (a tile: 64 halves or 32 floats) are
// staged in LDS, every operand in the order that it has in memory:
//   k-major:  one row m (or n) is 128 bytes, 8 chunks of 16; a fragment is one
//             16-byte read (8 halves for one 16x16x32 instruction, 4 floats
//             for four 16x16x4);
//   otherwise one inner index k is a row of TM (or TN) elements; a fragment of
//             halves is two transposing 8-byte reads, one of floats four
//             4-byte reads.
// Both orders give lane group g = lane / 16 the same inner indices (8 g to
// 8 g + 7, or 4 g to 4 g + 3, of a 64-byte slice), so they can be mixed.
// Chunks lie at a position XORed with a function of their row (Operand::swz),
// which spreads a fragment read's lanes over all banks.
//
// Columns of the wave are dealt to instructions so that tiles 2j and 2j + 1
// together give a lane 8 consecutive ones: row 4 p + r of tile t is column
// 32 (t / 2) + 8 p + 4 (t % 2) + r of the wave where b is k-major, and
// 32 (t / 2) + 8 p + 4 ((t + p) % 2) + r otherwise (there the four 8-byte
// pieces that a row of the transposing read takes, and its four rows, then
// fall on different banks; odd lane groups swap the two tiles' sums).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>
#include <utility>

#include "layer_device.hpp"

namespace ar {

typedef float f32x4v __attribute__((ext_vector_type(4)));
typedef int32_t i32x4v __attribute__((ext_vector_type(4)));
typedef short s16x4v __attribute__((ext_vector_type(4)));
typedef short s16x8v __attribute__((ext_vector_type(8)));
typedef f16 f16x8v __attribute__((ext_vector_type(8)));
typedef bf16 bf16x8v __attribute__((ext_vector_type(8)));

// One 64-byte slice of inner length of a 16 x 16 product; the operands are
// the lanes' 16 bytes.
template <typename T>
__device__ __forceinline__ f32x4v mma(const i32x4v& rows_n, const i32x4v& rows_m, f32x4v acc) {
  if constexpr (elem_of<T>() == kBF16) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8v, rows_n),
                                                   __builtin_bit_cast(bf16x8v, rows_m), acc, 0, 0, 0);
  } else if constexpr (elem_of<T>() == kF16) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8v, rows_n),
                                                  __builtin_bit_cast(f16x8v, rows_m), acc, 0, 0, 0);
  } else {
    const f32x4v n4 = __builtin_bit_cast(f32x4v, rows_n), m4 = __builtin_bit_cast(f32x4v, rows_m);
#pragma unroll
    for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(n4[e], m4[e], acc, 0, 0, 0);
    return acc;
  }
}

// The same in place, with the sums pinned to accumulation registers: for the
// wave tile whose 256 sums fill them.  Left to itself the compiler moves such
// sums between the two halves of the register file in the loop.  It does not
// know these to be matrix instructions, so the wait states that it would
// insert are the caller's: mma_ready() after ordinary instructions may have
// written an operand (in the loops none does: fragments come from LDS, and
// tests/test_gemm_code.py looks at what was compiled), mma_done() before the
// sums are read.
template <typename T>
__device__ __forceinline__ void mma_pinned(const i32x4v& rows_n, const i32x4v& rows_m, f32x4v& acc) {
  if constexpr (elem_of<T>() == kBF16) {
    asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(acc) : "v"(rows_n), "v"(rows_m));
  } else {
    static_assert(elem_of<T>() == kF16, "floats take tiles whose sums are not pinned");
    asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+a"(acc) : "v"(rows_n), "v"(rows_m));
  }
}
__device__ __forceinline__ void mma_ready() { asm volatile("s_nop 1"); }
// For the sums of the last three rows of products: those that may still be on
// their way, and some more.
__device__ __forceinline__ void mma_done(f32x4v (&a)[8], f32x4v (&b)[8], f32x4v (&c)[8]) {
  asm volatile("s_nop 15\n\ts_nop 15"
               : "+a"(a[0]), "+a"(a[1]), "+a"(a[2]), "+a"(a[3]), "+a"(a[4]), "+a"(a[5]), "+a"(a[6]), "+a"(a[7])::"memory");
  asm volatile("" : "+a"(b[0]), "+a"(b[1]), "+a"(b[2]), "+a"(b[3]), "+a"(b[4]), "+a"(b[5]), "+a"(b[6]), "+a"(b[7]));
  asm volatile("" : "+a"(c[0]), "+a"(c[1]), "+a"(c[2]), "+a"(c[3]), "+a"(c[4]), "+a"(c[5]), "+a"(c[6]), "+a"(c[7]));
}

// Pinned sums, moved to ordinary registers here and not before: the compiler
// would move all 256 at the loop's end, most of them on to memory.
__device__ __forceinline__ f32x4v unpinned(const f32x4v& a) {
  f32x4v v;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float x;
    asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(x) : "a"(a[e]));
    v[e] = x;
  }
  return v;
}

// 16 bytes that start on any element.
template <typename T>
__device__ __forceinline__ i32x4v load_whole(const void* p) {
  typedef T U __attribute__((ext_vector_type(16 / int(sizeof(T))), aligned(sizeof(T))));
  typedef T W __attribute__((ext_vector_type(16 / int(sizeof(T)))));
  return __builtin_bit_cast(i32x4v, W(*static_cast<const U*>(p)));
}

// 16 bytes of a row that has 16 at least, elements past `have` zero (have may be
// negative: p lies behind the row's end): the row's last 16 bytes are loaded
// (load_end), without a branch, so that the loads of several chunks go out
// together, and then shifted (end_chunk).
template <typename T>
__host__ __device__ __forceinline__ const T* end_at(const T* p, int64_t have) {
  constexpr int V = 16 / int(sizeof(T));
  return p + ((have < V ? int(have) : V) - V);
}
template <typename T>
__device__ __forceinline__ i32x4v load_end(const T* p, int64_t have) {
  return load_whole<T>(end_at(p, have));
}
template <typename T>
__device__ __forceinline__ i32x4v end_chunk(const i32x4v& raw, int64_t have) {
  constexpr int V = 16 / int(sizeof(T));
  const int h = have < V ? int(have) : V;
  typedef uint64_t L __attribute__((ext_vector_type(2)));
  const L x = __builtin_bit_cast(L, raw);
  const int bits = h > 0 ? (V - h) * 8 * int(sizeof(T)) : 128;  // to drop
  const uint64_t lo = bits >= 64 ? x[1] >> (bits & 63) : bits ? x[0] >> bits | x[1] << (64 - bits) : x[0];
  const L y = {bits >= 128 ? 0 : lo, bits >= 64 ? 0 : x[1] >> bits};
  return __builtin_bit_cast(i32x4v, y);
}
// The same element by element, of a shorter row.
template <typename T>
__device__ __forceinline__ i32x4v short_chunk(const T* p, int64_t have) {
  constexpr int V = 16 / int(sizeof(T));
  const int h = have < V ? int(have) : V;
  typedef T W __attribute__((ext_vector_type(V)));
  W w;
#pragma unroll
  for (int i = 0; i < V; ++i) w[i] = i < h ? p[i] : T(0);
  return __builtin_bit_cast(i32x4v, w);
}

// f(0), f(1), ... f(N - 1) with the index a constant in each.
template <typename F, int... I>
__device__ __forceinline__ void unrolled(F&& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}

__device__ __forceinline__ uint32_t lds_offset(const char* p) {
  return uint32_t(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const char*)p));
}

// 64 lanes' 16 bytes from base + voff to 1024 consecutive bytes of LDS, past
// the registers.  The compiler's own form of this instruction makes every
// later LDS read wait for it; here the caller waits (wait_all), one tile
// later.  It has no register outputs, and nothing else here uses m0.  base must
// be settled().
// lds_target() names the place, one instruction at least before.
__device__ __forceinline__ void lds_target(uint32_t lds) { asm volatile("s_mov_b32 m0, %0" ::"s"(lds)); }
__device__ __forceinline__ void load_to_lds(const char* base, uint32_t voff) {
  asm volatile("global_load_lds_dwordx4 %0, %1" ::"v"(voff), "s"(base));
}

// All but the last LOADS of this wave's loads have arrived, its LDS reads and
// writes are done, and so it is with the workgroup's other waves.
template <int LOADS>
__device__ __forceinline__ void wait_all() {
  static_assert(LOADS < 64, "the counter's range");
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((LOADS & 15) | ((LOADS >> 4) << 14) | 0x70);  // vmcnt(LOADS) lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// The same of this wave alone.
template <int LOADS>
__device__ __forceinline__ void wait_own() {
  static_assert(LOADS < 64, "the counter's range");
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((LOADS & 15) | ((LOADS >> 4) << 14) | 0x70);  // vmcnt(LOADS) lgkmcnt(0)
  asm volatile("" ::: "memory");
}

// The workgroup's LDS writes are done; loads into registers may be on their way.
__device__ __forceinline__ void meet() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// An address that is the same for all lanes, in scalar registers that a load to
// LDS may read: five wait states after a vector instruction wrote them, which
// the compiler does not know to insert before the assembly that reads them.
__device__ __forceinline__ const char* settled(const char* p) {
  const uint64_t v = reinterpret_cast<uint64_t>(p);
  uint32_t lo = __builtin_amdgcn_readfirstlane(uint32_t(v)), hi = __builtin_amdgcn_readfirstlane(uint32_t(v >> 32));
  asm volatile("s_nop 4" : "+s"(lo), "+s"(hi));
  return reinterpret_cast<const char*>(uint64_t(hi) << 32 | lo);
}

// An operand's tile: R rows of the output, 128 bytes of inner length each.
// FIRST: the operand b, whose rows are dealt to instructions as above.
template <typename T, bool KMAJOR, bool FIRST, int R, int THREADS>
struct Operand {
  static constexpr int kElems = 16 / int(sizeof(T));          // elements of a chunk
  static constexpr int kInner = kTileKBytes / int(sizeof(T));  // inner indices of a tile
  static constexpr int kChunks = R * 8;
  static constexpr int kSlots = kChunks / THREADS;
  static constexpr int kRowChunks = KMAJOR ? 8 : R / kElems;   // chunks of a row of the tile
  static constexpr int kRowBytes = 16 * kRowChunks;
  static constexpr int kSlotRows = THREADS / kRowChunks;       // tile rows between a thread's slots
  static constexpr int kBytes = R * kTileKBytes;
  static_assert(kSlots * THREADS == kChunks && kSlotRows * kRowChunks == THREADS, "whole slots");

  // Chunk c of tile row r lies at position c ^ swz(r).
  __host__ __device__ static __forceinline__ int swz(int r) {
    if constexpr (KMAJOR) return FIRST ? (r & 3) | ((r >> 1) & 4) : r & 7;
    else if constexpr (sizeof(T) == 2) return FIRST ? ((r & 1) << 2) | ((r >> 1) & 1) : (r & 3) << 1;
    else return FIRST ? ((r >> 2) & 1) | (r & 8) : (r & 12);
  }

  const char* base;   // element (first row, first inner index of the split)
  int64_t ld;         // bytes between rows of the matrix
  int32_t rows;       // rows of the output left from the tile's first one
  bool wide;          // whether the matrix' rows have 16 bytes
  uint32_t voff[kSlots];

  // Byte offsets of this thread's chunks from the tile's first element.  A
  // chunk of rows past the last is read from the last (k-major) or the first
  // (otherwise): its products land in sums that are never stored.
  __host__ __device__ __forceinline__ void init(const T* p, int64_t ld_elems, int64_t row0, int64_t k0, int64_t nrows, int64_t inner, int tid) {
    ld = ld_elems * int64_t(sizeof(T));
    rows = int32_t(nrows - row0 < R ? nrows - row0 : R);
    wide = (KMAJOR ? inner : nrows) >= kElems;
    base = reinterpret_cast<const char*>(p) +
           (KMAJOR ? row0 * ld + k0 * int64_t(sizeof(T)) : k0 * ld + row0 * int64_t(sizeof(T)));
#pragma unroll
    for (int i = 0; i < kSlots; ++i) {
      const int s = i * THREADS + tid, r = s / kRowChunks, c = (s % kRowChunks) ^ swz(r);
      if constexpr (KMAJOR) voff[i] = uint32_t(r < rows ? r : rows - 1) * uint32_t(ld) + uint32_t(c * 16);
      else voff[i] = uint32_t(r) * uint32_t(ld) + uint32_t(c * kElems < rows ? c * 16 : 0);
    }
  }

  // Bytes from an inner tile to the next.
  __host__ __device__ __forceinline__ int64_t step() const { return KMAJOR ? int64_t(kTileKBytes) : kInner * ld; }
  // The start of inner tile t.
  __host__ __device__ __forceinline__ const char* at(int32_t t) const {
    return base + t * step();
  }

  // The asynchronous load of this thread's chunk i of a whole tile (p: its
  // start) into LDS: its target, and then the load itself.
  __device__ __forceinline__ void aim(int i, uint32_t lds, int wave) const {
    lds_target(lds + uint32_t(i * THREADS + wave * 64) * 16);
  }
  __device__ __forceinline__ void issue(const char* p, int i) const { load_to_lds(p, voff[i]); }

  // A tile into registers.  One that is not the last, of an operand that is
  // open (tiles_open in layers.hpp), is loaded without a check, so that the loads
  // go out together: what it takes from behind a row's end are elements of the
  // matrix' next rows, or lie between rows, and land in sums that are never stored.
  __host__ __device__ __forceinline__ void load(i32x4v (&reg)[kSlots], int32_t t) const {
    const char* p = at(t);
#pragma unroll
    for (int i = 0; i < kSlots; ++i) reg[i] = load_whole<T>(p + voff[i]);
  }
  // Tile t, of which k_have inner indices exist.  Rows past the last one
  // (k-major): that one's, whose products are never stored; inner indices past
  // the last one (otherwise): zeros.
  __host__ __device__ __forceinline__ void load_checked(i32x4v (&reg)[kSlots], int32_t t, int64_t k_have, int tid) const {
    const T* p[kSlots];
    int64_t have[kSlots];
#pragma unroll
    for (int i = 0; i < kSlots; ++i) {
      const int s = i * THREADS + tid, r = s / kRowChunks, c = (s % kRowChunks) ^ swz(r);
      const bool there = KMAJOR || r < k_have;
      const int64_t row = KMAJOR ? (r < rows ? r : rows - 1) : (there ? r : 0);
      p[i] = reinterpret_cast<const T*>(at(t) + row * ld + c * 16);
      have[i] = KMAJOR ? k_have - c * kElems : rows - c * kElems;
      if (!there && have[i] > 0) {  // a chunk of the tile's first row is loaded and dropped whole
        p[i] += have[i];
        have[i] = 0;
      }
    }
    if (wide) {
#pragma unroll
      for (int i = 0; i < kSlots; ++i) reg[i] = load_end(p[i], have[i]);
#pragma unroll
      for (int i = 0; i < kSlots; ++i) reg[i] = end_chunk<T>(reg[i], have[i]);
    } else {
#pragma unroll
      for (int i = 0; i < kSlots; ++i) reg[i] = short_chunk(p[i], have[i]);
    }
  }
  __device__ __forceinline__ void store(const i32x4v (&reg)[kSlots], char* lds, int tid) const {
#pragma unroll
    for (int i = 0; i < kSlots; ++i) *reinterpret_cast<i32x4v*>(lds + (i * THREADS + tid) * 16) = reg[i];
  }
  // A tile, of which something exists, into LDS.
  __device__ __forceinline__ void copy(int32_t t, int64_t k_have, char* lds, int tid) const {
    i32x4v reg[kSlots];
    load_checked(reg, t, k_have, tid);
    store(reg, lds, tid);
  }
};

// Reads of a wave's fragments from an operand's tile in LDS.
template <typename T, bool KMAJOR, bool FIRST, int R>
struct Fragments {
  static constexpr int kRowBytes = KMAJOR ? kTileKBytes : R * int(sizeof(T));
  uint32_t off[4];

  // w0: the wave's first row in the tile, a multiple of 16 where the operand is
  // k-major and of 64 otherwise (its chunks' places repeat after 64 rows).
  __device__ __forceinline__ void init(int w0, int lane) {
    const int i = lane & 15, g = lane >> 4;
    using Op = Operand<T, KMAJOR, FIRST, R, R>;
    if constexpr (KMAJOR) {
      const int row = w0 + (FIRST ? 8 * (i >> 2) + (i & 3) : i);  // of tile t = 0; the others keep swz
      off[0] = uint32_t(row * kTileKBytes + ((g ^ Op::swz(row)) * 16));
      off[1] = off[0] ^ 64;
    } else if constexpr (sizeof(T) == 2) {
      const int k = 8 * g + (i >> 2);  // and k + 4: the same swz
      const int p = i & 3;             // the 8-byte piece that this lane fetches
#pragma unroll
      for (int odd = 0; odd < 2; ++odd) {
        const int col = w0 + (FIRST ? 8 * p + 4 * ((odd ^ p) & 1) : 16 * odd + 4 * p);
        const int c = col / 8;
        off[odd] = uint32_t(k * kRowBytes + ((c ^ Op::swz(k)) * 16) + (col % 8) * 2);
      }
    } else {
      const int p = i >> 2;
#pragma unroll
      for (int odd = 0; odd < 2; ++odd) {
        const int col = w0 + (FIRST ? 8 * p + 4 * ((odd ^ p) & 1) : 16 * odd + 4 * p) + (i & 3);
        const int c = col / 4;
        const int k = 4 * g;  // to 4 g + 3: the same swz; slice 1 is 16 rows further
        off[odd] = uint32_t(k * kRowBytes + ((c ^ Op::swz(k)) * 16) + (col % 4) * 4);
      }
    }
  }

  // The fragment of tile t (16 rows of the wave), slice s.
  __device__ __forceinline__ i32x4v read(const char* lds, int t, int s) const {
    if constexpr (KMAJOR) {
      const int row = FIRST ? 32 * (t >> 1) + 4 * (t & 1) : 16 * t;
      return *reinterpret_cast<const i32x4v*>(lds + off[s] + row * kTileKBytes);
    } else if constexpr (sizeof(T) == 2) {
      // tiles 2j and 2j + 1 take 32 rows: 64 bytes = 4 chunks of a tile row;
      // the XOR of swz stays within 8 chunks (see off), so whole groups of 8
      // chunks are added and the lower bit of j is XORed in
      const int j = t >> 1;
      const char* p = lds + ((off[t & 1] ^ uint32_t((j & 1) * 64)) + uint32_t((j >> 1) * 128 + s * 32 * kRowBytes));
      typedef __attribute__((address_space(3))) s16x4v Lds4;
      const s16x4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds4*)p);
      const s16x4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds4*)(p + 4 * kRowBytes));
      return __builtin_bit_cast(i32x4v, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
      // 32 rows are 128 bytes: 8 chunks; the XOR stays within 16
      const int j = t >> 1;
      const char* p = lds + ((off[t & 1] ^ uint32_t((j & 1) * 128)) + uint32_t((j >> 1) * 256 + s * 16 * kRowBytes));
      i32x4v v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = *reinterpret_cast<const int32_t*>(p + e * kRowBytes);
      return v;
    }
  }
};

// Order of the tiles: each XCD (workgroups go round the eight) takes a
// contiguous share of a list that walks the columns in groups of 8 rows of
// tiles, so that its L2 serves the operands that its tiles share.
__device__ __forceinline__ void tile_of(uint32_t id, uint32_t tm, uint32_t tn, uint32_t& m, uint32_t& n) {
  const uint32_t total = tm * tn, x = id & 7, per = total >> 3, more = total & 7;
  const uint32_t t = x * per + (x < more ? x : more) + (id >> 3);
  constexpr uint32_t G = 8;
  const uint32_t group = t / (G * tn), first = group * G;
  const uint32_t h = tm - first < G ? tm - first : G, in = t - group * G * tn;
  m = first + in % h;
  n = in / h;
}

// The epilogue of a whole tile from a wave's registers: this lane's sums, the
// first of which are those of row m, column n.  swap: the sums of tiles 2j and
// 2j + 1 lie the other way round (SWAPS: in some lane).  BIAS: there may be one.
template <typename T, int MT, int NT, bool BIAS, bool SWAPS>
__device__ __forceinline__ void direct(const GemmArgs& g, f32x4v (&acc)[MT][NT], bool swap, int32_t m, int32_t n, uint32_t part_of) {
  constexpr int kPairs = NT / 2, kUnits = MT * kPairs, kAhead = 4;
  const Epilogue& e = g.e;
  float b[kPairs][8];  // zeros without a bias, and where parts of a product are joined later
  if constexpr (BIAS) {
#pragma unroll
    for (int j = 0; j < kPairs; ++j) {
      if (g.splits > 1) {
#pragma unroll
        for (int k = 0; k < 8; ++k) b[j][k] = 0.0f;
      } else {
        load_bias<T, 8>(b[j], e, n + 32 * j);
      }
    }
  }
  auto biased = [&](float (&v)[8], int j) {
    if constexpr (BIAS) {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] += b[j][k];
    }
  };
  auto sum = [](const f32x4v& a) {
    if constexpr (MT * NT == 64) return unpinned(a);
    else return a;
  };
  // Of a lane whose sums lie the other way round what is read and written is
  // exchanged, not the sums: the compiler would do that for all of them at once,
  // beyond the registers.
  typedef uint32_t U4 __attribute__((ext_vector_type(4)));
  auto swapped = [&](U4 w) { return SWAPS && swap ? U4{w[2], w[3], w[0], w[1]} : w; };
  auto swap_halves = [&](U4& a, U4& b) {
    const U4 c = a;
    if (SWAPS) a = swap ? b : a;
    if (SWAPS) b = swap ? c : b;
  };
  auto store = [&](auto* to, const float (&v)[8]) {
    using Y = std::remove_pointer_t<decltype(to)>;
    if constexpr (sizeof(Y) == 4) {
      const int other = SWAPS && swap ? 4 : 0;
      store_group<4>(to + other, {v[0], v[1], v[2], v[3]});
      store_group<4>(to + (4 - other), {v[4], v[5], v[6], v[7]});
    } else {
      typedef Y H __attribute__((ext_vector_type(8)));
      typedef U4 Any __attribute__((aligned(2)));
      *reinterpret_cast<Any*>(to) = swapped(__builtin_bit_cast(U4, H{Y(v[0]), Y(v[1]), Y(v[2]), Y(v[3]), Y(v[4]), Y(v[5]), Y(v[6]), Y(v[7])}));
    }
  };
  // f(row, pair, values) for each unit of 8 columns
  auto units = [&](auto&& f) {
    unrolled([&](auto index) {
      constexpr int i = decltype(index)::value / kPairs, j = decltype(index)::value % kPairs;
      const f32x4v x = sum(acc[i][2 * j]), y = sum(acc[i][2 * j + 1]);
      float v[8] = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
      f(i, j, v);
      __builtin_amdgcn_sched_barrier(0);
    }, std::make_integer_sequence<int, kUnits>{});
  };
  auto write = [&](auto* to, int64_t ld) {
    to += int64_t(m) * ld + n;
    units([&](int i, int j, float (&v)[8]) {
      biased(v, j);
      store(to + i * (16 * ld) + 32 * j, v);
    });
  };
  __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): the loads to LDS that nobody waits for
  if (g.splits > 1) {
    write(g.part + int64_t(part_of) * e.M * g.ldp, g.ldp);
    return;
  }
  if (e.res) {
    Residual<8> res[2][kAhead];  // of this group of units and of the next
    auto fetch = [&](auto index) {
      constexpr int x = decltype(index)::value;
#pragma unroll
      for (int q = 0; q < kAhead; ++q) {
        Residual<8> r[1];
        load_residuals<T, 8, 1>(r, e, m + (x * kAhead + q) / kPairs * 16, 0, n + (x * kAhead + q) % kPairs * 32);
        res[x & 1][q] = r[0];
      }
      __builtin_amdgcn_sched_barrier(0);
    };
    static_assert(kUnits % kAhead == 0, "whole groups");
    fetch(std::integral_constant<int, 0>{});
    auto finish = [&](auto* to) {
      to += int64_t(m) * e.ldy + n;
      unrolled([&](auto index) {
        constexpr int x = decltype(index)::value;
        if constexpr ((x + 1) * kAhead < kUnits) fetch(std::integral_constant<int, x + 1>{});
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
          const int i = (x * kAhead + q) / kPairs, j = (x * kAhead + q) % kPairs;
          const f32x4v c = sum(acc[i][2 * j]), d = sum(acc[i][2 * j + 1]);
          float v[1][8] = {{c[0], c[1], c[2], c[3], d[0], d[1], d[2], d[3]}};
          biased(v[0], j);
          Residual<8> r[1] = {res[x & 1][q]};
          if (sizeof(*to) == 4) swap_halves(r[0].first, r[0].second);
          else r[0].first = swapped(r[0].first);
          add_residuals<T, 8, 1>(v, r, e, 0);
          store(to + i * (16 * e.ldy) + 32 * j, v[0]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }, std::make_integer_sequence<int, kUnits / kAhead>{});
    };
    if (e.y_f32) finish(static_cast<float*>(e.y));
    else finish(static_cast<T*>(e.y));
  } else if (e.y_f32) {
    write(static_cast<float*>(e.y), e.ldy);
  } else {
    write(static_cast<T*>(e.y), e.ldy);
  }
}

// The same with every stage, for pinned sums: a loop over the rows of the
// instructions' tiles, whose sums a chain of branches fetches from their
// registers, so that the code of the stages is there once (for every sum, it
// would not fit the instruction cache).  What the stages add to 8192 x 4096 x
// 4096 bf16, 182 us: relu or silu 8, the tanh form of gelu 10 and with a bias and
// z kept 16, gelu 19 and 23, dropout, bias and residual 27.
template <typename T, int MT, int NT>
__device__ __forceinline__ void direct_full(const GemmArgs& g, const f32x4v (&acc)[MT][NT], int32_t m, int32_t n) {
  constexpr int kPairs = NT / 2;
  const Epilogue& e = g.e;
  float b[kPairs][8];
#pragma unroll
  for (int j = 0; j < kPairs; ++j) load_bias<T, 8>(b[j], e, n + 32 * j);
  const bool wide = sizeof(T) == 4 || e.y_f32;
  Residual<8> res[kPairs], next[kPairs];
  auto fetch = [&](int32_t row) {
    const char* const p = static_cast<const char*>(e.res) + ((int64_t(row) * e.ldr + n) << (wide ? 2 : 1));
    using Half = typename Residual<8>::Half;
#pragma unroll
    for (int j = 0; j < kPairs; ++j) next[j].first = *reinterpret_cast<const Half*>(p + (wide ? 128 : 64) * j);
    if (wide) {
#pragma unroll
      for (int j = 0; j < kPairs; ++j) next[j].second = *reinterpret_cast<const Half*>(p + 128 * j + 16);
    }
  };
  __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): the loads to LDS that nobody waits for
  if (e.res) fetch(m);
#pragma unroll 1
  for (int i = 0; i < MT; ++i) {
    float v[kPairs][8];
    unrolled([&](auto index) {
      constexpr int x = decltype(index)::value;
      if (x == i) {
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          const f32x4v c = unpinned(acc[x][j]);
#pragma unroll
          for (int k = 0; k < 4; ++k) v[j / 2][j % 2 * 4 + k] = c[k];
        }
      }
    }, std::make_integer_sequence<int, MT>{});
    const int32_t row = m + 16 * i;
    auto store = [&](auto* to, int64_t ld) {
      to += int64_t(row) * ld + n;
#pragma unroll
      for (int j = 0; j < kPairs; ++j) store_group<8>(to + 32 * j, v[j]);
    };
#pragma unroll
    for (int j = 0; j < kPairs; ++j)
#pragma unroll
      for (int k = 0; k < 8; ++k) v[j][k] += b[j][k];
    if (e.res) {
#pragma unroll
      for (int j = 0; j < kPairs; ++j) res[j] = next[j];
      if (i + 1 < MT) fetch(row + 16);
    }
    if (e.z) store(static_cast<T*>(e.z), e.ldz);
    activate<T>(v, e.act);
    if (e.drop.on) {
#pragma unroll
      for (int j = 0; j < kPairs; ++j) drop_some<8>(v[j], e.drop, e.drop.row0 + uint32_t(row), uint32_t(n + 32 * j));
    }
    add_residuals<T, 8, kPairs>(v, res, e, 0);
    if (e.y_f32) store(static_cast<float*>(e.y), e.ldy);
    else store(static_cast<T*>(e.y), e.ldy);
  }
}

// Where the tiles of an operand lie: one after the other along the inner length.
struct Straight {
  template <typename Op>
  __device__ __forceinline__ const char* at(const Op& op, int32_t t) const { return op.at(t); }
  // from the tile before t to t, which is below whole or not there
  template <typename Op>
  __device__ __forceinline__ void move(const char*& p, const Op& op, int32_t t, int32_t whole) const {
    p += t < whole ? op.step() : 0;
  }
};

// The products of `whole` tiles of the inner length, added to acc.  Operands take
// the 2 D + 1 places in LDS in turn: a of tile 0, b of tile 0, a of tile 1, and
// so on.  Slice 0 of tile t is multiplied while slice 1 is read, and slice 1
// while slice 0 of tile t + 1 is.  Once every wave has read the whole of tile t,
// b of t + D is loaded to where a of t lay, and then a of t + D + 1 to where b of t
// lay; the waves' next meeting waits for tile t + 2 and before.  fa and fb are the
// fragments of both slices, whose contents do not matter before and after.
// ALONE: the operands' tiles are one wave's own, in LDS that no other touches,
// and nobody meets.
template <typename T, int MT, int NT, int D, bool ALONE = false, typename OpA, typename OpB, typename FragA, typename FragB, typename Where>
__device__ __forceinline__ void multiply_ring(f32x4v (&acc)[MT][NT], const OpA& a, const OpB& b, const FragA& ra,
                                              const FragB& rb, i32x4v (&fa)[2][MT], i32x4v (&fb)[2][NT], char* lds, int wave,
                                              int32_t whole, const Where& where) {
  constexpr uint32_t kPlace = OpA::kBytes, kRing = (2 * D + 1) * kPlace;
  constexpr bool kPinned = MT * NT == 64;
  constexpr int kReads = MT + NT, kProducts = MT * NT, kLoadsA = OpA::kSlots, kLoadsB = OpB::kSlots;
  static_assert(kLoadsA == kLoadsB && OpB::kBytes == kPlace, "operands of one size");
  const uint32_t lds0 = lds_offset(lds);
  auto after = [](uint32_t place) { return place == kRing - kPlace ? 0 : place + kPlace; };
  // fragment x of slice s, first those of b
  auto read = [&](int s, uint32_t at_a, uint32_t at_b, int x) {
    if (x < NT) fb[s][x] = rb.read(lds + at_b, x, s);
    else fa[s][x - NT] = ra.read(lds + at_a, x - NT, s);
  };
  auto product = [&](int s, int x) {
    const int i = x / NT, j = x % NT;
    if constexpr (kPinned) mma_pinned<T>(fb[s][j], fa[s][i], acc[i][j]);
    else acc[i][j] = mma<T>(fb[s][j], fa[s][i], acc[i][j]);
  };
  // all of an operand's tile t, or of the last one
  auto load_all = [&](const auto& op, int32_t t, uint32_t at) {
    const char* p = settled(where.at(op, t < whole ? t : whole - 1));
#pragma unroll
    for (int x = 0; x < kLoadsA; ++x) {
      op.aim(x, lds0 + at, wave);
      asm volatile("s_nop 0");
      op.issue(p, x);
    }
  };
  uint32_t at_a = 0, at_b = kPlace;
  if (whole > 0) {
#pragma unroll
    for (int x = 0; x <= 2 * D; ++x) {
      if (x % 2 == 0) load_all(a, x / 2, uint32_t(x) * kPlace);
      else load_all(b, x / 2, uint32_t(x) * kPlace);
    }
    if constexpr (ALONE) wait_own<(2 * D - 1) * kLoadsA>();
    else wait_all<(2 * D - 1) * kLoadsA>();
#pragma unroll
    for (int x = 0; x < kReads; ++x) read(0, at_a, at_b, x);
  }
  // The instruction stream of a tile: between two matrix instructions goes
  // at most one other of each kind, so that the matrix unit always has its
  // next one, and the loads are spread, since each keeps the address unit
  // busy for 16 cycles.  Slice 1 is read within the first half of slice 0's
  // products; after kMeet of them the waves meet.  The last tiles run the
  // same stream: their loads take the last tile again, which nobody reads.
  // Alone, a wave has its whole tile read by then, and a load goes with each product.
  constexpr int kMeet = ALONE ? kProducts / 2 : kProducts * 5 / 8;
  constexpr int kReadGap = kProducts / 2 / kReads, kReadGap1 = kProducts * 3 / 4 / kReads;
  constexpr int kGapB = ALONE ? 1 : kProducts >= 64 ? 5 : 2, kGapA = ALONE ? 1 : kProducts >= 64 ? 6 : 3;
  constexpr int kMeetA = kMeet + kGapB * kLoadsB;
  static_assert(kReadGap >= 1 && kMeetA + kGapA * kLoadsA + ALONE <= 2 * kProducts, "everything within a tile");
  const char* pb = settled(where.at(b, whole > D ? D : whole - 1));
  const char* pa = settled(where.at(a, whole > D + 1 ? D + 1 : whole - 1));
  for (int32_t t = 0; t < whole; ++t) {
    const uint32_t next_a = after(at_b), next_b = after(next_a);
    const char* const from_a = settled(pa);
    const char* const from_b = settled(pb);
    if constexpr (kPinned) mma_ready();
    unrolled([&](auto index) {
      constexpr int x = decltype(index)::value, y = x - kProducts, zb = x - kMeet, za = x - kMeetA;
      if constexpr (x < kProducts && x % kReadGap == 0 && x / kReadGap < kReads) read(1, at_a, at_b, x / kReadGap);
      if constexpr (x == kMeet && !ALONE) wait_all<(2 * D - 3) * kLoadsA>();
      if constexpr (x == kMeet && ALONE) wait_own<(2 * D - 3) * kLoadsA>();
      if constexpr (y >= 0 && y % kReadGap1 == 0 && y / kReadGap1 < kReads) read(0, next_a, next_b, y / kReadGap1);
      if constexpr (!ALONE) {
        if constexpr (zb >= 0 && za < 0 && zb % kGapB == 0) b.aim(zb / kGapB, lds0 + at_a, wave);
        if constexpr (zb >= 0 && za < 0 && zb % kGapB == 1) b.issue(from_b, zb / kGapB);
        if constexpr (za >= 0 && za / kGapA < kLoadsA && za % kGapA == 0) a.aim(za / kGapA, lds0 + at_b, wave);
        if constexpr (za >= 0 && za / kGapA < kLoadsA && za % kGapA == 1) a.issue(from_a, za / kGapA);
      } else {  // each load goes out before the next one's target is named
        if constexpr (zb >= 1 && zb <= kLoadsB) b.issue(from_b, zb - 1);
        if constexpr (za >= 1 && za <= kLoadsA) a.issue(from_a, za - 1);
        if constexpr (zb >= 0 && zb < kLoadsB) b.aim(zb, lds0 + at_a, wave);
        if constexpr (za >= 0 && za < kLoadsA) a.aim(za, lds0 + at_b, wave);
      }
      product(x / kProducts, x % kProducts);
      __builtin_amdgcn_sched_barrier(0);
    }, std::make_integer_sequence<int, 2 * kProducts>{});
    where.move(pb, b, t + D + 1, whole);
    where.move(pa, a, t + D + 2, whole);
    at_a = next_a;
    at_b = next_b;
  }
}

// LDS of a workgroup: five places, each for one operand of a tile.
constexpr int ring_bytes(int tile) { return 5 * tile * kTileKBytes; }

// What a kernel's epilogue has, each with less code and fewer registers than the
// next: kSums a residual, kBiased also a bias, kFull everything.
enum Stages { kSums, kBiased, kFull };

// Part `part` of tile `tile` of a product.
template <typename T, bool AK, bool BK, int MT, int NT, int WM, int WN, bool ASYNC, Stages STAGES>
__device__ __forceinline__ void gemm_tile(const GemmArgs& g, uint32_t tile, uint32_t part_of, char* lds) {
  constexpr int THREADS = WM * WN * 64, TM = WM * MT * 16, TN = WN * NT * 16;
  using OpA = Operand<T, AK, false, TM, THREADS>;
  using OpB = Operand<T, BK, true, TN, THREADS>;
  constexpr uint32_t kPlace = OpA::kBytes, kRing = 5 * kPlace;
  static_assert(OpB::kBytes == kPlace, "places of one size");
  constexpr int kInner = OpA::kInner;
  constexpr bool kPinned = MT * NT == 64;

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / WN, wn = wave % WN;
  uint32_t im, in;
  tile_of(tile, uint32_t(g.tiles_m), uint32_t(g.tiles_n), im, in);
  const int32_t m0 = int32_t(im) * TM, n0 = int32_t(in) * TN;
  const int32_t k0 = int32_t(part_of) * g.k_split;
  const int32_t klen = g.K - k0 < g.k_split ? g.K - k0 : g.k_split;

  OpA a;
  OpB b;
  a.init(static_cast<const T*>(g.a), g.lda, m0, k0, g.e.M, g.K, tid);
  b.init(static_cast<const T*>(g.b), g.ldb, n0, k0, g.e.N, g.K, tid);
  static_assert(MT % 4 == 0 && NT % 4 == 0, "the waves' first rows are multiples of 64");
  Fragments<T, AK, false, TM> ra;
  Fragments<T, BK, true, TN> rb;
  ra.init(wm * MT * 16, lane);
  rb.init(wn * NT * 16, lane);

  f32x4v acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = f32x4v{0.0f, 0.0f, 0.0f, 0.0f};

  const int32_t tiles = (klen + kInner - 1) / kInner;
  if constexpr (ASYNC) {
    const int32_t whole = klen / kInner;
    i32x4v fa[2][MT], fb[2][NT];
    multiply_ring<T, MT, NT, 2>(acc, a, b, ra, rb, fa, fb, lds, wave, whole, Straight{});
    if (whole < tiles) {  // what is left of the inner length, through registers
      wait_all<0>();
      a.copy(whole, klen - int64_t(whole) * kInner, lds, tid);
      b.copy(whole, klen - int64_t(whole) * kInner, lds + kPlace, tid);
      wait_all<0>();
#pragma unroll
      for (int s = 0; s < 2; ++s) {
#pragma unroll
        for (int x = 0; x < NT; ++x) fb[s][x] = rb.read(lds + kPlace, x, s);
#pragma unroll
        for (int x = 0; x < MT; ++x) fa[s][x] = ra.read(lds, x, s);
      }
      if constexpr (kPinned) mma_ready();
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int j = 0; j < NT; ++j) {
            if constexpr (kPinned) mma_pinned<T>(fb[s][j], fa[s][i], acc[i][j]);
            else acc[i][j] = mma<T>(fb[s][j], fa[s][i], acc[i][j]);
          }
    }
    if constexpr (kPinned) mma_done(acc[MT - 1], acc[MT - 2], acc[MT - 3]);
  } else {
    // Tiles go through registers, two sets of them: while tile t is
    // multiplied, t + 2 is on its way and t + 1, which has arrived, is written
    // to the other half of LDS, after which t + 3 is asked for.
    i32x4v xa0[OpA::kSlots], xb0[OpB::kSlots], xa1[OpA::kSlots], xb1[OpB::kSlots];
    auto fetch = [&](i32x4v (&xa)[OpA::kSlots], i32x4v (&xb)[OpB::kSlots], int32_t t) {
      a.load_checked(xa, t, klen - int64_t(t) * kInner, tid);
      b.load_checked(xb, t, klen - int64_t(t) * kInner, tid);
    };
    auto place = [&](const i32x4v (&xa)[OpA::kSlots], const i32x4v (&xb)[OpB::kSlots], int half) {
      a.store(xa, lds + half * 2 * kPlace, tid);
      b.store(xb, lds + half * 2 * kPlace + kPlace, tid);
    };
    auto multiply = [&](int half) {
      const char* at = lds + half * 2 * kPlace;
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        i32x4v fa[MT], fb[NT];
#pragma unroll
        for (int i = 0; i < MT; ++i) fa[i] = ra.read(at, i, s);
#pragma unroll
        for (int j = 0; j < NT; ++j) fb[j] = rb.read(at + kPlace, j, s);
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int j = 0; j < NT; ++j) acc[i][j] = mma<T>(fb[j], fa[i], acc[i][j]);
      }
    };
    const bool open = g.open;
    int32_t t = 0;
    if (open && tiles > 4) {
      a.load(xa0, 0);
      b.load(xb0, 0);
      a.load(xa1, 1);
      b.load(xb1, 1);
      place(xa0, xb0, 0);
      a.load(xa0, 2);
      b.load(xb0, 2);
      meet();
      for (; t + 5 < tiles; t += 2) {  // t + 4 is not the last
        multiply(0);
        place(xa1, xb1, 1);
        a.load(xa1, t + 3);
        b.load(xb1, t + 3);
        meet();
        multiply(1);
        place(xa0, xb0, 0);
        a.load(xa0, t + 4);
        b.load(xb0, t + 4);
        meet();
      }
      // t + 1 and t + 2 are in the registers; t + 3 is the last or the last but one
      multiply(0);
      place(xa1, xb1, 1);
      if (t + 4 < tiles) {
        a.load(xa1, t + 3);
        b.load(xb1, t + 3);
      } else {
        fetch(xa1, xb1, t + 3);
      }
      meet();
      multiply(1);
      place(xa0, xb0, 0);
      if (t + 4 < tiles) fetch(xa0, xb0, t + 4);
      meet();
      multiply(0);
      place(xa1, xb1, 1);
      meet();
      multiply(1);
      if (t + 4 < tiles) {
        place(xa0, xb0, 0);
        meet();
        multiply(0);
      }
    } else {  // few tiles, or rows far apart: two tiles at a time, the next two on their way
      auto get = [&](i32x4v (&xa)[OpA::kSlots], i32x4v (&xb)[OpB::kSlots], int32_t at) {
        if (open && at + 1 < tiles) {
          a.load(xa, at);
          b.load(xb, at);
        } else if (at < tiles) {
          fetch(xa, xb, at);
        }
      };
      get(xa0, xb0, 0);
      get(xa1, xb1, 1);
      for (; t < tiles; t += 2) {
        if (t > 0) meet();
        place(xa0, xb0, 0);
        if (t + 1 < tiles) place(xa1, xb1, 1);
        get(xa0, xb0, t + 2);
        get(xa1, xb1, t + 3);
        meet();
        multiply(0);
        if (t + 1 < tiles) multiply(1);
      }
    }
  }

  // A whole tile's sums leave from the lanes that hold them: of tiles 2j, 2j + 1 a lane has 8 columns
  // (32 j + 8 p on) of a row, and four lanes have 64 bytes of halves together,
  // whose line the next columns fill.  16384 x 1024 x 1024 bf16 30 us, through LDS
  // 40 (the passes below wait for each step by themselves).
  const bool whole = m0 + TM <= g.e.M && n0 + TN <= g.e.N;
  if (STAGES != kFull && whole) {
    direct<T, MT, NT, STAGES == kBiased, !BK>(g, acc, !BK && (lane & 16), m0 + wm * MT * 16 + (lane & 15), n0 + wn * NT * 16 + 8 * (lane >> 4), part_of);
    return;
  }
  if constexpr (STAGES == kFull && kPinned) {
    if (whole) {
      direct_full<T, MT, NT>(g, acc, m0 + wm * MT * 16 + (lane & 15), n0 + wn * NT * 16 + 8 * (lane >> 4));
      return;
    }
  }

  // At the matrix' edges, and from small tiles with every stage, the sums leave
  // through LDS, each wave by itself in its share of the
  // buffers: a lane of tiles 2j, 2j + 1 writes its 8 columns (32 j + 8 p on)
  // of a row as one 32-byte unit, at a place XORed with the row so that 16
  // rows fall on different banks, and then takes 8 columns of one row whose
  // other columns its neighbours take: whole lines of y, z and the residual.
  constexpr int kUnits = NT * 2;                                // 8-column units of a wave's row
  constexpr int kRounds = MT > 4 ? MT / 4 : 1, kTilesRound = MT / kRounds;
  constexpr int kShare = kTilesRound * 16 * kUnits * 32;        // bytes of a wave's share
  constexpr int kPassRows = 64 / kUnits, kPasses = kTilesRound * 16 / kPassRows, kAhead = 4;
  static_assert(kTilesRound * kRounds == MT && kPasses % (2 * kAhead) == 0 && uint32_t(kShare * WM * WN) <= kRing, "whole rounds");
  char* share = lds + wave * kShare;
  const bool swap = !BK && (lane & 16);
  const int32_t unit = lane % kUnits, n = n0 + wn * NT * 16 + 8 * unit;
  const int have = g.e.N - n, back = have < 8 ? 8 - have : 0;
  float* part = g.part + int64_t(part_of) * g.e.M * g.ldp + n;  // ldp is a multiple of 8
  float bias[8];
  if constexpr (STAGES != kSums) load_bias<T, 8>(bias, g.e, n, have > 0 ? back : 0);
  auto sum = [](const f32x4v& a) {
    if constexpr (kPinned) return unpinned(a);
    else return a;
  };
  auto spread = [&](auto round) {
    constexpr int first = decltype(round)::value * kTilesRound;
#pragma unroll
    for (int i = 0; i < kTilesRound; ++i) {
#pragma unroll
      for (int j = 0; j < NT / 2; ++j) {
        const f32x4v x = sum(acc[first + i][2 * j]), y = sum(acc[first + i][2 * j + 1]);
        const int r = 16 * i + (lane & 15), u = (4 * j + (lane >> 4)) ^ (r & (kUnits - 1));
        f32x4v* q = reinterpret_cast<f32x4v*>(share + (r * kUnits + u) * 32);
        q[swap ? 1 : 0] = x;
        q[swap ? 0 : 1] = y;
      }
    }
  };
  wait_all<0>();
#pragma unroll 1
  for (int round = 0; round < kRounds; ++round) {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    static_assert(kRounds <= 2, "rounds");
    if (round == 0) spread(std::integral_constant<int, 0>{});
    else spread(std::integral_constant<int, kRounds - 1>{});
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    const int32_t mw = m0 + (wm * MT + round * kTilesRound) * 16 + lane / kUnits;
    auto unit_at = [&](int r) { return share + (r * kUnits + (unit ^ (r & (kUnits - 1)))) * 32; };
    if (have > 0 && (g.e.N >= 8 || g.splits > 1)) {
      // the residual of half the passes is on its way while half are worked on
      Residual<8> res0[kAhead], res1[kAhead];
      auto fetch = [&](Residual<8> (&res)[kAhead], int pass) {
        if (g.splits == 1) load_residuals<T, 8, kAhead>(res, g.e, mw + pass * kPassRows, kPassRows, n - back);
      };
      auto finish = [&](const Residual<8> (&res)[kAhead], int pass) {
        float v[kAhead][8];
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
          const f32x4v* w = reinterpret_cast<const f32x4v*>(unit_at((pass + q) * kPassRows + lane / kUnits));
          const f32x4v x = w[0], y = w[1];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            v[q][i] = x[i];
            v[q][4 + i] = y[i];
          }
        }
        const int32_t m = mw + pass * kPassRows;
        if (g.splits > 1) {
#pragma unroll
          for (int q = 0; q < kAhead; ++q)
            if (m + q * kPassRows < g.e.M) store_group<8>(part + int64_t(m + q * kPassRows) * g.ldp, v[q]);
        } else {
          emit<T, 8, kAhead, STAGES != kSums, STAGES == kFull>(v, bias, res, g.e, m, kPassRows, n, back);
        }
      };
      fetch(res0, 0);
#pragma unroll 1
      for (int pass = 0; pass < kPasses; pass += 2 * kAhead) {
        fetch(res1, pass + kAhead);
        finish(res0, pass);
        if (pass + 2 * kAhead < kPasses) fetch(res0, pass + 2 * kAhead);
        finish(res1, pass + kAhead);
      }
    } else if (have > 0) {  // rows shorter than a unit
#pragma unroll 1
      for (int pass = 0; pass < kPasses; pass += kAhead) {
        const int32_t m = mw + pass * kPassRows;
        if (m >= g.e.M) break;
        auto sum = [&](int q, int i) {
          return reinterpret_cast<const float*>(unit_at((pass + q) * kPassRows + lane / kUnits))[i];
        };
        emit_tail<T, 8, kAhead, STAGES != kSums, STAGES == kFull>(sum, g.e, m, kPassRows, n, have);
      }
    }
  }
}

template <typename T, bool AK, bool BK, int MT, int NT, int WM, int WN, bool ASYNC, Stages STAGES>
__global__ __launch_bounds__(WM* WN * 64, MT * NT <= 16 ? 2 : 1) void gemm_kernel(GemmArgs g) {
  __shared__ __attribute__((aligned(1024))) char lds[ring_bytes(WM * MT * 16)];
  gemm_tile<T, AK, BK, MT, NT, WM, WN, ASYNC, STAGES>(g, blockIdx.x, blockIdx.y, lds);
}

// The gradient's two products in one launch: x's workgroups begin at x_from,
// w's at w_from, one of which is 0; the other is a multiple of 8, so that both
// orders of tiles (tile_of) go round the XCDs alike.
template <typename T, int MT, int NT, bool ASYNC>
__global__ __launch_bounds__(256, MT * NT <= 16 ? 2 : 1) void gemm_pair_kernel(GemmArgs x, GemmArgs w, uint32_t x_from,
                                                                                uint32_t w_from) {
  __shared__ __attribute__((aligned(1024))) char lds[ring_bytes(2 * MT * 16)];
  const uint32_t tx = uint32_t(x.tiles_m) * uint32_t(x.tiles_n), tw = uint32_t(w.tiles_m) * uint32_t(w.tiles_n);
  if (x_from > w_from ? blockIdx.x >= x_from : blockIdx.x < w_from) {
    const uint32_t id = blockIdx.x - x_from, part = id / tx;
    if (part < uint32_t(x.splits)) gemm_tile<T, true, false, MT, NT, 2, 2, ASYNC, kSums>(x, id - part * tx, part, lds);
  } else {
    const uint32_t id = blockIdx.x - w_from, part = id / tw;
    if (part < uint32_t(w.splits)) gemm_tile<T, false, false, MT, NT, 2, 2, ASYNC, kSums>(w, id - part * tw, part, lds);
  }
}

template <typename T, bool AK, bool BK, Stages STAGES>
int launch_stages(const GemmArgs& g, bool aligned, int32_t shape, hipStream_t st) {
  const dim3 grid(uint32_t(g.tiles_m) * uint32_t(g.tiles_n), uint32_t(g.splits));
  if (shape == kTile256) {
    if constexpr (sizeof(T) == 2) {
      if (!aligned) return int(hipErrorInvalidValue);
      gemm_kernel<T, AK, BK, 8, 8, 2, 2, true, STAGES><<<grid, dim3(256), 0, st>>>(g);
    } else {
      return int(hipErrorInvalidValue);
    }
  } else if (aligned) {
    gemm_kernel<T, AK, BK, 4, 4, 2, 2, true, STAGES><<<grid, dim3(256), 0, st>>>(g);
  } else {
    gemm_kernel<T, AK, BK, 4, 4, 2, 2, false, STAGES><<<grid, dim3(256), 0, st>>>(g);
  }
  return int(hipGetLastError());
}

// The gradient's products have a residual at most; parts are joined later with
// the whole epilogue.
template <typename T>
int launch_gemm_of(const GemmArgs& g, bool a_kmajor, bool b_kmajor, bool aligned, int32_t shape, void* stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (a_kmajor && b_kmajor) {
    const bool full = g.splits == 1 && (g.e.z || g.e.act != kActNone || g.e.drop.on);
    return full ? launch_stages<T, true, true, kFull>(g, aligned, shape, st) : launch_stages<T, true, true, kBiased>(g, aligned, shape, st);
  }
  if (b_kmajor || g.e.bias || g.e.z || g.e.act != kActNone || g.e.drop.on) return int(hipErrorInvalidValue);
  return a_kmajor ? launch_stages<T, true, false, kSums>(g, aligned, shape, st)
                  : launch_stages<T, false, false, kSums>(g, aligned, shape, st);
}

// The product with the longer parts first.
template <typename T>
int launch_pair_of(const GemmArgs& x, const GemmArgs& w, bool aligned, int32_t shape, void* stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  const uint32_t nx = uint32_t(x.tiles_m) * uint32_t(x.tiles_n) * uint32_t(x.splits);
  const uint32_t nw = uint32_t(w.tiles_m) * uint32_t(w.tiles_n) * uint32_t(w.splits);
  const bool x_first = x.k_split >= w.k_split;
  const uint32_t x_from = x_first ? 0 : (nw + 7) / 8 * 8, w_from = x_first ? (nx + 7) / 8 * 8 : 0;
  const dim3 grid(x_first ? w_from + nw : x_from + nx);
  if (shape == kTile256) {
    if constexpr (sizeof(T) == 2) {
      if (!aligned) return int(hipErrorInvalidValue);
      gemm_pair_kernel<T, 8, 8, true><<<grid, dim3(256), 0, st>>>(x, w, x_from, w_from);
    } else {
      return int(hipErrorInvalidValue);
    }
  } else if (aligned) {
    gemm_pair_kernel<T, 4, 4, true><<<grid, dim3(256), 0, st>>>(x, w, x_from, w_from);
  } else {
    gemm_pair_kernel<T, 4, 4, false><<<grid, dim3(256), 0, st>>>(x, w, x_from, w_from);
  }
  return int(hipGetLastError());
}

}  // namespace ar
