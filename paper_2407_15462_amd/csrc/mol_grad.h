// Pieces shared by the two forms of the score gradient.
#pragma once

#include <algorithm>

#include "mol_tile.h"

namespace mol {
namespace grad {

// Sums of partial results: out[o] = sum over s < S of in[s * stride + o], o < L,
// as float32 (added to what an earlier slab left in acc) and, where wanted, in the
// output's type.  o of batch o / in_len goes to element out_at + o % in_len of
// that batch of out_len in the output.
struct SumJob {
  const float* in;
  long L, stride;
  int S;
  float* acc;              // NULL, or float32 sums kept between slabs
  int add;
  void* out;               // NULL, or the output
  int bf16;
  long in_len, out_len, out_at;
  int cols_log2;           // (set by the launcher) columns of a block: 256, 64 or 16
};
constexpr int kSumJobs = 8;   // one an output
struct SumArgs {
  int n;
  long first[kSumJobs + 1];    // first block of each job
  SumJob job[kSumJobs];
};
struct SumList {
  SumArgs a{};
  hipStream_t st;
  explicit SumList(hipStream_t s) : st(s) {}
  void add(const SumJob& j);
  hipError_t run();
};

// The bf16 form on 16-bit matrix instructions (mol_score_grad_bf16.hip).
bool bf16_supported(const DevProb& pr);
size_t bf16_bytes(const DevProb& pr);      // of a call
size_t bf16_most(const DevProb& pr);       // of every call with the same shape and no more queries or items; 0: none takes this form
hipError_t launch_bf16(const DevProb& pr, const float* dphi, const mol_score_grads& o, char* ws, hipStream_t st);

// K splits of a product of `waves` waves a part with `chunks` K chunks: about 2048
// waves in all, with two chunks a split up to 64 splits (a short product is a chain of
// latencies) and `least` beyond (each split is a part to write and to add).
inline long most_splits(long chunks, long least) { return std::max(std::min(chunks / 2, 64l), chunks / least); }
inline int split_of(long waves, long chunks, long least) {
  const long want = (2048 + waves / 2) / waves;
  return static_cast<int>(std::max(1l, std::min(want, most_splits(chunks, least))));
}
// Bytes of the parts of such a product of `out` bytes: two splits or more leave at
// most 2730 tiles of 32 x 64 floats (n splits of w waves, n w <= 2048 + w / 2 and 2 w <= n w).
inline size_t most_parts(size_t out, long chunks, long least) {
  const long n = most_splits(chunks, least);
  return n < 2 ? 0 : std::min<size_t>(2730ul * 8192, n * out);
}

// high halves of a and b: their first bf16 terms by truncation
__device__ __forceinline__ uint32_t high_halves(float a, float b) {
  return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
}
__device__ __forceinline__ float rest(float a) { return a - __uint_as_float(__float_as_uint(a) & 0xFFFF0000u); }

// eight values as bf16 terms, two values a word
template <int TERMS>
struct Terms {
  uint4 t[TERMS];
};
template <int TERMS>
__device__ __forceinline__ Terms<TERMS> split(const float (&x)[8]) {
  Terms<TERMS> o;
  float v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = x[e];
#pragma unroll
  for (int k = 0; k < TERMS; ++k) {
    o.t[k] = make_uint4(high_halves(v[0], v[1]), high_halves(v[2], v[3]), high_halves(v[4], v[5]), high_halves(v[6], v[7]));
    if (k + 1 < TERMS)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = rest(v[e]);
  }
  return o;
}
template <int TERMS>
__device__ __forceinline__ tile::f32x4_t mfma_terms(uint4 a, const Terms<TERMS>& b, tile::f32x4_t c) {
#pragma unroll
  for (int k = TERMS - 1; k >= 0; --k) c = tile::mfma_bf16(a, b.t[k], c);   // small terms first
  return c;
}

// Stores a wave's tile of a product: element (4 g + i, c) of each 16x16 block, rows
// from m0 to m and columns from t0 to d, as a part's float32 or as the output's type.
template <typename T, int RB, int CB>
__device__ __forceinline__ void put_tile(void* out, long base, int m0, int m, int t0, int d, int direct,
                                         const tile::f32x4_t (&acc)[RB][CB]) {
  const int c = threadIdx.x & 15, g = threadIdx.x / 16 % 4;
  auto each = [&](auto put) {
#pragma unroll
    for (int r = 0; r < RB; ++r)
#pragma unroll
      for (int t = 0; t < CB; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int row = m0 + 16 * r + 4 * g + i, x = t0 + 16 * t + c;
          if (row < m && x < d) put(base + static_cast<long>(row) * d + x, acc[r][t][i]);
        }
  };
  if (sizeof(T) == 2 && direct)
    each([&](long at, float v) { static_cast<bf16_t*>(out)[at] = __builtin_bit_cast(uint16_t, static_cast<__bf16>(v)); });
  else
    each([&](long at, float v) { static_cast<float*>(out)[at] = v; });
}

// A product's tiles of 32 rows and 64 columns, a wave each: `rows` by `cols` of them
// and z (splits, and item components of dX).  Waves are numbered through, so that
// four of any of them make a workgroup.
struct Tiles {
  int rows, cols, z;
  __host__ __device__ long count() const { return static_cast<long>(rows) * cols * z; }
};
__device__ __forceinline__ int3 tile_of(const Tiles& t, uint32_t unit) {
  const uint32_t rest = unit / static_cast<uint32_t>(t.rows), z = rest / static_cast<uint32_t>(t.cols);
  return make_int3(unit - rest * t.rows, rest - z * t.cols, z);
}

typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4_t lds_s16x4_t;

// The transposing read: each group of 16 lanes reads 4 rows of 16 elements (8
// bytes a lane, rows lane / 4) and gets column lane, its 4 rows in order
__device__ __forceinline__ uint2 read_tr(const void* lds) {
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                       (lds_s16x4_t*)(__attribute__((address_space(3))) const void*)lds));
}

// Rows of X or Q as the K of a bf16 product: a chunk of 32 of them, 64 columns wide.
constexpr int kRowB = 9;                             // 16-byte words of an LDS row of 64 columns (and one: other banks)
constexpr int kTileB = 32 * kRowB;                   // of a wave's chunk of X or Q

// Lane l of a wave has piece l % 8 (8 columns) of rows l / 8 + 8 j of a chunk.
template <bool VEC>
struct RowTile {
  int rows, d, row, col;
  __device__ __forceinline__ RowTile(int rows_, int d_, int t0) : rows(rows_), d(d_) {
    const int lane = threadIdx.x & 63;
    row = lane >> 3;
    col = min(t0 + 8 * (lane & 7), VEC ? d - 8 : d - 1);   // (past d: others, for products that are not stored)
  }
  __device__ __forceinline__ void fetch(uint4 (&v)[4], const bf16_t* base, int k0) const {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bf16_t* p = base + (static_cast<uint64_t>(min(k0 + 8 * j + row, rows - 1)) * static_cast<uint32_t>(d) + col);
      if constexpr (VEC) {
        v[j] = *reinterpret_cast<const uint4*>(p);
      } else {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
          w[e] = p[min(2 * e, d - 1 - col)] | static_cast<uint32_t>(p[min(2 * e + 1, d - 1 - col)]) << 16;
        v[j] = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
  }
  // (rows past the end: zeros, as ds is there)
  __device__ __forceinline__ void put(const uint4 (&v)[4], uint4* sh, int k0) const {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      sh[(8 * j + row) * kRowB + (threadIdx.x & 7)] = k0 + 8 * j + row < rows ? v[j] : make_uint4(0, 0, 0, 0);
  }
};
// column 16 t + c of the chunk, K slots 8 g ..
__device__ __forceinline__ uint4 column_of(const uint4* sh, int t, int c, int g) {
  const unsigned char* p =
      reinterpret_cast<const unsigned char*>(sh) + (8 * g + (c >> 2)) * (16 * kRowB) + 8 * (c & 3) + 32 * t;
  const uint2 a = read_tr(p), b = read_tr(p + 4 * 16 * kRowB);
  return make_uint4(a.x, a.y, b.x, b.y);
}

}  // namespace grad
}  // namespace mol
