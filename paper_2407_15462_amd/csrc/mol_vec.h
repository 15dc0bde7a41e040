// Runs of elements at any element alignment, and sums over teams of lanes, for
// the kernels that work on whole rows (norms, dropout, the gated scan).
#pragma once

#include "mol_device.h"

namespace mol {
namespace vec {

// Vector loads and stores of addresses that are aligned to an element only (the
// hardware takes them; a row of an odd size starts anywhere).
template <int BYTES, int ALIGN>
struct Mem;
#define MOL_MEM(BYTES, ALIGN, TYPE)                                            \
  template <>                                                                  \
  struct Mem<BYTES, ALIGN> {                                                   \
    typedef TYPE __attribute__((aligned(ALIGN), may_alias)) type;              \
  };
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
MOL_MEM(4, 2, uint32_t)
MOL_MEM(8, 2, u32x2_t)
MOL_MEM(16, 2, u32x4_t)
MOL_MEM(8, 4, u32x2_t)
MOL_MEM(16, 4, u32x4_t)
#undef MOL_MEM

// float32 -> bf16, nearest even; NaN stays NaN
__device__ __forceinline__ bf16_t to_bf16(float f) { return __builtin_bit_cast(bf16_t, static_cast<__bf16>(f)); }
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  typedef float f32x2_t __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
  const f32x2_t v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2_t));
}

// Whether a call's inputs are to be read past the caches: if they are more than the last-level
// cache's 256 MB.  Measured: dropout of 134M bfloat16 elements with residual (512 MB read) 117 us, 137
// through the caches; of 30M float32 ones (114 MB) 46, and 36 through the caches, which hold them.
inline bool streams(size_t bytes) { return bytes >= 256ul << 20; }

// N elements as they lie in memory.
template <typename T, int N>
struct Raw {
  static constexpr int kWords = N * sizeof(T) / 4;
  uint32_t w[kWords];
  __device__ __forceinline__ float at(int e) const {
    if constexpr (sizeof(T) == 4)
      return __uint_as_float(w[e]);
    else
      return __uint_as_float(e & 1 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = 0;
  }
  // all N; ONCE: past the caches, for tensors that they do not hold (see streams())
  template <bool ONCE = false>
  __device__ __forceinline__ void load(const T* p) {
    constexpr int kStep = kWords < 4 ? kWords : 4;
#pragma unroll
    for (int i = 0; i < kWords; i += kStep) {
      const auto* at = reinterpret_cast<const typename Mem<kStep * 4, sizeof(T)>::type*>(p + i * 4 / sizeof(T));
      typename Mem<kStep * 4, sizeof(T)>::type v;
      if constexpr (ONCE)
        v = __builtin_nontemporal_load(at);
      else
        v = *at;
      if constexpr (kStep == 1)
        w[i] = v;
      else
#pragma unroll
        for (int j = 0; j < kStep; ++j) w[i + j] = v[j];
    }
  }
  // the first n (none for n <= 0), zeros behind them
  template <bool ONCE = false>
  __device__ __forceinline__ void load(const T* p, int n) {
    if (n >= N) return load<ONCE>(p);
    zero();
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (e < n) {
        if constexpr (sizeof(T) == 4)
          w[e] = __float_as_uint(p[e]);
        else
          w[e / 2] |= static_cast<uint32_t>(p[e]) << (e & 1) * 16;
      }
  }
};

// N values to memory, each rounded once: all, or the first n
template <bool ONCE = false, typename T, int N>
__device__ __forceinline__ void store(T* p, const float (&v)[N]) {
  constexpr int kWords = Raw<T, N>::kWords, kStep = kWords < 4 ? kWords : 4;
  uint32_t w[kWords];
#pragma unroll
  for (int i = 0; i < kWords; ++i) {
    if constexpr (sizeof(T) == 4)
      w[i] = __float_as_uint(v[i]);
    else
      w[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
  }
#pragma unroll
  for (int i = 0; i < kWords; i += kStep) {
    typename Mem<kStep * 4, sizeof(T)>::type x;
    if constexpr (kStep == 1)
      x = w[i];
    else
#pragma unroll
      for (int j = 0; j < kStep; ++j) x[j] = w[i + j];
    auto* to = reinterpret_cast<typename Mem<kStep * 4, sizeof(T)>::type*>(p + i * 4 / sizeof(T));
    if constexpr (ONCE)
      __builtin_nontemporal_store(x, to);
    else
      *to = x;
  }
}
template <bool ONCE = false, typename T, int N>
__device__ __forceinline__ void store(T* p, const float (&v)[N], int n) {
  if (n >= N) return store<ONCE>(p, v);
#pragma unroll
  for (int e = 0; e < N; ++e)
    if (e < n) {
      if constexpr (sizeof(T) == 4)
        p[e] = v[e];
      else
        p[e] = to_bf16(v[e]);
    }
}

// Sum over the team of `lanes` (a power of two up to 64, the same in all of the
// wave) lanes that this lane belongs to; every lane gets the same bits.
template <int CTRL>
__device__ __forceinline__ float moved(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ float team_sum(float v, int lanes) {
  if (lanes > 1) v += moved<0xB1>(v);     // lane ^ 1
  if (lanes > 2) v += moved<0x4E>(v);     // lane ^ 2
  if (lanes > 4) v += moved<0x141>(v);    // 7 - lane of 8
  if (lanes > 8) v += moved<0x140>(v);    // 15 - lane of 16
  if (lanes > 16) v += __shfl_xor(v, 16);
  if (lanes > 32) v += __shfl_xor(v, 32);
  return v;
}

}  // namespace vec
}  // namespace mol
