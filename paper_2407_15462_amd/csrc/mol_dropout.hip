// Dropout from a counter-based generator:
//   y_i = residual_i + (kept_i ? x_i / (1 - p) : 0)
// with the mask formed where it is used, and formed again by the gradient (the
// same call on dy).  Element i takes half e = j mod 8 of the four 32-bit words of
// Philox 4x32 with 10 rounds (Salmon et al., "Parallel random numbers: as easy as
// 1, 2, 3", SC 2011), j = offset + i, for the counter (j / 8, step, 0) and the key
// seed, and is kept if these 16 bits are at least 65,536 p.
//
// Bound by memory: a thread takes 8 elements, one counter, at a time.  Its 10
// rounds are 20 64-bit products, which for 32 bits an element would take as long as the
// memory does (bfloat16).  Measured: 134M bf16 elements 81 to 86 us (6.3 TB/s), with a residual 121 to 129 (6.2 to
// 6.6), both read past the caches (91 and 137 through them; see streams()); 524,288 in 2.7 us, of a call's 6.4.
#include <algorithm>

#include "mol_kernels.h"
#include "mol_vec.h"

namespace mol {

namespace {

using vec::Raw;

struct DropArgs {
  long n;
  const void* x;
  const void* residual;    // of y's type, or NULL
  void* y;
  uint64_t block0;         // counter of element 0
  uint32_t key0, key1, threshold;
  uint32_t step;
  const int32_t* step_ptr;
  float scale;
};

struct Words {
  uint32_t w[4];
};
__device__ __forceinline__ Words philox(uint64_t place, uint32_t step, uint32_t k0, uint32_t k1) {
  uint32_t c0 = static_cast<uint32_t>(place), c1 = static_cast<uint32_t>(place >> 32), c2 = step, c3 = 0;
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = static_cast<uint64_t>(c0) * 0xD2511F53u, b = static_cast<uint64_t>(c2) * 0xCD9E8D57u;
    c0 = static_cast<uint32_t>(b >> 32) ^ c1 ^ k0;
    c1 = static_cast<uint32_t>(b);
    c2 = static_cast<uint32_t>(a >> 32) ^ c3 ^ k1;
    c3 = static_cast<uint32_t>(a);
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return {{c0, c1, c2, c3}};
}

}  // namespace

template <typename T, typename TO, bool RES, bool ONCE>
__global__ __launch_bounds__(256) void k_dropout(DropArgs a) {
  const T* x = static_cast<const T*>(a.x);
  const TO* res = static_cast<const TO*>(a.residual);
  TO* y = static_cast<TO*>(a.y);
  const uint32_t step = a.step_ptr ? static_cast<uint32_t>(*a.step_ptr) : a.step;
  const long blocks = (a.n + 7) / 8, stride = static_cast<long>(gridDim.x) * 256;
  for (long i = static_cast<long>(blockIdx.x) * 256 + threadIdx.x; i < blocks; i += stride) {
    const int n = static_cast<int>(min(8l, a.n - 8 * i));
    Raw<T, 8> v;
    Raw<TO, 8> r;
    v.template load<ONCE>(x + 8 * i, n);
    if (RES) r.template load<ONCE>(res + 8 * i, n);
    const Words w = philox(a.block0 + i, step, a.key0, a.key1);
    float o[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t bits = e & 1 ? w.w[e / 2] >> 16 : w.w[e / 2] & 0xFFFFu;
      o[e] = bits >= a.threshold ? v.at(e) * a.scale : 0.f;
      if (RES) o[e] += r.at(e);
    }
    vec::store(y + 8 * i, o, n);
  }
}

uint32_t dropout_threshold(double p) { return static_cast<uint32_t>(p * 65536.0 + 0.5); }

hipError_t launch_dropout(const void* x, int x_dtype, int64_t n, uint32_t threshold, uint64_t seed, uint64_t offset,
                          uint32_t step, const int32_t* step_ptr, const void* residual, void* y, int y_dtype,
                          hipStream_t st) {
  DropArgs a{};
  a.n = n;
  a.x = x;
  a.residual = residual;
  a.y = y;
  a.block0 = offset / 8;
  a.key0 = static_cast<uint32_t>(seed);
  a.key1 = static_cast<uint32_t>(seed >> 32);
  a.threshold = threshold;
  a.step = step;
  a.step_ptr = step_ptr;
  a.scale = static_cast<float>(65536.0 / (65536.0 - threshold));
  const bool once = vec::streams(static_cast<size_t>(n) * ((x_dtype == MOL_BF16 ? 2 : 4) + (residual ? (y_dtype == MOL_BF16 ? 2 : 4) : 0)));
  const unsigned grid = static_cast<unsigned>(std::min<int64_t>((n + 2047) / 2048, 1 << 20));
  auto go = [&](auto t, auto to) {
    using T = decltype(t);
    using TO = decltype(to);
    auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(grid), dim3(256), 0, st, a); };
    if (residual)
      once ? run(k_dropout<T, TO, true, true>) : run(k_dropout<T, TO, true, false>);
    else
      once ? run(k_dropout<T, TO, false, true>) : run(k_dropout<T, TO, false, false>);
    return hipGetLastError();
  };
  if (x_dtype == MOL_BF16) return y_dtype == MOL_BF16 ? go(bf16_t{}, bf16_t{}) : go(bf16_t{}, 0.f);
  return y_dtype == MOL_BF16 ? go(0.f, bf16_t{}) : go(0.f, 0.f);
}

}  // namespace mol
