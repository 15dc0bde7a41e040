// One AdamW step over many tensors (decoupled weight decay), with float32 or
// 8-bit states:
//   m' = beta1 m + (1 - beta1) g',  v' = beta2 v + (1 - beta2) g'^2,
//   p' = p (1 - lr wd) - lr (m' / bc1) / (sqrt(v' / bc2) + eps).
//
// Bound by memory: every buffer is read or written once (28 bytes an element in
// float32, 16 with 8-bit states, bf16 gradients and a bf16 copy): 3 M elements of
// 24 float32 tensors in 16 us (5.2 TB/s), 173 M with 8-bit states in 520 us (5.3 TB/s,
// a copy runs at 4.6); with step and rate on the GPU 17 and 524.  A launch takes up to kMaxTensors tensors, described in
// its arguments; workgroups have chunks of kChunk elements, found by a search
// over the tensors' first chunks.  A wave has 256 elements, one block
// of an 8-bit state, at a time, four a lane: the block's largest magnitude is a
// reduction in registers, and the loads of its kChunk / 1024 blocks are issued together.
//
// 8-bit states hold e4m3 codes of m and of sqrt(v) (whose range is half of
// v's in powers of two) relative to the largest of 256, 2^-9 / 448 of it at the
// least.  The rounding is stochastic, by adding 16 random bits below the last
// one that is kept: a mix of 32 bits of the element's place, the seed and the step.
#include <algorithm>
#include <cmath>

#include "mol_tile.h"

namespace mol {

using namespace tile;

namespace {

constexpr int kMaxTensors = 30;      // descriptors of a launch: 3.9 KB of arguments
constexpr int kRounds = 4;           // blocks of 256 a wave takes
constexpr int kChunk = 1024 * kRounds;

struct AdamwDesc {
  long n;
  const void *p, *g, *m, *v;
  const float *m_scale, *v_scale;
  void *p_out, *m_out, *v_out;
  float *m_scale_out, *v_scale_out;
  void* copy_out;
  float weight_decay;
  uint32_t rng_lo, rng_hi;
  uint16_t form;                     // bits: 0 bf16 parameter, 1 bf16 gradient, 2 8-bit states
  uint16_t vec;                      // every buffer allows loads of four elements
};

struct AdamwArgs {
  int count;
  int first[kMaxTensors + 1];        // first chunk of each tensor
  float beta1, one_beta1, beta2, one_beta2, eps;
  float lr, step_size, root;         // step_size = lr / bc1, root = 1 / sqrt(bc2)
  double log_beta1, log_beta2;
  uint32_t seed, mixed;              // mixed: of seed and step
  const float* grad_scale;
  const float* lr_ptr;
  const int32_t* step_ptr;
  AdamwDesc t[kMaxTensors];
};
static_assert(sizeof(AdamwArgs) <= 4096, "kernel arguments");

// A 32-bit mix: shifts and multipliers that C. Wellons published in 2018, from a search
// for the least bias of two multiplications.  The other odd factors spread the step
// (2^32 over the golden ratio) and the place's high word (from A. Appleby's public-domain hash, 2011).
__host__ __device__ inline uint32_t mix32(uint32_t x) {
  x = (x ^ (x >> 16)) * 0x7FEB352Du;
  x = (x ^ (x >> 15)) * 0x846CA68Bu;
  return x ^ (x >> 16);
}
__host__ __device__ inline uint32_t mix_seed(uint32_t seed, uint32_t step) { return mix32(seed ^ step * 0x9E3779B9u); }

// Four elements from `i` on, zeros from n on.
template <typename T>
__device__ __forceinline__ void load4(const void* base, long i, long n, bool vec, float (&x)[4]) {
  const T* p = static_cast<const T*>(base) + i;
  if (vec && i + 4 <= n) {
    if constexpr (sizeof(T) == 4) {
      const float4 v = *reinterpret_cast<const float4*>(p);
      x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
    } else {
      const uint2 v = *reinterpret_cast<const uint2*>(p);
      x[0] = __uint_as_float(v.x << 16);
      x[1] = __uint_as_float(v.x & 0xFFFF0000u);
      x[2] = __uint_as_float(v.y << 16);
      x[3] = __uint_as_float(v.y & 0xFFFF0000u);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = i + e < n ? to_f32(p[e]) : 0.f;
  }
}
__device__ __forceinline__ uint32_t load_codes(const void* base, long i, long n, bool vec) {
  const uint8_t* p = static_cast<const uint8_t*>(base) + i;
  if (vec && i + 4 <= n) return *reinterpret_cast<const uint32_t*>(p);
  uint32_t c = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (i + e < n) c |= static_cast<uint32_t>(p[e]) << (8 * e);
  return c;
}
__device__ __forceinline__ void store_f32(void* base, long i, long n, bool vec, const float (&x)[4]) {
  float* p = static_cast<float*>(base) + i;
  if (vec && i + 4 <= n) {
    *reinterpret_cast<float4*>(p) = float4{x[0], x[1], x[2], x[3]};
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (i + e < n) p[e] = x[e];
  }
}
__device__ __forceinline__ void store_bf16(void* base, long i, long n, bool vec, const float (&x)[4]) {
  bf16_t* p = static_cast<bf16_t*>(base) + i;
  const uint2 w = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
  if (vec && i + 4 <= n) {
    *reinterpret_cast<uint2*>(p) = w;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (i + e < n) p[e] = static_cast<bf16_t>((e < 2 ? w.x : w.y) >> (16 * (e & 1)));
  }
}
__device__ __forceinline__ void store_codes(void* base, long i, long n, bool vec, uint32_t c) {
  uint8_t* p = static_cast<uint8_t*>(base) + i;
  if (vec && i + 4 <= n) {
    *reinterpret_cast<uint32_t*>(p) = c;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (i + e < n) p[e] = static_cast<uint8_t>(c >> (8 * e));
  }
}

// largest magnitude of a wave from each lane's, as bits (ordered as the numbers
// are, NaN above all), in all lanes
template <int ROR>
__device__ __forceinline__ uint32_t ror_bits(uint32_t v) {
  return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), 0x120 + ROR, 0xf, 0xf, true));
}
__device__ __forceinline__ float wave_top(uint32_t v) {
  v = max(v, ror_bits<8>(v));
  v = max(v, ror_bits<4>(v));
  v = max(v, ror_bits<2>(v));
  v = max(v, ror_bits<1>(v));
  const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = max(a[0], a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return __uint_as_float(max(b[0], b[1]));
}

// the four values of a word of codes
__device__ __forceinline__ void decode(uint32_t c, float scale, float (&x)[4]) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(c, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(c, true);
  x[0] = lo[0] * scale;
  x[1] = lo[1] * scale;
  x[2] = hi[0] * scale;
  x[3] = hi[1] * scale;
}

// codes of a block's four values a lane, and its scale (448 / top overflows
// for a top below 2^-119: such a block is stored as zeros).  The conversion adds the top bits of r below the last bit that it keeps
// and cuts the rest off: up with the chance r16 / 2^16 of what is cut off, also
// among the subnormal codes.
template <bool POSITIVE>
__device__ __forceinline__ uint32_t encode4(const float (&x)[4], const uint32_t (&r)[4], float top, float& scale) {
  const bool some = top > 0x1p-119f && top <= 3.4e38f;        // (false for NaN)
  scale = some ? top * (1.f / 448.f) : top <= 0x1p-119f ? 0.f : __builtin_nanf("");
  const float rt = __builtin_amdgcn_rcpf(top), q = 448.f * rt, inv = fmaf(fmaf(-q, top, 448.f), rt, q);   // 448 / top
  float y[4];
#pragma unroll
  for (int e = 0; e < 4; ++e)
    y[e] = __builtin_amdgcn_fmed3f(x[e] * inv, POSITIVE ? (x[e] > 0.f ? 0x1p-9f : 0.f) : -448.f, 448.f);
  int c = __builtin_amdgcn_cvt_sr_fp8_f32(y[0], r[0], 0, 0);
  c = __builtin_amdgcn_cvt_sr_fp8_f32(y[1], r[1], c, 1);
  c = __builtin_amdgcn_cvt_sr_fp8_f32(y[2], r[2], c, 2);
  c = __builtin_amdgcn_cvt_sr_fp8_f32(y[3], r[3], c, 3);
  return some ? static_cast<uint32_t>(c) : 0;
}

// sqrt(v) of v >= 0.  The hardware's root takes numbers below 2^-126 for 0, and a
// gradient of 1e-19 leaves a v of 1e-41: small ones are taken 2^64 times as large.
// EXACT (the root is stored): the last bit put right by one step from the reciprocal root.
template <bool EXACT>
__device__ __forceinline__ float root_of(float v) {
  const bool small = v < 0x1p-96f;
  const float x = small ? v * 0x1p64f : v;
  float r;
  if constexpr (EXACT) {
    const float y = __builtin_amdgcn_rsqf(fmaxf(x, 0x1p-126f)), t = x * y;
    r = fmaf(fmaf(-t, t, x), 0.5f * y, t);
  } else {
    r = __builtin_amdgcn_sqrtf(x);
  }
  return small ? r * 0x1p-32f : r;
}

struct Rates {
  float decay_lr, step_size, root;
  uint32_t mixed;
};

// One chunk of a tensor.
template <typename TP, typename TG, bool E8>
__device__ __forceinline__ void step_chunk(const AdamwArgs& a, const AdamwDesc& t, const Rates& rt, float gs, long c0) {
#pragma clang fp contract(off)
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const float keep = 1.f - rt.decay_lr * t.weight_decay;
  const bool vec = t.vec;
  float p[kRounds][4], g[kRounds][4], m[E8 ? 1 : kRounds][4], v[E8 ? 1 : kRounds][4];
  uint32_t mc[kRounds], vc[kRounds];
  float ms[kRounds], vs[kRounds];
#pragma unroll
  for (int k = 0; k < kRounds; ++k) {
    const long i = c0 + (k * 4 + wave) * 256 + lane * 4;
    load4<TP>(t.p, i, t.n, vec, p[k]);
    load4<TG>(t.g, i, t.n, vec, g[k]);
    if constexpr (E8) {
      mc[k] = load_codes(t.m, i, t.n, vec);
      vc[k] = load_codes(t.v, i, t.n, vec);
      const bool any = i < t.n;
      ms[k] = any ? t.m_scale[i >> 8] : 0.f;
      vs[k] = any ? t.v_scale[i >> 8] : 0.f;
    } else {
      load4<float>(t.m, i, t.n, vec, m[k]);
      load4<float>(t.v, i, t.n, vec, v[k]);
    }
  }
#pragma unroll
  for (int k = 0; k < kRounds; ++k) {
    const long i0 = c0 + (k * 4 + wave) * 256, i = i0 + lane * 4;
    if (i0 >= t.n) break;                                     // (a wave's own block)
    float mk[4], vk[4], root[4];
    if constexpr (E8) {
      decode(mc[k], ms[k], mk);
      decode(vc[k], vs[k], vk);
    }
    uint32_t top_m = 0, top_v = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float gg = g[k][e] * gs;
      const float m0 = E8 ? mk[e] : m[E8 ? 0 : k][e], v0 = E8 ? vk[e] * vk[e] : v[E8 ? 0 : k][e];
      mk[e] = a.beta1 * m0 + a.one_beta1 * gg;
      vk[e] = a.beta2 * v0 + a.one_beta2 * gg * gg;
      root[e] = root_of<E8>(vk[e]);
      const float x = rt.step_size * mk[e] * __builtin_amdgcn_rcpf(fmaf(root[e], rt.root, a.eps));
      p[k][e] = p[k][e] * keep - x;
      if constexpr (E8) {
        top_m = max(top_m, __float_as_uint(mk[e]) & 0x7FFFFFFFu);
        top_v = max(top_v, __float_as_uint(root[e]) & 0x7FFFFFFFu);
      }
    }
    if constexpr (sizeof(TP) == 4)
      store_f32(t.p_out, i, t.n, vec, p[k]);
    else
      store_bf16(t.p_out, i, t.n, vec, p[k]);
    if (t.copy_out) store_bf16(t.copy_out, i, t.n, vec, p[k]);
    if constexpr (E8) {
      uint32_t rm[4], rv[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        // the element's place, 64 bits: the high word moves the seed
        const uint64_t at = (static_cast<uint64_t>(t.rng_hi) << 32 | t.rng_lo) + static_cast<uint64_t>(i + e);
        const uint32_t h = mix32(static_cast<uint32_t>(at) ^ rt.mixed ^ static_cast<uint32_t>(at >> 32) * 0x85EBCA6Bu);
        rm[e] = h << 16;
        rv[e] = h & 0xFFFF0000u;
      }
      float sm, sv;
      const uint32_t cm = encode4<false>(mk, rm, wave_top(top_m), sm);
      const uint32_t cv = encode4<true>(root, rv, wave_top(top_v), sv);
      store_codes(t.m_out, i, t.n, vec, cm);
      store_codes(t.v_out, i, t.n, vec, cv);
      if (lane == 0) {
        t.m_scale_out[i0 >> 8] = sm;
        t.v_scale_out[i0 >> 8] = sv;
      }
    } else {
      store_f32(t.m_out, i, t.n, vec, mk);
      store_f32(t.v_out, i, t.n, vec, vk);
    }
  }
}

}  // namespace

__global__ __launch_bounds__(256) void k_adamw(AdamwArgs a) {
  const int chunk = blockIdx.x;
  int lo = 0, hi = a.count;                       // first[lo] <= chunk < first[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (a.first[mid] <= chunk) lo = mid; else hi = mid;
  }
  const AdamwDesc& t = a.t[lo];
  const float gs = a.grad_scale ? *a.grad_scale : 1.f;
  Rates rt{a.lr, a.step_size, a.root, a.mixed};
  if (a.lr_ptr || a.step_ptr) {
    // rates of a step whose number or rate is known only on the device
    __shared__ Rates sh;
    if (threadIdx.x == 0) {
      const float lr = a.lr_ptr ? *a.lr_ptr : a.lr;
      sh = rt;
      if (a.step_ptr) {
        const int step = max(*a.step_ptr, 1);
        sh.step_size = static_cast<float>(static_cast<double>(lr) / -expm1(step * a.log_beta1));
        sh.root = static_cast<float>(1.0 / sqrt(-expm1(step * a.log_beta2)));
        sh.mixed = mix_seed(a.seed, static_cast<uint32_t>(step));
      } else {
        sh.step_size = a.step_size * lr;          // (step_size: 1 / bc1 where lr_ptr is given)
      }
      sh.decay_lr = lr;
    }
    __syncthreads();
    rt = sh;
  }
  const long c0 = static_cast<long>(chunk - a.first[lo]) * kChunk;
  switch (t.form) {
    case 0: step_chunk<float, float, false>(a, t, rt, gs, c0); break;
    case 1: step_chunk<bf16_t, float, false>(a, t, rt, gs, c0); break;
    case 2: step_chunk<float, bf16_t, false>(a, t, rt, gs, c0); break;
    case 3: step_chunk<bf16_t, bf16_t, false>(a, t, rt, gs, c0); break;
    case 4: step_chunk<float, float, true>(a, t, rt, gs, c0); break;
    case 5: step_chunk<bf16_t, float, true>(a, t, rt, gs, c0); break;
    case 6: step_chunk<float, bf16_t, true>(a, t, rt, gs, c0); break;
    default: step_chunk<bf16_t, bf16_t, true>(a, t, rt, gs, c0); break;
  }
}

static uint16_t allows_vec(const mol_adamw_tensor& t) {
  auto bits = [](const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n; };
  const size_t np = t.param_dtype == MOL_BF16 ? 8 : 16, ng = t.grad_dtype == MOL_BF16 ? 8 : 16;
  const size_t ns = t.state == MOL_STATE_E4M3 ? 4 : 16;
  return !(bits(t.p, np) | bits(t.p_out, np) | bits(t.g, ng) | bits(t.m, ns) | bits(t.v, ns) | bits(t.m_out, ns) |
           bits(t.v_out, ns) | bits(t.copy_out, 8));
}

hipError_t launch_adamw(const mol_adamw& o, const mol_adamw_tensor* tensors, int n_tensors, hipStream_t st) {
  const double bc1 = 1.0 - std::pow(o.beta1, o.step), bc2 = 1.0 - std::pow(o.beta2, o.step);
  for (int at = 0; at < n_tensors;) {
    AdamwArgs a;
    a.beta1 = static_cast<float>(o.beta1);
    a.one_beta1 = static_cast<float>(1.0 - o.beta1);     // (in float32 1 - 0.999f is off by 5e-5 of itself)
    a.beta2 = static_cast<float>(o.beta2);
    a.one_beta2 = static_cast<float>(1.0 - o.beta2);
    a.eps = static_cast<float>(o.eps);
    a.lr = static_cast<float>(o.lr);
    a.step_size = static_cast<float>((o.lr_ptr ? 1.0 : o.lr) / bc1);
    a.root = static_cast<float>(1.0 / std::sqrt(bc2));
    a.log_beta1 = std::log(o.beta1);                     // (-inf for 0: expm1 gives -1)
    a.log_beta2 = std::log(o.beta2);
    a.seed = o.seed;
    a.mixed = mix_seed(o.seed, static_cast<uint32_t>(o.step));
    a.grad_scale = o.grad_scale;
    a.lr_ptr = o.lr_ptr;
    a.step_ptr = o.step_ptr;
    a.count = 0;
    long chunks = 0;
    for (; at < n_tensors && a.count < kMaxTensors; ++at) {
      const mol_adamw_tensor& t = tensors[at];
      if (t.n == 0) continue;
      const long more = (t.n + kChunk - 1) / kChunk;
      if (a.count && chunks + more > (1l << 23)) break;   // (a grid holds 2^32 threads)
      AdamwDesc& d = a.t[a.count];
      d = AdamwDesc{t.n, t.p, t.g, t.m, t.v, t.m_scale, t.v_scale, t.p_out, t.m_out, t.v_out, t.m_scale_out,
                    t.v_scale_out, t.copy_out, t.weight_decay, static_cast<uint32_t>(t.rng_offset),
                    static_cast<uint32_t>(t.rng_offset >> 32), 0, allows_vec(t)};
      d.form = (t.param_dtype == MOL_BF16) | (t.grad_dtype == MOL_BF16) << 1 | (t.state == MOL_STATE_E4M3) << 2;
      a.first[a.count++] = static_cast<int>(chunks);
      chunks += more;
    }
    a.first[a.count] = static_cast<int>(chunks);
    if (chunks == 0) continue;
    hipLaunchKernelGGL(k_adamw, dim3(static_cast<unsigned>(chunks)), dim3(256), 0, st, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace mol
