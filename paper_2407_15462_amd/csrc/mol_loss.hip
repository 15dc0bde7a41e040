// Sampled-softmax loss of dense score rows and its gradient (Eq. 4):
//   z_i = inv_temp phi_i,  loss = log sum_kept e^{z_i} - z_t,
//   dphi_i = weight inv_temp (e^{z_i} / sum - [i = t]).
// Column i is kept unless its id is negative or it repeats the positive's id.
//
// Bound by memory: a row is read once and written once.  A workgroup holds a
// whole row in registers, kRegs values a thread (64, 256 or 1024 threads: rows
// of up to 2176, 8704 or 34,816 columns), in few enough of them that two
// workgroups of 1024 share a CU and one's loads run under the other's stores.
// Longer rows are cut into parts, whose maxima and sums a first launch
// leaves in the workspace and a second one joins, reading the row again (from
// the last-level cache where the batch's scores fit it).  Rows start at any
// element, so that loads are 4 bytes a lane, kRegs of them in flight.
// Measured: 1024 rows of 32,771 take 70 us (3.8 TB/s; a copy of as much 59),
// 128 rows of 128 5 us, of a call's 10.  Rows in parts: 128 of 100,003 42 + 46 us, 1024 of
// 65,537 147 + 203 (a copy of as much: 22 and 118).
// Maximum, sum and loss are float32.
#include <algorithm>

#include "mol_kernels.h"

namespace mol {

namespace {

constexpr int kRegs = 34;
constexpr float kLog2E = 1.4426950408889634f, kLog2ELo = 1.925963033500e-8f, kLn2 = 0.6931471805599453f;

// e^x, x <= 0: 2^t with t = x log2(e) in two parts, since float32's rounding of
// t alone is an error of |t| 2^-24 in the result
__device__ __forceinline__ float exp_neg(float x) {
  const float t = x * kLog2E;
  const float r = fmaf(x, kLog2ELo, fmaf(x, kLog2E, -t));
  const float e = __builtin_amdgcn_exp2f(t);
  return e == 0.f ? 0.f : fmaf(e, r * kLn2, e);   // (0 for x = -inf, whose r is NaN)
}

// e^{z - m}; 0 for z = -inf, also where the whole row is (its sum is then 0, its loss NaN)
__device__ __forceinline__ float weight(float z, float m) { return z == -__builtin_inff() ? 0.f : exp_neg(z - m); }

__device__ __forceinline__ float wave_max(float v) {
  for (int o = 32; o; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
  return v;
}
__device__ __forceinline__ float wave_sum(float v) {
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
  return v;
}
template <int NT>
__device__ __forceinline__ float block_max(float v, float* sh) {
  v = wave_max(v);
  if constexpr (NT > 64) {
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
    __syncthreads();
    v = sh[0];
    for (int i = 1; i < NT / 64; ++i) v = fmaxf(v, sh[i]);
    __syncthreads();
  }
  return v;
}
template <int NT>
__device__ __forceinline__ float block_sum(float v, float* sh) {
  v = wave_sum(v);
  if constexpr (NT > 64) {
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
    __syncthreads();
    v = sh[0];
    for (int i = 1; i < NT / 64; ++i) v += sh[i];
    __syncthreads();
  }
  return v;
}

struct LossArgs {
  int B, N;
  const float* phi;          // dphi may be the same buffer
  const int32_t* target;
  const int32_t* ids;
  float inv_temp;
  const float* row_weight;
  float* loss;
  float* dphi;
  int parts, part_len;       // long rows
  float* ws;                 // [B][parts][2] maxima and sums, then [B] z_t
};

struct Row {
  int t;                     // the positive's column
  int32_t tid;               // its id
  bool dead;                 // no positive: loss and gradient are zero
};
__device__ __forceinline__ Row row_of(const LossArgs& a, int b) {
  Row r;
  r.t = a.target[b];
  r.dead = static_cast<uint32_t>(r.t) >= static_cast<uint32_t>(a.N);
  r.tid = 0;
  if (!r.dead && a.ids) {
    r.tid = a.ids[r.t];
    r.dead = r.tid < 0;
  }
  return r;
}
__device__ __forceinline__ bool kept(const LossArgs& a, const Row& r, int i) {
  if (!a.ids) return true;
  const int32_t id = a.ids[i];
  return id >= 0 && (i == r.t || id != r.tid);
}

}  // namespace

// One workgroup a row.  A left-out column is held as -inf: its exponential is 0,
// and a gradient whose exponential is 0 is written as 0 whatever the row's sum is.
template <int NT>
__global__ __launch_bounds__(NT, NT == 1024 ? 8 : 4) void k_softmax_loss(LossArgs a) {
  __shared__ float sh[NT / 64];
  const int b = blockIdx.x, tid = threadIdx.x;
  const long at = static_cast<long>(b) * a.N;
  const float* phi = a.phi + at;
  float* out = a.dphi ? a.dphi + at : nullptr;
  const Row r = row_of(a, b);
  if (r.dead) {
    if (out)
      for (int i = tid; i < a.N; i += NT) out[i] = 0.f;
    if (a.loss && tid == 0) a.loss[b] = 0.f;
    return;
  }
  const float zt = a.inv_temp * phi[r.t];
  // columns k NT + tid for the k < full, and one of the rest
  const int full = a.N / NT, il = full * NT + tid;
  const bool rest = il < a.N;
  float z[kRegs], zl = -__builtin_inff();
#pragma unroll
  for (int k = 0; k < kRegs; ++k)
    if (k < full) z[k] = phi[k * NT + tid];
  if (rest) zl = phi[il];
  float m = -__builtin_inff();
#pragma unroll
  for (int k = 0; k < kRegs; ++k)
    if (k < full) {
      z[k] = kept(a, r, k * NT + tid) ? a.inv_temp * z[k] : -__builtin_inff();
      m = fmaxf(m, z[k]);
    }
  if (rest) {
    zl = kept(a, r, il) ? a.inv_temp * zl : -__builtin_inff();
    m = fmaxf(m, zl);
  }
  m = block_max<NT>(m, sh);
  zl = weight(zl, m);
  float s = zl;                                            // (a NaN, which the maximum passes over, shows here)
#pragma unroll
  for (int k = 0; k < kRegs; ++k)
    if (k < full) {
      z[k] = weight(z[k], m);
      s += z[k];
    }
  s = block_sum<NT>(s, sh);
  if (a.loss && tid == 0) a.loss[b] = logf(s) + (m - zt);
  if (!out) return;
  const float w = (a.row_weight ? a.row_weight[b] : 1.f) * a.inv_temp, q = 1.f / s;
  auto grad = [&](int i, float e) { return i == r.t ? w * (e * q - 1.f) : e == 0.f ? 0.f : w * (e * q); };
#pragma unroll
  for (int k = 0; k < kRegs; ++k)
    if (k < full) out[k * NT + tid] = grad(k * NT + tid, z[k]);
  if (rest) out[il] = grad(il, zl);
}

// Long rows, first launch: maximum and sum of part blockIdx.x of row blockIdx.y.
__global__ __launch_bounds__(256) void k_softmax_part(LossArgs a) {
  __shared__ float sh[4];
  const int b = blockIdx.y, tid = threadIdx.x;
  const float* phi = a.phi + static_cast<long>(b) * a.N;
  const Row r = row_of(a, b);
  if (r.dead) return;
  const int i0 = blockIdx.x * a.part_len, i1 = min(a.N - i0, a.part_len) + i0;
  float m = -__builtin_inff(), s = 0.f;                    // of this thread's columns
  constexpr int U = 8;
  for (long base = i0; base < i1; base += U * 256) {
    float v[U], top = m;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long i = base + u * 256 + tid;
      v[u] = -__builtin_inff();
      if (i < i1 && kept(a, r, static_cast<int>(i))) v[u] = a.inv_temp * phi[i];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) top = fmaxf(top, v[u]);
    if (top > m) {
      s *= exp_neg(m - top);
      m = top;
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      s += weight(v[u], m);                                     // (NaN is not passed over)
  }
  const float all = block_max<256>(m, sh);
  // (a part of nothing but -inf has the sum 0)
  s = block_sum<256>(m == -__builtin_inff() && !(s != s) ? 0.f : s * exp_neg(m - all), sh);
  if (tid == 0) {
    float* dst = a.ws + (static_cast<long>(b) * a.parts + blockIdx.x) * 2;
    dst[0] = all;
    dst[1] = s;
    if (blockIdx.x == 0) a.ws[2l * a.B * a.parts + b] = a.inv_temp * phi[r.t];
  }
}

// Second launch: joins the parts of its row, writes its part's gradient.
__global__ __launch_bounds__(256) void k_softmax_join(LossArgs a) {
  __shared__ float sh[4];
  const int b = blockIdx.y, tid = threadIdx.x;
  const long at = static_cast<long>(b) * a.N;
  const Row r = row_of(a, b);
  const int i0 = blockIdx.x * a.part_len, i1 = min(a.N - i0, a.part_len) + i0;
  if (r.dead) {
    if (a.dphi)
      for (long i = i0 + tid; i < i1; i += 256) a.dphi[at + i] = 0.f;
    if (a.loss && blockIdx.x == 0 && tid == 0) a.loss[b] = 0.f;
    return;
  }
  const float* part = a.ws + static_cast<long>(b) * a.parts * 2;
  float m = -__builtin_inff(), s = 0.f;
  for (int k = tid; k < a.parts; k += 256) m = fmaxf(m, part[2 * k]);
  m = block_max<256>(m, sh);
  for (int k = tid; k < a.parts; k += 256) {
    const float pm = part[2 * k], ps = part[2 * k + 1];
    s += pm == -__builtin_inff() && ps == 0.f ? 0.f : ps * exp_neg(pm - m);
  }
  s = block_sum<256>(s, sh);
  if (a.loss && blockIdx.x == 0 && tid == 0) a.loss[b] = logf(s) + (m - a.ws[2l * a.B * a.parts + b]);
  if (!a.dphi) return;
  const float w = (a.row_weight ? a.row_weight[b] : 1.f) * a.inv_temp, q = 1.f / s;
  constexpr int U = 8;
  for (long base = i0; base < i1; base += U * 256) {
    float v[U];
    uint32_t keep = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long i = base + u * 256 + tid;
      v[u] = 0.f;
      if (i < i1) {
        v[u] = a.phi[at + i];
        keep |= static_cast<uint32_t>(kept(a, r, static_cast<int>(i))) << u;
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long i = base + u * 256 + tid;
      if (i >= i1) continue;
      const float e = (keep >> u) & 1 ? weight(a.inv_temp * v[u], m) : 0.f;
      a.dphi[at + i] = i == r.t ? w * (e * q - 1.f) : e == 0.f ? 0.f : w * (e * q);
    }
  }
}

// ---------------------------------------------------------------------------
namespace {

// A row's parts: none where one workgroup holds it; else parts of about 8192
// columns, fewer and longer ones where the batch fills the card anyway.
int loss_parts(int B, int N) {
  if (N <= 1024 * kRegs) return 1;
  const long most = (N + 8191l) / 8192, want = (1024l + B - 1) / B;
  return static_cast<int>(std::max<long>(2, std::min(most, want)));
}

}  // namespace

size_t softmax_loss_bytes(int B, int N) {
  const int parts = loss_parts(B, N);
  return parts == 1 ? 0 : (4ul * B * (2ul * parts + 1) + 255) / 256 * 256;
}

// the most of up to B rows of up to N columns: rows of ceil(1024 / B) parts, of which B times
// as many pass 1024 by up to B - 1, two at least and one for 8192 columns at most
size_t softmax_loss_most(int B, int N) {
  if (N <= 1024 * kRegs) return 0;
  const size_t b = B, parts = std::max(2 * b, std::min(b * ((N + 8191ul) / 8192), 1023 + b));
  return (4 * (2 * parts + b) + 255) / 256 * 256;
}

hipError_t launch_softmax_loss(int B, int N, const float* phi, const int32_t* target, const int32_t* ids,
                               float inv_temp, const float* row_weight, float* loss, float* dphi, void* ws,
                               hipStream_t st) {
  LossArgs a{B, N, phi, target, ids, inv_temp, row_weight, loss, dphi, loss_parts(B, N), 0, static_cast<float*>(ws)};
  if (a.parts == 1) {
    if (N <= 64 * kRegs)
      hipLaunchKernelGGL(k_softmax_loss<64>, dim3(B), dim3(64), 0, st, a);
    else if (N <= 256 * kRegs)
      hipLaunchKernelGGL(k_softmax_loss<256>, dim3(B), dim3(256), 0, st, a);
    else
      hipLaunchKernelGGL(k_softmax_loss<1024>, dim3(B), dim3(1024), 0, st, a);
    return hipGetLastError();
  }
  a.part_len = static_cast<int>((static_cast<long>(N) + a.parts - 1) / a.parts);
  a.parts = static_cast<int>((static_cast<long>(N) + a.part_len - 1) / a.part_len);   // (none of them empty)
  hipLaunchKernelGGL(k_softmax_part, dim3(a.parts, B), dim3(256), 0, st, a);
  hipLaunchKernelGGL(k_softmax_join, dim3(a.parts, B), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace mol
