// Gradient of the MoL scores (Eq. 1 / Eq. 2 with the gating MLP of Appendix
// A.3) for every input, any supported shape and both storage types, in float32
// throughout: bf16 outputs are rounded once, at the end.
//
// With g = dphi, per pair (query, item):
//   dl_p = g pi_p (s_p - phi)             dh = W2^T dl
//   du   = dh sig (1 + u (1 - sig))       ds = g pi + W1^T du
// and sums of dl, du, du s^T, dl h^T, ds X and ds Q over pairs.
//
// 1. k_score_grad recomputes the chain and goes back through it.  A workgroup
//    of 8 waves has TI items and walks over blocks of QB queries, QB TI = 128
//    pairs: the waves form the tile's dot products (as k_mol_f32 does) in LDS,
//    then each wave takes 16 items of one query through the chain on 16x16x4
//    f32 MFMAs.  Lane (c = lane % 16, g = lane / 16) holds item c's components
//    p = RUN g + mu, mu < RUN = PV / 4, the layout in which s, dl (K = p) and
//    h, du (K = j, four hidden units of each 16) are B operands as they stand,
//    so that the four products with W1, W2 and their transposes exchange
//    nothing between lanes.  dW1 = sum du s^T and dW2 = sum dl h^T have K = the
//    items: s and dl are read back from LDS, h and du go through a small block
//    of the wave's, four items a lane.  The two sums stay in registers for the
//    whole walk (JTG blocks of 16 hidden units; a wider MLP takes a launch for
//    every JTG blocks, of which only the first writes ds, da_q and da_x), as
//    does da_x.  The workgroup's sums go to the workspace.
// 2. ds goes there too, [Px][B Pq][items], as float32, and k_grad_products forms
//    dQ = sum ds X and dX = sum ds Q on matrix cores from it, with rows of X and Q as
//    K, as they lie (bf16 problems: ds in three bf16 terms, which are exact).
// 3. k_sum_parts adds the partial sums in a fixed order.
// Items are taken in slabs, so that ds and what else grows with them stay within kSlabBytes.
//
// What bounds it: the f32 matrix rate, 12 P H + 2 P d flop a pair, and for few pairs
// the latencies of a workgroup's one or two tiles (weights, dot products, the
// chain and back, the sums: 50 us at P = H = 64).  Measured in float32: 32 x 129
// pairs of 4 x 4, H = 32 13 + 7 + 5 us (pairs, products, sums), 24 a call; 200 x 4000 of
// them 121 + 54 + 15 (pairs at 54 TFLOP/s, a large product at 144); 8 x 6112 of
// 8 x 8, H = 64 66 + 22 + 8.  In bf16: 128 x 1000 of 16 x 4, H = 64 112 + 24 + 11; 128 x 1000 of
// 8 x 8, H = 256, whose four groups of hidden units repeat the chain, 4 x 345 + 24 + 19;
// 1024 x 2048 of 8 x 8, H = 64 in two slabs of 698 + 111 + 19.
#include <algorithm>

#include "mol_grad.h"

namespace mol {

using namespace tile;
using namespace grad;

namespace {

constexpr int kWaves = 8, kThreads = 64 * kWaves, kPairs = 16 * kWaves;
constexpr int kSumFloats = kWaves * 2 * 4 * 256;     // of the waves' sums in LDS: four blocks of two matrices
// Of a slab's ds and partial sums: a million pairs of 64 components, whose
// ds alone is 268 MB (see the bf16 form).
constexpr size_t kSlabBytes = size_t(288) << 20;

// JTG, blocks of 16 hidden units whose sums a workgroup keeps.  Up to 64 units of up to 16
// components leave registers for a second workgroup on the CU (launch bounds of four waves
// a SIMD): one's dot products run beside the other's chain (200 x 4000: 161 -> 131 us).
template <int PV>
constexpr int group_tiles(bool few) { return PV == 64 || (PV == 16 && few) ? 4 : 8; }
template <int PV, int JTG>
constexpr int wgs_per_cu() { return PV == 16 && JTG == 4 ? 2 : 1; }

__device__ __forceinline__ f32x4_t mfma_f32(float a, float b, f32x4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4_t mfma_f32x4(float4 a, float4 b, f32x4_t c) {
  c = mfma_f32(a.x, b.x, c);
  c = mfma_f32(a.y, b.y, c);
  c = mfma_f32(a.z, b.z, c);
  return mfma_f32(a.w, b.w, c);
}

// 16 bytes (or their zero-padded tail) of a row of `d` elements from element t
template <typename T, bool VEC>
__device__ __forceinline__ uint4 row16(const T* row, int t, int d) {
  constexpr int E = 16 / sizeof(T);
  if constexpr (VEC) {
    const uint4 v = *reinterpret_cast<const uint4*>(row + min(t, d - E));
    return t < d ? v : make_uint4(0, 0, 0, 0);
  } else {
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const T x = row[min(t + e, d - 1)];
      uint32_t bits;
      if constexpr (sizeof(T) == 4) bits = __float_as_uint(x);
      else bits = x;
      if (t + e >= d) bits = 0;
      if constexpr (sizeof(T) == 4) w[e] = bits;
      else w[e / 2] |= bits << (16 * (e & 1));
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
}
template <typename T>
__device__ __forceinline__ f32x4_t mma16(uint4 a, uint4 b, f32x4_t c) {
  if constexpr (sizeof(T) == 4)
    return mfma_f32x4(__builtin_bit_cast(float4, a), __builtin_bit_cast(float4, b), c);
  else
    return mfma_bf16(a, b, c);
}

struct GradDims {
  int QB, upq_log2;        // queries of a tile, log2 of its 16-item units a query
  int TI, TIP;             // items of a tile, floats of an LDS row of s
  int n0, ns;              // the slab's first item, its items (a multiple of TI)
  int qsplits;             // query ranges: blockIdx.y
  int group;               // hidden units 16 JTG group .. of dW1, dW2
  long m;                  // B Pq
};

// Per-workgroup sums in the workspace.
struct GradParts {
  float* ds;               // [Px][B Pq][ns]
  float* da_q;             // [ns / 16][B][P]
  float* da_x;             // [qsplits][ns][P]
  float* dW1;              // [workgroups][H][P]
  float* dW2;              // [workgroups][P][H]
  float* db1;              // [workgroups][H]
  float* db2;              // [workgroups][P]
};

template <int PV>
constexpr int op_tiles() { return PV / 16; }   // 1 KB blocks of prepared weights per 16 hidden units and matrix

// floats of LDS; weights: the four prepared operand matrices, us: the units' u
template <int PV>
size_t grad_lds(int JT, bool weights, bool us, const GradDims& dm) {
  return (weights ? 4ul * JT * op_tiles<PV>() * 256 : 0) + 16ul * JT + dm.QB * PV + dm.TI * (PV + 4) +
         static_cast<size_t>(dm.QB) * PV * dm.TIP + (us ? 256ul * kWaves * JT : 0) + kWaves * 2 * 256 + PV + 256;
}

// prepared operands of 16x16x4 f32 MFMAs, 64 lanes x 4 floats a block:
// W1 and W2T (A operands with K = p), W2 and W1T (K = j), see k_mol_f32
template <typename T, int PV>
__device__ __forceinline__ float prepared(const T* W1, const T* W2, int P, int H, int which, int jt, int m, int lane,
                                          int e) {
  constexpr int RUN = PV / 4;
  const int c = lane & 15, g = lane >> 4;
  if (which < 2) {
    const int j = 16 * jt + c, p = RUN * g + 4 * m + e;
    if (j >= H || p >= P) return 0.f;
    return which == 0 ? to_f32(W1[j * P + p]) : to_f32(W2[p * H + j]);
  }
  const int p = RUN * (c >> 2) + 4 * m + (c & 3), j = 16 * jt + 4 * g + e;
  if (j >= H || p >= P) return 0.f;
  return which == 2 ? to_f32(W2[p * H + j]) : to_f32(W1[j * P + p]);
}

}  // namespace

// The four prepared matrices in the workspace, for MLPs too wide for LDS.
template <typename T, int PV>
__global__ __launch_bounds__(256) void k_grad_weights(DevProb pr, int JT, float* __restrict__ out) {
  const int i = blockIdx.x * 256 + threadIdx.x, per = JT * op_tiles<PV>() * 256;
  if (i >= 4 * per) return;
  const int which = i / per, r = i - which * per, e = r & 3, lane = (r >> 2) & 63, blk = r >> 8;
  out[i] = prepared<T, PV>(static_cast<const T*>(pr.W1), static_cast<const T*>(pr.W2), pr.P, pr.H, which,
                           blk / op_tiles<PV>(), blk % op_tiles<PV>(), lane, e);
}

template <typename T, int PV, bool VEC, int JTG>
__global__ __launch_bounds__(kThreads, (2 * wgs_per_cu<PV, JTG>())) void k_score_grad(DevProb pr, GradDims dm, const float* __restrict__ dphi,
                                                            const float* __restrict__ wglob,
                                                            float* __restrict__ uglob, GradParts out) {
  constexpr int RUN = PV / 4, PT = PV / 16, E = 16 / sizeof(T), KCH = 4 * E;
  extern __shared__ __attribute__((aligned(16))) float smf[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c = lane & 15, g = lane >> 4;
  const int P = pr.P, H = pr.H, d = pr.d, N = pr.N, JT = (H + 15) / 16;
  const int QB = dm.QB, TI = dm.TI, TIP = dm.TIP;
  const int wsize = JT * PT * 256;
  float* sW = smf;                                                     // prepared weights, or nothing
  float* sB1 = sW + (wglob ? 0 : 4 * wsize);
  float* sC = sB1 + 16 * JT;                                           // a_q + b2, -inf past P
  float* sAx = sC + QB * PV;
  float* sS = sAx + TI * (PV + 4);
  float* sU = sS + QB * PV * TIP + (wave * JT) * 256 + lane * 4;       // the lane's u, 16 bytes a block
  float* sT0 = sS + QB * PV * TIP + (uglob ? 0 : 256 * kWaves * JT);
  const long wg = static_cast<long>(blockIdx.y) * gridDim.x + blockIdx.x;
  float4* gU = reinterpret_cast<float4*>(uglob) + (wg * kWaves + wave) * JT * 64 + lane;   // the same, where LDS has no room
  float* sT = sT0 + wave * 512;                                        // du and h of 16 hidden units, [16][16 items] each
  uint32_t* sOff = reinterpret_cast<uint32_t*>(sT0 + kWaves * 512);    // ds offset of p
  int* sRow = reinterpret_cast<int*>(sOff + PV);                       // s row of each query vector (QB P_q <= 256)
  const float4* w1 = reinterpret_cast<const float4*>(wglob ? wglob : sW) + lane;
  const float4* w2t = w1 + wsize / 4;
  const float4* w2 = w2t + wsize / 4;
  const float4* w1t = w2 + wsize / 4;
  const T* X = static_cast<const T*>(pr.X);
  const T* Q = static_cast<const T*>(pr.Q);

  if (!wglob) {
#pragma unroll
    for (int which = 0; which < 4; ++which)
      for (int i = tid; i < wsize; i += kThreads) {
        const int blk = i >> 8;
        sW[which * wsize + i] = prepared<T, PV>(static_cast<const T*>(pr.W1), static_cast<const T*>(pr.W2), P, H, which,
                                                blk / PT, blk % PT, (i >> 2) & 63, i & 3);
      }
  }
  for (int i = tid; i < 16 * JT; i += kThreads) sB1[i] = i < H ? pr.b1[i] : 0.f;
  for (int i = tid; i < QB * PV * TIP; i += kThreads) sS[i] = 0.f;
  for (int i = tid; i < PV; i += kThreads)
    sOff[i] = i < P ? static_cast<uint32_t>((i % pr.Px * dm.m + i / pr.Px) * dm.ns) : 0xFFFFFFFFu;
  for (int i = tid; i < (QB * pr.Pq + 31) / 32 * 32; i += kThreads)
    sRow[i] = i < QB * pr.Pq ? (i / pr.Pq * PV + i % pr.Pq * pr.Px) * TIP : -1;
  const int i0 = blockIdx.x * TI;                                      // the tile's first item of the slab
  auto item_of = [&](int i) { return min(dm.n0 + i0 + i, N - 1); };
  for (int i = tid; i < TI * (PV + 4); i += kThreads) {
    const int n = i / (PV + 4), p = i - n * (PV + 4);
    sAx[i] = p < P ? pr.a_x[static_cast<long>(item_of(n)) * P + p] : 0.f;
  }

  const int q = wave >> dm.upq_log2, it = 16 * (wave & ((1 << dm.upq_log2) - 1)) + c;
  const int slot = i0 + it;                                            // of the slab
  const bool has_item = dm.n0 + slot < N;
  f32x4_t aw1[JTG][PT] = {}, aw2[JTG][PT] = {};
  float ab1[JTG] = {}, dax[RUN] = {};
  const int nqb = (pr.B + QB - 1) / QB;
  const int qb0 = static_cast<int>(static_cast<long>(nqb) * blockIdx.y / dm.qsplits);
  const int qb1 = static_cast<int>(static_cast<long>(nqb) * (blockIdx.y + 1) / dm.qsplits);
  for (int qb = qb0; qb < qb1; ++qb) {
    const int b0 = qb * QB, nq = min(QB, pr.B - b0);
    __syncthreads();                                                   // the previous tile's units are done
    for (int i = tid; i < QB * PV; i += kThreads) {
      const int p = i % PV, b = min(b0 + i / PV, pr.B - 1);
      sC[i] = p < P ? pr.a_q[static_cast<long>(b) * P + p] + pr.b2[p] : -__builtin_inff();
    }
    const int b = b0 + q;
    const bool live = q < nq && has_item;
    const float gr = live ? dphi[static_cast<long>(b) * N + dm.n0 + slot] : 0.f;
    // 1. dot products: jobs of (item component, 16 R items, 16 R vector rows)
    constexpr int R = PV == 16 ? 1 : 2;                                // (few components: as many jobs as waves)
    const int nvec = nq * pr.Pq, nrt = (nvec + 16 * R - 1) / (16 * R), nct = TI / (16 * R);
    for (int job = wave; job < pr.Px * nrt * nct; job += kWaves) {
      const int ct = job % nct, jr = job / nct, px = jr / nrt, rt = jr - px * nrt;
      const T *qr[R], *xr[R];
#pragma unroll
      for (int r = 0; r < R; ++r) {
        qr[r] = Q + (static_cast<long>(b0) * pr.Pq + min(16 * (R * rt + r) + c, nvec - 1)) * d;
        xr[r] = X + (static_cast<long>(px) * N + item_of(16 * (R * ct + r) + c)) * d;
      }
      f32x4_t acc[R][R] = {};
      int k0 = 0;
      if constexpr (PV < 64) {
        // (registers for four chunks in flight)
        for (; k0 + 4 * KCH <= d; k0 += 4 * KCH) {
          uint4 x[4][R], y[4][R];
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int r = 0; r < R; ++r) {
              x[e][r] = row16<T, VEC>(xr[r], k0 + e * KCH + g * E, d);
              y[e][r] = row16<T, VEC>(qr[r], k0 + e * KCH + g * E, d);
            }
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
              for (int h = 0; h < R; ++h) acc[r][h] = mma16<T>(y[e][r], x[e][h], acc[r][h]);
        }
      }
      for (; k0 < d; k0 += KCH) {
        uint4 x[R], y[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
          x[r] = row16<T, VEC>(xr[r], k0 + g * E, d);
          y[r] = row16<T, VEC>(qr[r], k0 + g * E, d);
        }
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
          for (int h = 0; h < R; ++h) acc[r][h] = mma16<T>(y[r], x[h], acc[r][h]);
      }
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const int v = 16 * (R * rt + r) + 4 * g;
        const int4 row = *reinterpret_cast<const int4*>(sRow + v);
        const int ro[4] = {row.x, row.y, row.z, row.w};
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (v + i < nvec) {
            float* dst = sS + ro[i] + px * TIP + 16 * R * ct + c;
#pragma unroll
            for (int h = 0; h < R; ++h) dst[16 * h] = acc[r][h][i];
          }
      }
    }
    __syncthreads();

    // 2. the wave's unit (queries past the batch: g = 0 on the last tile's s)
    float dl[RUN];
    f32x4_t ds[PT];
    float4 sv[PT];                                                     // s[16 pt + c][4 g ..]: K = items
    {
      float s[RUN];
      const float* src = sS + (q * PV + RUN * g) * TIP + it;
#pragma unroll
      for (int mu = 0; mu < RUN; ++mu) s[mu] = src[mu * TIP];
#pragma unroll
      for (int pt = 0; pt < PT; ++pt)
        sv[pt] = *reinterpret_cast<const float4*>(sS + (q * PV + 16 * pt + c) * TIP + it - c + 4 * g);
      f32x4_t l[PT];
      const float* ax = sAx + it * (PV + 4) + RUN * g;
#pragma unroll
      for (int pt = 0; pt < PT; ++pt) {
        const float4 cq = *reinterpret_cast<const float4*>(sC + q * PV + RUN * g + 4 * pt);
        const float4 a = *reinterpret_cast<const float4*>(ax + 4 * pt);
        l[pt] = f32x4_t{cq.x + a.x, cq.y + a.y, cq.z + a.z, cq.w + a.w};
      }
      for (int jt = 0; jt < JT; ++jt) {
        const float4 bj = *reinterpret_cast<const float4*>(sB1 + 16 * jt + 4 * g);
        f32x4_t u = f32x4_t{bj.x, bj.y, bj.z, bj.w};
#pragma unroll
        for (int m = 0; m < PT; ++m)
          u = mfma_f32x4(w1[(jt * PT + m) * 64], float4{s[4 * m], s[4 * m + 1], s[4 * m + 2], s[4 * m + 3]}, u);
        if (uglob) gU[jt * 64] = float4{u[0], u[1], u[2], u[3]};
        else *reinterpret_cast<float4*>(sU + jt * 256) = float4{u[0], u[1], u[2], u[3]};
        float h[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
          h[i] = u[i] * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * u[i]));
#pragma unroll
        for (int pt = 0; pt < PT; ++pt)
          l[pt] = mfma_f32x4(w2[(jt * PT + pt) * 64], float4{h[0], h[1], h[2], h[3]}, l[pt]);
      }
      float mx = l[0][0];
#pragma unroll
      for (int mu = 0; mu < RUN; ++mu) mx = fmaxf(mx, l[mu / 4][mu % 4]);
      mx = max_groups(mx);
      float den = 0.f, num = 0.f;
#pragma unroll
      for (int mu = 0; mu < RUN; ++mu) {
        const float w = __builtin_amdgcn_exp2f(kLog2e * (l[mu / 4][mu % 4] - mx));   // 0 past P
        l[mu / 4][mu % 4] = w;
        den += w;
        num = fmaf(w, s[mu], num);
      }
      const float rden = 1.f / sum_groups(den), phi = sum_groups(num) * rden, gw = gr * rden;
#pragma unroll
      for (int mu = 0; mu < RUN; ++mu) {
        const float gpi = gw * l[mu / 4][mu % 4];
        ds[mu / 4][mu % 4] = gpi;
        dl[mu] = gpi * (s[mu] - phi);
        dax[mu] += dl[mu];
      }
    }
    // dl in the place of the unit's s, read back with K = items
    {
      float* dst = sS + (q * PV + RUN * g) * TIP + it;
#pragma unroll
      for (int mu = 0; mu < RUN; ++mu) dst[mu * TIP] = dl[mu];
    }
    wave_lds_sync();
    float4 dv[PT];
    float rowsum = 0.f;                                                // sum over the items, p = 16 g' + c of lane group g'
#pragma unroll
    for (int pt = 0; pt < PT; ++pt) {
      dv[pt] = *reinterpret_cast<const float4*>(sS + (q * PV + 16 * pt + c) * TIP + it - c + 4 * g);
      const float t = sum_groups((dv[pt].x + dv[pt].y) + (dv[pt].z + dv[pt].w));
      if (g == pt) rowsum = t;
    }
    if (dm.group == 0 && q < nq && 16 * g + c < P && g < PT)
      out.da_q[(static_cast<long>((i0 >> 4) + (wave & ((1 << dm.upq_log2) - 1))) * pr.B + b) * P + 16 * g + c] = rowsum;

    for (int jg = 0; jg < JT; jg += JTG) {
      const bool mine = jg == dm.group * JTG;                          // accumulates dW1, dW2
#pragma unroll
      for (int jj = 0; jj < JTG; ++jj) {
        const int jt = jg + jj;
        if (jt >= JT) break;
        f32x4_t dh = {};
#pragma unroll
        for (int m = 0; m < PT; ++m)
          dh = mfma_f32x4(w2t[(jt * PT + m) * 64], float4{dl[4 * m], dl[4 * m + 1], dl[4 * m + 2], dl[4 * m + 3]}, dh);
        float4 u;
        if (uglob) u = gU[jt * 64];
        else u = *reinterpret_cast<const float4*>(sU + jt * 256);
        const float uu[4] = {u.x, u.y, u.z, u.w};
        float du[4], h[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float sig = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * uu[i]));
          h[i] = uu[i] * sig;
          du[i] = dh[i] * fmaf(h[i], 1.f - sig, sig);                  // sig (1 + u (1 - sig))
        }
        if (dm.group == 0) {
#pragma unroll
          for (int pt = 0; pt < PT; ++pt)
            ds[pt] = mfma_f32x4(w1t[(jt * PT + pt) * 64], float4{du[0], du[1], du[2], du[3]}, ds[pt]);
        }
        if (mine) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            sT[(4 * g + i) * 16 + c] = du[i];
            sT[256 + (4 * g + i) * 16 + c] = h[i];
          }
          wave_lds_sync();
          const float4 duv = *reinterpret_cast<const float4*>(sT + c * 16 + 4 * g);
          const float4 hv = *reinterpret_cast<const float4*>(sT + 256 + c * 16 + 4 * g);
          ab1[jj] += (duv.x + duv.y) + (duv.z + duv.w);
#pragma unroll
          for (int pt = 0; pt < PT; ++pt) {
            aw1[jj][pt] = mfma_f32x4(duv, sv[pt], aw1[jj][pt]);
            aw2[jj][pt] = mfma_f32x4(dv[pt], hv, aw2[jj][pt]);
          }
          wave_lds_sync();
        }
      }
    }
    if (dm.group == 0 && q < nq) {
      // pairs past the corpus end are stored as zeros (g = 0)
      const long base = static_cast<long>(b) * pr.Pq * dm.ns + slot;
#pragma unroll
      for (int mu = 0; mu < RUN; ++mu) {
        const uint32_t off = sOff[RUN * g + mu];
        const float v = ds[mu / 4][mu % 4];
        if (RUN * g + mu < P) out.ds[base + off] = v;
      }
    }
  }

  // the workgroup's sums, in the place of the rest: four blocks of dW1 and of dW2 of
  // every wave at a time ([wave][2][4][64][4]), added and stored by four elements a thread
  float* acc = smf;
  float* acc1 = smf + kSumFloats;                                      // [wave][JTG][16] of db1
  const int live_tiles = min(JTG, JT - dm.group * JTG);
  __syncthreads();
#pragma unroll
  for (int jj = 0; jj < JTG; ++jj) {
    const float t = sum_groups(ab1[jj]);
    if (g == 0) acc1[(wave * JTG + jj) * 16 + c] = t;
  }
#pragma unroll
  for (int b0 = 0; b0 < JTG * PT; b0 += 4) {
    if (b0 >= live_tiles * PT) break;
    if (b0) __syncthreads();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      f32x4_t* to = reinterpret_cast<f32x4_t*>(acc) + (wave * 8 + k) * 64 + lane;
      to[0] = aw1[(b0 + k) / PT][(b0 + k) % PT];
      to[256] = aw2[(b0 + k) / PT][(b0 + k) % PT];
    }
    __syncthreads();
    f32x4_t t = {};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) t += reinterpret_cast<const f32x4_t*>(acc)[w * 512 + tid];
    // (block (jj, pt) of matrix `which`; element r of lane l: row 4 (l / 16) + r, column l % 16)
    const int which = tid >> 8, blk = b0 + ((tid >> 6) & 3), jj = blk / PT, pt = blk - jj * PT;
    const int row = 4 * g, jb = 16 * (dm.group * JTG + jj);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int j = which ? jb + c : jb + row + r, p = which ? 16 * pt + row + r : 16 * pt + c;
      if (j < H && p < P) {
        if (which) out.dW2[(wg * P + p) * H + j] = t[r];
        else out.dW1[(wg * H + j) * P + p] = t[r];
      }
    }
  }
  for (int i = tid; i < 16 * JTG; i += kThreads) {
    const int j = 16 * dm.group * JTG + i;
    float t = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) t += acc1[w * JTG * 16 + i];
    if (j < H) out.db1[wg * H + j] = t;
  }
  if (dm.group) return;
  // db2: da_x summed over the items, then over the waves
#pragma unroll
  for (int mu = 0; mu < RUN; ++mu) {
    float t = dax[mu];
    t += row_ror<8>(t);
    t += row_ror<4>(t);
    t += row_ror<2>(t);
    t += row_ror<1>(t);
    if (c == mu % 16) ab1[0] = t;                                      // (RUN <= 16: lane c keeps component c)
  }
  __syncthreads();
  if (c < RUN) acc[wave * PV + RUN * g + c] = ab1[0];
  __syncthreads();
  for (int i = tid; i < P; i += kThreads) {
    float t = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) t += acc[w * PV + i];
    out.db2[wg * P + i] = t;
  }
  // da_x: the waves of a tile's queries in turn
  for (int w = 0; w < QB; ++w) {
    __syncthreads();
    if (q == w) {
#pragma unroll
      for (int mu = 0; mu < RUN; ++mu) {
        float* o = acc + it * (PV + 1) + RUN * g + mu;
        *o = w ? *o + dax[mu] : dax[mu];
      }
    }
  }
  __syncthreads();
  for (int i = tid; i < TI * P; i += kThreads) {
    const int n = i / P, p = i - n * P;
    out.da_x[(static_cast<long>(blockIdx.y) * dm.ns + i0 + n) * P + p] = acc[n * (PV + 1) + p];
  }
}

// ---------------------------------------------------------------------------
// Products with ds on matrix cores: out[m][t] = sum_k A[m][k] Bt[t][k].
// COLS false (dQ): m = (b, pq), k = (px, item): A rows run along k.
// COLS true (dX): one px a batch, m = item, k = (b, pq): A columns run along m.
// A wave has 32 rows and 64 columns; K chunks of `KCH` are split into ranges, z % splits,
// whose sums are separate parts.
struct GemmDims {
  int m, d;
  long lda;                // elements of a row of ds
  long a_px;               // elements between item components of ds
  int k_px, kvalid;        // K of one px (padded), rows of X or Q that exist
  int npx;                 // px of the K loop (dQ) or of the batch (dX)
  long b_px;               // elements between px of X (dQ)
  int splits;
  long out_px, out_split;  // elements between px (dX), between splits
  int direct;              // one split: out is the output itself
  Tiles tiles;
};
template <typename T, bool COLS, bool VEC>
__device__ __forceinline__ void product_tile(const GemmDims& gd, uint32_t unit, const float* __restrict__ ds,
                                             const T* __restrict__ rows, void* __restrict__ out, uint4* sh) {
  constexpr int E = 16 / sizeof(T), KCH = 4 * E, RB = 2, CB = 4;
  const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  const int3 at = tile_of(gd.tiles, unit);
  const int m0 = at.x * 16 * RB, t0 = at.y * 16 * CB, z = at.z;
  const int split = z % gd.splits, px0 = COLS ? z / gd.splits : 0;
  const int per = gd.k_px / KCH, chunks = COLS ? per : per * gd.npx;
  const int k0 = static_cast<int>(static_cast<long>(chunks) * split / gd.splits);
  const int k1 = static_cast<int>(static_cast<long>(chunks) * (split + 1) / gd.splits);
  f32x4_t acc[RB][CB] = {};
  int row[RB], col[CB];
#pragma unroll
  for (int r = 0; r < RB; ++r) row[r] = min(m0 + 16 * r + c, gd.m - 1);
#pragma unroll
  for (int t = 0; t < CB; ++t) col[t] = min(t0 + 16 * t + c, gd.d - 1);
  const RowTile<VEC> rt(gd.kvalid, gd.d, t0);
  struct Chunk {
    float a[RB][E];
    uint4 b[CB];
  };
  auto fetch = [&](Chunk& v, int ch) {
    const int px = COLS ? px0 : ch / per, kc = (COLS ? ch : ch - px * per) * KCH, k = kc + g * E;
    const float* A = ds + px * gd.a_px;
#pragma unroll
    for (int r = 0; r < RB; ++r) {
      if constexpr (COLS) {
#pragma unroll
        for (int e = 0; e < E; ++e) v.a[r][e] = A[min(k + e, gd.kvalid - 1) * gd.lda + row[r]];
      } else {
#pragma unroll
        for (int e = 0; e < E; e += 4) {
          const float4 x = *reinterpret_cast<const float4*>(A + row[r] * gd.lda + k + e);
          v.a[r][e] = x.x;
          v.a[r][e + 1] = x.y;
          v.a[r][e + 2] = x.z;
          v.a[r][e + 3] = x.w;
        }
      }
    }
    const T* B = COLS ? rows : rows + px * gd.b_px;
    if constexpr (sizeof(T) == 2) {
      rt.fetch(v.b, B, kc);
    } else {
      // (four rows of 16 columns a load)
      uint32_t w[CB][4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float* p = B + static_cast<long>(min(k + e, gd.kvalid - 1)) * gd.d;
#pragma unroll
        for (int t = 0; t < CB; ++t) w[t][e] = __float_as_uint(p[col[t]]);
      }
#pragma unroll
      for (int t = 0; t < CB; ++t) v.b[t] = make_uint4(w[t][0], w[t][1], w[t][2], w[t][3]);
    }
  };
  auto use = [&](const Chunk& v, int ch) {
    const int kc = (COLS ? ch : ch % per) * KCH, left = gd.kvalid - kc - g * E;   // rows past the end: zeros, as ds is there
    uint4 bv[CB];
    if constexpr (sizeof(T) == 2) {
      rt.put(v.b, sh, kc);
      wave_lds_sync();
#pragma unroll
      for (int t = 0; t < CB; ++t) bv[t] = column_of(sh, t, c, g);
    } else {
#pragma unroll
      for (int t = 0; t < CB; ++t)
        bv[t] = make_uint4(left > 0 ? v.b[t].x : 0, left > 1 ? v.b[t].y : 0, left > 2 ? v.b[t].z : 0, left > 3 ? v.b[t].w : 0);
    }
#pragma unroll
    for (int r = 0; r < RB; ++r) {
      float a[E];
#pragma unroll
      for (int e = 0; e < E; ++e) a[e] = !COLS || e < left ? v.a[r][e] : 0.f;
      if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int t = 0; t < CB; ++t) acc[r][t] = mfma_f32x4(float4{a[0], a[1], a[2], a[3]}, __builtin_bit_cast(float4, bv[t]), acc[r][t]);
      } else {
        // exact, in three terms; small products first
        const Terms<3> at = grad::split<3>(a);
#pragma unroll
        for (int k = 2; k >= 0; --k)
#pragma unroll
          for (int t = 0; t < CB; ++t) acc[r][t] = mfma_bf16(at.t[k], bv[t], acc[r][t]);
      }
    }
    if constexpr (sizeof(T) == 2) wave_lds_sync();                     // read before the next chunk is written
  };
  // (two sets of registers in turn: copies of one would wait for its loads)
  Chunk v0, v1;
  if (k0 < k1) fetch(v0, k0);
  for (int ch = k0; ch < k1; ch += 2) {
    fetch(v1, min(ch + 1, k1 - 1));
    use(v0, ch);
    fetch(v0, min(ch + 2, k1 - 1));
    if (ch + 1 < k1) use(v1, ch + 1);
  }
  put_tile<T>(out, px0 * gd.out_px + split * gd.out_split, m0, gd.m, t0, gd.d, gd.direct, acc);
}

// ---------------------------------------------------------------------------
// Both products, side by side: the first tiles are dQ's.  (In bf16 at 1024 x 2048
// pairs of 8 x 8 one launch of both is 13 us shorter than two.)
// VEC: rows of X and Q of whole 16-byte words (bf16).
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void k_grad_products(GemmDims q, GemmDims x, const float* __restrict__ ds,
                                                       const T* __restrict__ X, const T* __restrict__ Q,
                                                       void* __restrict__ out_q, void* __restrict__ out_x) {
  __shared__ __attribute__((aligned(16))) uint4 sh[4][sizeof(T) == 2 ? kTileB : 1];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t unit = blockIdx.x * 4 + wave, nq = static_cast<uint32_t>(q.tiles.count());
  if (unit < nq)
    product_tile<T, false, VEC>(q, unit, ds, X, out_q, sh[wave]);
  else if (unit - nq < static_cast<uint32_t>(x.tiles.count()))
    product_tile<T, true, VEC>(x, unit - nq, ds, Q, out_x, sh[wave]);
}

// ---------------------------------------------------------------------------
// Sums of partial results (SumJob).  A block has 256, 64 or 16 columns, and
// one, 4 or 16 runs of the parts of each: the more parts there are, the fewer columns.
__global__ __launch_bounds__(256) void k_sum_parts(SumArgs a) {
  __shared__ float sh[256];
  for (long blk0 = blockIdx.x; blk0 < a.first[a.n]; blk0 += gridDim.x) {
    int j = 0;
    while (j + 1 < a.n && a.first[j + 1] <= blk0) ++j;
    const SumJob& s = a.job[j];
    const int cols = 1 << s.cols_log2, runs = 256 >> s.cols_log2;
    const int lane = threadIdx.x & (cols - 1), run = threadIdx.x >> s.cols_log2;
    const long o = (blk0 - a.first[j]) * cols + lane;
    float v = 0.f;
    const int k0 = static_cast<int>(static_cast<long>(s.S) * run / runs);
    const int k1 = static_cast<int>(static_cast<long>(s.S) * (run + 1) / runs);
    if (o < s.L) {
#pragma unroll 8
      for (int k = k0; k < k1; ++k) v += s.in[k * s.stride + o];
    }
    if (runs > 1) {
      sh[threadIdx.x] = v;
      __syncthreads();
      v = 0.f;
      if (run == 0)
        for (int k = 0; k < runs; ++k) v += sh[k * cols + lane];
      __syncthreads();
    }
    if (o >= s.L || run) continue;
    if (s.add) v += s.acc[o];
    if (s.acc) s.acc[o] = v;
    if (s.out) {
      const long bt = o / s.in_len, at = bt * s.out_len + s.out_at + (o - bt * s.in_len);
      if (s.bf16)
        static_cast<bf16_t*>(s.out)[at] = __builtin_bit_cast(uint16_t, static_cast<__bf16>(v));
      else
        static_cast<float*>(s.out)[at] = v;
    }
  }
}

namespace grad {

void SumList::add(const SumJob& j) {
  SumJob& s = a.job[a.n] = j;
  s.cols_log2 = j.S <= 16 && j.L >= 4096 ? 8 : j.S <= 128 ? 6 : 4;
  a.first[a.n + 1] = a.first[a.n] + ((j.L + (1l << s.cols_log2) - 1) >> s.cols_log2);
  ++a.n;
}

hipError_t SumList::run() {
  // (a grid holds 2^32 threads)
  const unsigned blocks = static_cast<unsigned>(std::min<long>(a.first[a.n], 1l << 22));
  if (a.n) hipLaunchKernelGGL(k_sum_parts, dim3(blocks), dim3(256), 0, st, a);
  a.n = 0;
  return hipGetLastError();
}

}  // namespace grad

// ---------------------------------------------------------------------------
// Host side.
namespace {

struct GradPlan {
  GradDims dm;
  int JT, jtg, groups, slab, slabs;
  bool wlds, ulds;                      // prepared weights and the units' u in LDS
  size_t lds;
  int sp_q, sp_x;                       // K splits of dQ and dX
  size_t off_w, off_u, off_ds, off_daq, off_dax, off_dw1, off_dw2, off_db1, off_db2, off_pq, off_px, off_acc, bytes;
  long a_daq, a_dw1, a_dw2, a_db1, a_db2, a_dq;   // floats into the sums over slabs
  int wgs;
  int cus;                              // workgroups that run at once
  size_t wg_bytes;                      // of a workgroup's sums, and of u where LDS has no room
};

int queries_of(long B) { return B >= 4 ? 4 : B >= 2 ? 2 : 1; }

// What a plan owes to the shape and to QB, the queries of a tile.
template <int PV>
GradPlan plan_shape(const DevProb& pr, int QB) {
  GradPlan f{};
  f.JT = (pr.H + 15) / 16;
  f.jtg = group_tiles<PV>(f.JT <= 4);
  f.groups = (f.JT + f.jtg - 1) / f.jtg;
  GradDims& dm = f.dm;
  dm.QB = QB;
  dm.upq_log2 = dm.QB == 4 ? 1 : dm.QB == 2 ? 2 : 3;
  dm.TI = kPairs / dm.QB;
  dm.TIP = dm.TI + 4;
  // LDS has room for both up to P H = 4096; u is the less to read from the caches
  constexpr size_t most = 160 * 1024 / 4;
  f.ulds = grad_lds<PV>(f.JT, true, true, dm) <= most;
  f.wlds = grad_lds<PV>(f.JT, true, f.ulds, dm) <= most;
  if (!f.wlds) f.ulds = grad_lds<PV>(f.JT, false, true, dm) <= most;
  f.lds = grad_lds<PV>(f.JT, f.wlds, f.ulds, dm) * 4;
  // the final sums take the same place: dW1 and dW2 by four blocks, db1, then [TI][PV + 1] of da_x
  f.lds = std::max<size_t>(f.lds, 4 * (kSumFloats + 16ul * kWaves * f.jtg));
  f.lds = std::max<size_t>(f.lds, 4ul * dm.TI * (PV + 1));
  f.cus = PV == 16 && f.jtg == 4 && f.lds <= 80 * 1024 ? 512 : 256;
  f.wg_bytes = 4ul * (2ul * pr.H * pr.P + pr.H + pr.P) + (f.ulds ? 0 : 1024ul * kWaves * f.JT);
  return f;
}
// bytes of an item of a slab: ds, da_x, and what a tile's workgroup leaves (its sums and u)
size_t item_bytes(const DevProb& pr, const GradPlan& f, long B) {
  return 4ul * pr.P * (B + 1) + (f.wg_bytes + f.dm.TI - 1) / f.dm.TI;
}
// K of a product's chunk, and the least chunks of a long product's split: 128 items or query vectors
template <typename T>
constexpr int kChunk = 64 / sizeof(T);
template <typename T>
constexpr int kLeast = 128 / kChunk<T>;

template <typename T, int PV>
GradPlan plan_grad(const DevProb& pr) {
  GradPlan f = plan_shape<PV>(pr, queries_of(pr.B));
  GradDims& dm = f.dm;
  dm.m = static_cast<long>(pr.B) * pr.Pq;
  const long tiles = (static_cast<long>(pr.N) + dm.TI - 1) / dm.TI;
  const long fit = std::max<long>(1, static_cast<long>(kSlabBytes / (item_bytes(pr, f, pr.B) * dm.TI)));
  f.slabs = static_cast<int>((tiles + fit - 1) / fit);
  f.slab = static_cast<int>((tiles + f.slabs - 1) / f.slabs * dm.TI);
  f.slabs = static_cast<int>((static_cast<long>(pr.N) + f.slab - 1) / f.slab);
  dm.ns = f.slab;
  const int st = f.slab / dm.TI, nqb = (pr.B + dm.QB - 1) / dm.QB;
  dm.qsplits = std::max(1, std::min(nqb, f.cus / st));
  f.wgs = st * dm.qsplits;
  const long cg = (pr.d + 63) / 64;
  f.sp_q = split_of((dm.m + 31) / 32 * cg, static_cast<long>(pr.Px) * f.slab / kChunk<T>, kLeast<T>);
  f.sp_x = split_of((f.slab + 31l) / 32 * cg * pr.Px, (dm.m + 31) / 32 * 32 / kChunk<T>, kLeast<T>);
  auto up = [](size_t v) { return (v + 255) / 256 * 256; };
  size_t at = 0;
  const size_t P = pr.P, H = pr.H;
  f.off_w = at;   at = up(at + (f.wlds ? 0 : 16ul * f.JT * (PV / 16) * 256));
  f.off_u = at;   at = up(at + (f.ulds ? 0 : 1024ul * f.wgs * kWaves * f.JT));
  f.off_ds = at;  at = up(at + 4ul * pr.Px * dm.m * f.slab);
  f.off_daq = at; at = up(at + 4ul * (f.slab / 16) * pr.B * P);
  f.off_dax = at; at = up(at + 4ul * dm.qsplits * f.slab * P);
  f.off_dw1 = at; at = up(at + 4ul * f.wgs * H * P);
  f.off_dw2 = at; at = up(at + 4ul * f.wgs * H * P);
  f.off_db1 = at; at = up(at + 4ul * f.wgs * H);
  f.off_db2 = at; at = up(at + 4ul * f.wgs * P);
  f.off_pq = at;  at = up(at + 4ul * f.sp_q * dm.m * pr.d);
  f.off_px = at;  at = up(at + (f.sp_x > 1 ? 4ul * f.sp_x * pr.Px * static_cast<size_t>(f.slab) * pr.d : 0));
  f.a_daq = 0;
  f.a_dw1 = f.a_daq + static_cast<long>(pr.B) * P;
  f.a_dw2 = f.a_dw1 + static_cast<long>(H * P);
  f.a_db1 = f.a_dw2 + static_cast<long>(H * P);
  f.a_db2 = f.a_db1 + static_cast<long>(H);
  f.a_dq = f.a_db2 + static_cast<long>(P);
  f.off_acc = at; at = up(at + 4ul * (f.a_dq + (f.slabs > 1 ? dm.m * pr.d : 0)));
  f.bytes = at;
  return f;
}

// The most that plan_grad takes of the same shape with no more queries or items: each
// term bounds a part of the workspace by what grows with B and N alone, for the batches of each QB.
template <typename T, int PV>
size_t most_grad(const DevProb& pr) {
  size_t most = 0;
  for (int QB = 1; QB <= queries_of(pr.B); QB *= 2) {
    const GradPlan f = plan_shape<PV>(pr, QB);
    const size_t B = std::min<long>(pr.B, QB == 4 ? pr.B : 2 * QB - 1), m = B * pr.Pq, P = pr.P, TI = f.dm.TI;
    const size_t tiles = (pr.N + TI - 1) / TI, items = tiles * TI, item = item_bytes(pr, f, B);
    // ds, da_x of one range of queries and the workgroups' sums; da_q is a sixteenth of ds
    const size_t slab = std::min(item * items, std::max(kSlabBytes, TI * item));
    // more ranges of queries: f.cus workgroups at most
    const size_t nqb = (B + QB - 1) / QB;
    const size_t ranges = f.wg_bytes * std::min<size_t>(f.cus, nqb * tiles) + 4 * P * std::min(f.cus * TI, nqb * items);
    const size_t q = 4 * m * pr.d, chunks = (m + 31) / 32 * 32 / kChunk<T>;
    const size_t products = std::max(q, most_parts(q, pr.Px * items / kChunk<T>, kLeast<T>)) +
                            most_parts(4 * pr.Px * items * pr.d, chunks, kLeast<T>);
    const size_t weights = f.wlds ? 0 : 16ul * f.JT * (PV / 16) * 256;
    most = std::max(most, weights + slab + slab / 16 + ranges + products + 4 * B * P + f.wg_bytes + q + 16 * 256);
  }
  return (most + 255) / 256 * 256;
}

template <typename T, int PV>
hipError_t run_grad(const DevProb& pr, const float* dphi, const mol_score_grads& o, char* ws, hipStream_t st) {
  const GradPlan f = plan_grad<T, PV>(pr);
  const int bf = sizeof(T) == 2;
  GradDims dm = f.dm;
  auto F = [&](size_t off) { return reinterpret_cast<float*>(ws + off); };
  GradParts parts{F(f.off_ds), F(f.off_daq), F(f.off_dax), F(f.off_dw1), F(f.off_dw2),
                  F(f.off_db1), F(f.off_db2)};
  float* acc = F(f.off_acc);
  const float* wglob = nullptr;
  if (!f.wlds) {
    wglob = F(f.off_w);
    hipLaunchKernelGGL((k_grad_weights<T, PV>), dim3(4 * f.JT * (PV / 16)), dim3(256), 0, st, pr, f.JT, F(f.off_w));
  }
  const bool vec = (pr.d * sizeof(T)) % 16 == 0 &&
                   ((reinterpret_cast<uintptr_t>(pr.Q) | reinterpret_cast<uintptr_t>(pr.X)) & 15) == 0;
  const T* X = static_cast<const T*>(pr.X);
  const T* Q = static_cast<const T*>(pr.Q);
  constexpr int few = group_tiles<PV>(true), many = group_tiles<PV>(false);
  auto kern = f.jtg == few ? (vec ? &k_score_grad<T, PV, true, few> : &k_score_grad<T, PV, false, few>)
                           : (vec ? &k_score_grad<T, PV, true, many> : &k_score_grad<T, PV, false, many>);
  hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize,
                                     static_cast<int>(f.lds));
  if (e != hipSuccess) return e;
  const int cg = (pr.d + 63) / 64;   // column tiles
  SumList sums(st);
  for (int sl = 0; sl < f.slabs; ++sl) {
    const bool last = sl + 1 == f.slabs;
    dm.n0 = sl * f.slab;
    const int items = std::min(f.slab, pr.N - dm.n0);
    for (int grp = 0; grp < f.groups; ++grp) {
      dm.group = grp;
      if (grp && !o.dW1 && !o.dW2 && !o.db1) break;
      hipLaunchKernelGGL(kern, dim3(f.slab / dm.TI, dm.qsplits), dim3(kThreads), f.lds, st, pr, dm, dphi, wglob,
                         f.ulds ? nullptr : F(f.off_u), parts);
    }
    const long P = pr.P, H = pr.H, BP = pr.B * P;
    const long per_px = static_cast<long>(items) * pr.d;
    if (o.dQ || o.dX) {
      const int m = static_cast<int>(dm.m);
      // a product of one split (of dQ: and one slab) is stored as the output's type
      const bool dir_q = f.sp_q == 1 && f.slabs == 1, dir_x = f.sp_x == 1;
      const GemmDims gq{m, pr.d, f.slab, dm.m * f.slab, f.slab, items, pr.Px, static_cast<long>(pr.N) * pr.d, f.sp_q, 0,
                        dm.m * pr.d, dir_q, Tiles{(m + 31) / 32, cg, o.dQ ? f.sp_q : 0}};
      const GemmDims gx{items, pr.d, f.slab, dm.m * f.slab, (m + 31) / 32 * 32, m, pr.Px, 0, f.sp_x,
                        dir_x ? static_cast<long>(pr.N) * pr.d : per_px, per_px * pr.Px, dir_x,
                        Tiles{(items + 31) / 32, cg, o.dX ? f.sp_x * pr.Px : 0}};
      void* to_q = dir_q ? o.dQ : F(f.off_pq);
      void* to_x = dir_x ? static_cast<T*>(o.dX) + static_cast<long>(dm.n0) * pr.d : static_cast<void*>(F(f.off_px));
      const long units = gq.tiles.count() + gx.tiles.count();
      auto products = vec || !bf ? &k_grad_products<T, true> : &k_grad_products<T, sizeof(T) != 2>;
      hipLaunchKernelGGL(products, dim3(static_cast<unsigned>((units + 3) / 4)), dim3(256), 0, st, gq, gx, parts.ds,
                         X + static_cast<long>(dm.n0) * pr.d, Q, to_q, to_x);
    }
    if (o.dQ && (f.sp_q > 1 || f.slabs > 1))
      sums.add({F(f.off_pq), dm.m * pr.d, dm.m * pr.d, f.sp_q, f.slabs > 1 ? acc + f.a_dq : nullptr, sl > 0,
                last ? o.dQ : nullptr, bf, dm.m * pr.d, dm.m * pr.d, 0});
    if (o.dX && f.sp_x > 1)
      sums.add({F(f.off_px), per_px * pr.Px, per_px * pr.Px, f.sp_x, nullptr, 0, o.dX, bf, per_px,
                static_cast<long>(pr.N) * pr.d, static_cast<long>(dm.n0) * pr.d});
    if (o.da_q)
      sums.add({parts.da_q, BP, BP, f.slab / 16, acc + f.a_daq, sl > 0, last ? o.da_q : nullptr, 0, BP, BP, 0});
    if (o.da_x)
      sums.add({parts.da_x, items * P, f.slab * P, dm.qsplits, nullptr, 0, o.da_x, 0, items * P, items * P,
                static_cast<long>(dm.n0) * P});
    if (o.dW1)
      sums.add({parts.dW1, H * P, H * P, f.wgs, acc + f.a_dw1, sl > 0, last ? o.dW1 : nullptr, bf, H * P, H * P, 0});
    if (o.dW2)
      sums.add({parts.dW2, H * P, H * P, f.wgs, acc + f.a_dw2, sl > 0, last ? o.dW2 : nullptr, bf, H * P, H * P, 0});
    if (o.db1) sums.add({parts.db1, H, H, f.wgs, acc + f.a_db1, sl > 0, last ? o.db1 : nullptr, 0, H, H, 0});
    if (o.db2) sums.add({parts.db2, P, P, f.wgs, acc + f.a_db2, sl > 0, last ? o.db2 : nullptr, 0, P, P, 0});
    if ((e = sums.run()) != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

size_t score_grad_bytes(const DevProb& pr) {
  if (bf16_supported(pr)) return bf16_bytes(pr);
  if (pr.dtype == MOL_BF16)
    return (pr.P <= 16 ? plan_grad<bf16_t, 16>(pr) : pr.P <= 32 ? plan_grad<bf16_t, 32>(pr) : plan_grad<bf16_t, 64>(pr)).bytes;
  return (pr.P <= 16 ? plan_grad<float, 16>(pr) : pr.P <= 32 ? plan_grad<float, 32>(pr) : plan_grad<float, 64>(pr)).bytes;
}

size_t score_grad_most(const DevProb& pr) {
  if (bf16_supported(pr)) return bf16_most(pr);
  const size_t general =
      pr.dtype == MOL_BF16
          ? (pr.P <= 16 ? most_grad<bf16_t, 16>(pr) : pr.P <= 32 ? most_grad<bf16_t, 32>(pr) : most_grad<bf16_t, 64>(pr))
          : (pr.P <= 16 ? most_grad<float, 16>(pr) : pr.P <= 32 ? most_grad<float, 32>(pr) : most_grad<float, 64>(pr));
  return std::max(general, bf16_most(pr));   // (a shorter corpus may take the bf16 form)
}

hipError_t launch_score_grad(const DevProb& pr, const float* dphi, const mol_score_grads& o, void* ws, hipStream_t st) {
  if (bf16_supported(pr)) return launch_bf16(pr, dphi, o, static_cast<char*>(ws), st);
  auto f = pr.dtype == MOL_BF16
               ? (pr.P <= 16 ? &run_grad<bf16_t, 16> : pr.P <= 32 ? &run_grad<bf16_t, 32> : &run_grad<bf16_t, 64>)
               : (pr.P <= 16 ? &run_grad<float, 16> : pr.P <= 32 ? &run_grad<float, 32> : &run_grad<float, 64>);
  return f(pr, dphi, o, static_cast<char*>(ws), st);
}

}  // namespace mol
