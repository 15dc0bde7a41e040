// Gradient of the MoL scores for bf16 problems of up to 8 x 8 components and 64
// hidden units, or 8 x 4 and 128, on bf16 matrix instructions (mol_score_grad.hip has the
// formulas and every other shape).
//
// Precision.  W1 and W2 are bf16, exact.  What meets them on the way to the
// float32 outputs (s, h and dl) is split into three bf16 terms, 8 + 8 + 8 bits by
// truncation: exact, so that a product is as good as a float32 one at three
// bf16 MFMAs (of 8 times the f32 rate).  Three values that only bf16 outputs are
// made of take two terms, 16 bits: du on its way to ds, ds itself, and both factors
// of dW1 and dW2 (the products of two second terms are left out).  An output's error
// against 64 bits stays that of its own rounding to 8 bits (128 x 1031 of 8 x 8: dQ
// 1.656e-3 in the norm, as from float32 operations), but one element in 80 to 230 of dQ, dX, dW1
// and dW2 rounds to the other neighbour; and a sum whose terms cancel to less than
// 2^-8 of their size keeps fewer than 8 bits.  A third term of ds would be half as much
// again to write and read, one of the factors has no room in LDS.  MOL_FLAG_F32_GATING takes
// the general form, which has none of these roundings.
//
// A wave takes units of 16 items of one query, independent of the other waves.
// Lane (c = lane % 16, g = lane / 16) holds item c's slots (g, mu), mu < RUN,
// of components pq = NPQ g + mu / PXP, px = mu % PXP: the dot products come out
// of the MFMA in that layout (row 4 g + i of A is query component NPQ g + i, i
// < NPQ; the other rows repeat it), and nothing is exchanged between lanes
// up to the sums over items.  u^T = W1 s and dh^T = W2^T dl have K = the slots (K slot 8 g + e of
// block m is (g, 8 m + e)), l^T += W2 h and ds^T += W1^T du have K = hidden
// units (K slot 8 g + e of block m is j = 32 m + 16 (e / 4) + 4 g + e % 4, where
// the accumulators of u and dh have them), and their output row 4 g + i of
// tile pt is the lane's own slot (g, 4 pt + i).  W1 and W2 sit in LDS once,
// as [j][slot] and [slot][j]; the transposed operands are read by the
// transposing LDS read.  dW1 = sum du s^T and dW2 = sum dl h^T have K = items: the four
// factors are written item by item (two terms each) and read transposed too.
// dW1, dW2, db1 and da_x stay in registers over all of the wave's units.
//
// ds goes to the workspace as two bf16 terms, by blocks of 16 items, [px][item
// block][b pq][16 first terms, 16 second terms]: 64-byte rows that both products read
// whole.  dQ = sum ds X reads rows (K = items); dX = sum ds Q (K = b pq) takes them through LDS
// and the transposing read.
//
// Measured, 1024 x 2048 pairs of 8 x 8, d = H = 64, in two slabs: 763 us a call,
// 203 TFLOP/s; under the profiler, a tenth slower, a slab's pairs take 283 to 312 us,
// products 95 to 107 (5.4 TB/s of ds), sums 17 to 20.  128 x 1031 of 8 x 8, d = 32: 63 + 18 + 9.  The pairs are bound by issue and latency: a unit
// is 914 vector, 49 transcendental, 124 matrix and 121 LDS instructions, its
// 256 registers leave two waves a SIMD, and these issue vector instructions 40 % of
// the time.  The general form, on f32 matrix instructions, takes 698 us for a slab's
// pairs.
#include <algorithm>
#include <type_traits>

#include "mol_grad.h"

namespace mol {

using namespace tile;
using namespace grad;

namespace {

constexpr int kWaves = 8, kThreads = 64 * kWaves;
// Of a slab's ds and partial sums: a million pairs of 64 components, whose
// ds alone is 268 MB (1024 x 2048 pairs: two such slabs 770 us, three of 187 MB, whose
// workgroups fill 220 of the 256 CUs, 882).
constexpr size_t kSlabBytes = size_t(288) << 20;
constexpr int kAhead = 2;                          // blocks of 32 of d loaded ahead
constexpr int kJT = 4;                             // hidden tiles of 16 that LDS holds h and du of
constexpr int kH = 16 * kJT;

// Elements t .. t + 7 of a row of `d` at base + off bytes, of which base is the
// same for the whole wave; past the row's end zeros, or other elements of it
template <bool VEC>
__device__ __forceinline__ uint4 row16_of(const bf16_t* base, uint32_t off, int t, int d, bool zero) {
  const char* p = reinterpret_cast<const char*>(base);
  if constexpr (VEC) {                                                // (d is a multiple of 8)
    const uint4 v = *reinterpret_cast<const uint4*>(p + (off + 2u * min(t, d - 8)));
    return !zero || t < d ? v : make_uint4(0, 0, 0, 0);
  } else {
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t x = *reinterpret_cast<const bf16_t*>(p + (off + 2u * min(t + e, d - 1)));
      w[e / 2] |= (!zero || t + e < d ? x : 0u) << (16 * (e & 1));
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
}
// A lane's offset, unknown to the compiler from here on: it would otherwise keep
// the 64-bit sums of every base and offset in registers over the whole loop.
__device__ __forceinline__ uint32_t fresh(uint32_t off) {
  asm volatile("" : "+v"(off));
  return off;
}
template <typename T>
__device__ __forceinline__ const T& at32(const T* base, uint32_t bytes) {
  return *reinterpret_cast<const T*>(reinterpret_cast<const char*>(base) + bytes);
}

// x[slot] summed over the 16 lanes of a row, lane c with the sum of slot c mod
// RUN: at each step a lane passes on one half of its slots and keeps the
// other, so that 16 slots take 15 additions and not 64
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
template <int HALF, int CTRL, int LEN>
__device__ __forceinline__ void fold(float (&v)[LEN], bool upper) {
#pragma unroll
  for (int i = 0; i < HALF; ++i) {
    const float keep = upper ? v[i + HALF] : v[i], pass = upper ? v[i] : v[i + HALF];
    v[i] = keep + dpp<CTRL>(pass);
  }
}
template <int RUN>
__device__ __forceinline__ float sum_items(const float (&x)[RUN], int c) {
  constexpr int kRor8 = 0x128, kHalfMirror = 0x141, kReverse4 = 0x1B, kSwap2 = 0xB1;   // lane c ^ 8, c ^ 7, c ^ 3, c ^ 1
  float v[RUN];
#pragma unroll
  for (int i = 0; i < RUN; ++i) v[i] = x[i];
  if constexpr (RUN >= 16) fold<8, kRor8>(v, c & 8);
  if constexpr (RUN >= 8) fold<4, kHalfMirror>(v, c & 4);
  fold<2, kReverse4>(v, c & 2);
  fold<1, kSwap2>(v, c & 1);
  float t = v[0];
  if constexpr (RUN < 16) t += dpp<kRor8>(t);
  if constexpr (RUN < 8) t += dpp<0x124>(t);                           // (rotated by 4)
  return t;
}

struct Bf16Dims {
  int QB;            // waves that share 16 items: queries a step
  int n0, ns, items; // the slab's first item, its padded length (a multiple of 32) and its items
  int nb;            // its blocks of 16
  int qsplits;       // query ranges
  int kl;            // blocks of 32 of d that the items' rows have in LDS
  long m;            // B Pq
};
struct Bf16Parts {
  uint32_t* ds;      // [Px][nb][m][16]
  float* da_q;       // [nb][B][P]
  float* da_x;       // [qsplits][ns][P]
  float* dW1;        // [workgroups][H][P]
  float* dW2;        // [workgroups][P][H]
  float* db1;        // [workgroups][H]
  float* db2;        // [workgroups][P]
};

// LDS bytes of a wave: s or dl, h and du by tiles of 16 slots or hidden units
// (16 items x 32 bytes, first and second terms), k in the place of du
template <int RUN>
constexpr int wave_bytes() { return 1024 * (2 * (RUN / 4) + 2 * kJT); }
// W1 [j][slot] and W2 [slot][j], rows without padding
template <int RUN, int HALVES>
constexpr int weight_bytes() { return 2 * HALVES * kH * 4 * RUN * 2; }
template <int RUN, int HALVES>
constexpr int lds_bytes() { return weight_bytes<RUN, HALVES>() + kWaves * wave_bytes<RUN>(); }
// Bytes of a block of 32 of the items' rows in LDS, [px][4][16 items][16 bytes]
constexpr int x_bytes(int pxp) { return pxp * 1024; }
static_assert(lds_bytes<4, 1>() >= 4 * kWaves * 16 * 16 && lds_bytes<16, 1>() >= 4 * kWaves * 16 * 64, "the sums of da_x fit");

}  // namespace

// XL: the workgroup's waves share 16 items, whose rows lie in LDS (2: as far as there is room).  FULL 1 or 2: P_q = 4
// NPQ, P_x = PXP, every row allows 16-byte reads (H a multiple of 4) and H is
// at most 32 FULL: no branches in a unit, which leaves its order to the compiler.
// HALVES 2: 65 to 128 hidden units.  u stays in registers on the way forward, and the way
// back takes 64 of them at a time: h and du of those to LDS, and their part of dW1 and dW2
// (512 x 2000 pairs of 8 x 4, d = H = 128: 331 us; a call 410, 865 in the general form).
template <int NPQ, int PXP, int XL, int FULL, int HALVES>
__global__ __launch_bounds__(kThreads, 2) void k_score_grad_bf16(DevProb pr, Bf16Dims dm,
                                                                 const float* __restrict__ dphi, Bf16Parts out) {
  constexpr int RUN = NPQ * PXP, SLOTS = 4 * RUN, PT = RUN / 4, KB = RUN > 8 ? RUN / 8 : 1, HU = HALVES * kH;
  extern __shared__ __attribute__((aligned(16))) unsigned char smb[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c = lane & 15, g = lane >> 4;
  const int P = pr.P, H = pr.H, d = pr.d, N = pr.N, JT2 = FULL ? FULL : (H + 31) / 32, nch = 4 * (XL == 2 ? dm.kl : (d + 31) / 32);
  const int Pq = FULL ? 4 * NPQ : pr.Pq, Px = FULL ? PXP : pr.Px;
  unsigned char* sW1 = smb;
  unsigned char* sW2 = sW1 + 2 * HU * SLOTS;
  unsigned char* waves = sW2 + 2 * HU * SLOTS;
  unsigned char* mine = waves + wave * wave_bytes<RUN>();
  unsigned char* sS = mine;                                           // s by tiles: first terms, second terms
  unsigned char* sD = sS + 1024 * PT;                                 // dl
  unsigned char* sH = sD + 1024 * PT;                                 // h
  unsigned char* sU = sH + 1024 * kJT;                                // k (float32, as the lanes have it), then du
  uint4* sX = reinterpret_cast<uint4*>(waves + kWaves * wave_bytes<RUN>());
  auto component = [&](int slot) {                                    // p of a slot, -1 for none
    const int pq = NPQ * (slot / RUN) + slot % RUN / PXP, px = slot % PXP;
    return pq < Pq && px < Px ? pq * Px + px : -1;
  };
  // byte of an element of W1 (row j) and W2 (row a slot): the 8-byte pieces of a
  // row are rotated by two for each row, so that rows meet different banks
  auto w1_at = [](int j, int sl) { return j * (2 * SLOTS) + ((2 * sl + 16 * j) & (2 * SLOTS - 1)); };
  auto w2_at = [](int sl, int j) { return sl * (2 * HU) + ((2 * j + 16 * sl) & (2 * HU - 1)); };
  const bool vec = FULL || (d % 8 == 0 && ((reinterpret_cast<uintptr_t>(pr.Q) | reinterpret_cast<uintptr_t>(pr.X)) & 15) == 0);
  auto row16 = [&](const bf16_t* base, uint32_t off, int t, bool zero) {
    return vec ? row16_of<true>(base, off, t, d, zero) : row16_of<false>(base, off, t, d, zero);
  };

  const int q = wave % dm.QB, blk = blockIdx.x * (kWaves / dm.QB) + wave / dm.QB;   // the wave's query of a step, its block
  const bool has_blk = blk < dm.nb;
  const int slot = 16 * min(blk, dm.nb - 1) + c;                                    // its item of the slab
  const bool has_item = has_blk && slot < dm.items;
  const int n = min(dm.n0 + slot, N - 1);
  const int row_pq = min(NPQ * (c >> 2) + min(c & 3, NPQ - 1), Pq - 1);             // the component of A row c
  // offsets of a lane in 32 bits (the launcher sees to it), from bases that are the wave's
  const bf16_t* X = static_cast<const bf16_t*>(pr.X);
  const long x_px = static_cast<long>(N) * d;
  const uint32_t x_off = 2u * static_cast<uint32_t>(n) * d, q_off = 2u * row_pq * d, ax_off = 4u * static_cast<uint32_t>(n) * P;
  {
    const bf16_t* W1 = static_cast<const bf16_t*>(pr.W1);
    const bf16_t* W2 = static_cast<const bf16_t*>(pr.W2);
    for (int i = tid; i < HU * SLOTS; i += kThreads) {
      const int j = i / SLOTS, sl = i - j * SLOTS, p = component(sl);
      const bool in = j < H && p >= 0;
      *reinterpret_cast<bf16_t*>(sW1 + w1_at(j, sl)) = in ? W1[j * P + p] : 0;
      *reinterpret_cast<bf16_t*>(sW2 + w2_at(sl, j)) = in ? W2[p * H + j] : 0;
    }
    if constexpr (XL != 0) {
      // (zeros past d would do no good here: Q has them)
      for (int i = tid; i < PXP * nch * 16; i += kThreads) {
        const int it = i & 15, ch = (i >> 4) % nch, px = (i >> 4) / nch;
        const int item = min(dm.n0 + 16 * static_cast<int>(blockIdx.x) + it, N - 1);
        sX[i] = row16(X + min(px, Px - 1) * x_px, 2u * static_cast<uint32_t>(item) * d, 8 * ch, false);
      }
    }
  }
  __syncthreads();

  // where the lane's slots lie in a tile array: 8 bytes (16 of RUN > 4), halves of a row swapped from item 8 on
  auto place = [&](int sl) { return (sl >> 4) * 1024 + c * 32 + ((((sl >> 3) & 1) ^ (c >> 3)) << 4) + ((sl & 4) << 1); };
  // the transposing read of a tile: rows 4 g .. of items
  const int tr = (4 * g + (c >> 2)) * 32 + ((((c & 3) >> 1) ^ (g >> 1)) << 4) + ((c & 1) << 3);

  // the wave's part of the workgroup's dW1 (waves 0 to 3) or dW2: hidden tiles j0 .., slot tiles pt0 ..
  constexpr int JW = PT == 4 ? 2 : 1, PW = PT == 1 ? 1 : 2;
  const int sub = wave & 3, j0 = PT == 4 ? 2 * (sub >> 1) : sub, pt0 = PT == 4 ? 2 * (sub & 1) : 0;
  const bool second = wave >= 4;
  f32x4_t aw[HALVES][JW][PW] = {}, ab1[HALVES * kJT] = {};
  float dax[RUN] = {};
  // what a unit reads from its query's rows, loaded a step ahead
  uint4 qf[kAhead];
  float gr = 0.f, gr_next = 0.f;
  auto fetch = [&](int b) {
    const bf16_t* Q = static_cast<const bf16_t*>(pr.Q) + static_cast<long>(b) * Pq * d;
    gr_next = at32(dphi + static_cast<long>(b) * N, fresh(4u * n));
    const uint32_t qo = fresh(q_off);
#pragma unroll
    for (int k = 0; k < kAhead; ++k) qf[k] = row16(Q, qo, 32 * k + 8 * g, true);
  };
  const int steps = (pr.B + dm.QB - 1) / dm.QB;
  const int st0 = static_cast<int>(static_cast<long>(steps) * blockIdx.y / dm.qsplits);
  const int st1 = static_cast<int>(static_cast<long>(steps) * (blockIdx.y + 1) / dm.qsplits);
  if (has_blk && st0 * dm.QB + q < pr.B) fetch(st0 * dm.QB + q);
  for (int st = st0; st < st1; ++st) {
    const int b = st * dm.QB + q;
    const bool busy = has_blk && b < pr.B;                            // (the same for the whole wave)
    Terms<3> a[KB];                                                   // of s, then of dl
    f32x4_t ds[PT], ur[HALVES == 2 ? 2 * kJT : 1];
    // (not indented: the way forward, before the first half; the way back, a half; ds, after the last)
#pragma unroll
    for (int half = 0; half < HALVES; ++half) {
    if (busy) {
    if (half == 0) {
    gr = has_item ? gr_next : 0.f;
    // a_q, a_x and b2, for l
    f32x4_t l[PT], lx[PT], b2[PT];
    {
      const float* aq = pr.a_q + static_cast<long>(b) * P;
      const uint32_t ao = fresh(ax_off), go = fresh(4u * RUN * g);
#pragma unroll
      for (int pt = 0; pt < PT; ++pt) {
        if constexpr (FULL) {
          l[pt] = at32(reinterpret_cast<const f32x4_t*>(aq), go + 16u * pt);
          lx[pt] = at32(reinterpret_cast<const f32x4_t*>(pr.a_x), ao + go + 16u * pt);
          b2[pt] = at32(reinterpret_cast<const f32x4_t*>(pr.b2), go + 16u * pt);
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int mu = 4 * pt + i, p = min(NPQ * g + mu / PXP, Pq - 1) * Px + min(mu % PXP, Px - 1);
            l[pt][i] = at32(aq, 4u * p);
            lx[pt][i] = at32(pr.a_x, ao + 4u * p);
            const float v = at32(pr.b2, 4u * p);
            b2[pt][i] = NPQ * g + mu / PXP < Pq && mu % PXP < Px ? v : -__builtin_inff();   // no component
          }
        }
      }
    }
    // s: one MFMA row tile of query components against the 16 items, each item component
    float s[RUN];
    {
      f32x4_t acc[PXP] = {};
      const bf16_t* Q = static_cast<const bf16_t*>(pr.Q) + static_cast<long>(b) * Pq * d;
      const uint32_t qo = fresh(q_off), xo = fresh(x_off);
      auto block = [&](int k, uint4 qv, bool lds) {                   // (zeros of Q past d meet X's own, finite, elements)
        uint4 xv[PXP];
        const bf16_t* Xp = X;
#pragma unroll
        for (int px = 0; px < PXP; ++px, Xp += px < Px ? x_px : 0)
          xv[px] = lds ? sX[(px * nch + 4 * k + g) * 16 + c] : row16(Xp, xo, 32 * k + 8 * g, false);
#pragma unroll
        for (int px = 0; px < PXP; ++px) acc[px] = mfma_bf16(qv, xv[px], acc[px]);
      };
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
        if (32 * k < d) block(k, qf[k], XL != 0);
      int k = kAhead;
      if constexpr (XL == 2)
        for (; k < dm.kl; ++k) block(k, row16(Q, qo, 32 * k + 8 * g, true), true);
      for (; 32 * k < d; ++k) block(k, row16(Q, qo, 32 * k + 8 * g, true), XL == 1);
#pragma unroll
      for (int px = 0; px < PXP; ++px)
#pragma unroll
        for (int i = 0; i < NPQ; ++i) s[i * PXP + px] = acc[px][i];
    }
    // forward
    // (b1 and b2 come from the caches each time: LDS and registers are full)
    f32x4_t b1[HALVES * kJT];
    {
      const uint32_t go = fresh(16u * g);
#pragma unroll
      for (int jt = 0; jt < HALVES * kJT; ++jt) {
        if constexpr (FULL) {
          const f32x4_t v = at32(reinterpret_cast<const f32x4_t*>(pr.b1), min(go + 64u * jt, 4u * H - 16u));
          b1[jt] = 16 * jt + 4 * g < H ? v : f32x4_t{0.f, 0.f, 0.f, 0.f};
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float v = at32(pr.b1, min(go + 64u * jt + 4u * i, 4u * H - 4u));
            b1[jt][i] = 16 * jt + 4 * g + i < H ? v : 0.f;
          }
        }
      }
    }
#pragma unroll
    for (int pt = 0; pt < PT; ++pt) {
      l[pt] = l[pt] + lx[pt] + b2[pt];
    }
    auto slots8 = [&](const float (&x)[RUN], int m) {
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = 8 * m + e < RUN ? x[(8 * m + e) % RUN] : 0.f;
      return split<3>(v);
    };
    auto store_slots = [&](unsigned char* to) {                       // two terms, item by item
#pragma unroll
      for (int m = 0; m < KB; ++m)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          unsigned char* at = to + place(RUN * g + 8 * m) + 512 * k;
          if constexpr (RUN >= 8)
            *reinterpret_cast<uint4*>(at) = a[m].t[k];
          else
            *reinterpret_cast<uint2*>(at) = make_uint2(a[m].t[k].x, a[m].t[k].y);
        }
    };
#pragma unroll
    for (int m = 0; m < KB; ++m) a[m] = slots8(s, m);
    store_slots(sS);
#pragma unroll
    for (int j2 = 0; j2 < HALVES * kJT / 2; ++j2) {
      if (j2 >= JT2) break;
      float h[8];
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        const int jt = 2 * j2 + hf;
        f32x4_t u = b1[jt];
#pragma unroll
        for (int m = 0; m < KB; ++m) {
          uint4 w;
          const unsigned char* at = sW1 + w1_at(16 * jt + c, RUN * g + 8 * m);
          if constexpr (RUN >= 8) {
            w = *reinterpret_cast<const uint4*>(at);
          } else {
            const uint2 w2 = *reinterpret_cast<const uint2*>(at);
            w = make_uint4(w2.x, w2.y, 0, 0);
          }
          u = mfma_terms<3>(w, a[m], u);
        }
        if constexpr (HALVES == 2) ur[jt] = u;
        float kk[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float sig = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * u[i]));
          h[4 * hf + i] = u[i] * sig;
          kk[i] = fmaf(h[4 * hf + i], 1.f - sig, sig);                // sig (1 + u (1 - sig))
        }
        if constexpr (HALVES == 1) *reinterpret_cast<float4*>(sU + 1024 * jt + 16 * lane) = float4{kk[0], kk[1], kk[2], kk[3]};
      }
      const Terms<3> ht = split<3>(h);
      if constexpr (HALVES == 1) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          *reinterpret_cast<uint2*>(sH + 1024 * (2 * j2) + 512 * k + place(4 * g)) = make_uint2(ht.t[k].x, ht.t[k].y);
          *reinterpret_cast<uint2*>(sH + 1024 * (2 * j2 + 1) + 512 * k + place(4 * g)) = make_uint2(ht.t[k].z, ht.t[k].w);
        }
      }
#pragma unroll
      for (int pt = 0; pt < PT; ++pt) {
        // row c of tile pt: slot RUN (c / 4) + 4 pt + c % 4
        const int sl = RUN * (c >> 2) + 4 * pt + (c & 3);
        const uint2 w0 = *reinterpret_cast<const uint2*>(sW2 + w2_at(sl, 32 * j2 + 4 * g));
        const uint2 w1 = *reinterpret_cast<const uint2*>(sW2 + w2_at(sl, 32 * j2 + 16 + 4 * g));
        l[pt] = mfma_terms<3>(make_uint4(w0.x, w0.y, w1.x, w1.y), ht, l[pt]);
      }
    }
    // softmax, dl
    float dl[RUN];
    {
      float mx = l[0][0];
#pragma unroll
      for (int mu = 0; mu < RUN; ++mu) mx = fmaxf(mx, l[mu / 4][mu % 4]);
      mx = max_groups(mx);
      float den = 0.f, num = 0.f;
#pragma unroll
      for (int mu = 0; mu < RUN; ++mu) {
        const float w = __builtin_amdgcn_exp2f(kLog2e * (l[mu / 4][mu % 4] - mx));   // 0 in the slots of no component
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
#pragma unroll
    for (int m = 0; m < KB; ++m) a[m] = slots8(dl, m);
    store_slots(sD);
    // the next unit's operands, behind which there is still the way back
    if (st + 1 < st1 && b + dm.QB < pr.B) fetch(b + dm.QB);
    // da_q: sums over the 16 items, lane c of the group gets slot c's (c mod RUN)
    {
      const float t = sum_items<RUN>(dl, c);
      const int pq = NPQ * g + c / PXP, px = c % PXP;
      if (c < RUN && pq < Pq && px < Px) out.da_q[(static_cast<long>(blk) * pr.B + b) * P + pq * Px + px] = t;
    }
    }
    // back through 64 hidden units of the MLP
#pragma unroll
      for (int l2 = 0; l2 < kJT / 2; ++l2) {
        const int j2 = half * (kJT / 2) + l2;
        if (j2 >= JT2) break;
        float du[8], h[8];
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          const int jt = 2 * j2 + hf;
          f32x4_t dh = {};
#pragma unroll
          for (int m = 0; m < KB; ++m) {
            // A row j = 16 jt + c, K = slots RUN g + 8 m + e: columns of W2's rows
            const int sl = RUN * g + 8 * m + (c >> 2), j = 16 * jt + 4 * (c & 3);
            const uint2 w0 = read_tr(sW2 + w2_at(sl, j));
            const uint2 w1 = RUN >= 8 ? read_tr(sW2 + w2_at(sl + 4, j)) : make_uint2(0, 0);
            dh = mfma_terms<3>(make_uint4(w0.x, w0.y, w1.x, w1.y), a[m], dh);
          }
          float kk[4];
          if constexpr (HALVES == 1) {
            const float4 k = *reinterpret_cast<const float4*>(sU + 1024 * jt + 16 * lane);
            kk[0] = k.x, kk[1] = k.y, kk[2] = k.z, kk[3] = k.w;
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float u = ur[jt][i], sig = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * u));
              h[4 * hf + i] = u * sig;
              kk[i] = fmaf(h[4 * hf + i], 1.f - sig, sig);
            }
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            du[4 * hf + i] = dh[i] * kk[i];
            ab1[jt][i] += du[4 * hf + i];
          }
        }
        auto store_hidden = [&](unsigned char* to, const Terms<2>& x) {
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            *reinterpret_cast<uint2*>(to + 1024 * (2 * l2) + 512 * k + place(4 * g)) = make_uint2(x.t[k].x, x.t[k].y);
            *reinterpret_cast<uint2*>(to + 1024 * (2 * l2 + 1) + 512 * k + place(4 * g)) = make_uint2(x.t[k].z, x.t[k].w);
          }
        };
        const Terms<2> dt = split<2>(du);
        store_hidden(sU, dt);                                         // (in the place of k, which the wave has read)
        if constexpr (HALVES == 2) store_hidden(sH, split<2>(h));
#pragma unroll
        for (int pt = 0; pt < PT; ++pt) {
          // A row slot RUN (c / 4) + 4 pt + c % 4, K = j: columns of W1's rows
          const int j = 32 * j2 + 4 * g + (c >> 2), sl = RUN * (c & 3) + 4 * pt;
          const uint2 w0 = read_tr(sW1 + w1_at(j, sl)), w1 = read_tr(sW1 + w1_at(j + 16, sl));
          ds[pt] = mfma_terms<2>(make_uint4(w0.x, w0.y, w1.x, w1.y), dt, ds[pt]);
        }
      }
    // ds as two terms; lanes of a pair of items exchange them, the even one takes the first terms of both
    if (half + 1 == HALVES) {
      const uint32_t pick = c & 1 ? 0x03020706u : 0x05040100u;        // (own word low in the permute)
      uint32_t* to = out.ds + (static_cast<long>(blk) * dm.m + static_cast<long>(b) * Pq) * 16;
      const uint32_t to_off = fresh(4u * (16 * NPQ * g + ((c & 1) << 3) + (c >> 1)));
      const long px_step = static_cast<long>(dm.nb) * dm.m * 16;
#pragma unroll
      for (int px = 0; px < PXP; ++px, to += px_step)
#pragma unroll
      for (int i = 0; i < NPQ; ++i) {
        const int mu = i * PXP + px;
        const float v = ds[mu / 4][mu % 4];
        const uint32_t hi = __builtin_bit_cast(uint16_t, static_cast<__bf16>(v));
        const uint32_t lo = __builtin_bit_cast(uint16_t, static_cast<__bf16>(v - __uint_as_float(hi << 16)));
        const uint32_t own = hi | lo << 16;
        const uint32_t other =                                         // quad_perm 1,0,3,2
            static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(own), 0xB1, 0xf, 0xf, true));
        // even: (own low, other low); odd: (other high, own high)
        const uint32_t w = __builtin_amdgcn_perm(other, own, pick);
        if (FULL || (NPQ * g + i < Pq && px < Px)) const_cast<uint32_t&>(at32(to, to_off + 64u * i)) = w;
      }
    }
    } else if (half == 0) {
      // no unit: factors of zeros
      for (int i = lane; i < wave_bytes<RUN>() / 16; i += 64) reinterpret_cast<uint4*>(mine)[i] = make_uint4(0, 0, 0, 0);
    }
    // (these barriers wait for LDS alone: the stores of ds and the next operands stay in flight)
    ring_barrier<63>();
    // dW1 += du s^T, dW2^T += h dl^T over the eight units' items, two units a K block:
    // slots 8 g + e are items 4 g + e % 4 of the one and the other
    if (half * kJT + j0 < 2 * JT2) {
      const unsigned char* u0 = waves + tr;
      const unsigned char* pj = u0 + 1024 * (2 * PT + (second ? 0 : kJT) + j0);      // h or du
      const unsigned char* pp = u0 + 1024 * ((second ? PT : 0) + pt0);               // dl or s
#pragma unroll 1
      for (int u = 0; u < kWaves; u += 2, pj += 2 * wave_bytes<RUN>(), pp += 2 * wave_bytes<RUN>()) {
        uint4 fj[JW][2], fp[PW][2];
        auto pair = [&](const unsigned char* at) {
          const uint2 x = read_tr(at), y = read_tr(at + wave_bytes<RUN>());
          return make_uint4(x.x, x.y, y.x, y.y);
        };
#pragma unroll
        for (int k = 0; k < 2; ++k) {
#pragma unroll
          for (int j = 0; j < JW; ++j) fj[j][k] = pair(pj + 1024 * j + 512 * k);
#pragma unroll
          for (int i = 0; i < PW; ++i) fp[i][k] = pair(pp + 1024 * i + 512 * k);
        }
#pragma unroll
        for (int k = 2; k >= 0; --k)                                  // small products first
#pragma unroll
          for (int j = 0; j < JW; ++j)
#pragma unroll
            for (int i = 0; i < PW; ++i) aw[half][j][i] = mfma_bf16(fj[j][k == 2], fp[i][k == 1], aw[half][j][i]);
      }
    }
    ring_barrier<63>();                                               // read before the next units, or halves, write
    }
  }

  // the workgroup's sums
  const long wg = static_cast<long>(blockIdx.y) * gridDim.x + blockIdx.x;
#pragma unroll
  for (int half = 0; half < HALVES; ++half)
#pragma unroll
    for (int j = 0; j < JW; ++j)
#pragma unroll
      for (int i = 0; i < PW; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          // rows: hidden units, 4 g + r of a tile; columns: slots, c (of dW2 too, as its transpose)
          const int jj = kH * half + 16 * (j0 + j) + 4 * g + r, p = component(16 * (pt0 + i) + c);
          if (jj < H && p >= 0) {
            if (second) out.dW2[(wg * P + p) * H + jj] = aw[half][j][i][r];
            else out.dW1[(wg * H + jj) * P + p] = aw[half][j][i][r];
          }
        }
  float* acc = reinterpret_cast<float*>(smb);                         // (in the place of everything in LDS)
#pragma unroll
  for (int jt = 0; jt < HALVES * kJT; ++jt)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float t = ab1[jt][i];
      t += row_ror<8>(t);
      t += row_ror<4>(t);
      t += row_ror<2>(t);
      t += row_ror<1>(t);
      if (c == 0) acc[wave * HU + 16 * jt + 4 * g + i] = t;
    }
  // (db2: da_x summed over the items)
  float* acc2 = acc + kWaves * HU;
  {
    const float t = sum_items<RUN>(dax, c);
    if (c < RUN) acc2[wave * SLOTS + RUN * g + c] = t;
  }
  __syncthreads();
  for (int i = tid; i < H; i += kThreads) {
    float t = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) t += acc[w * HU + i];
    out.db1[wg * H + i] = t;
  }
  for (int i = tid; i < SLOTS; i += kThreads) {
    float t = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) t += acc2[w * SLOTS + i];
    const int p = component(i);
    if (p >= 0) out.db2[wg * P + p] = t;
  }
  __syncthreads();
  // da_x: the waves of a block's queries in turn
  float* sx = acc + wave / dm.QB * (16 * SLOTS);                      // [blocks][16 items][slots]
  for (int w = 0; w < dm.QB; ++w) {
    __syncthreads();
    if (q == w) {
#pragma unroll
      for (int mu = 0; mu < RUN; ++mu) {
        float* o = sx + c * SLOTS + ((RUN * g + mu) ^ c);             // (spread over the banks)
        *o = w ? *o + dax[mu] : dax[mu];
      }
    }
  }
  __syncthreads();
  const int nblk = min(kWaves / dm.QB, dm.nb - static_cast<int>(blockIdx.x) * (kWaves / dm.QB));
  for (int i = tid; i < nblk * 16 * SLOTS; i += kThreads) {
    const int it = i / SLOTS, sl = i - it * SLOTS, p = component(sl);
    if (p >= 0)
      out.da_x[(static_cast<long>(blockIdx.y) * dm.ns + 16 * blockIdx.x * (kWaves / dm.QB) + it) * P + p] =
          acc[it * SLOTS + (sl ^ (it & 15))];
  }
}

// ---------------------------------------------------------------------------
// dQ and dX on matrix cores from ds: 32 rows and 64 columns a wave, K split.
// The rows of X and Q are the products' K: a chunk of 32 of them, 64 columns wide,
// goes through the wave's LDS and the transposing read.
struct GemmBf16 {
  int m, nb, d, npx;
  int splits;
  int items;         // of the slab: rows of X (dQ), rows of the output (dX)
  long x_px;         // dQ: elements between item components of X
  int direct;        // one split: out is the output itself
  long out_px;       // dX: elements between item components of out
  Tiles tiles;
};
constexpr int kTileA = 256;                          // 16-byte words of a wave's chunk of ds

// dQ[m][t] = sum over px and items of ds X; z: the split
template <bool VEC>
__device__ __forceinline__ void dq_tile(const GemmBf16& gd, uint32_t unit, const uint32_t* __restrict__ ds,
                                        const bf16_t* __restrict__ X, void* __restrict__ out, uint4* sh) {
  constexpr int RB = 2, CB = 4;
  const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  const int3 at = tile_of(gd.tiles, unit);
  const int m0 = at.x * 16 * RB, t0 = at.y * 16 * CB, z = at.z;
  const int per = gd.nb / 2, chunks = per * gd.npx;  // a chunk: two blocks of items
  const int k0 = static_cast<int>(static_cast<long>(chunks) * z / gd.splits);
  const int k1 = static_cast<int>(static_cast<long>(chunks) * (z + 1) / gd.splits);
  f32x4_t acc[RB][CB] = {};
  // Lane (c, g) reads piece g of row c of both blocks, rows of 64 bytes, whole;
  // the halves of the wave are then swapped to first terms (items 8 g .. of the
  // chunk) and second terms.
  const uint32_t* a[RB];
#pragma unroll
  for (int r = 0; r < RB; ++r) a[r] = ds + static_cast<long>(min(m0 + 16 * r + c, gd.m - 1)) * 16 + 4 * g;
  const RowTile<VEC> rows(gd.items, gd.d, t0);
  const long a_blk = 16l * gd.m;
  struct Chunk {
    uint4 a[RB][2], b[CB];
  };
  auto fetch = [&](Chunk& v, int ch) {                                // (px by px, the blocks follow each other)
    const int px = ch / per, k = ch - px * per;
#pragma unroll
    for (int r = 0; r < RB; ++r)
#pragma unroll
      for (int e = 0; e < 2; ++e) v.a[r][e] = *reinterpret_cast<const uint4*>(a[r] + (2l * ch + e) * a_blk);
    rows.fetch(v.b, X + px * gd.x_px, 32 * k);
  };
  auto use = [&](const Chunk& v, int ch) {
    rows.put(v.b, sh, 32 * (ch % per));
    wave_lds_sync();
    uint4 bv[CB];
#pragma unroll
    for (int t = 0; t < CB; ++t) bv[t] = column_of(sh, t, c, g);
#pragma unroll
    for (int r = 0; r < RB; ++r) {
      const uint4 x = v.a[r][0], y = v.a[r][1];
      const auto p0 = __builtin_amdgcn_permlane32_swap(x.x, y.x, false, false);
      const auto p1 = __builtin_amdgcn_permlane32_swap(x.y, y.y, false, false);
      const auto p2 = __builtin_amdgcn_permlane32_swap(x.z, y.z, false, false);
      const auto p3 = __builtin_amdgcn_permlane32_swap(x.w, y.w, false, false);
      const uint4 h = make_uint4(p0[0], p1[0], p2[0], p3[0]), l = make_uint4(p0[1], p1[1], p2[1], p3[1]);
#pragma unroll
      for (int t = 0; t < CB; ++t) acc[r][t] = mfma_bf16(l, bv[t], acc[r][t]);
#pragma unroll
      for (int t = 0; t < CB; ++t) acc[r][t] = mfma_bf16(h, bv[t], acc[r][t]);
    }
    wave_lds_sync();
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
  put_tile<bf16_t>(out, static_cast<long>(z) * gd.m * gd.d, m0, gd.m, t0, gd.d, gd.direct, acc);
}

// dX[px][n][t] = sum over (b, pq) of ds Q: rows of ds of a block of items, 32
// at a time, through the wave's LDS and the transposing read as well
// (z: px and split; sh: [block][32 rows][64 bytes], then the rows of Q)
template <bool VEC>
__device__ __forceinline__ void dx_tile(const GemmBf16& gd, uint32_t unit, const uint32_t* __restrict__ ds,
                                        const bf16_t* __restrict__ Q, void* __restrict__ out, uint4* sh) {
  constexpr int RB = 2, CB = 4;
  const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
  const int3 at = tile_of(gd.tiles, unit);                      // (no workgroup barrier below)
  const int blk0 = at.x * RB, t0 = at.y * 16 * CB, z = at.z;
  const int px = z / gd.splits, split = z - px * gd.splits;
  const int chunks = (gd.m + 31) / 32;
  const int k0 = static_cast<int>(static_cast<long>(chunks) * split / gd.splits);
  const int k1 = static_cast<int>(static_cast<long>(chunks) * (split + 1) / gd.splits);
  f32x4_t acc[RB][CB] = {};
  const uint4* a[RB];
#pragma unroll
  for (int r = 0; r < RB; ++r)
    a[r] = reinterpret_cast<const uint4*>(ds + (static_cast<long>(px) * gd.nb + min(blk0 + r, gd.nb - 1)) * gd.m * 16);
  const RowTile<VEC> rows(gd.m, gd.d, t0);
  struct Chunk {
    uint4 a[RB][2], b[CB];
  };
  const long last = static_cast<long>(gd.m) * 4 - 1;                  // 16-byte pieces of a block's rows
  auto fetch = [&](Chunk& v, int ch) {
#pragma unroll
    for (int r = 0; r < RB; ++r)
#pragma unroll
      for (int e = 0; e < 2; ++e) v.a[r][e] = a[r][min(ch * 128l + e * 64 + lane, last)];
    rows.fetch(v.b, Q, 32 * ch);
  };
  // K slots 8 g + e: rows 8 g + e
  const unsigned char* mine = reinterpret_cast<const unsigned char*>(sh) + (8 * g + (c >> 2)) * 64 + 8 * (c & 3);
  auto use = [&](const Chunk& v, int ch) {
#pragma unroll
    for (int r = 0; r < RB; ++r)
#pragma unroll
      for (int e = 0; e < 2; ++e)                                     // (rows past b pq: zeros, as Q's are)
        sh[r * 128 + e * 64 + lane] = ch * 128l + e * 64 + lane <= last ? v.a[r][e] : make_uint4(0, 0, 0, 0);
    rows.put(v.b, sh + kTileA, 32 * ch);
    wave_lds_sync();
    uint4 bv[CB];
#pragma unroll
    for (int t = 0; t < CB; ++t) bv[t] = column_of(sh + kTileA, t, c, g);
#pragma unroll
    for (int r = 0; r < RB; ++r) {
      const unsigned char* p = mine + r * 2048;
      const uint2 h0 = read_tr(p), h1 = read_tr(p + 256), l0 = read_tr(p + 32), l1 = read_tr(p + 288);
      const uint4 h = make_uint4(h0.x, h0.y, h1.x, h1.y), l = make_uint4(l0.x, l0.y, l1.x, l1.y);
#pragma unroll
      for (int t = 0; t < CB; ++t) acc[r][t] = mfma_bf16(l, bv[t], acc[r][t]);
#pragma unroll
      for (int t = 0; t < CB; ++t) acc[r][t] = mfma_bf16(h, bv[t], acc[r][t]);
    }
    wave_lds_sync();
  };
  Chunk v0, v1;
  if (k0 < k1) fetch(v0, k0);
  for (int ch = k0; ch < k1; ch += 2) {
    fetch(v1, min(ch + 1, k1 - 1));
    use(v0, ch);
    fetch(v0, min(ch + 2, k1 - 1));
    if (ch + 1 < k1) use(v1, ch + 1);
  }
  put_tile<bf16_t>(out, (static_cast<long>(split) * gd.npx + px) * gd.out_px, 16 * blk0, gd.items, t0, gd.d, gd.direct,
                         acc);
}

// Both products, side by side: the first tiles are dQ's.
// VEC: rows of X and Q of whole 16-byte words.
template <bool VEC>
__global__ __launch_bounds__(256) void k_grad_products_bf16(GemmBf16 q, GemmBf16 x, const uint32_t* __restrict__ ds,
                                                            const bf16_t* __restrict__ X, const bf16_t* __restrict__ Q,
                                                            void* __restrict__ out_q, void* __restrict__ out_x) {
  __shared__ __attribute__((aligned(16))) uint4 sh[4][kTileB + kTileA];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t unit = blockIdx.x * 4 + wave, nq = static_cast<uint32_t>(q.tiles.count());
  if (unit < nq)
    dq_tile<VEC>(q, unit, ds, X, out_q, sh[wave]);
  else if (unit - nq < static_cast<uint32_t>(x.tiles.count()))
    dx_tile<VEC>(x, unit - nq, ds, Q, out_x, sh[wave]);
}

// ---------------------------------------------------------------------------
namespace grad {

namespace {

struct Bf16Plan {
  Bf16Dims dm;
  int slab, slabs, wgx, wgs;
  int sp_q, sp_x;
  size_t off_ds, off_daq, off_dax, off_dw1, off_dw2, off_db1, off_db2, off_pq, off_px, off_acc, bytes;
  long a_dw1, a_dw2, a_db1, a_db2, a_dq;       // floats into the sums over slabs
};

// waves that share 16 items, and the bytes of an item of a slab: ds, da_x and what the workgroups leave
int queries_of(long B) { return B >= 8 ? 8 : B >= 4 ? 4 : B >= 2 ? 2 : 1; }
size_t wg_bytes(const DevProb& pr) { return 4ul * (2ul * pr.H * pr.P + pr.H + pr.P); }
size_t item_bytes(const DevProb& pr, long B, int QB) {
  return 4ul * pr.P * (B + 1) + (wg_bytes(pr) * QB + 16 * kWaves - 1) / (16 * kWaves);
}

Bf16Plan plan(const DevProb& pr) {
  Bf16Plan f{};
  Bf16Dims& dm = f.dm;
  dm.QB = queries_of(pr.B);
  dm.m = static_cast<long>(pr.B) * pr.Pq;
  const long blocks = (pr.N + 31l) / 32;                              // slabs of whole pairs of 16 items
  const long fit = std::max<long>(1, static_cast<long>(kSlabBytes / (32 * item_bytes(pr, pr.B, dm.QB))));
  f.slabs = static_cast<int>((blocks + fit - 1) / fit);
  f.slab = static_cast<int>((blocks + f.slabs - 1) / f.slabs * 32);
  f.slabs = static_cast<int>((static_cast<long>(pr.N) + f.slab - 1) / f.slab);
  dm.ns = f.slab;
  dm.nb = f.slab / 16;
  const int steps = (pr.B + dm.QB - 1) / dm.QB, per = kWaves / dm.QB;
  f.wgx = (dm.nb + per - 1) / per;
  dm.qsplits = std::max(1, std::min(steps, 256 / f.wgx));
  f.wgs = f.wgx * dm.qsplits;
  const long cg = (pr.d + 63) / 64;
  f.sp_q = split_of((dm.m + 31) / 32 * cg, static_cast<long>(pr.Px) * dm.nb / 2, 4);
  f.sp_x = split_of(static_cast<long>(dm.nb) / 2 * cg * pr.Px, (dm.m + 31) / 32, 4);
  auto up = [](size_t v) { return (v + 255) / 256 * 256; };
  size_t at = 0;
  const size_t P = pr.P, H = pr.H;
  f.off_ds = at;  at = up(at + 4ul * pr.Px * dm.m * f.slab);
  f.off_daq = at; at = up(at + 4ul * dm.nb * pr.B * P);
  f.off_dax = at; at = up(at + 4ul * dm.qsplits * f.slab * P);
  f.off_dw1 = at; at = up(at + 4ul * f.wgs * H * P);
  f.off_dw2 = at; at = up(at + 4ul * f.wgs * H * P);
  f.off_db1 = at; at = up(at + 4ul * f.wgs * H);
  f.off_db2 = at; at = up(at + 4ul * f.wgs * P);
  f.off_pq = at;  at = up(at + 4ul * f.sp_q * dm.m * pr.d);
  f.off_px = at;  at = up(at + (f.sp_x > 1 ? 4ul * f.sp_x * pr.Px * f.slab * pr.d : 0));
  f.a_dw1 = static_cast<long>(pr.B) * P;
  f.a_dw2 = f.a_dw1 + static_cast<long>(H * P);
  f.a_db1 = f.a_dw2 + static_cast<long>(H * P);
  f.a_db2 = f.a_db1 + static_cast<long>(H);
  f.a_dq = f.a_db2 + static_cast<long>(P);
  f.off_acc = at; at = up(at + 4ul * (f.a_dq + (f.slabs > 1 ? dm.m * pr.d : 0)));
  f.bytes = at;
  return f;
}

template <int NPQ, int PXP, int HALVES>
hipError_t launch_pairs(const DevProb& pr, const Bf16Plan& f, Bf16Dims dm, const float* dphi,
                        const Bf16Parts& parts, hipStream_t st) {
  auto aligned = [](const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; };
  const bool full = pr.Pq == 4 * NPQ && pr.Px == PXP && pr.d % 8 == 0 && aligned(pr.Q) && aligned(pr.X) && aligned(pr.a_q) &&
                    aligned(pr.a_x) && aligned(pr.b1) && aligned(pr.b2) && pr.H % 4 == 0;
  // the items' rows in LDS where the workgroup has one block of items: whole, or the first
  // blocks of 32 that there is room for (the loaded-ahead ones at least)
  constexpr int base = lds_bytes<NPQ * PXP, HALVES>(), room = (160 * 1024 - base) / x_bytes(PXP);
  static_assert(room >= kAhead, "LDS");
  const int blocks = (pr.d + 31) / 32;
  dm.kl = dm.QB == kWaves ? std::min(blocks, room) : 0;
  const int lds = base + dm.kl * x_bytes(PXP);
  auto of = [&](auto xl) {
    constexpr int XL = decltype(xl)::value, all = 2 * HALVES;
    return full ? (HALVES == 1 && pr.H <= 32 ? &k_score_grad_bf16<NPQ, PXP, XL, 1, 1> : &k_score_grad_bf16<NPQ, PXP, XL, all, HALVES>)
                : &k_score_grad_bf16<NPQ, PXP, XL, 0, HALVES>;
  };
  auto kern = dm.kl == 0 ? of(std::integral_constant<int, 0>())
              : dm.kl == blocks ? of(std::integral_constant<int, 1>()) : of(std::integral_constant<int, 2>());
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(kern, dim3(f.wgx, dm.qsplits), dim3(kThreads), lds, st, pr, dm, dphi, parts);
  return hipGetLastError();
}

}  // namespace

// (a problem that asks for float32 gets it throughout)
static bool bf16_shape(const DevProb& pr) {
  return pr.dtype == MOL_BF16 && !(pr.flags & MOL_FLAG_F32_GATING) && pr.Pq <= 8 &&
         (pr.H <= kH ? pr.Px <= 8 : pr.H <= 2 * kH && pr.Px <= 4);
}
bool bf16_supported(const DevProb& pr) {
  // (a lane's offsets from its wave's bases in 32 bits)
  return bf16_shape(pr) && static_cast<long>(pr.N) * pr.d < (1l << 31) && static_cast<long>(pr.N) * pr.P < (1l << 30);
}

size_t bf16_bytes(const DevProb& pr) { return plan(pr).bytes; }

// Each term bounds a part of plan()'s workspace by what grows with B and N alone, for
// the batches of each QB: slabs, splits and ranges of the queries fall as well as rise with them.
size_t bf16_most(const DevProb& pr) {
  if (!bf16_shape(pr)) return 0;
  size_t most = 0;
  for (int QB = 1; QB <= queries_of(pr.B); QB *= 2) {
    const size_t B = std::min<long>(pr.B, QB == 8 ? pr.B : 2 * QB - 1), m = B * pr.Pq, P = pr.P;
    const size_t items = (pr.N + 31ul) / 32 * 32, item = item_bytes(pr, B, QB), wg = wg_bytes(pr);
    // ds, da_x of one range of queries and the workgroups' sums; da_q is a sixteenth of ds
    const size_t slab = std::min(item * items, std::max(kSlabBytes, 32 * item)) + wg;
    // more ranges of queries: 256 workgroups at most
    const size_t steps = (B + QB - 1) / QB, wgs = std::min<size_t>(256, steps * (items * QB / (16 * kWaves) + 1));
    const size_t ranges = wg * wgs + 4 * P * std::min<size_t>(256ul * 16 * kWaves / QB, steps * items);
    const size_t q = 4 * m * pr.d;
    const size_t products = std::max(q, most_parts(q, pr.Px * items / 32, 4)) + most_parts(4 * pr.Px * items * pr.d, (m + 31) / 32, 4);
    most = std::max(most, slab + slab / 16 + ranges + products + 4 * B * P + wg + q + 16 * 256);
  }
  return (most + 255) / 256 * 256;
}

hipError_t launch_bf16(const DevProb& pr, const float* dphi, const mol_score_grads& o, char* ws, hipStream_t st) {
  const Bf16Plan f = plan(pr);
  Bf16Dims dm = f.dm;
  auto F = [&](size_t off) { return reinterpret_cast<float*>(ws + off); };
  const Bf16Parts parts{reinterpret_cast<uint32_t*>(ws + f.off_ds), F(f.off_daq), F(f.off_dax), F(f.off_dw1),
                        F(f.off_dw2), F(f.off_db1), F(f.off_db2)};
  float* acc = F(f.off_acc);
  auto pairs = pr.H > kH ? (pr.Pq <= 4 ? &launch_pairs<1, 4, 2> : &launch_pairs<2, 4, 2>)
               : pr.Px > 4 ? &launch_pairs<2, 8, 1>
                           : (pr.Pq <= 4 ? &launch_pairs<1, 4, 1> : &launch_pairs<2, 4, 1>);
  const int cg = (pr.d + 63) / 64;
  const long P = pr.P, H = pr.H, BP = pr.B * P;
  SumList sums(st);
  for (int sl = 0; sl < f.slabs; ++sl) {
    const bool last = sl + 1 == f.slabs;
    dm.n0 = sl * f.slab;
    dm.items = std::min(f.slab, pr.N - dm.n0);
    hipError_t e;
    if ((e = pairs(pr, f, dm, dphi, parts, st)) != hipSuccess) return e;
    const long per_px = static_cast<long>(dm.items) * pr.d;
    if (o.dQ || o.dX) {
      // a product of one split (of dQ: and one slab) is stored as bf16
      const bool dir_q = f.sp_q == 1 && f.slabs == 1, dir_x = f.sp_x == 1;
      const int m = static_cast<int>(dm.m);
      const GemmBf16 gq{m, dm.nb, pr.d, pr.Px, f.sp_q, dm.items, static_cast<long>(pr.N) * pr.d, dir_q, 0,
                        Tiles{(m + 31) / 32, cg, o.dQ ? f.sp_q : 0}};
      const GemmBf16 gx{m, dm.nb, pr.d, pr.Px, f.sp_x, dm.items, 0, dir_x,
                        dir_x ? static_cast<long>(pr.N) * pr.d : per_px, Tiles{(dm.nb + 1) / 2, cg, o.dX ? f.sp_x * pr.Px : 0}};
      void* to_q = dir_q ? o.dQ : F(f.off_pq);
      void* to_x = dir_x ? static_cast<bf16_t*>(o.dX) + static_cast<long>(dm.n0) * pr.d : static_cast<void*>(F(f.off_px));
      const bf16_t* X = static_cast<const bf16_t*>(pr.X) + static_cast<long>(dm.n0) * pr.d;
      const bf16_t* Q = static_cast<const bf16_t*>(pr.Q);
      const bool vec = pr.d % 8 == 0 && ((reinterpret_cast<uintptr_t>(pr.X) | reinterpret_cast<uintptr_t>(pr.Q)) & 15) == 0;
      const long units = gq.tiles.count() + gx.tiles.count();
      auto products = vec ? &k_grad_products_bf16<true> : &k_grad_products_bf16<false>;
      hipLaunchKernelGGL(products, dim3(static_cast<unsigned>((units + 3) / 4)), dim3(256), 0, st, gq, gx, parts.ds, X, Q,
                         to_q, to_x);
    }
    if (o.dQ && (f.sp_q > 1 || f.slabs > 1))
      sums.add({F(f.off_pq), dm.m * pr.d, dm.m * pr.d, f.sp_q, f.slabs > 1 ? acc + f.a_dq : nullptr, sl > 0,
                last ? o.dQ : nullptr, 1, dm.m * pr.d, dm.m * pr.d, 0});
    if (o.dX && f.sp_x > 1)
      sums.add({F(f.off_px), per_px * pr.Px, per_px * pr.Px, f.sp_x, nullptr, 0, o.dX, 1, per_px,
                static_cast<long>(pr.N) * pr.d, static_cast<long>(dm.n0) * pr.d});
    if (o.da_q)
      sums.add({parts.da_q, BP, BP, dm.nb, acc, sl > 0, last ? o.da_q : nullptr, 0, BP, BP, 0});
    if (o.da_x)
      sums.add({parts.da_x, dm.items * P, f.slab * P, dm.qsplits, nullptr, 0, o.da_x, 0, dm.items * P, dm.items * P,
                static_cast<long>(dm.n0) * P});
    if (o.dW1)
      sums.add({parts.dW1, H * P, H * P, f.wgs, acc + f.a_dw1, sl > 0, last ? o.dW1 : nullptr, 1, H * P, H * P, 0});
    if (o.dW2)
      sums.add({parts.dW2, H * P, H * P, f.wgs, acc + f.a_dw2, sl > 0, last ? o.dW2 : nullptr, 1, H * P, H * P, 0});
    if (o.db1) sums.add({parts.db1, H, H, f.wgs, acc + f.a_db1, sl > 0, last ? o.db1 : nullptr, 0, H, H, 0});
    if (o.db2) sums.add({parts.db2, P, P, f.wgs, acc + f.a_db2, sl > 0, last ? o.db2 : nullptr, 0, P, P, 0});
    if ((e = sums.run()) != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace grad

}  // namespace mol
