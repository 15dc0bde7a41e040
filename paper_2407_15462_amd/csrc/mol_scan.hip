// A gated linear recurrence over histories, and its gradient.  For each channel of
// each history (tokens offsets[b] .. offsets[b + 1] - 1 of packed rows):
//   f_t = 1 / (1 + e^{-gate_t}),  h_t = f_t h_{t-1} + (1 - f_t) x_t,  h_{-1} = h0
// and back, with D_t = dL / dh_t in all, E_t = f_t D_t, E behind the last token = dlast:
//   D_t = dh_t + E_{t+1},  dx_t = (1 - f_t) D_t,  dgate_t = f_t (1 - f_t) (h_{t-1} - x_t) D_t,  dh0 = E_0
//
// Both are linear maps of the state that comes in, state -> A state + H, which join:
// the scan cuts the packed tokens, wherever histories end, into chunks of equal length,
// each read once.  A workgroup holds a chunk of 128 channels (two a lane): each
// wave, or part of a wave where there are few channels, takes a slice of S tokens
// and runs through it from state 0, keeping every token's A and H; slices are
// joined in LDS; the workgroup publishes the chunk's (A, H), gets the state that comes
// in from the chunks before, and writes h = A state + H.  A history's first
// token starts from h0 with A = 0, so that nothing crosses from one history to the next.
//
// The state that comes in is formed in an order that the sizes and offsets fix: the
// state at the end of the group of kGroup chunks before (published by the
// group's last chunk), then the (A, H) of the chunks since, in order; both only from the chunk in
// which the history starts.  So a long history is a chain of one wait a group, and
// short ones are none at all.
//
// Waiting is sure to end: workgroups take their chunks by a ticket, in order, so that
// a chunk's predecessors belong to workgroups that run or have ended, and each
// publishes its (A, H) before it waits for anything.  A published pair is one
// 64-bit word, whose top bit (the sign of A, which is not negative) says that it is there.
#include <algorithm>

#include "mol_kernels.h"
#include "mol_vec.h"

namespace mol {

namespace {

using vec::Raw;

constexpr int kWaves = 8, kThreads = 64 * kWaves;
constexpr int kGroup = 32;                // chunks of a group
constexpr int kSlots = kGroup / kWaves;   // whose pairs a wave reads
constexpr float kLog2E = 1.4426950408889634f, kLog2ELo = 1.925963033500e-8f, kLn2 = 0.6931471805599453f;

struct ScanArgs {
  int T, d, B;
  int chunks, groups;      // of tokens; of channels (128 or what there are)
  int lanes_log2;          // lanes of a row
  const void* gate;
  const void* x;
  const int32_t* offsets;  // or NULL: one history of all tokens
  const float* h0;
  void* h;                 // forward: written; back: read
  int h_bf16;              // forward
  float* last;             // forward: the last states, or NULL
  const void* dh;          // back, or NULL
  const float* dlast;
  void* dgate;
  void* dx;
  float* dh0;
  uint32_t* ticket;        // workspace
  int2* plan;              // of each chunk: the first history that it holds tokens of, and the chunk
                           // that the state coming in starts from (the chunk itself: none comes in)
  uint64_t* pairs;         // [chunks][d]
  uint64_t* states;        // [chunks / kGroup][d]
};

__device__ __forceinline__ int offset_at(const ScanArgs& a, int i) {
  if (!a.offsets) return i ? a.T : 0;
  return min(max(a.offsets[i], 0), a.T);
}

struct Gate {
  float f, rest;           // sigmoid(gate), sigmoid(-gate)
};
__device__ __forceinline__ Gate gate_of(float g) {
  const float n = -fabsf(g), t = n * kLog2E;
  const float r = fmaf(n, kLog2ELo, fmaf(n, kLog2E, -t));
  const float e0 = __builtin_amdgcn_exp2f(t);
  const float e = e0 == 0.f ? 0.f : fmaf(e0, r * kLn2, e0);    // e^{-|g|}
  const float s = __builtin_amdgcn_rcpf(1.f + e), q = e * s;
  return g >= 0.f ? Gate{s, q} : Gate{q, s};
}

// a v, and 0 for a = 0 whatever v is (another history's state)
__device__ __forceinline__ float through(float a, float v) { return a == 0.f ? 0.f : a * v; }

__device__ __forceinline__ void publish(uint64_t* p, float a, float h) {
  const uint64_t v = static_cast<uint64_t>(__float_as_uint(a) | 0x80000000u) << 32 | __float_as_uint(h);
  __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uint64_t look(const uint64_t* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ bool there(uint64_t v) { return v >> 63; }
__device__ __forceinline__ float a_of(uint64_t v) { return __uint_as_float(static_cast<uint32_t>(v >> 32) & 0x7FFFFFFFu); }
__device__ __forceinline__ float h_of(uint64_t v) { return __uint_as_float(static_cast<uint32_t>(v)); }

// two channels, or the one that there is
template <bool EVEN, typename T>
__device__ __forceinline__ void put(T* p, const float (&v)[2], int n) {
  if (EVEN)
    vec::store(p, v);
  else
    vec::store(p, v, n);
}

// First history that has tokens at t or behind: the number of ends offsets[1 .. B] up to t,
// by a wave, 64 ways a step.
__device__ __forceinline__ int ends_up_to(const ScanArgs& a, int t) {
  const int lane = threadIdx.x & 63;
  int lo = 0, hi = a.B;                    // the count is in [lo, hi]
  while (lo < hi) {
    const int step = (hi - lo + 63) / 64;
    const int i = lo + lane * step;        // ends i + 1 .. : is end i + 1 up to t?
    const bool in = i < hi && offset_at(a, i + 1) <= t;
    const int n = __popcll(__ballot(in));
    if (n == 0) return lo;
    lo = lo + (n - 1) * step + 1;
    hi = min(hi, lo + step - 1);
  }
  return lo;
}

}  // namespace

// What the chunks need to know of the histories, the workspace cleared, and the last
// states (or the first states' gradients) of histories without tokens.
template <bool BACK>
__global__ __launch_bounds__(256) void k_scan_plan(ScanArgs a, int chunk_len) {
  const long tid = static_cast<long>(blockIdx.x) * 256 + threadIdx.x, all = static_cast<long>(gridDim.x) * 256;
  const int lane = threadIdx.x & 63;
  if (a.ticket && tid == 0) *a.ticket = 0;
  const long words = (static_cast<long>(a.chunks) + a.chunks / kGroup) * a.d;      // (states lie behind pairs)
  for (long i = tid; i < words; i += all) a.pairs[i] = 0;
  for (long c = tid / 64; c < a.chunks; c += all / 64) {
    int first, from = static_cast<int>(c);
    if (!BACK) {
      const int t = static_cast<int>(c) * chunk_len;
      first = ends_up_to(a, t);
      if (first < a.B) {
        const int start = offset_at(a, first);
        if (start < t) from = start / chunk_len;
      }
    } else {
      const int end = a.T - static_cast<int>(c) * chunk_len, t = max(0, end - chunk_len);
      first = ends_up_to(a, t);
      // the history of the chunk's last token, where the run back begins
      const int b = ends_up_to(a, end - 1);
      if (b < a.B && offset_at(a, b) < end) {
        const int stop = offset_at(a, b + 1);
        if (stop > end) from = (a.T - stop) / chunk_len;
      }
    }
    if (lane == 0) a.plan[c] = make_int2(first, from);
  }
  float* out = BACK ? a.dh0 : a.last;
  const float* in = BACK ? a.dlast : a.h0;
  if (!out) return;
  for (long b0 = tid / 64 * 64; b0 < a.B; b0 += all) {
    const int b = static_cast<int>(b0) + lane;
    uint64_t m = __ballot(b < a.B && offset_at(a, b) >= offset_at(a, b + 1));
    for (; m; m &= m - 1) {
      const long at = (b0 + __builtin_ctzll(m)) * a.d;
      for (int c = lane; c < a.d; c += 64) out[at + c] = in ? in[at + c] : 0.f;
    }
  }
}

// UNI: a wave's lanes share their slice (more than 64 channels), so that what depends on
// the token alone is a scalar.  EVEN: an even number of channels, so that lanes
// without channels of their own can read others'.
template <bool BACK, typename T, typename TH, int S, bool UNI, bool EVEN>
__global__ __launch_bounds__(kThreads, 4) void k_scan(ScanArgs a) {
  constexpr int kMost = UNI ? kWaves * S : kWaves * S * 16;    // tokens of a chunk (4 lanes a row at least)
  constexpr int kBlock = S < 8 ? S : 8;                        // tokens whose loads are in flight together on the way out
  __shared__ uint32_t flags[kMost / S];                        // of a slice: the tokens at which a history begins, those at which
                                                               // it ends << 16 (in the scan's direction)
  __shared__ int begin_b[kMost], end_b[kMost];                 // whose
  __shared__ float sum_a[kWaves][128], sum_h[kWaves][128];     // [wave][channel]
  __shared__ float in_a[kWaves][128], in_h[kWaves][128], in_s[128];
  __shared__ int my_ticket;

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int lanes = UNI ? 64 : 1 << a.lanes_log2, per_wave = UNI ? 1 : 64 >> a.lanes_log2;
  const int sub = UNI ? 0 : lane >> a.lanes_log2;              // which slice of the wave's
  const int slice = wave * per_wave + sub, slices = kWaves * per_wave, len = slices * S;
  int unit = blockIdx.x;
  if (a.chunks > 1) {
    if (tid == 0) my_ticket = __hip_atomic_fetch_add(a.ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    unit = __builtin_amdgcn_readfirstlane(my_ticket);
  }
  const int chunk = unit / a.groups, cg = unit - chunk * a.groups, d = a.d;
  const int row_lane = UNI ? lane : lane & (lanes - 1);
  const int ch = cg * 128 + 2 * row_lane, nch = d - ch;        // this lane's channels: 2 or 1 (or none)
  const uint32_t from_ch = EVEN ? min(ch, d - 2) : min(ch, d - 1);

  // tokens in the scan's direction: i = 0 .. len - 1 of the chunk stands for token
  // first + i, or first - i on the way back
  const int first = BACK ? a.T - 1 - chunk * len : chunk * len;
  const int lo = BACK ? max(0, first + 1 - len) : first;
  const int hi = BACK ? first + 1 : min(a.T, first + len);
  const int live_lo = __builtin_amdgcn_readfirstlane(max(lo, offset_at(a, 0)));
  const int live_hi = __builtin_amdgcn_readfirstlane(min(hi, offset_at(a, a.B)));

  for (int i = tid; i < slices; i += kThreads) flags[i] = 0;
  __syncthreads();
  int2 plan = a.chunks > 1 ? a.plan[chunk] : make_int2(0, 0);
  plan.x = __builtin_amdgcn_readfirstlane(plan.x);
  plan.y = __builtin_amdgcn_readfirstlane(plan.y);
  for (int b = plan.x + tid; b < a.B; b += kThreads) {
    const int s = offset_at(a, b), e = offset_at(a, b + 1);
    if (a.chunks > 1 && s >= hi) break;
    if (s >= e) {
      // (without a plan's launch, histories without tokens are seen to here)
      float* out = BACK ? a.dh0 : a.last;
      const float* in = BACK ? a.dlast : a.h0;
      if (a.chunks == 1 && out)
        for (int c = cg * 128; c < min(d, cg * 128 + 128); ++c)
          out[static_cast<long>(b) * d + c] = in ? in[static_cast<long>(b) * d + c] : 0.f;
      continue;
    }
    const int tb = BACK ? e - 1 : s, te = BACK ? s : e - 1;
    if (tb >= lo && tb < hi) {
      const int i = BACK ? first - tb : tb - first;
      begin_b[i] = b;
      atomicOr(&flags[i / S], 1u << i % S);
    }
    if (te >= lo && te < hi) {
      const int i = BACK ? first - te : te - first;
      end_b[i] = b;
      atomicOr(&flags[i / S], 0x10000u << i % S);
    }
  }
  __syncthreads();
  uint32_t flag = flags[slice];
  if (UNI) flag = __builtin_amdgcn_readfirstlane(flag);
  const int t_first = BACK ? first - slice * S : first + slice * S;
  auto token = [&](int s) { return BACK ? t_first - s : t_first + s; };
  auto live = [&](int s) { return token(s) >= live_lo && token(s) < live_hi; };
  // Rows that are no history's are not read (another's stands in): what comes of
  // them is not written, and the next history begins anew.
  const int read_lo = live_lo < live_hi ? live_lo : lo, read_hi = live_lo < live_hi ? live_hi : hi;
  auto load = [&](auto& r, const auto* base, int t) {
    const auto* p = base + static_cast<int64_t>(min(max(t, read_lo), read_hi - 1)) * d + from_ch;
    if (EVEN)
      r.load(p);
    else
      r.load(p, nch);
  };

  // the slice from state 0: p[s] = A, q[s] = H; on the way back of D_t
  Raw<T, 2> gate[S];
  float p[S][2], q[S][2];
  float A[2] = {1.f, 1.f}, H[2] = {0.f, 0.f};
  {
    Raw<T, 2> xr[BACK ? 1 : S];
    Raw<TH, 2> dr[BACK ? S : 1];
#pragma unroll
    for (int s = 0; s < S; ++s) {
      load(gate[s], static_cast<const T*>(a.gate), token(s));
      if constexpr (BACK) {
        dr[s].zero();
        if (a.dh) load(dr[s], static_cast<const TH*>(a.dh), token(s));
      } else {
        load(xr[s], static_cast<const T*>(a.x), token(s));
      }
    }
#pragma unroll
    for (int s = 0; s < S; ++s) {
      if (flag >> s & 1) {
        const float* in = BACK ? a.dlast : a.h0;
        const long at = static_cast<long>(begin_b[slice * S + s]) * d + ch;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          A[e] = 0.f;
          H[e] = in && e < nch ? in[at + e] : 0.f;
        }
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const Gate g = gate_of(gate[s].at(e));
        if constexpr (BACK) {
          p[s][e] = A[e];
          q[s][e] = dr[s].at(e) + H[e];
          A[e] *= g.f;
          H[e] = g.f * q[s][e];
        } else {
          p[s][e] = A[e] *= g.f;
          q[s][e] = H[e] = fmaf(g.f, H[e], g.rest * xr[s].at(e));
        }
      }
    }
  }

  // slices joined: (A, H) of all slices before this one, within the wave, then over waves
  float before_a[2] = {1.f, 1.f}, before_h[2] = {0.f, 0.f}, wave_a[2], wave_h[2];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    float ca = A[e], chh = H[e];                 // inclusive over slices of the wave
    if (!UNI) {
      for (int o = lanes; o < 64; o <<= 1) {
        const float ua = __shfl_up(ca, o), uh = __shfl_up(chh, o);
        if (lane >= o) {
          chh += through(ca, uh);
          ca = through(ca, ua);
        }
      }
      const float ua = __shfl_up(ca, lanes), uh = __shfl_up(chh, lanes);
      if (sub) before_a[e] = ua, before_h[e] = uh;
    }
    wave_a[e] = ca;
    wave_h[e] = chh;
    if (sub == per_wave - 1) {
      sum_a[wave][2 * row_lane + e] = ca;
      sum_h[wave][2 * row_lane + e] = chh;
    }
  }
  __syncthreads();
  float pre_a[2] = {1.f, 1.f}, pre_h[2] = {0.f, 0.f};           // of the waves before
  for (int w = 0; w < wave; ++w)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const float wa = sum_a[w][2 * row_lane + e], wh = sum_h[w][2 * row_lane + e];
      pre_h[e] = wh + through(wa, pre_h[e]);
      pre_a[e] = through(wa, pre_a[e]);
    }
  float all_a[2], all_h[2];                                     // of the chunk (the last wave's last slice)
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    all_h[e] = wave_h[e] + through(wave_a[e], pre_h[e]);
    all_a[e] = through(wave_a[e], pre_a[e]);
  }
  const bool speaks = wave == kWaves - 1 && sub == per_wave - 1;
  if (a.chunks > 1 && speaks)
#pragma unroll
    for (int e = 0; e < 2; ++e)
      if (e < nch) publish(a.pairs + static_cast<long>(chunk) * a.d + ch + e, all_a[e], all_h[e]);

  // the state that comes in
  float state[2] = {0.f, 0.f};
  if (plan.y < chunk) {
    const int group0 = chunk / kGroup * kGroup, from = max(plan.y, group0);
    float ra[2] = {1.f, 1.f}, rh[2] = {0.f, 0.f};
    uint64_t got[kSlots][2];
    bool missing = false;
#pragma unroll
    for (int k = 0; k < kSlots; ++k) {
      const int j = group0 + wave * kSlots + k;
#pragma unroll
      for (int e = 0; e < 2; ++e)
        got[k][e] = j >= from && j < chunk && e < nch ? look(a.pairs + static_cast<long>(j) * a.d + ch + e) : ~0ull;
    }
    do {
      missing = false;
#pragma unroll
      for (int k = 0; k < kSlots; ++k) {
        const int j = group0 + wave * kSlots + k;
#pragma unroll
        for (int e = 0; e < 2; ++e)
          if (!there(got[k][e])) {
            got[k][e] = look(a.pairs + static_cast<long>(j) * a.d + ch + e);
            missing = missing || !there(got[k][e]);
          }
      }
      if (missing) __builtin_amdgcn_s_sleep(2);
    } while (missing);
#pragma unroll
    for (int k = 0; k < kSlots; ++k) {
      const int j = group0 + wave * kSlots + k;
      if (j >= from && j < chunk)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float wa = a_of(got[k][e]);
          rh[e] = h_of(got[k][e]) + through(wa, rh[e]);
          ra[e] = through(wa, ra[e]);
        }
    }
    if (sub == 0)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        in_a[wave][2 * row_lane + e] = ra[e];
        in_h[wave][2 * row_lane + e] = rh[e];
      }
    if (wave == 0 && plan.y < group0 && sub == 0)
#pragma unroll
      for (int e = 0; e < 2; ++e)
        if (e < nch) {
          const uint64_t* w = a.states + static_cast<long>(chunk / kGroup - 1) * a.d + ch + e;
          uint64_t v = look(w);
          while (!there(v)) {
            __builtin_amdgcn_s_sleep(2);
            v = look(w);
          }
          in_s[2 * row_lane + e] = h_of(v);
        }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      state[e] = plan.y < group0 ? in_s[2 * row_lane + e] : 0.f;
      for (int w = 0; w < kWaves; ++w)
        state[e] = in_h[w][2 * row_lane + e] + through(in_a[w][2 * row_lane + e], state[e]);
    }
  }
  if (a.chunks > 1 && chunk % kGroup == kGroup - 1 && speaks)
#pragma unroll
    for (int e = 0; e < 2; ++e)
      if (e < nch)
        publish(a.states + static_cast<long>(chunk / kGroup) * a.d + ch + e, 0.f, all_h[e] + through(all_a[e], state[e]));
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    state[e] = pre_h[e] + through(pre_a[e], state[e]);          // over the waves before,
    state[e] = before_h[e] + through(before_a[e], state[e]);    // and the wave's slices before
  }

  // out
  if (nch <= 0) return;
  if constexpr (!BACK) {
#pragma unroll
    for (int s = 0; s < S; ++s) {
      if (flag >> s & 1) state[0] = state[1] = 0.f;
      if (!live(s)) continue;
      const float v[2] = {fmaf(p[s][0], state[0], q[s][0]), fmaf(p[s][1], state[1], q[s][1])};
      const int64_t row = static_cast<int64_t>(token(s)) * d;
      if (a.h_bf16)
        put<EVEN>(static_cast<bf16_t*>(a.h) + row + from_ch, v, nch);
      else
        put<EVEN>(static_cast<float*>(a.h) + row + from_ch, v, nch);
      if (a.last && (flag >> (16 + s) & 1)) put<EVEN>(a.last + static_cast<long>(end_b[slice * S + s]) * d + from_ch, v, nch);
    }
  } else {
    // (the gates are formed again: kept from above they would take S more registers for each channel)
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
      for (int i = 0; i < Raw<T, 2>::kWords; ++i) asm volatile("" : "+v"(gate[s].w[i]));
#pragma unroll
    for (int s0 = 0; s0 < S; s0 += kBlock) {
      Raw<T, 2> xr[kBlock];
      Raw<TH, 2> hr[kBlock];
#pragma unroll
      for (int i = 0; i < kBlock; ++i) {
        load(xr[i], static_cast<const T*>(a.x), token(s0 + i));
        // (of a history's first token not used)
        const TH* before = static_cast<const TH*>(a.h) + static_cast<int64_t>(max(token(s0 + i) - 1, 0)) * d + from_ch;
        if (EVEN)
          hr[i].load(before);
        else
          hr[i].load(before, nch);
      }
#pragma unroll
      for (int i = 0; i < kBlock; ++i) {
        const int s = s0 + i;
        const int64_t row = static_cast<int64_t>(token(s)) * d;
        if (flag >> s & 1) state[0] = state[1] = 0.f;
        if (!live(s)) {                        // rows of no history: no loss depends on them
          const float none[2] = {0.f, 0.f};
          if (token(s) >= 0) {
            put<EVEN>(static_cast<T*>(a.dgate) + row + from_ch, none, nch);
            put<EVEN>(static_cast<T*>(a.dx) + row + from_ch, none, nch);
          }
          continue;
        }
        float prev[2] = {hr[i].at(0), hr[i].at(1)}, dg[2], dx[2], out[2];
        const bool stops = flag >> (16 + s) & 1;
        const long b = stops ? end_b[slice * S + s] : 0;
        if (stops)
#pragma unroll
          for (int e = 0; e < 2; ++e) prev[e] = a.h0 && e < nch ? a.h0[b * d + ch + e] : 0.f;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const Gate g = gate_of(gate[s].at(e));
          const float D = fmaf(p[s][e], state[e], q[s][e]);
          dx[e] = g.rest * D;
          out[e] = g.f * D;
          dg[e] = out[e] * g.rest * (prev[e] - xr[i].at(e));
        }
        put<EVEN>(static_cast<T*>(a.dgate) + row + from_ch, dg, nch);
        put<EVEN>(static_cast<T*>(a.dx) + row + from_ch, dx, nch);
        if (stops && a.dh0) put<EVEN>(a.dh0 + b * d + from_ch, out, nch);
      }
    }
  }
}

// One token of every history: the new states, and h in its type.
struct StepArgs {
  long n;
  const void* gate;
  const void* x;
  const float* state;
  float* state_out;
  void* h;                 // or NULL
  int h_bf16;
};
template <typename T, int VE>
__global__ __launch_bounds__(256) void k_gated_step(StepArgs a) {
  const long i = (static_cast<long>(blockIdx.x) * 256 + threadIdx.x) * VE;
  if (i >= a.n) return;
  const int n = static_cast<int>(min(static_cast<long>(VE), a.n - i));
  Raw<T, VE> g, x;
  Raw<float, VE> h;
  g.load(static_cast<const T*>(a.gate) + i, n);
  x.load(static_cast<const T*>(a.x) + i, n);
  h.load(a.state + i, n);
  float o[VE];
#pragma unroll
  for (int e = 0; e < VE; ++e) {
    const Gate f = gate_of(g.at(e));
    o[e] = fmaf(f.f, h.at(e), f.rest * x.at(e));
  }
  vec::store(a.state_out + i, o, n);
  if (!a.h) return;
  if (a.h_bf16)
    vec::store(static_cast<bf16_t*>(a.h) + i, o, n);
  else
    vec::store(static_cast<float*>(a.h) + i, o, n);
}

namespace {

// tokens of a slice: what two workgroups of a CU have registers for
template <bool BACK>
constexpr int slice_len() {
  return BACK ? 8 : 16;
}
struct ScanShape {
  int lanes_log2, len, chunks, groups;
};
ScanShape scan_shape(int T, int d, int S) {
  ScanShape s{};
  s.lanes_log2 = 2;
  while (s.lanes_log2 < 6 && (2 << s.lanes_log2) < d) ++s.lanes_log2;
  s.len = kWaves * (64 >> s.lanes_log2) * S;
  s.chunks = static_cast<int>((static_cast<long>(T) + s.len - 1) / s.len);
  s.groups = (d + 127) / 128;
  return s;
}
constexpr size_t kScanAlign = 256;
size_t up(size_t n) { return (n + kScanAlign - 1) / kScanAlign * kScanAlign; }
size_t shape_bytes(const ScanShape& s, int d) {
  if (s.chunks <= 1) return 0;
  return kScanAlign + up(s.chunks * sizeof(int2)) + (static_cast<size_t>(s.chunks) + s.chunks / kGroup) * d * sizeof(uint64_t);
}

template <bool BACK, typename T, typename TH>
hipError_t run_scan(ScanArgs a, void* ws, hipStream_t st) {
  constexpr int S = slice_len<BACK>();
  const ScanShape s = scan_shape(a.T, a.d, S);
  a.chunks = s.chunks;
  a.groups = s.groups;
  a.lanes_log2 = s.lanes_log2;
  if (s.chunks == 0) {                       // no tokens: no history has any
    hipLaunchKernelGGL((k_scan_plan<BACK>), dim3(static_cast<unsigned>(std::min(a.B / 64 + 1, 1024))), dim3(256), 0, st, a, s.len);
    return hipGetLastError();
  }
  if (s.chunks > 1) {
    char* w = static_cast<char*>(ws);
    a.ticket = reinterpret_cast<uint32_t*>(w);
    a.plan = reinterpret_cast<int2*>(w + kScanAlign);
    a.pairs = reinterpret_cast<uint64_t*>(w + kScanAlign + up(s.chunks * sizeof(int2)));
    a.states = a.pairs + static_cast<long>(s.chunks) * a.d;
    const long want = std::max<long>(static_cast<long>(s.chunks) * a.d / 1024, s.chunks / 4);
    hipLaunchKernelGGL((k_scan_plan<BACK>), dim3(static_cast<unsigned>(std::min(want + 1, 1024l))), dim3(256), 0, st, a, s.len);
  }
  const unsigned grid = static_cast<unsigned>(s.chunks) * s.groups;
  const bool even = a.d % 2 == 0;
  if (s.lanes_log2 == 6 && even)
    hipLaunchKernelGGL((k_scan<BACK, T, TH, S, true, true>), dim3(grid), dim3(kThreads), 0, st, a);
  else if (s.lanes_log2 == 6)
    hipLaunchKernelGGL((k_scan<BACK, T, TH, S, true, false>), dim3(grid), dim3(kThreads), 0, st, a);
  else if (even)
    hipLaunchKernelGGL((k_scan<BACK, T, TH, S, false, true>), dim3(grid), dim3(kThreads), 0, st, a);
  else
    hipLaunchKernelGGL((k_scan<BACK, T, TH, S, false, false>), dim3(grid), dim3(kThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace

size_t gated_scan_bytes(int T, int d) {
  return std::max(shape_bytes(scan_shape(T, d, slice_len<false>()), d), shape_bytes(scan_shape(T, d, slice_len<true>()), d));
}
long gated_scan_blocks(int T, int d) {
  const ScanShape s = scan_shape(T, d, std::min(slice_len<false>(), slice_len<true>()));
  return static_cast<long>(s.chunks) * s.groups;
}

hipError_t launch_gated_scan(const void* gate, const void* x, int x_dtype, int T, int d, const int32_t* offsets, int B,
                             const float* h0, void* h, int h_dtype, float* last, void* ws, hipStream_t st) {
  ScanArgs a{};
  a.T = T;
  a.d = d;
  a.B = B;
  a.gate = gate;
  a.x = x;
  a.offsets = offsets;
  a.h0 = h0;
  a.h = h;
  a.h_bf16 = h_dtype == MOL_BF16;
  a.last = last;
  return x_dtype == MOL_BF16 ? run_scan<false, bf16_t, bf16_t>(a, ws, st) : run_scan<false, float, float>(a, ws, st);
}

hipError_t launch_gated_scan_grad(const void* gate, const void* x, int x_dtype, const void* h, const void* dh, int h_dtype,
                                  int T, int d, const int32_t* offsets, int B, const float* h0, const float* dlast,
                                  void* dgate, void* dx, float* dh0, void* ws, hipStream_t st) {
  ScanArgs a{};
  a.T = T;
  a.d = d;
  a.B = B;
  a.gate = gate;
  a.x = x;
  a.offsets = offsets;
  a.h0 = h0;
  a.h = const_cast<void*>(h);
  a.dh = dh;
  a.dlast = dlast;
  a.dgate = dgate;
  a.dx = dx;
  a.dh0 = dh0;
  if (x_dtype == MOL_BF16)
    return h_dtype == MOL_BF16 ? run_scan<true, bf16_t, bf16_t>(a, ws, st) : run_scan<true, bf16_t, float>(a, ws, st);
  return h_dtype == MOL_BF16 ? run_scan<true, float, bf16_t>(a, ws, st) : run_scan<true, float, float>(a, ws, st);
}

hipError_t launch_gated_step(const void* gate, const void* x, int x_dtype, int64_t n, const float* state, float* state_out,
                             void* h, int h_dtype, hipStream_t st) {
  StepArgs a{n, gate, x, state, state_out, h, h_dtype == MOL_BF16};
  constexpr int VE = 4;
  const unsigned grid = static_cast<unsigned>((n + 256 * VE - 1) / (256 * VE));
  if (x_dtype == MOL_BF16)
    hipLaunchKernelGGL((k_gated_step<bf16_t, VE>), dim3(grid), dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((k_gated_step<float, VE>), dim3(grid), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace mol
