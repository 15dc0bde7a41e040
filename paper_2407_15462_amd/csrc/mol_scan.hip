// A gated linear recurrence over histories, and its gradient.  For each channel of
// each history (tokens offsets[b] .. offsets[b + 1] - 1 of packed rows):
//   f_t = 1 / (1 + e^{-gate_t}),  h_t = f_t h_{t-1} + (1 - f_t) x_t,  h_{-1} = h0
// and back, with D_t = dL / dh_t in all, E_t = f_t D_t, E behind the last token = dlast:
//   D_t = dh_t + E_{t+1},  dx_t = (1 - f_t) D_t,  dgate_t = f_t (1 - f_t) (h_{t-1} - x_t) D_t,  dh0 = E_0
//
// Both are linear maps of the state that comes in, state -> A state + H, which join:
// the scan cuts the packed tokens, wherever histories end, into chunks of equal length,
// each read once.  A workgroup holds a chunk of 128 channels (two a lane): each
// wave, or part of a wave where there are few channels, takes a slice of S tokens and
// runs through it from state 0, for its (A, H); slices are joined in LDS; the
// workgroup publishes the chunk's (A, H), gets the state that comes in from the
// chunks before, and runs through the tokens once more, which it kept in registers, for
// what it writes.  A history's first token starts from h0, with a mark for A, so that
// nothing crosses from one history to the next.  (A = 0 is no such mark: it is a product of gates
// below float32's range, through which a NaN or an infinity stays what it is, since f is never 0.)
//
// The state that comes in is formed in an order that sizes and offsets alone fix: the
// state at the end of the kSuper chunks before (a chain of waits along a long history),
// then the (A, H) of the groups of kGroup chunks since, then those of the
// group's chunks; each only from the chunk in which the history starts, so that short
// histories wait for little.
//
// Waiting is sure to end: workgroups take their chunks by a ticket, in order, so that
// a chunk's predecessors belong to workgroups that run or have ended, and what each
// publishes needs nothing but what those before it publish.  A published pair is one
// 64-bit word, whose top bit (the sign of A, which is not negative) says that it is there.
//
// Measured, bf16: 1024 histories of 262,144 tokens of 512 channels 191 to 207 us (3.9 to 4.2 TB/s), back 305 to 309
// (5.2 TB/s, where a copy of as much reaches 5.0); one history of 131,072 x 1024 200 to 208, back (x 512) 173 to 180; 64
// histories of 20,000 x 512 32.  Inputs of 256 MB and more are read and written past the caches (through them 217, 318,
// 225 and 182, where these took the larger figures).  What bounds it: back,
// memory; forward, the waits (27 to 45 us in a build without them) and, at more than half of the vector rate, two
// gates an element (27 instructions).  Tried and slower forward: every token's A and H kept in place of the second
// run (half as many tokens a slice: 225 to 231 where this took 219), workgroups that stay and load their next chunk
// ahead (226 to 311: a wait is then for workgroups at another place of their turn), a ninth wave for the waits,
// tickets of their own for every 128 channels (238: neighbours in memory drift apart in time).
#include <algorithm>
#include <cfloat>
#include <type_traits>

#include "mol_kernels.h"
#include "mol_vec.h"

namespace mol {

namespace {

using vec::Raw;

constexpr int kWaves = 8, kThreads = 64 * kWaves;
constexpr int kGroup = 8, kSuper = 64;    // chunks
static_assert(kGroup - 1 < kWaves && kSuper / kGroup - 1 < kWaves, "a wave waits for one pair of each kind");

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
  uint32_t* ticket;        // workspace (of more than one chunk)
  int2* plan;              // of each chunk: the first history that it holds tokens of, and the chunk
                           // that the state coming in starts from (the chunk itself: none comes in)
  uint64_t* pairs;         // [chunks][d] (A, H)
  uint64_t* group_pairs;   // [chunks / kGroup][d]
  uint64_t* states;        // [chunks / kSuper][d] (0, state)
  long words;              // of the three together
  bool once;               // rows are read past the caches
  bool empties;            // the scan's own launch sees to histories without tokens
};

__device__ __forceinline__ int offset_at(const ScanArgs& a, int i) {
  if (!a.offsets) return i ? a.T : 0;
  return min(max(a.offsets[i], 0), a.T);
}

// f = sigmoid(g) and rest = sigmoid(-g), which 1 - f would not give near f = 1; far out
// e^{-g} stays finite (f is 2^-126 there), and NaN stays NaN
template <typename T>
__device__ __forceinline__ void gates_of(float g, float& f, float& rest) {
  float e;
  if (sizeof(T) == 2) {
    // (the product's rounding makes e off by a relative |g| 2^-24, where the gate itself is known to 2^-9 |g|)
    e = __builtin_amdgcn_exp2f(__builtin_elementwise_minimum(g * -kLog2E, 126.f));
  } else {
    g = __builtin_elementwise_minimum(__builtin_elementwise_maximum(g, -87.f), 120.f);
    const float t = g * -kLog2E, r = fmaf(g, -kLog2ELo, fmaf(g, -kLog2E, -t));
    e = __builtin_amdgcn_exp2f(t);
    e = fmaf(e, r * kLn2, e);
  }
  f = __builtin_amdgcn_rcpf(1.f + e);
  rest = e * f;
}

// The A of tokens among which a history begins is NaN, as it is behind a NaN gate (whose H is NaN as well, so that what
// comes in changes nothing); others' are from 0 to 1.  So the A of tokens behind others is the product of both.
constexpr float kBegins = __builtin_nanf("");
// What is left of v behind tokens of A = a: a v; nothing where a history begins there, whatever v is (another
// history's state); and a v that is not finite as it is, since no product of gates is 0.
__device__ __forceinline__ float through(float a, float v) { return a != a ? 0.f : fabsf(v) <= FLT_MAX ? a * v : v; }

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
template <bool EVEN, bool ONCE, typename T>
__device__ __forceinline__ void put(T* p, const float (&v)[2], int n) {
  if (EVEN)
    vec::store<ONCE>(p, v);
  else
    vec::store<ONCE>(p, v, n);
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
  for (long i = tid; i < a.words; i += all) a.pairs[i] = 0;
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
  // (eight histories a wave and turn: enough waves for rows of many that are empty, few turns for many that are not)
  for (long b0 = tid / 64 * 8; b0 < a.B; b0 += all / 8) {
    const int b = static_cast<int>(b0) + lane;
    uint64_t m = __ballot(lane < 8 && b < a.B && offset_at(a, b) >= offset_at(a, b + 1));
    for (; m; m &= m - 1) {
      const long at = (b0 + __builtin_ctzll(m)) * a.d;
#pragma unroll 4
      for (int c = lane; c < a.d; c += 64) out[at + c] = in ? in[at + c] : 0.f;
    }
  }
}

// UNI: a wave's lanes share their slice (more than 64 channels), so that what depends on
// the token alone is a scalar.  EVEN: an even number of channels, so that lanes
// without channels of their own can read others'.  ONCE: rows are read and written past the caches.
template <bool BACK, typename T, typename TH, int S, bool UNI, bool EVEN, bool ONCE>
__global__ __launch_bounds__(kThreads, 4) void k_scan(ScanArgs a) {
  constexpr int kMost = kWaves * S * (UNI ? 1 : 16);            // tokens of a chunk (4 lanes a row at least)
  constexpr int kBlock = BACK ? 8 : S;                         // tokens whose x and h are in flight together on the way out
  __shared__ uint32_t begins[kMost / S], ends[kMost / S];      // of a slice: the tokens at which a history begins and ends
  __shared__ int begin_b[kMost], end_b[kMost];                 // (in the scan's direction), and whose
  __shared__ float sum_a[kWaves][128], sum_h[kWaves][128];       // [wave][channel]: of the unit's slices
  __shared__ float in_a[kWaves][128], in_h[kWaves][128], come[128];
  __shared__ int my_ticket;

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid / 64), d = a.d;
  const int lanes = UNI ? 64 : 1 << a.lanes_log2, per_wave = UNI ? 1 : 64 >> a.lanes_log2;
  const int len = kWaves * per_wave * S;
  int ticket = blockIdx.x;
  if (a.chunks > 1) {
    if (tid == 0) my_ticket = __hip_atomic_fetch_add(a.ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    ticket = __builtin_amdgcn_readfirstlane(my_ticket);
  }
  const int chunk = __builtin_amdgcn_readfirstlane(ticket / a.groups), cg = ticket - chunk * a.groups;
  // tokens in the scan's direction: i = 0 .. len - 1 stands for token first + i, or first - i on the way back
  const int first = BACK ? a.T - 1 - chunk * len : chunk * len;
  const int lo = BACK ? max(0, first + 1 - len) : first;
  const int hi = BACK ? first + 1 : min(a.T, first + len);

  const int sub = UNI ? 0 : lane >> a.lanes_log2;              // which slice of the wave's
  const int slice = wave * per_wave + sub;
  const int row_lane = UNI ? lane : lane & (lanes - 1);
  const int ch = cg * 128 + 2 * row_lane, nch = d - ch;        // this lane's channels: 2 or 1 (or none)
  const uint32_t from_ch = min(ch, EVEN ? d - 2 : d - 1);      // where it reads
  Raw<T, 2> gate[S];
  Raw<T, 2> xr[BACK ? 1 : S];
  Raw<TH, 2> dr[BACK ? S : 1];
  auto row_at = [&](auto* base, int row) {                     // this lane's channels of a row
    typedef std::remove_reference_t<decltype(*base)> E;
    typedef std::conditional_t<std::is_const_v<E>, const char, char> Byte;
    return reinterpret_cast<E*>(reinterpret_cast<Byte*>(base + static_cast<int64_t>(row) * d) +
                                from_ch * static_cast<uint32_t>(sizeof(E)));
  };
  auto load = [&](auto& r, const auto* base, int t) {
    if (EVEN)
      r.template load<ONCE>(row_at(base, t));
    else
      r.template load<ONCE>(row_at(base, t), d - static_cast<int>(from_ch));
  };
  const int t_first = BACK ? first - slice * S : first + slice * S;
  auto token = [&](int s) { return BACK ? t_first - s : t_first + s; };
  // Rows that are no history's are read as well (and past the tensor's ends others
  // in their place): what comes of them is not written, and the next history begins anew.
#pragma unroll
  for (int s = 0; s < S; ++s) {
    const int t = min(max(token(s), 0), a.T - 1);
    load(gate[s], static_cast<const T*>(a.gate), t);
    if constexpr (BACK) {
      dr[s].zero();
      if (a.dh) load(dr[s], static_cast<const TH*>(a.dh), t);
    } else {
      load(xr[s], static_cast<const T*>(a.x), t);
    }
  }
  const int live_lo = __builtin_amdgcn_readfirstlane(max(lo, offset_at(a, 0)));
  const int live_hi = __builtin_amdgcn_readfirstlane(min(hi, offset_at(a, a.B)));
  auto live = [&](int s) { return token(s) >= live_lo && token(s) < live_hi; };
  for (int i = tid; i < kWaves * per_wave; i += kThreads) begins[i] = ends[i] = 0;
  __syncthreads();
  int2 plan = a.chunks > 1 ? a.plan[chunk] : make_int2(0, 0);
  plan.x = __builtin_amdgcn_readfirstlane(plan.x);
  plan.y = __builtin_amdgcn_readfirstlane(plan.y);
  for (int b0 = plan.x + wave * 64; b0 < a.B; b0 += kThreads) {
    const int b = b0 + lane;
    const int s = b < a.B ? offset_at(a, b) : a.T, e = b < a.B ? offset_at(a, b + 1) : a.T;
    if (a.chunks > 1 && __all(s >= hi)) break;
    if (s < e) {
      const int tb = BACK ? e - 1 : s, te = BACK ? s : e - 1;
      if (tb >= lo && tb < hi) {
        const int i = BACK ? first - tb : tb - first;
        begin_b[i] = b;
        atomicOr(&begins[i / S], 1u << i % S);
      }
      if (te >= lo && te < hi) {
        const int i = BACK ? first - te : te - first;
        end_b[i] = b;
        atomicOr(&ends[i / S], 1u << i % S);
      }
    }
    // (histories without tokens, unless a launch of the plan's sees to them)
    float* out = BACK ? a.dh0 : a.last;
    const float* in = BACK ? a.dlast : a.h0;
    if (a.empties && out)
      for (uint64_t m = __ballot(b < a.B && s >= e); m; m &= m - 1) {
        const long at = static_cast<long>(b0 + __builtin_ctzll(m)) * d;
        for (int c = cg * 128 + lane; c < min(d, cg * 128 + 128); c += 64) out[at + c] = in ? in[at + c] : 0.f;
      }
  }
  const int group0 = chunk / kGroup * kGroup, super0 = chunk / kSuper * kSuper;
  const int from = min(plan.y, chunk);
  const int from1 = max(from, group0);                         // chunks whose pairs are needed: from1 .. chunk - 1,
  const int from2 = max(from, super0) / kGroup;                // groups: from2 .. group0 / kGroup - 1 (where from < group0),
  const bool old = from < super0;                              // and the state in front of the super
  __syncthreads();
  uint32_t begin = begins[slice], end = ends[slice];
  if (UNI) begin = __builtin_amdgcn_readfirstlane(begin), end = __builtin_amdgcn_readfirstlane(end);
  // the state (back: E) that a history begins with at token s of the slice
  auto start = [&](int s, float (&v)[2]) {
    const float* in = BACK ? a.dlast : a.h0;
    const long at = static_cast<long>(begin_b[slice * S + s]) * d + ch;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      v[e] = in && e < nch ? in[at + e] : 0.f;
      asm volatile("" : "+v"(v[e]));                         // (waited for here, not by tokens without a beginning)
    }
  };
  // the slice from state 0
  float A[2] = {1.f, 1.f}, H[2] = {0.f, 0.f};
  auto run = [&](auto marked) {
#pragma unroll
    for (int s = 0; s < S; ++s) {
      if (marked && (begin >> s & 1)) {
        A[0] = A[1] = kBegins;
        start(s, H);
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float f, rest;
        gates_of<T>(gate[s].at(e), f, rest);
        A[e] *= f;
        if constexpr (BACK)
          H[e] = f * (dr[s].at(e) + H[e]);
        else
          H[e] = fmaf(f, H[e], rest * xr[s].at(e));
      }
    }
  };
  // (slices in which no history begins, nearly all, have a form without the tests)
  if (__any(begin))
    run(std::true_type{});
  else
    run(std::false_type{});
  // What follows forms the gates again, from the rows as they lie in registers: half as many as
  // every token's A and H would take, so that a slice can be twice as long.
#pragma unroll
  for (int s = 0; s < S; ++s)
#pragma unroll
    for (int i = 0; i < Raw<T, 2>::kWords; ++i) asm volatile("" : "+v"(gate[s].w[i]));

  // slices joined: (A, H) of the wave's slices before this one, and of the wave
  float before_a[2] = {1.f, 1.f}, before_h[2] = {0.f, 0.f};
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    float ca = A[e], chh = H[e];                             // inclusive over slices of the wave
    if (!UNI) {
      for (int o = lanes; o < 64; o <<= 1) {
        const float ua = __shfl_up(ca, o), uh = __shfl_up(chh, o);
        if (lane >= o) {
          chh += through(ca, uh);
          ca *= ua;
        }
      }
      const float ua = __shfl_up(ca, lanes), uh = __shfl_up(chh, lanes);
      if (sub) before_a[e] = ua, before_h[e] = uh;
    }
    if (sub == per_wave - 1) {
      sum_a[wave][2 * row_lane + e] = ca;
      sum_h[wave][2 * row_lane + e] = chh;
    }
  }
  __syncthreads();                                           // sums
  float pre_a[2], pre_h[2], all_a[2], all_h[2];              // of the waves before, and with this one (the last: of all)
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    pre_a[e] = 1.f, pre_h[e] = 0.f;
    for (int v = 0; v < wave; ++v) {
      const float wa = sum_a[v][2 * row_lane + e], wh = sum_h[v][2 * row_lane + e];
      pre_h[e] = wh + through(wa, pre_h[e]);
      pre_a[e] *= wa;
    }
    const float wa = sum_a[wave][2 * row_lane + e], wh = sum_h[wave][2 * row_lane + e];
    all_h[e] = wh + through(wa, pre_h[e]);
    all_a[e] = wa * pre_a[e];
  }
  const bool speaks = a.chunks > 1 && wave == kWaves - 1 && sub == 0;
  if (speaks)
#pragma unroll
    for (int e = 0; e < 2; ++e)
      if (e < nch) publish(a.pairs + static_cast<long>(chunk) * d + ch + e, all_a[e], all_h[e]);
  // the state that comes in: each wave gets a pair of the group's chunks, then one of the super's groups
  float state[2] = {0.f, 0.f};
  // (A, H) of the pairs i0 .. i1 - 1, pair j0 + v by wave v, joined
  auto gather = [&](const uint64_t* base, int i0, int i1, int j0, float (&fa)[2], float (&fh)[2]) {
    if (j0 + wave >= i0 && j0 + wave < i1 && sub == 0) {
      const uint64_t* at = base + static_cast<long>(j0 + wave) * d + ch;
      uint64_t got[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) got[e] = e < nch ? look(at + e) : ~0ull;
      while (__any(!there(got[0]) || !there(got[1]))) {
        // (the channels' words were written together: until the first is there, only it is looked for)
        for (;;) {
          bool yes = true;
          if (row_lane == 0) yes = there(got[0] = look(at));
          if (__all(yes)) break;
          __builtin_amdgcn_s_sleep(4);
        }
#pragma unroll
        for (int e = 0; e < 2; ++e)
          if (!there(got[e])) got[e] = look(at + e);
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        in_a[wave][2 * row_lane + e] = a_of(got[e]);
        in_h[wave][2 * row_lane + e] = h_of(got[e]);
      }
    }
    __syncthreads();
    for (int i = i0; i < i1; ++i)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float wa = in_a[i - j0][2 * row_lane + e];
        fh[e] = in_h[i - j0][2 * row_lane + e] + through(wa, fh[e]);
        fa[e] *= wa;
      }
    __syncthreads();
  };
  if (a.chunks > 1) {
    float ga[2] = {1.f, 1.f}, gh[2] = {0.f, 0.f};
    if (from1 < chunk) gather(a.pairs, from1, chunk, group0, ga, gh);
    if (speaks && chunk % kGroup == kGroup - 1)
#pragma unroll
      for (int e = 0; e < 2; ++e)
        if (e < nch)
          publish(a.group_pairs + static_cast<long>(chunk / kGroup) * d + ch + e, all_a[e] * ga[e],
                  all_h[e] + through(all_a[e], gh[e]));
    if (from < group0) {
      float sa[2] = {1.f, 1.f}, sh[2] = {0.f, 0.f};
      if (old) {
        if (wave == kWaves - 1 && sub == 0) {
          const uint64_t* at = a.states + static_cast<long>(chunk / kSuper - 1) * d + ch;
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            uint64_t v = e < nch ? look(at + e) : ~0ull;
            while (!there(v)) {
              __builtin_amdgcn_s_sleep(1);
              v = look(at + e);
            }
            come[2 * row_lane + e] = h_of(v);
          }
        }
      }
      if (from2 < group0 / kGroup) gather(a.group_pairs, from2, group0 / kGroup, super0 / kGroup, sa, sh);
      if (old) {
        __syncthreads();
        state[0] = come[2 * row_lane], state[1] = come[2 * row_lane + 1];
        __syncthreads();
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) state[e] = sh[e] + through(sa[e], state[e]);
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) state[e] = gh[e] + through(ga[e], state[e]);
    if (speaks && chunk % kSuper == kSuper - 1)
#pragma unroll
      for (int e = 0; e < 2; ++e)
        if (e < nch)
          publish(a.states + static_cast<long>(chunk / kSuper) * d + ch + e, 0.f, all_h[e] + through(all_a[e], state[e]));
  }
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    state[e] = pre_h[e] + through(pre_a[e], state[e]);
    state[e] = before_h[e] + through(before_a[e], state[e]);
  }

  // out
  const int t_last = token(S - 1);
  const bool plain = !begin && !end && min(t_first, t_last) >= live_lo && max(t_first, t_last) < live_hi;
  auto out = [&](auto marked) {
#pragma unroll
    for (int s0 = 0; s0 < S; s0 += kBlock) {
      Raw<T, 2> xo[kBlock];
      Raw<TH, 2> hr[kBlock];
      if constexpr (BACK)
#pragma unroll
        for (int i = 0; i < kBlock; ++i) {
          load(xo[i], static_cast<const T*>(a.x), max(token(s0 + i), 0));
          load(hr[i], static_cast<const TH*>(a.h), max(token(s0 + i) - 1, 0));    // (of a history's first token not used)
        }
#pragma unroll
      for (int i = 0; i < kBlock; ++i) {
        const int s = s0 + i;
        if (marked && (begin >> s & 1)) start(s, state);
        const bool stops = marked && (end >> s & 1);
        float f[2], rest[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) gates_of<T>(gate[s].at(e), f[e], rest[e]);
        if constexpr (!BACK) {
#pragma unroll
          for (int e = 0; e < 2; ++e) state[e] = fmaf(f[e], state[e], rest[e] * xr[s].at(e));
          if ((marked && !live(s)) || nch <= 0) continue;
          if (a.h_bf16)
            put<EVEN, ONCE>(row_at(static_cast<bf16_t*>(a.h), token(s)), state, nch);
          else
            put<EVEN, ONCE>(row_at(static_cast<float*>(a.h), token(s)), state, nch);
          if (stops && a.last) put<EVEN, false>(row_at(a.last, end_b[slice * S + s]), state, nch);
        } else {
          float prev[2] = {hr[i].at(0), hr[i].at(1)}, dg[2], dx[2];
          const int b = stops ? end_b[slice * S + s] : 0;
          if (stops)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              prev[e] = a.h0 && e < nch ? a.h0[static_cast<long>(b) * d + ch + e] : 0.f;
              asm volatile("" : "+v"(prev[e]));
            }
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float D = dr[s].at(e) + state[e];
            dx[e] = rest[e] * D;
            state[e] = f[e] * D;
            dg[e] = state[e] * rest[e] * (prev[e] - xo[i].at(e));
          }
          if ((marked && token(s) < 0) || nch <= 0) continue;
          if (marked && !live(s)) dg[0] = dg[1] = dx[0] = dx[1] = 0.f;   // rows of no history: no loss depends on them
          put<EVEN, ONCE>(row_at(static_cast<T*>(a.dgate), token(s)), dg, nch);
          put<EVEN, ONCE>(row_at(static_cast<T*>(a.dx), token(s)), dx, nch);
          if (stops && a.dh0) put<EVEN, false>(row_at(a.dh0, b), state, nch);
        }
      }
    }
  };
  if (__all(plain))
    out(std::false_type{});
  else
    out(std::true_type{});
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
    float f, rest;
    gates_of<T>(g.at(e), f, rest);
    o[e] = fmaf(f, h.at(e), rest * x.at(e));
  }
  vec::store(a.state_out + i, o, n);
  if (!a.h) return;
  if (a.h_bf16)
    vec::store(static_cast<bf16_t*>(a.h) + i, o, n);
  else
    vec::store(static_cast<float*>(a.h) + i, o, n);
}

namespace {

// Tokens of a slice: 16, or 32 (as many as registers hold, forward in bfloat16) where that leaves
// every CU a workgroup.  The longer, the fewer waits, each of which costs a workgroup the latencies of a store
// and a load that pass the caches (262,144 x 512 through the caches: 219 us, with 24 tokens 230; 20,000 x 512 32, with 16 33); the
// shorter, the more workgroups (6400 x 256: 15 us a call, with 32 tokens 20).
constexpr int kSlice = 16, kLongSlice = 32;
constexpr long kManyUnits = 256;

struct ScanShape {
  int lanes_log2, len, chunks, groups;
};
int row_lanes_log2(int d) {
  int n = 2;
  while (n < 6 && (2 << n) < d) ++n;
  return n;
}
ScanShape scan_shape(int T, int d, int S) {
  ScanShape s{};
  s.lanes_log2 = row_lanes_log2(d);
  s.len = kWaves * (64 >> s.lanes_log2) * S;
  s.chunks = static_cast<int>((static_cast<long>(T) + s.len - 1) / s.len);
  s.groups = (d + 127) / 128;
  return s;
}
constexpr size_t kScanAlign = 256;
size_t up(size_t n) { return (n + kScanAlign - 1) / kScanAlign * kScanAlign; }
long pair_words(const ScanShape& s, int d) {
  return (static_cast<long>(s.chunks) + s.chunks / kGroup + s.chunks / kSuper) * d;
}
size_t shape_bytes(const ScanShape& s, int d) {
  return s.chunks <= 1 ? 0 : kScanAlign + up(s.chunks * sizeof(int2)) + pair_words(s, d) * sizeof(uint64_t);
}
template <bool BACK, typename T, typename TH, bool UNI, int S>
hipError_t run_scan_slices(ScanArgs a, void* ws, hipStream_t st) {
  const ScanShape s = scan_shape(a.T, a.d, S);
  a.chunks = s.chunks;
  a.groups = s.groups;
  a.lanes_log2 = s.lanes_log2;
  // The plan's launch: of one chunk, and of no tokens, there is none to make, but histories without tokens.  A few
  // of these the scan's workgroups see to (4096 histories with 100 tokens x 512: 33 us a call, with theirs 194).
  ScanArgs plan = a;
  plan.words = 0;
  bool wanted = s.chunks != 1 || a.B > 32;
  a.empties = !wanted;
  if (s.chunks > 1) {
    char* w = static_cast<char*>(ws);
    a.ticket = reinterpret_cast<uint32_t*>(w);
    a.plan = reinterpret_cast<int2*>(w + kScanAlign);
    a.pairs = reinterpret_cast<uint64_t*>(w + kScanAlign + up(s.chunks * sizeof(int2)));
    a.group_pairs = a.pairs + static_cast<long>(s.chunks) * a.d;
    a.states = a.group_pairs + static_cast<long>(s.chunks / kGroup) * a.d;
    a.words = pair_words(s, a.d);
    plan = a;
  } else {
    plan.chunks = 0;
    wanted = wanted && (BACK ? a.dh0 : a.last);
  }
  if (wanted) {
    const long want = std::max({plan.words / 1024, plan.chunks / 4l, a.B / 32l});
    hipLaunchKernelGGL((k_scan_plan<BACK>), dim3(static_cast<unsigned>(std::min(want + 1, 1024l))), dim3(256), 0, st, plan, s.len);
  }
  if (s.chunks == 0) return hipGetLastError();
  const unsigned grid = static_cast<unsigned>(s.chunks) * s.groups;
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(grid), dim3(kThreads), 0, st, a); };
  if (a.d % 2) {
    go(k_scan<BACK, T, TH, S, UNI, false, false>);
  } else if constexpr (UNI) {
    a.once ? go(k_scan<BACK, T, TH, S, UNI, true, true>) : go(k_scan<BACK, T, TH, S, UNI, true, false>);
  } else {
    go(k_scan<BACK, T, TH, S, UNI, true, false>);
  }
  return hipGetLastError();
}
template <bool BACK, typename T, typename TH>
hipError_t run_scan(const ScanArgs& a, void* ws, hipStream_t st) {
  if (row_lanes_log2(a.d) < 6) return run_scan_slices<BACK, T, TH, false, kSlice>(a, ws, st);
  if constexpr (!BACK && sizeof(T) == 2) {
    const ScanShape s = scan_shape(a.T, a.d, kLongSlice);
    if (static_cast<long>(s.chunks) * s.groups >= kManyUnits)
      return run_scan_slices<BACK, T, TH, true, kLongSlice>(a, ws, st);
  }
  return run_scan_slices<BACK, T, TH, true, kSlice>(a, ws, st);
}

}  // namespace

size_t gated_scan_bytes(int T, int d) {
  return shape_bytes(scan_shape(T, d, kSlice), d);                // (of the shortest slices)
}
long gated_scan_blocks(int T, int d) {
  const ScanShape s = scan_shape(T, d, kSlice);
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
  a.once = vec::streams(static_cast<size_t>(T) * d * (x_dtype == MOL_BF16 ? 4 : 8));
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
  a.once = vec::streams(static_cast<size_t>(T) * d * ((x_dtype == MOL_BF16 ? 4 : 8) + (h_dtype == MOL_BF16 ? 2 : 4) * (dh ? 2 : 1)));
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
