// Embedding rows by id and the gradient of their tables.
//
// Lookup: out[c][t][:] = scale table[c][ids[t]][:], a zero row for an id
// outside [0, V).  Bound by memory: a thread moves 16 bytes of output, four
// of them in flight, and consecutive threads share a row (131,072 rows of 64
// from each of 8 float32 tables to bf16: 61 us, 6.6 TB/s, where a copy runs at 4.6).
//
// Gradient: table_grad[c][v][:] = scale sum_{t: ids[t] = v} grad[c][t][:].
//  1. The tokens are sorted by id, stably: up to kSortRank of them by counting,
//     else in least-significant-digit radix passes over (id, t) pairs, of up to
//     11 bits, a histogram and a scatter launch each.  Empty slots sort behind every row (key V).
//  2. Each workgroup takes a span of sorted tokens and a column slice of a
//     table.  Teams of LPR lanes (16 bytes a lane) walk K tokens each, with
//     four rows in flight, and keep the running sum of the current id in
//     registers (float32).  A run that lies in one team's tokens is written
//     at once; pieces of a run that crosses teams are joined in LDS, and
//     pieces that cross spans go to the workspace.
//     In the same launch, other workgroups write the zero rows: they look the
//     ids of their rows up in the sorted list (a 64-way search, then a bitmap
//     in LDS), so that every row is written once and nothing is cleared first.
//  3. The few runs that cross spans are joined from the workspace.
// Every sum is formed in an order that ids and sizes fix: no atomics on
// floats, the same bits every time.  Bound by memory where rows have few tokens: grad is
// read once and table_grad written once.
// Measured: 262,144 tokens of 4 x 128 bf16 onto 24,186 float32 rows take 29 us
// for the sort, 68 for the sums (4.7 TB/s) and 8 for the join, 112 a call; 65,536 of
// 8 x 32 onto 674,044 rows 30, 139 (5.2 TB/s, nine tenths of it zero rows) and 5.
// Many tokens a row cost more than as many rows, in two chains of latencies: the workgroup
// that looks for a block of zero rows reads every token of them, 256 a step, and the join
// walks the spans of a run one by one.  262,144 tokens onto 1000 rows of 8: 338 us (34 with
// accumulate, which has no zero rows), of 128: 73 (38); a million of 64 bf16 on a single row: 1674 (539),
// spread over 1000 rows 387 (76), over a million 201 (194).
// The sort's passes are chains of latencies (5 us a histogram, 9 a scatter).
// Sorted chunks of 4096 merged by rank took 53 us against 31 at 65,536 tokens, and
// rows cleared beside the sort slowed it by what the sums gained.  Spans that end
// where runs do, with nothing to join, took 12 us against 6 + 4 at 1024 tokens of 512.
#include <algorithm>
#include <type_traits>

#include "mol_kernels.h"

namespace mol {

namespace {

// Tokens at most that are sorted by counting (1024: 3.7 us, 4096: 6.8, 8192: 12.4,
// 16,384: 38; the radix passes take 21 from 8193 on, one workgroup's took 6.8 at 1024).
constexpr int kSortRank = 8192;
constexpr int kSortThreads = 256;     // of a block of the radix passes
constexpr int kSortWaves = kSortThreads / 64;
constexpr int kSortU = 8;             // loads in flight
constexpr int kMinBits = 8, kMaxBits = 11;   // digit of a radix pass
constexpr int kSortBlock = kSortThreads * kSortU;   // tokens a block takes at least
constexpr int kSortBlocks = 128;      // blocks at most

template <typename T>
struct Elem;
template <>
struct Elem<float> {
  static constexpr int kVec = 4;      // elements of 16 bytes
};
template <>
struct Elem<bf16_t> {
  static constexpr int kVec = 8;
};

// float32 -> bf16, nearest even; NaN stays NaN
__device__ __forceinline__ bf16_t to_bf16(float f) {
  return __builtin_bit_cast(bf16_t, static_cast<__bf16>(f));
}
__device__ __forceinline__ void put(float& o, float v) { o = v; }
__device__ __forceinline__ void put(bf16_t& o, float v) { o = to_bf16(v); }

template <typename T, int N>
struct alignas(sizeof(T) * N > 16 ? 16 : sizeof(T) * N) Pack {
  T v[N];
};

// lanes of the wave (of `live`) whose low BITS bits of `digit` equal this lane's
template <int BITS>
__device__ __forceinline__ uint64_t same_digit(uint32_t digit, uint64_t live) {
  uint64_t m = live;
#pragma unroll
  for (int b = 0; b < BITS; ++b) {
    const bool on = (digit >> b) & 1;
    const uint64_t x = __ballot(on);
    m &= on ? x : ~x;
  }
  return m;
}

__device__ __forceinline__ uint32_t key_of(int32_t id, int V) {
  return static_cast<uint32_t>(id) < static_cast<uint32_t>(V) ? static_cast<uint32_t>(id) : static_cast<uint32_t>(V);
}

// inclusive sum over the lanes of a wave
__device__ __forceinline__ uint32_t wave_scan(uint32_t v, int lane) {
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t u = __shfl_up(v, o);
    if (lane >= o) v += u;
  }
  return v;
}

}  // namespace

// ---------------------------------------------------------------------------
// Lookup.  VE elements a thread and step (1: any alignment), U steps in flight.
// A block starts at vector blockIdx.x * 256 * U of its table's T * nv.
template <typename TI, typename TO, int VE>
__global__ __launch_bounds__(256) void k_embed_lookup(const TI* __restrict__ table, int V, int d, int nv,
                                                      const int32_t* __restrict__ ids, int T, float scale,
                                                      TO* __restrict__ out) {
  constexpr int U = 4;
  const long base = static_cast<long>(blockIdx.x) * (256 * U), total = static_cast<long>(T) * nv;
  const int t0 = static_cast<int>(base / nv);
  const uint32_t r0 = static_cast<uint32_t>(base - static_cast<long>(t0) * nv);
  const TI* tab = table + static_cast<long>(blockIdx.y) * V * d;
  TO* dst = out + static_cast<long>(blockIdx.y) * T * d;
  int32_t id[U];
  uint32_t col[U];
  bool live[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint32_t local = r0 + u * 256 + threadIdx.x;
    const uint32_t dt = local / static_cast<uint32_t>(nv);
    col[u] = (local - dt * nv) * VE;
    live[u] = base + u * 256 + threadIdx.x < total;
    id[u] = live[u] ? ids[t0 + dt] : -1;
  }
  Pack<TI, VE> x[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const bool ok = static_cast<uint32_t>(id[u]) < static_cast<uint32_t>(V);
    if (ok) {
      x[u] = *reinterpret_cast<const Pack<TI, VE>*>(tab + static_cast<long>(id[u]) * d + col[u]);
    } else {
#pragma unroll
      for (int e = 0; e < VE; ++e) x[u].v[e] = 0;
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (!live[u]) continue;
    const bool ok = static_cast<uint32_t>(id[u]) < static_cast<uint32_t>(V);
    Pack<TO, VE> y;
#pragma unroll
    for (int e = 0; e < VE; ++e) put(y.v[e], ok ? scale * to_f32(x[u].v[e]) : 0.f);
    *reinterpret_cast<Pack<TO, VE>*>(dst + (base + u * 256 + threadIdx.x) * VE) = y;
  }
}

// ---------------------------------------------------------------------------
// Sorting few tokens: a token's place is the number of those before it in the
// order of (key, token), counted against all keys in LDS.  A workgroup has 16
// tokens, and lane (c = lane % 16, q = lane / 16) of wave w counts every 16th
// four keys, from 4 w + q on, for token c.
__global__ __launch_bounds__(256) void k_sort_rank(const int32_t* __restrict__ ids, int T, int V,
                                                   uint2* __restrict__ out) {
  extern __shared__ __attribute__((aligned(16))) uint32_t keys[];   // 64 ceil(T / 64), then [16][16] counts
  const int tid = threadIdx.x, c = tid & 15, part = tid >> 4;
  const int Tp = (T + 63) / 64 * 64, i0 = blockIdx.x * 16;
  for (int b = tid; b < Tp; b += 256 * kSortU) {
    int32_t id[kSortU];
#pragma unroll
    for (int u = 0; u < kSortU; ++u) id[u] = ids[min(b + 256 * u, T - 1)];
#pragma unroll
    for (int u = 0; u < kSortU; ++u) {
      const int i = b + 256 * u;
      if (i < Tp) keys[i] = i < T ? key_of(id[u], V) : 0xFFFFFFFFu;
    }
  }
  __syncthreads();
  const uint32_t mine = keys[min(i0 + c, T - 1)];
  // keys of tokens before the workgroup's count where they are mine or less, of those
  // behind it where they are less; its own 16 (four fours) by place
  const uint4* four = reinterpret_cast<const uint4*>(keys);
  const int own = i0 / 4, all = Tp / 4;
  uint32_t n = 0;
  int m = part;
#pragma unroll 4
  for (; m < own; m += 16) {
    const uint4 k = four[m];
    n += (k.x <= mine) + (k.y <= mine) + (k.z <= mine) + (k.w <= mine);
  }
  if (m < own + 4) {
    const uint4 k = four[m];
    const int before = i0 + c - 4 * m;                                // of the four
    n += (before > 0 ? k.x <= mine : k.x < mine) + (before > 1 ? k.y <= mine : k.y < mine) +
         (before > 2 ? k.z <= mine : k.z < mine) + (before > 3 ? k.w <= mine : k.w < mine);
    m += 16;
  }
#pragma unroll 4
  for (; m < all; m += 16) {
    const uint4 k = four[m];
    n += (k.x < mine) + (k.y < mine) + (k.z < mine) + (k.w < mine);
  }
  uint32_t* counts = keys + Tp;
  counts[part * 16 + c] = n;
  __syncthreads();
  if (tid < 16 && i0 + tid < T) {
    uint32_t at = 0;
#pragma unroll
    for (int k = 0; k < 16; ++k) at += counts[k * 16 + tid];
    out[at] = make_uint2(mine, i0 + tid);
  }
}

// a token's (key, place); in: NULL for the ids themselves
__device__ __forceinline__ uint2 token(const int32_t* __restrict__ ids, const uint2* __restrict__ in, long i, int V) {
  return in ? in[i] : make_uint2(key_of(ids[i], V), static_cast<uint32_t>(i));
}

// counts[block][bin] of the digit at `shift`
__global__ __launch_bounds__(kSortThreads) void k_sort_hist(const int32_t* __restrict__ ids,
                                                            const uint2* __restrict__ in, long T, int V, int per,
                                                            int shift, int bits, uint32_t* __restrict__ counts) {
  __shared__ uint32_t hist[1 << kMaxBits];
  const int bins = 1 << bits;
  for (int i = threadIdx.x; i < bins; i += kSortThreads) hist[i] = 0;
  __syncthreads();
  const long i0 = static_cast<long>(blockIdx.x) * per, i1 = min(T, i0 + per);
  for (long b = i0 + threadIdx.x; b < i1; b += kSortThreads * kSortU) {
    uint32_t k[kSortU];
#pragma unroll
    for (int u = 0; u < kSortU; ++u) k[u] = token(ids, in, min(b + u * kSortThreads, i1 - 1), V).x;
#pragma unroll
    for (int u = 0; u < kSortU; ++u)
      if (b + u * kSortThreads < i1) atomicAdd(&hist[(k[u] >> shift) & (bins - 1)], 1u);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < bins; i += kSortThreads) counts[static_cast<long>(blockIdx.x) * bins + i] = hist[i];
}

// Stable scatter of one pass: wave w of block j takes the w-th part of the
// block's tokens, in order, and its tokens of a digit follow those of the
// digits below, of the blocks before and of the waves before.
template <int BITS>
__global__ __launch_bounds__(kSortThreads) void k_sort_scatter(const int32_t* __restrict__ ids,
                                                               const uint2* __restrict__ in, long T, int V, int per,
                                                               int shift, int nb,
                                                               const uint32_t* __restrict__ counts,
                                                               uint2* __restrict__ out) {
  constexpr int bins = 1 << BITS, PT = bins / kSortThreads;          // thread tid has bins PT tid ..
  // a wave adds the counts of 256 bins (and of 256 more), four a lane, over a part of the blocks
  constexpr int kGroups = bins / 256, kParts = kGroups < kSortWaves ? kSortWaves / kGroups : 1;
  __shared__ uint32_t hist[kSortWaves][bins];
  __shared__ __attribute__((aligned(16))) uint32_t sums[2][kParts][bins];
  __shared__ uint32_t carry[kSortWaves];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int mine = blockIdx.x;
  const long i0 = min(T, static_cast<long>(mine) * per + static_cast<long>(w) * (per / kSortWaves));
  const long i1 = min(T, i0 + per / kSortWaves);
  uint2 tok[kSortU];                                   // the wave's next tokens
  auto fetch = [&](long b) {
#pragma unroll
    for (int u = 0; u < kSortU; ++u) tok[u] = token(ids, in, min(b + u * 64 + lane, T - 1), V);
  };
  fetch(i0);
  // totals of every bin and those of the blocks before
#pragma unroll
  for (int grp = w / kParts; grp < kGroups; grp += kSortWaves / kParts) {
    const int part = w % kParts, j0 = nb * part / kParts, j1 = nb * (part + 1) / kParts;
    uint4 t = make_uint4(0, 0, 0, 0), f = t;
    auto add = [&](auto width) {
      constexpr int U = decltype(width)::value;
      for (int j = j0; j < j1; j += U) {
        uint4 n[U];                                                    // (other XCDs' counts: a trip past L2)
#pragma unroll
        for (int u = 0; u < U; ++u)
          n[u] = *reinterpret_cast<const uint4*>(counts + static_cast<long>(min(j + u, j1 - 1)) * bins + grp * 256 + 4 * lane);
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const uint32_t in_t = j + u < j1 ? 0xFFFFFFFFu : 0u, in_f = j + u < min(j1, mine) ? 0xFFFFFFFFu : 0u;
          t = make_uint4(t.x + (n[u].x & in_t), t.y + (n[u].y & in_t), t.z + (n[u].z & in_t), t.w + (n[u].w & in_t));
          f = make_uint4(f.x + (n[u].x & in_f), f.y + (n[u].y & in_f), f.z + (n[u].z & in_f), f.w + (n[u].w & in_f));
        }
      }
    };
    if (j1 - j0 <= 4) add(std::integral_constant<int, 4>());
    else add(std::integral_constant<int, 32>());
    *reinterpret_cast<uint4*>(&sums[0][part][grp * 256 + 4 * lane]) = t;
    *reinterpret_cast<uint4*>(&sums[1][part][grp * 256 + 4 * lane]) = f;
  }
  __syncthreads();
  uint32_t tot[PT] = {}, before[PT] = {};
#pragma unroll
  for (int part = 0; part < kParts; ++part)
#pragma unroll
    for (int k = 0; k < PT; ++k) {
      tot[k] += sums[0][part][PT * tid + k];
      before[k] += sums[1][part][PT * tid + k];
    }
#pragma unroll
  for (int k = 0; k < PT; ++k)
#pragma unroll
    for (int j = 0; j < kSortWaves; ++j) hist[j][PT * tid + k] = 0;
  uint32_t sum = 0;
#pragma unroll
  for (int k = 0; k < PT; ++k) sum += tot[k];
  const uint32_t incl = wave_scan(sum, lane);
  if (lane == 63) carry[w] = incl;
  __syncthreads();
  for (long b = i0; b < i1; b += 64 * kSortU) {
    if (b > i0) fetch(b);
#pragma unroll
    for (int u = 0; u < kSortU; ++u)
      if (b + u * 64 + lane < i1) atomicAdd(&hist[w][(tok[u].x >> shift) & (bins - 1)], 1u);
  }
  if (i1 - i0 > 64 * kSortU) fetch(i0);
  uint32_t start = incl - sum;
#pragma unroll
  for (int j = 0; j < kSortWaves; ++j) start += j < w ? carry[j] : 0;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < PT; ++k) {
    uint32_t at = start + before[k];
    start += tot[k];
#pragma unroll
    for (int j = 0; j < kSortWaves; ++j) {
      const uint32_t n = hist[j][PT * tid + k];
      hist[j][PT * tid + k] = at;
      at += n;
    }
  }
  __syncthreads();
  for (long b = i0; b < i1; b += 64 * kSortU) {
    if (b > i0) fetch(b);
#pragma unroll
    for (int u = 0; u < kSortU; ++u) {
      const bool live = b + u * 64 + lane < i1;
      const uint32_t digit = (tok[u].x >> shift) & (bins - 1);
      const uint64_t m = same_digit<BITS>(digit, __ballot(live));
      const int rank = __popcll(m & ((1ull << lane) - 1));
      const uint32_t at = hist[w][digit] + rank;
      __builtin_amdgcn_wave_barrier();
      if (live && rank == 0) hist[w][digit] += __popcll(m);
      __builtin_amdgcn_wave_barrier();
      if (live) out[at] = tok[u];
    }
  }
}

// ---------------------------------------------------------------------------
// Row sums over the sorted tokens.
struct GradArgs {
  long T;
  int C, V, d;
  int lpr_log2, slices;     // lanes a row, column slices (lpr * VE columns each)
  int K;                    // tokens a team
  int spans;                // of (256 / lpr) * K tokens
  int zrows, zblocks;       // rows of a block of the zero rows, blocks a table
  float scale;
  int accumulate;
};

// the row's columns from `col` on: sum (times scale) to table_grad
template <typename TO, int VE>
__device__ __forceinline__ void write_row(const GradArgs& a, TO* __restrict__ out, int c, uint32_t v, int col,
                                          const float* s) {
  Pack<TO, VE>* dst = reinterpret_cast<Pack<TO, VE>*>(out + (static_cast<long>(c) * a.V + v) * a.d + col);
  Pack<TO, VE> y;
  if (a.accumulate) y = *dst;
#pragma unroll
  for (int e = 0; e < VE; ++e) put(y.v[e], a.accumulate ? fmaf(a.scale, s[e], to_f32(y.v[e])) : a.scale * s[e]);
  *dst = y;
}

// part: [spans][2][C][d]: the piece of the run that enters a span, and of the one that leaves it
template <typename TI, typename TO, int VE>
__global__ __launch_bounds__(256) void k_embed_grad(GradArgs a, const TI* __restrict__ grad,
                                                    const uint2* __restrict__ sorted, float* __restrict__ part,
                                                    TO* __restrict__ out) {
  __shared__ __attribute__((aligned(16))) float head[256 * VE], tail[256 * VE];
  // of a team, bit 0: its first run entered it, 1: that run ended in it, 2: its last run, begun in it, goes on
  __shared__ int state[256];
  const int tid = threadIdx.x;
  const long seg_blocks = static_cast<long>(a.spans) * a.slices * a.C;
  if (blockIdx.x >= seg_blocks) {
    // zero rows: rows [v0, v1) of table c that no token has
    uint32_t* seen = reinterpret_cast<uint32_t*>(state);     // 256 words: zrows <= 8192
    __shared__ long first;
    const long zb = blockIdx.x - seg_blocks;
    const int c = static_cast<int>(zb / a.zblocks);
    const long v0 = (zb - static_cast<long>(c) * a.zblocks) * a.zrows, v1 = min(v0 + a.zrows, static_cast<long>(a.V));
    seen[tid] = 0;
    if (tid < 64) {
      // first token whose id is v0 or more: 64 probes a round
      long lo = 0, hi = a.T;                       // tokens before lo are below, those from hi on are not
      while (hi > lo) {
        const long step = (hi - lo + 63) / 64, at = lo + step * tid;
        const bool below = at < hi && sorted[at].x < static_cast<uint32_t>(v0);
        const int n = __popcll(__ballot(below));   // (the probes below are the first n)
        if (n == 0) { hi = lo; break; }
        const long nhi = n < 64 ? min(hi, lo + step * n) : hi;
        lo = lo + step * (n - 1) + 1;
        hi = nhi;
      }
      if (tid == 0) first = lo;
    }
    __syncthreads();
    for (long i = first + tid; i < a.T; i += 256) {
      const uint32_t k = sorted[i].x;
      if (k >= static_cast<uint32_t>(v1)) break;
      const uint32_t r = k - static_cast<uint32_t>(v0);
      atomicOr(&seen[r >> 5], 1u << (r & 31));
    }
    __syncthreads();
    Pack<TO, VE> z;
#pragma unroll
    for (int e = 0; e < VE; ++e) z.v[e] = 0;
    const uint32_t nv = a.d / VE, n = static_cast<uint32_t>(v1 - v0) * nv;
    Pack<TO, VE>* dst = reinterpret_cast<Pack<TO, VE>*>(out + (static_cast<long>(c) * a.V + v0) * a.d);
    for (uint32_t i = tid; i < n; i += 256) {
      const uint32_t r = i / nv;
      if (!((seen[r >> 5] >> (r & 31)) & 1)) dst[i] = z;
    }
    return;
  }
  // blocks of one span follow each other: its tokens' rows of all tables and slices
  const int span = static_cast<int>(blockIdx.x / (a.slices * a.C));
  const int rest = static_cast<int>(blockIdx.x - static_cast<long>(span) * (a.slices * a.C));
  const int c = rest / a.slices, slice = rest - c * a.slices;
  const int lpr = 1 << a.lpr_log2, teams = 256 >> a.lpr_log2, team = tid >> a.lpr_log2;
  const int col = (slice * lpr + (tid & (lpr - 1))) * VE;
  const bool live = col < a.d;
  const int lcol = min(col, a.d - VE);            // idle lanes repeat the last columns
  const long s0 = static_cast<long>(span) * teams * a.K, s1 = min(s0 + static_cast<long>(teams) * a.K, a.T);
  const long p0 = min(s0 + static_cast<long>(team) * a.K, s1), p1 = min(p0 + a.K, s1);
  const TI* g = grad + static_cast<long>(c) * a.T * a.d + lcol;
  float sum[VE];
#pragma unroll
  for (int e = 0; e < VE; ++e) sum[e] = 0.f;
  int st = 0;
  if (p0 < p1) {
    const uint32_t kfirst = sorted[p0].x;
    const bool entered = p0 > 0 && sorted[p0 - 1].x == kfirst;
    const uint32_t knext = p1 < a.T ? sorted[p1].x : 0xFFFFFFFFu;
    uint32_t cur = kfirst;
    bool first_run = entered;                      // the current run began before the team's tokens
    if (entered) st |= 1;
    auto flush = [&](bool ended) {                 // the current run, complete here unless it entered or goes on
      if (first_run) {
#pragma unroll
        for (int e = 0; e < VE; ++e) head[tid * VE + e] = sum[e];
        if (ended) st |= 2;
      } else if (!ended) {
#pragma unroll
        for (int e = 0; e < VE; ++e) tail[tid * VE + e] = sum[e];
        st |= 4;
      } else if (live && cur < static_cast<uint32_t>(a.V)) {
        write_row<TO, VE>(a, out, c, cur, col, sum);
      }
      first_run = false;
    };
    constexpr int U = 4;
    for (long p = p0; p < p1; p += U) {
      uint2 tok[U];
      Pack<TI, VE> x[U];
#pragma unroll
      for (int u = 0; u < U; ++u) tok[u] = sorted[min(p + u, p1 - 1)];
#pragma unroll
      for (int u = 0; u < U; ++u)
        x[u] = *reinterpret_cast<const Pack<TI, VE>*>(g + static_cast<long>(tok[u].y) * a.d);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (p + u >= p1) break;
        if (tok[u].x != cur) {
          flush(true);
          cur = tok[u].x;
#pragma unroll
          for (int e = 0; e < VE; ++e) sum[e] = 0.f;
        }
#pragma unroll
        for (int e = 0; e < VE; ++e) sum[e] += to_f32(x[u].v[e]);
      }
    }
    flush(knext != cur);
  }
  if ((tid & (lpr - 1)) == 0) state[team] = st;
  __syncthreads();
  // the runs that cross teams: the team where one began (team 0: also the one
  // that entered the span) adds the following teams' first pieces
  const int used = s1 > s0 ? static_cast<int>((s1 - s0 + a.K - 1) / a.K) : 0;   // teams with tokens
  const int me = tid & (lpr - 1);
  const long pcol = static_cast<long>(c) * a.d + col, prow = static_cast<long>(a.C) * a.d;
  for (int w = 0; w < 2; ++w) {
    const bool enter = w == 0;                     // the run that entered the span, then the runs begun here
    if (enter ? !(team == 0 && (st & 1)) : !(st & 4)) continue;
    float s[VE];
#pragma unroll
    for (int e = 0; e < VE; ++e) s[e] = enter ? head[tid * VE + e] : tail[tid * VE + e];
    bool done = enter && (st & 2);
    for (int k = team + 1; k < used && !done; ++k) {
      // (the team after one whose run goes on was entered)
#pragma unroll
      for (int e = 0; e < VE; ++e) s[e] += head[((k << a.lpr_log2) + me) * VE + e];
      done = state[k] & 2;
    }
    if (!live) continue;
    if (enter || !done) {
      float* dst = part + (static_cast<long>(span) * 2 + (enter ? 0 : 1)) * prow + pcol;
#pragma unroll
      for (int e = 0; e < VE; ++e) dst[e] = s[e];
    } else {
      const uint32_t v = sorted[p1 - 1].x;
      if (v < static_cast<uint32_t>(a.V)) write_row<TO, VE>(a, out, c, v, col, s);
    }
  }
}

// The runs that cross spans.  A block has the run that leaves span blockIdx.x
// if it began there, and adds the pieces that entered the following spans.
template <typename TO>
__global__ __launch_bounds__(256) void k_embed_grad_join(GradArgs a, int span_tokens,
                                                         const uint2* __restrict__ sorted,
                                                         const float* __restrict__ part, TO* __restrict__ out) {
  const long s0 = static_cast<long>(blockIdx.x) * span_tokens, s1 = s0 + span_tokens;
  if (s1 >= a.T) return;
  const uint32_t v = sorted[s1 - 1].x;
  if (v >= static_cast<uint32_t>(a.V) || sorted[s1].x != v) return;
  if (s0 > 0 && sorted[s0].x == v && sorted[s0 - 1].x == v) return;   // began earlier
  // spans whose last token still has the id, then the one where it ends
  const long cd = static_cast<long>(a.C) * a.d;
  int last = blockIdx.x + 1;
  while ((last + 1l) * span_tokens < a.T && sorted[(last + 1l) * span_tokens - 1].x == v &&
         sorted[(last + 1l) * span_tokens].x == v)
    ++last;
  for (long i = static_cast<long>(blockIdx.y) * 256 + threadIdx.x; i < cd; i += 256l * gridDim.y) {
    float s = part[(blockIdx.x * 2l + 1) * cd + i];
#pragma unroll 8
    for (int k = blockIdx.x + 1; k <= last; ++k) s += part[k * 2l * cd + i];
    const int c = static_cast<int>(i / a.d), col = static_cast<int>(i - static_cast<long>(c) * a.d);
    write_row<TO, 1>(a, out, c, v, col, &s);
  }
}

// ---------------------------------------------------------------------------
// Host side.
namespace {

bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// elements a lane moves at once: 16 bytes of the narrower type where every row
// of both arrays starts on such a boundary, else one
template <typename TI, typename TO>
int vec_of(const void* a, const void* b, int d) {
  constexpr int VE = Elem<TI>::kVec > Elem<TO>::kVec ? Elem<TI>::kVec : Elem<TO>::kVec;
  return d % VE == 0 && aligned(a, 16) && aligned(b, 16) ? VE : 1;
}

int key_bits(int V) {
  int bits = 1;
  while (bits < 32 && (static_cast<uint32_t>(V) >> bits)) ++bits;   // keys 0 .. V
  return bits;
}

int sort_per(long T) {
  const long per = std::max<long>(kSortBlock, (T + kSortBlocks - 1) / kSortBlocks);
  return static_cast<int>((per + kSortBlock - 1) / kSortBlock * kSortBlock);
}

// Tokens of a team: the most that still gives every CU two workgroups (fewer
// pieces to join), 4 at least; few tokens in one span, with nothing to join (a call
// of 900 tokens of 4 x 32: 14.6 us in two spans or more, 12.0 in one).
int team_tokens(long T, int teams, long per_span) {
  if (T <= 16l * teams) return static_cast<int>(std::max<long>(4, (T + teams - 1) / teams));
  int K = 32;
  while (K > 4 && (T + teams * K - 1) / (teams * K) * per_span < 512) K /= 2;
  return K;
}

GradArgs grad_args(int C, int V, int d, long T, int VE) {
  GradArgs a;
  a.T = T;
  a.C = C;
  a.V = V;
  a.d = d;
  // lanes a row: the width that leaves the fewest lanes idle, the widest of those
  const int cols = (d + VE - 1) / VE;
  int best = 6, waste = 1 << 30;
  for (int l = 6; l >= 2; --l) {
    const int w = (cols + (1 << l) - 1) / (1 << l) * (1 << l) - cols;
    if (w < waste) {
      waste = w;
      best = l;
    }
  }
  a.lpr_log2 = best;
  a.slices = (cols + (1 << best) - 1) >> best;
  const int teams = 256 >> best;
  a.K = team_tokens(T, teams, static_cast<long>(a.slices) * C);
  a.spans = static_cast<int>((T + teams * a.K - 1) / (teams * a.K));
  return a;
}

}  // namespace

static size_t grad_layout(int C, int d, long T, size_t spans, size_t off[4]) {
  auto up = [](size_t v) { return (v + 255) / 256 * 256; };
  size_t at = 0;
  off[0] = at; at = up(at + 8ul * T);                      // sorted pairs
  off[1] = at; if (T > kSortRank) at = up(at + 8ul * T);    // the other side of the passes
  off[2] = at; if (T > kSortRank) at = up(at + 4ul * kSortBlocks * (1 << kMaxBits));
  off[3] = at;
  if (spans > 1) at = up(at + 8ul * spans * C * d);
  return at;
}

size_t embed_grad_bytes(int C, int V, int d, long T, size_t off[4]) {
  size_t spans = 0;
  for (int VE : {1, 4, 8}) spans = std::max<size_t>(spans, grad_args(C, V, d, T, VE).spans);
  return grad_layout(C, d, T, spans, off);
}

// Spans of up to T tokens: teams of 32 tokens make the most of the longest list, and
// fewer tokens a team (4 at least) are taken up to 512 workgroups, which at most doubles them.
size_t embed_grad_most(int C, int V, int d, long T) {
  size_t spans = 0, off[4];
  for (int VE : {1, 4, 8}) {
    const GradArgs a = grad_args(C, V, d, T, VE);
    const long teams = 256 >> a.lpr_log2, per_span = static_cast<long>(a.slices) * C;
    const long few = std::min((T + 4 * teams - 1) / (4 * teams), 2 * ((511 + per_span) / per_span));
    spans = std::max<size_t>(spans, std::max((T + 32 * teams - 1) / (32 * teams), few));
  }
  return grad_layout(C, d, T, spans, off);
}

template <typename TI, typename TO>
static hipError_t lookup_t(const void* table, int C, int V, int d, const int32_t* ids, int T, float scale, void* out,
                           hipStream_t st) {
  constexpr int VE = Elem<TI>::kVec > Elem<TO>::kVec ? Elem<TI>::kVec : Elem<TO>::kVec;
  const int ve = vec_of<TI, TO>(table, out, d), nv = d / ve;
  const long blocks = (static_cast<long>(T) * nv + 1023) / 1024;
  const dim3 grid(static_cast<unsigned>(blocks), C);
  auto kern = ve == 1 ? &k_embed_lookup<TI, TO, 1> : &k_embed_lookup<TI, TO, VE>;
  hipLaunchKernelGGL(kern, grid, dim3(256), 0, st, static_cast<const TI*>(table), V, d, nv, ids, T, scale,
                     static_cast<TO*>(out));
  return hipGetLastError();
}

hipError_t launch_embed_lookup(const void* table, int table_dtype, int C, int V, int d, const int32_t* ids, int T,
                               float scale, void* out, int out_dtype, hipStream_t st) {
  auto f = table_dtype == MOL_BF16 ? (out_dtype == MOL_BF16 ? &lookup_t<bf16_t, bf16_t> : &lookup_t<bf16_t, float>)
                                   : (out_dtype == MOL_BF16 ? &lookup_t<float, bf16_t> : &lookup_t<float, float>);
  return f(table, C, V, d, ids, T, scale, out, st);
}

static hipError_t launch_sort(const int32_t* ids, long T, int V, uint2* a, uint2* b, uint32_t* counts, hipStream_t st) {
  if (T <= kSortRank) {
    const size_t lds = ((T + 63) / 64 * 64 + 256) * 4;                // (33 KB at most)
    hipLaunchKernelGGL(k_sort_rank, dim3(static_cast<unsigned>((T + 15) / 16)), dim3(256), lds, st, ids,
                       static_cast<int>(T), V, a);
    return hipGetLastError();
  }
  const int bits = key_bits(V);
  const int passes = (bits + kMaxBits - 1) / kMaxBits, each = std::max(kMinBits, (bits + passes - 1) / passes);
  const int per = sort_per(T), nb = static_cast<int>((T + per - 1) / per);
  auto scatter = each == 8 ? &k_sort_scatter<8> : each == 9 ? &k_sort_scatter<9> : each == 10 ? &k_sort_scatter<10>
                                                                                              : &k_sort_scatter<11>;
  // the last pass ends in `a`
  const uint2* in = nullptr;
  for (int p = 0; p < passes; ++p) {
    uint2* to = (passes - p) % 2 ? a : b;
    hipLaunchKernelGGL(k_sort_hist, dim3(nb), dim3(kSortThreads), 0, st, ids, in, T, V, per, p * each, each, counts);
    hipLaunchKernelGGL(scatter, dim3(nb), dim3(kSortThreads), 0, st, ids, in, T, V, per, p * each, nb, counts, to);
    in = to;
  }
  return hipGetLastError();
}

template <typename TI, typename TO>
static hipError_t grad_t(const void* grad, int C, int V, int d, const int32_t* ids, long T, float scale,
                         int accumulate, void* out, char* ws, hipStream_t st) {
  constexpr int VE = Elem<TI>::kVec > Elem<TO>::kVec ? Elem<TI>::kVec : Elem<TO>::kVec;
  const int ve = vec_of<TI, TO>(grad, out, d);
  size_t off[4];
  embed_grad_bytes(C, V, d, T, off);
  uint2* sorted = reinterpret_cast<uint2*>(ws + off[0]);
  float* part = reinterpret_cast<float*>(ws + off[3]);
  if (T > 0) {
    const hipError_t e = launch_sort(ids, T, V, sorted, reinterpret_cast<uint2*>(ws + off[1]),
                                     reinterpret_cast<uint32_t*>(ws + off[2]), st);
    if (e != hipSuccess) return e;
  }
  GradArgs a = grad_args(C, V, d, T, ve);
  a.scale = scale;
  a.accumulate = accumulate;
  // zero rows: blocks of about 64 KB, as many rows as their bitmap holds at most
  const long fit = 65536 / (static_cast<long>(d) * static_cast<long>(sizeof(TO)));
  a.zrows = static_cast<int>(std::max<long>(1, std::min<long>({fit, 8192, V})));
  a.zblocks = accumulate ? 0 : static_cast<int>((V + a.zrows - 1l) / a.zrows);
  const long blocks = static_cast<long>(a.spans) * a.slices * C + static_cast<long>(a.zblocks) * C;
  if (blocks > 0) {
    auto kern = ve == 1 ? &k_embed_grad<TI, TO, 1> : &k_embed_grad<TI, TO, VE>;
    hipLaunchKernelGGL(kern, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, st, a, static_cast<const TI*>(grad),
                       sorted, part, static_cast<TO*>(out));
  }
  if (a.spans > 1) {
    const int y = static_cast<int>(std::min<long>((static_cast<long>(C) * d + 255) / 256, 64));
    hipLaunchKernelGGL(k_embed_grad_join<TO>, dim3(a.spans - 1, y), dim3(256), 0, st, a,
                       (256 >> a.lpr_log2) * a.K, sorted, part, static_cast<TO*>(out));
  }
  return hipGetLastError();
}

hipError_t launch_embed_grad(const void* grad, int grad_dtype, int C, int V, int d, const int32_t* ids, int T,
                             float scale, int accumulate, void* out, int out_dtype, void* ws, hipStream_t st) {
  auto f = grad_dtype == MOL_BF16 ? (out_dtype == MOL_BF16 ? &grad_t<bf16_t, bf16_t> : &grad_t<bf16_t, float>)
                                  : (out_dtype == MOL_BF16 ? &grad_t<float, bf16_t> : &grad_t<float, float>);
  return f(grad, C, V, d, ids, T, scale, accumulate, out, static_cast<char*>(ws), st);
}

}  // namespace mol
