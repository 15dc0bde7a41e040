// Rows normalised, and the gradients: layer norm (mean 0, variance 1, then scale
// and shift) and L2 normalisation of Eq. 2's components (length 1).
//
//   layer norm:  y = xhat gamma + beta,  xhat = (x - mean) rstd,  rstd = 1 / sqrt(var + eps)
//                dx = rstd (w - mean(w) - xhat mean(w xhat)),  w = dy gamma
//                dgamma = sum over rows of dy xhat,  dbeta = sum over rows of dy
//   L2:          y = x / r,  r = max(|x|, eps)
//                dx = (dy - y <y, dy>) / r   (dy / eps where |x| <= eps)
//
// Bound by memory: a row is read once into the registers of a team of lanes
// (both rows of a gradient), its statistics are formed there (variance about the mean,
// float32; a gradient forms them again from x rather than reading them), and it is
// written once.  Measured: layer norm of 262,144 x 512 bf16 93 to 100 us (5.4 TB/s, where a copy of
// as much runs at 5.0), its gradient 137 to 141 + 5 (5.5; through the caches 158 + 5); 172M float32 elements to bf16 rows
// of 32 of length 1 172 us (6.0).  Reading past the caches gains in gradients of large tensors only (streams();
// forwards it took 134 us for 100).  Where rows are few, their chains of loads and sums: 32 rows of 1024 take
// 3.5 us, the gradient of 4099 float32 rows of 777 14 to 16 + 4 (7 at the rate of large ones).
#include <algorithm>
#include <cfloat>
#include <type_traits>

#include "mol_kernels.h"
#include "mol_vec.h"

namespace mol {

namespace {

using vec::Raw;

enum { kLayer = 0, kLength = 1 };

// Rows go round teams of `lanes` lanes of a wave (TEAM 0), or of TEAM threads, a
// workgroup.  A lane holds E elements of a row: runs of VE, one run of every lanes VE.
struct RowArgs {
  long T;
  int d, lanes;
  float eps;
  const void* x;
  const float* gamma;      // or NULL: 1
  const float* beta;       // or NULL: 0
  void* y;
  int y_bf16;
  const void* dy;          // gradients
  float* dgamma;           // [2][d] of the workgroup, or of the call; NULL: not wanted
  float* dbeta;
  long part;               // floats from one workgroup's to the next
  bool once;               // gradients, teams of lanes: read past the caches
};

template <int TEAM>
struct Team {
  int lanes, lane;         // of a team
  float* sh;               // TEAM / 64 * N floats, for sums over waves
  // N sums over the team at once
  template <int N>
  __device__ __forceinline__ void sum(float (&v)[N]) const {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = vec::team_sum(v[i], TEAM ? 64 : lanes);
    if constexpr (TEAM > 64) {
      if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) sh[threadIdx.x / 64 * N + i] = v[i];
      __syncthreads();
#pragma unroll
      for (int i = 0; i < N; ++i) {
        v[i] = sh[i];
        for (int w = 1; w < TEAM / 64; ++w) v[i] += sh[w * N + i];
      }
      __syncthreads();
    }
  }
};

// What a lane knows of its place in every row.
template <int E, int VE>
struct Place {
  int col[E / VE], n[E / VE];      // first element of each run, and how many of the row's it holds
  int span, d;
  __device__ __forceinline__ Place(int lane, int lanes, int d_) : span(lanes * VE), d(d_) {
#pragma unroll
    for (int g = 0; g < E / VE; ++g) {
      col[g] = (g * lanes + lane) * VE;
      n[g] = min(VE, d - col[g]);
    }
  }
  // of the runs g of all lanes: all whole, none there
  __device__ __forceinline__ bool full(int g) const { return (g + 1) * span <= d; }
  __device__ __forceinline__ bool none(int g) const { return g * span >= d; }
};

// Powers of two that bring a row's squares back into range, for sums of
// squares out of it: exact, and seldom needed.
__device__ __forceinline__ float rescale(float ss) {
  return !(ss <= FLT_MAX) ? 0x1p-96f : ss < 0x1p-80f ? 0x1p96f : 1.f;
}

// The row centred (layer norm) and scaled by `scale`, and 1 / its size in that scale
template <int MODE, int TEAM, int E, int VE, bool WHOLE>
struct Stats {
  float x[E];              // scale (x - mean), 0 behind the row's end; L2: scale x
  float inv;               // layer norm: 1 / (scale sqrt(var + eps)); L2: 1 / (scale max(|x|, eps))
  float scale;
  bool flat;               // L2: |x| <= eps

  template <typename T>
  __device__ __forceinline__ void form(const Raw<T, VE> (&raw)[E / VE], const Place<E, VE>& at, const Team<TEAM>& team, int d,
                                       float eps) {
    float ss;
    scale = 1.f;
    for (bool again = false;; again = true) {                  // (one copy of the code, which runs once, seldom twice)
      ss = squares(raw, at, team, d, scale);
      const float want = rescale(MODE == kLayer ? ss + eps : ss);
      // (a layer norm's small rows need none: eps is added to their variance, in range as well)
      const bool needed = MODE == kLength ? want != 1.f : want < 1.f;
      if (again || !__any(needed)) break;
      if (needed) scale = want;
    }
    if (MODE == kLayer) {
      if (ss == 0.f) scale = 1.f;                              // (a constant row: x is 0 in any scale, and all that counts is eps)
      inv = 1.f / sqrtf(ss / d + eps * scale * scale);
      flat = false;
    } else {
      const float r = sqrtf(ss);
      flat = r <= eps * scale;
      inv = 1.f / (flat ? eps * scale : r);
    }
  }

 private:
  template <typename T>
  __device__ __forceinline__ float squares(const Raw<T, VE> (&raw)[E / VE], const Place<E, VE>& at, const Team<TEAM>& team,
                                           int d, float s) {
    float mean[1] = {0.f};
#pragma unroll
    for (int g = 0; g < E / VE; ++g)
#pragma unroll
      for (int e = 0; e < VE; ++e) x[g * VE + e] = raw[g].at(e);
#pragma unroll
    for (int i = 0; i < E; ++i) x[i] *= s;
    if (MODE == kLayer) {
#pragma unroll
      for (int i = 0; i < E; ++i) mean[0] += x[i];
      team.sum(mean);
      mean[0] /= d;
    }
    float ss[1] = {0.f};
#pragma unroll
    for (int g = 0; g < E / VE; ++g) {
      if (MODE == kLayer) {
        if (WHOLE || at.full(g)) {
#pragma unroll
          for (int e = 0; e < VE; ++e) x[g * VE + e] -= mean[0];
        } else {
#pragma unroll
          for (int e = 0; e < VE; ++e) x[g * VE + e] = e < at.n[g] ? x[g * VE + e] - mean[0] : 0.f;
        }
      }
#pragma unroll
      for (int e = 0; e < VE; ++e) ss[0] = fmaf(x[g * VE + e], x[g * VE + e], ss[0]);
    }
    team.sum(ss);
    return ss[0];
  }
};

// A row as it lies: runs that pass its end are read from where they would end with it
// (settle() puts that right), so that every lane loads whole runs and nothing branches.
template <bool ONCE = false, typename T, int E, int VE>
__device__ __forceinline__ void load_row(Raw<T, VE> (&r)[E / VE], const T* p, const Place<E, VE>& at, bool whole) {
  if (!whole && at.d < VE) {                           // (rows shorter than a run)
#pragma unroll
    for (int g = 0; g < E / VE; ++g) r[g].load(p + at.col[g], at.n[g]);
    return;
  }
#pragma unroll
  for (int g = 0; g < E / VE; ++g) r[g].template load<ONCE>(p + (whole ? at.col[g] : min(at.col[g], at.d - VE)));
}
// what was read for elements behind the row's end becomes 0, the last run's elements move to their places
template <typename T, int E, int VE>
__device__ __forceinline__ void settle(Raw<T, VE> (&r)[E / VE], const Place<E, VE>& at, bool whole) {
  if (whole || at.d < VE) return;
  constexpr int kPer = 4 / sizeof(T);                  // elements of a word
#pragma unroll
  for (int g = 0; g < E / VE; ++g) {
    if (at.full(g)) continue;
    if (at.d % VE) {                                   // by VE - n elements, of the lane whose run is cut
      const int k = at.n[g] > 0 ? VE - at.n[g] : 0;
#pragma unroll
      for (int by = 1; by < Raw<T, VE>::kWords; by <<= 1)
#pragma unroll
        for (int i = 0; i < Raw<T, VE>::kWords; ++i)
          r[g].w[i] = k / kPer & by ? (i + by < Raw<T, VE>::kWords ? r[g].w[i + by] : 0) : r[g].w[i];
      if (kPer == 2)
#pragma unroll
        for (int i = 0; i < Raw<T, VE>::kWords; ++i) {
          const uint32_t above = i + 1 < Raw<T, VE>::kWords ? r[g].w[i + 1] : 0;
          r[g].w[i] = k & 1 ? __builtin_amdgcn_alignbit(above, r[g].w[i], 16) : r[g].w[i];
        }
    }
#pragma unroll
    for (int i = 0; i < Raw<T, VE>::kWords; ++i) r[g].w[i] = at.n[g] > 0 ? r[g].w[i] : 0;
  }
}

template <int E, int VE>
__device__ __forceinline__ void store_row(void* out, int bf16, long row, int d, const Place<E, VE>& at, bool whole,
                                          const float (&v)[E]) {
#pragma unroll
  for (int g = 0; g < E / VE; ++g) {
    if (!whole && at.none(g)) continue;
    float o[VE];
#pragma unroll
    for (int e = 0; e < VE; ++e) o[e] = v[g * VE + e];
    const long to = row * d + at.col[g];
    auto put = [&](auto* y) {
      if (whole || at.full(g) || at.n[g] >= VE)
        vec::store(y + to, o);
      else if (d % VE)
        vec::store(y + to, o, at.n[g]);
    };
    if (bf16)
      put(static_cast<bf16_t*>(out));
    else
      put(static_cast<float*>(out));
  }
}

template <int E, int VE>
__device__ __forceinline__ void load_weights(float (&w)[E], const float* p, float otherwise, const Place<E, VE>& at,
                                             bool whole) {
  if (p) {
    Raw<float, VE> r[E / VE];
    load_row(r, p, at, whole);
    settle(r, at, whole);
#pragma unroll
    for (int i = 0; i < E; ++i) w[i] = r[i / VE].at(i % VE);
  } else {
#pragma unroll
    for (int i = 0; i < E; ++i) w[i] = otherwise;
  }
}

template <int TEAM>
constexpr int threads() {
  return TEAM ? TEAM : 256;
}

}  // namespace

template <int MODE, typename T, int TEAM, int E, bool WHOLE>
__global__ __launch_bounds__(threads<TEAM>()) void k_norm(RowArgs a) {
  constexpr int VE = 16 / sizeof(T);
  __shared__ float sh[TEAM ? TEAM / 64 : 1];
  const int lanes = TEAM ? TEAM : a.lanes, teams = TEAM ? 1 : 256 / lanes;
  const Team<TEAM> team{lanes, static_cast<int>(threadIdx.x) & (lanes - 1), sh};
  const Place<E, VE> at(team.lane, lanes, a.d);
  const T* x = static_cast<const T*>(a.x);
  float gamma[E], beta[E];
  if (MODE == kLayer) {
    load_weights(gamma, a.gamma, 1.f, at, WHOLE);
    load_weights(beta, a.beta, 0.f, at, WHOLE);
  }
  const long step = static_cast<long>(gridDim.x) * teams;
  // (the rows of a wave start together and end together, so that sums over lanes find them all)
  const long first = static_cast<long>(blockIdx.x) * teams;
  const int mine = TEAM ? 0 : threadIdx.x / lanes;
  Raw<T, VE> raw[E / VE], next[E / VE];
  load_row(raw, x + min(first + mine, a.T - 1) * a.d, at, WHOLE);
  for (long row = first; row < a.T; row += step) {
    if (row + step < a.T) load_row(next, x + min(row + step + mine, a.T - 1) * a.d, at, WHOLE);
    settle(raw, at, WHOLE);
    Stats<MODE, TEAM, E, VE, WHOLE> st;
    st.form(raw, at, team, a.d, a.eps);
#pragma unroll
    for (int i = 0; i < E; ++i) {
      st.x[i] *= st.inv;
      if (MODE == kLayer) st.x[i] = fmaf(st.x[i], gamma[i], beta[i]);
    }
    if (row + mine < a.T) store_row(a.y, a.y_bf16, row + mine, a.d, at, WHOLE, st.x);
#pragma unroll
    for (int g = 0; g < E / VE; ++g) raw[g] = next[g];
  }
}

// The weights' gradients are summed over a lane's rows in registers, over the
// workgroup's teams at the end, and over workgroups by a launch of sums.
template <int MODE, typename T, typename TG, int TEAM, int E, bool WHOLE, bool ONCE>
__global__ __launch_bounds__(threads<TEAM>()) void k_norm_grad(RowArgs a) {
  constexpr int VE = sizeof(T) == 2 && sizeof(TG) == 2 ? 8 : 4;
  extern __shared__ float dyn[];             // [4][2][d] where teams are joined
  __shared__ float sh[TEAM ? TEAM / 64 * 2 : 1];
  const int lanes = TEAM ? TEAM : a.lanes, teams = TEAM ? 1 : 256 / lanes;
  const Team<TEAM> team{lanes, static_cast<int>(threadIdx.x) & (lanes - 1), sh};
  const Place<E, VE> at(team.lane, lanes, a.d);
  const T* x = static_cast<const T*>(a.x);
  const TG* dy = static_cast<const TG*>(a.dy);
  // (float32 rows leave no registers for the row behind them; nor do 16 elements of each of 1024 threads, for
  // which gamma is read again with every row)
  constexpr bool kGamma = TEAM < 1024 || E == 8, kAhead = kGamma && VE == 8;
  float gamma[E], dgamma[E], dbeta[E];
  if (MODE == kLayer && kGamma) load_weights(gamma, a.gamma, 1.f, at, WHOLE);
#pragma unroll
  for (int i = 0; i < E; ++i) dgamma[i] = dbeta[i] = 0.f;
  const long step = static_cast<long>(gridDim.x) * teams;
  const long first = static_cast<long>(blockIdx.x) * teams;
  const int mine = TEAM ? 0 : threadIdx.x / lanes;
  Raw<T, VE> raw[E / VE], next[E / VE];
  Raw<TG, VE> graw[E / VE], gnext[E / VE];
  auto fetch = [&](Raw<T, VE>(&r)[E / VE], Raw<TG, VE>(&g)[E / VE], long row) {
    const long at_row = min(row + mine, a.T - 1) * a.d;
    load_row<ONCE>(r, x + at_row, at, WHOLE);
    load_row<ONCE>(g, dy + at_row, at, WHOLE);
  };
  if (kAhead) fetch(raw, graw, first);
  for (long row = first; row < a.T; row += step) {
    if (!kAhead)
      fetch(raw, graw, row);
    else if (row + step < a.T)
      fetch(next, gnext, row + step);
    if (MODE == kLayer && !kGamma) load_weights(gamma, a.gamma, 1.f, at, WHOLE);
    const bool live = row + mine < a.T;
    settle(raw, at, WHOLE);
    settle(graw, at, WHOLE);
    Stats<MODE, TEAM, E, VE, WHOLE> st;
    st.form(raw, at, team, a.d, a.eps);
    float w[E], c[2] = {0.f, 0.f};             // layer norm: sums of w and w xhat; L2: of y dy
#pragma unroll
    for (int g = 0; g < E / VE; ++g)
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        const int i = g * VE + e;
        const float v = graw[g].at(e);
        st.x[i] *= st.inv;
        if (MODE == kLayer) {
          w[i] = v * gamma[i];
          c[0] += w[i];
        } else {
          w[i] = v;
        }
        c[1] = fmaf(w[i], st.x[i], c[1]);
      }
    if (MODE == kLayer && live)
#pragma unroll
      for (int g = 0; g < E / VE; ++g)
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          dgamma[g * VE + e] = fmaf(graw[g].at(e), st.x[g * VE + e], dgamma[g * VE + e]);
          dbeta[g * VE + e] += graw[g].at(e);
        }
    team.sum(c);
    if (MODE == kLayer) {
      c[0] /= a.d;
      c[1] /= a.d;
    } else if (st.flat) {
      c[1] = 0.f;
    }
    // (L2 in two factors: 1 / |x| may be 2^-135 where dx is a normal number; layer norm's is 2^-128 and more)
    const bool two = MODE == kLength && st.scale < 1.f;
    const float inv = two ? st.inv : st.inv * st.scale, then = two ? st.scale : 1.f;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      w[i] = inv * fmaf(-st.x[i], c[1], MODE == kLayer ? w[i] - c[0] : w[i]);
      if (MODE == kLength) w[i] *= then;
    }
    if (live) store_row(a.y, a.y_bf16, row + mine, a.d, at, WHOLE, w);
    if (kAhead)
#pragma unroll
      for (int g = 0; g < E / VE; ++g) raw[g] = next[g], graw[g] = gnext[g];
  }
  if (MODE != kLayer || !a.dgamma) return;
  float* og = a.dgamma + blockIdx.x * a.part;
  float* ob = a.dbeta + blockIdx.x * a.part;
  if constexpr (TEAM == 0) {
    for (int o = lanes; o < 64; o <<= 1)
#pragma unroll
      for (int i = 0; i < E; ++i) {
        dgamma[i] += __shfl_xor(dgamma[i], o);
        dbeta[i] += __shfl_xor(dbeta[i], o);
      }
    float* mineg = dyn + threadIdx.x / 64 * 2 * a.d;
    if ((threadIdx.x & 63) < lanes)
#pragma unroll
      for (int g = 0; g < E / VE; ++g)
#pragma unroll
        for (int e = 0; e < VE; ++e)
          if (e < at.n[g]) {
            mineg[at.col[g] + e] = dgamma[g * VE + e];
            mineg[a.d + at.col[g] + e] = dbeta[g * VE + e];
          }
    __syncthreads();
    for (int i = threadIdx.x; i < a.d; i += 256) {
      const int s = 2 * a.d;
      og[i] = (dyn[i] + dyn[s + i]) + (dyn[2 * s + i] + dyn[3 * s + i]);
      ob[i] = (dyn[a.d + i] + dyn[s + a.d + i]) + (dyn[2 * s + a.d + i] + dyn[3 * s + a.d + i]);
    }
  } else {
#pragma unroll
    for (int g = 0; g < E / VE; ++g)
#pragma unroll
      for (int e = 0; e < VE; ++e)
        if (e < at.n[g]) {
          og[at.col[g] + e] = dgamma[g * VE + e];
          ob[at.col[g] + e] = dbeta[g * VE + e];
        }
  }
}

// The workgroups' parts [parts][2][d] summed: 16 columns of dgamma and dbeta by 64 runs of parts,
// the runs in order.
__global__ __launch_bounds__(1024) void k_norm_sums(const float* in, int parts, int d, float* dgamma, float* dbeta) {
  __shared__ float sh[64][17];
  const int c = threadIdx.x & 15, run = threadIdx.x / 16, col = blockIdx.x * 16 + c;
  float v = 0.f;
  if (col < 2 * d) {
#pragma unroll 8
    for (int k = run; k < parts; k += 64) v += in[static_cast<long>(k) * 2 * d + col];
  }
  sh[run][c] = v;
  __syncthreads();
  if (threadIdx.x < 64) {                              // four lanes a column
    const int col4 = threadIdx.x / 4, q = threadIdx.x & 3;
    float t = 0.f;
#pragma unroll
    for (int k = 0; k < 16; ++k) t += sh[16 * q + k][col4];
    t = vec::team_sum(t, 4);
    const int to = blockIdx.x * 16 + col4;
    if (q == 0 && to < 2 * d) (to < d ? dgamma[to] : dbeta[to - d]) = t;
  }
}

namespace {

struct RowPlan {
  int team, E, lanes;      // team 0: lanes of a wave
  int rows;                // of a workgroup at once
};
int pow2_up(int n) {
  int p = 1;
  while (p < n) p <<= 1;
  return p;
}
// A row's team is as small as its registers allow, since sums over fewer lanes take fewer
// steps, and a row of 64 lanes or less needs no barrier.
RowPlan row_plan(int d) {
  RowPlan p{};
  if (d <= 1024) {
    p.E = d <= 128 ? 8 : 16;
    p.lanes = pow2_up((d + p.E - 1) / p.E);
    p.rows = 256 / p.lanes;
  } else {
    p.team = d <= 4096 ? 256 : 1024;
    p.E = d <= 8 * p.team ? 8 : 16;
    p.lanes = p.team;
    p.rows = 1;
  }
  return p;
}
bool row_whole(const RowPlan& p, int d) { return d == p.lanes * p.E; }
// Workgroups.  Without gradients of weights each takes the rows that it holds at once, since
// a grid that stays drifts apart in memory (172M elements in rows of 32 to unit length: 174 us,
// with 2048 workgroups that stay 206; wide rows, which read as much of gamma and beta, stay).
// With them, whose parts each writes and a launch of sums reads, about as many as run at once,
// of two rows a team at least (512 in place of 1024 took 179 us at 262,144 x 512 through the caches, for 163).
long row_blocks(const RowPlan& p, long T, bool weights) {
  const long rows = weights ? 2 * p.rows : p.rows, want = (T + rows - 1) / rows;
  if (p.team == 1024) return std::min(want, weights ? 256l : 512l);
  return std::min(want, weights ? 1024l : 1l << 22);
}

template <int MODE, typename T, int TEAM, int E>
void run_norm(const RowArgs& a, long blocks, bool whole, hipStream_t st) {
  if (whole)
    hipLaunchKernelGGL((k_norm<MODE, T, TEAM, E, true>), dim3(blocks), dim3(threads<TEAM>()), 0, st, a);
  else
    hipLaunchKernelGGL((k_norm<MODE, T, TEAM, E, false>), dim3(blocks), dim3(threads<TEAM>()), 0, st, a);
}
template <int MODE, typename T>
hipError_t launch_norm_mode(RowArgs& a, hipStream_t st) {
  const RowPlan p = row_plan(a.d);
  a.lanes = p.lanes;
  const long blocks = row_blocks(p, a.T, false);
  const bool whole = row_whole(p, a.d);
  auto of = [&](auto e) {
    constexpr int E = decltype(e)::value;
    if (p.team == 256)
      run_norm<MODE, T, 256, E>(a, blocks, whole, st);
    else if (p.team)
      run_norm<MODE, T, 1024, E>(a, blocks, whole, st);
    else
      run_norm<MODE, T, 0, E>(a, blocks, whole, st);
  };
  p.E == 8 ? of(std::integral_constant<int, 8>{}) : of(std::integral_constant<int, 16>{});
  return hipGetLastError();
}

template <int MODE, typename T, typename TG, int TEAM, int E>
void run_norm_grad(const RowArgs& a, long blocks, bool whole, hipStream_t st) {
  const size_t lds = TEAM == 0 && MODE == kLayer && a.dgamma ? 8 * a.d * sizeof(float) : 0;
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(blocks), dim3(threads<TEAM>()), lds, st, a); };
  if constexpr (TEAM == 0) {
    if (a.once) {
      whole ? go(k_norm_grad<MODE, T, TG, TEAM, E, true, true>) : go(k_norm_grad<MODE, T, TG, TEAM, E, false, true>);
      return;
    }
  }
  whole ? go(k_norm_grad<MODE, T, TG, TEAM, E, true, false>) : go(k_norm_grad<MODE, T, TG, TEAM, E, false, false>);
}
template <int MODE, typename T, typename TG>
hipError_t launch_norm_grad_mode(RowArgs& a, float* dgamma, float* dbeta, float* ws, hipStream_t st) {
  const RowPlan p = row_plan(a.d);
  a.lanes = p.lanes;
  const long blocks = row_blocks(p, a.T, MODE == kLayer);     // (0 of no rows, whose sums are 0)
  const bool whole = row_whole(p, a.d), sums = dgamma && blocks != 1;
  a.dgamma = sums ? ws : dgamma;
  a.dbeta = sums ? ws + a.d : dbeta;
  a.part = sums ? 2l * a.d : 0;
  auto of = [&](auto e) {
    constexpr int E = decltype(e)::value;
    if (p.team == 256)
      run_norm_grad<MODE, T, TG, 256, E>(a, blocks, whole, st);
    else if (p.team)
      run_norm_grad<MODE, T, TG, 1024, E>(a, blocks, whole, st);
    else
      run_norm_grad<MODE, T, TG, 0, E>(a, blocks, whole, st);
  };
  if (blocks) p.E == 8 ? of(std::integral_constant<int, 8>{}) : of(std::integral_constant<int, 16>{});
  if (!sums) return hipGetLastError();
  hipLaunchKernelGGL(k_norm_sums, dim3((2 * a.d + 15) / 16), dim3(1024), 0, st, ws, static_cast<int>(blocks), a.d, dgamma, dbeta);
  return hipGetLastError();
}

}  // namespace

size_t norm_grad_bytes(long T, int d) {
  const long blocks = row_blocks(row_plan(d), T, true);
  return blocks > 1 ? static_cast<size_t>(blocks) * 2 * d * sizeof(float) : 0;
}
// of every call of no more rows and elements (the widest rows have fewer workgroups)
size_t norm_grad_most(long T, int d) { return std::max(norm_grad_bytes(T, d), norm_grad_bytes(T, std::min(d, 4096))); }

hipError_t launch_norm(int length, const void* x, int x_dtype, long T, int d, const float* gamma, const float* beta, float eps,
                       void* y, int y_dtype, hipStream_t st) {
  RowArgs a{};
  a.T = T;
  a.d = d;
  a.eps = eps;
  a.x = x;
  a.gamma = gamma;
  a.beta = beta;
  a.y = y;
  a.y_bf16 = y_dtype == MOL_BF16;
  if (length)
    return x_dtype == MOL_BF16 ? launch_norm_mode<kLength, bf16_t>(a, st) : launch_norm_mode<kLength, float>(a, st);
  return x_dtype == MOL_BF16 ? launch_norm_mode<kLayer, bf16_t>(a, st) : launch_norm_mode<kLayer, float>(a, st);
}

hipError_t launch_norm_grad(int length, const void* dy, int dy_dtype, const void* x, int x_dtype, long T, int d,
                            const float* gamma, float eps, void* dx, int dx_dtype, float* dgamma, float* dbeta, void* ws,
                            hipStream_t st) {
  RowArgs a{};
  a.T = T;
  a.d = d;
  a.eps = eps;
  a.x = x;
  a.dy = dy;
  a.gamma = gamma;
  a.y = dx;
  a.y_bf16 = dx_dtype == MOL_BF16;
  a.once = vec::streams(static_cast<size_t>(T) * d * ((x_dtype == MOL_BF16 ? 2 : 4) + (dy_dtype == MOL_BF16 ? 2 : 4)));
  float* w = static_cast<float*>(ws);
  auto types = [&](auto t, auto tg) {
    using T_ = decltype(t);
    using G_ = decltype(tg);
    return length ? launch_norm_grad_mode<kLength, T_, G_>(a, nullptr, nullptr, w, st)
                  : launch_norm_grad_mode<kLayer, T_, G_>(a, dgamma, dbeta, w, st);
  };
  if (x_dtype == MOL_BF16) return dy_dtype == MOL_BF16 ? types(bf16_t{}, bf16_t{}) : types(bf16_t{}, 0.f);
  return dy_dtype == MOL_BF16 ? types(0.f, bf16_t{}) : types(0.f, 0.f);
}

}  // namespace mol
