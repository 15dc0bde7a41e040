// Pieces shared by the two forms of the score gradient.
#pragma once

#include "mol_tile.h"

namespace mol {
namespace grad {

// Sums of partial results: out[o] = sum over s < S of in[s * stride + o], o < L,
// as float32 (added to what an earlier slab left in acc) and, where wanted, in the
// output's type.  o of batch o / in_len goes to element out_at + o % in_len of
// that batch of out_len in the output.
struct SumJob {
  const float* in;
  long L, stride;
  int S;
  float* acc;              // NULL, or float32 sums kept between slabs
  int add;
  void* out;               // NULL, or the output
  int bf16;
  long in_len, out_len, out_at;
  int wide;                // (set by the launcher) 256 columns a block
};
constexpr int kSumJobs = 8;   // one an output
struct SumArgs {
  int n;
  long first[kSumJobs + 1];    // first block of each job
  SumJob job[kSumJobs];
};
struct SumList {
  SumArgs a{};
  hipStream_t st;
  explicit SumList(hipStream_t s) : st(s) {}
  void add(const SumJob& j);
  hipError_t run();
};

// Q [m][d] -> qt [d][ldq] (rows from m to ldq zero) where qt is not NULL, and items
// [n0, n0 + items) of X [Px][N][d] -> xt [Px][d][ns] (zero from items to ns)
// where xt is not NULL, one launch.
template <typename T>
hipError_t launch_transposes(const DevProb& pr, long m, int ldq, T* qt, int n0, int items, int ns, T* xt,
                             hipStream_t st);

// The bf16 form on 16-bit matrix instructions (mol_score_grad_bf16.hip).
bool bf16_supported(const DevProb& pr);
size_t bf16_bytes(const DevProb& pr);
hipError_t launch_bf16(const DevProb& pr, const float* dphi, const mol_score_grads& o, char* ws, hipStream_t st);

// dQ and dX from ds in one launch or in two.  Together they fill the card where
// there is little of it (34 MB of ds: 18 us against 12 + 12); apart the second finds
// part of what the first read in the last-level cache (268 MB: 77 + 60 us against 259).
constexpr int kProductQ = 1, kProductX = 2;
inline bool products_together(size_t ds_bytes) { return ds_bytes <= (size_t(64) << 20); }

// Elements of a row of X or Q transposed: whole K blocks of 32, and 64 more, so that
// the rows that a load takes together (powers of two apart otherwise) are not
// all in the same channels of the L2 cache.
inline int padded_row(long n) { return static_cast<int>((n + 31) / 32 * 32 + 64); }

// K splits of a product of `waves` waves a part with `chunks` K chunks, `least` of them a part
inline int split_of(long waves, long chunks, long least) {
  const long want = (2048 + waves - 1) / waves, most = chunks / least;
  const long n = want < most ? want : most;
  return static_cast<int>(n < 1 ? 1 : n > 64 ? 64 : n);
}

}  // namespace grad
}  // namespace mol
