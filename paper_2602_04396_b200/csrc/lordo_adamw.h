// Internal interface between the host layer of the AdamW groups (lordo_adamw_api.cu) and their kernels (lordo_adamw.cu).
#pragma once
#include <algorithm>

#include "lordo_common.cuh"
#include "lordo_plan.h"

namespace lordo {

constexpr int kAwBlock = 256;    // elements per scale of the 8-bit moments
// Elements of one worker's tensor that a CTA of the step works on: 2048 (eight a thread) to 32768, about one for each of eight CTAs an SM where there are fewer.
inline long long aw_piece(long long elements) {
  const long long p = (elements / (kPlannedSms * 8) + 2047) / 2048 * 2048;
  return p < 2048 ? 2048 : p > 32768 ? 32768 : p;
}
constexpr int kAwOuter = 2048;   // elements of one worker's tensor that a CTA of the synchronisation works on, for all workers
constexpr int kAwTable = 512;    // tensors of one launch

// One tensor, built once and kept in the workspace. Arrays are [K][n]; X0, B are [n].
struct AwTensor {
  long long n, nb;         // elements of a worker, blocks of 256 among them
  void* W;
  void *m, *v;             // fp32, or E4M3 codes of m and sqrt(v)
  unsigned char *ms, *vs;  // [K][nb] exponents of the scales, biased by 127 (8 bits)
  float *X0, *B;
  float wd;
  int index;               // among the group's tensors
  // gradient by tokens, see lordo_embed.h
  long long d, cap;        // columns of a row (n is a multiple), most tokens of a worker
  const int2* segs;        // [K][n / d]
  const float* rows;       // [K][cap][d] sums, at the first sorted entry of their token
  const double* rowsq;     // [K][rowsq_count] sums of their squares
  const int* rowsq_count;
  // divides by d / 8 (lordo_plan.h); row_mul = 0 where d is no multiple of 8 or n too large
  unsigned row_mul;
  int row_shift;
};

// Gradients and the dealing of a launch, handed over as kernel arguments: no copy to the device, and nothing that a later call could overwrite.
struct AwTable {
  const void* G[kAwTable];       // [K][n], or null: the gradient lies in AwTensor.rows
  unsigned start[kAwTable + 1];  // first unit of work (piece, chunk) of every tensor among those of one worker
};

struct AwStep {
  float lr, b1, a1, b2, a2;  // a = 1 - b
  float omega, a_omega, eps;
  float inv_bc1, inv_bc2, root_inv_bc2;
  float one;                 // 1, as a number that the compiler does not know
  unsigned long long key;    // of the rounding, for this step
};

// Tensors [first, first + count) of a group are one launch.
struct AwLaunch {
  const AwTensor* tensors;  // of the launch
  int count, K;
  unsigned units;           // per worker
  int w_dt, g_dt, small;    // small: 8-bit moments
  int piece;                // elements behind a unit
};

struct AwClip {
  double* partial;     // [K][total]
  int chunk;           // elements of one worker's tensor behind a partial sum
  unsigned total, at;  // chunks of a worker in all launches, and before this one
  unsigned* tickets;   // scope 0: [K]; scope 1: [n_tensors][K]; zero before the first launch, and again after every step
  double rho;
  int scope, n_tensors;
  float* coef;         // [n_tensors][K]
  unsigned* status;
};
void launch_aw_norm(const AwLaunch& l, const AwTable& t, const AwClip& c, cudaStream_t st);
// coef: [tensor][K] with `stride` = K, one row for all with 0, or null (1)
void launch_aw_step(const AwLaunch& l, const AwTable& t, const float* coef, int stride, const AwStep& s, cudaStream_t st);

struct AwOuter {
  int sync_m, sync_v, nesterov;
  float eta, mu;
  unsigned long long key;
};
// start: [count + 1] first block of every tensor, in device memory
void launch_aw_outer(const AwLaunch& l, const unsigned* start, const AwOuter& o, cudaStream_t st);
// Worker 0's weights to the others and to X0; zero moments and outer momentum.
void launch_aw_init(const AwLaunch& l, const unsigned* start, cudaStream_t st);

}  // namespace lordo
