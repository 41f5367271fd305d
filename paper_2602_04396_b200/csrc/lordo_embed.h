// Internal interface of the token-sorted sums (lordo_embed.cu): used by the embedding's entry points and by the AdamW step of a table
// whose gradient is given by its tokens (lordo_adamw.cu).
#pragma once
#include "lordo_common.cuh"

namespace lordo {

// Scratch of one table: K workers with up to `cap` tokens each.
struct TokScratch {
  int2* buf[2];     // [K][cap] (token, position), by turns
  int2* segs;       // [K][V] first and last + 1 sorted entry of every token, 0 0 without one
  int* valid;       // [K] tokens inside [0, V)
  float* parts;     // [K][windows][2][d] sums of tokens whose entries lie in more than one window
  long long bytes;
};

// With base null only measures. Good for every T <= cap.
TokScratch tok_scratch(char* base, int K, long long V, long long d, long long cap);

struct TokProblem {
  const void* tokens;  // [K][T]
  int is64;
  int K;
  long long V, T, d;
  const void* dY;      // [K][T][d]
  int y_dt;
  float scale;
};

// Sorts every worker's tokens, ties by position, then dW[k][v] (in w_dt) = the sums, or += for the tokens that occur. Returns the launches.
int tok_dense(const TokProblem& p, const TokScratch& s, void* dW, int w_dt, int accumulate, cudaStream_t st);
// The same into rows[k][i] (fp32, [K][cap][d]) = the sum of the token whose first sorted entry is i; sq[k][0 .. *count) = sums of their
// squares, *count at most tok_row_blocks_max.
struct TokRows {
  float* rows;
  double* sq;
  int* count;
  long long cap;
};
long long tok_row_blocks_max(long long cap, long long d);
int tok_rows(const TokProblem& p, const TokScratch& s, const TokRows& r, cudaStream_t st);

// Argument checks: lordo_status. Limits are what the kernels' grids and 32-bit positions take.
int check_tokens(int K, int64_t V, int64_t d, int64_t T, int index);
inline bool misaligned(const void* p, int dt) { return (reinterpret_cast<uintptr_t>(p) & (dt == LORDO_F32 ? 3u : 1u)) != 0; }
inline bool misaligned_tokens(const void* p, int index) { return (reinterpret_cast<uintptr_t>(p) & (index == LORDO_I64 ? 7u : 3u)) != 0; }

}  // namespace lordo
