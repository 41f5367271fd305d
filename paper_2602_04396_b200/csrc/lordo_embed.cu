// Embedding lookup, and the table's gradient by sorted tokens:
//   out[k][t] = scale * W[k][tok[k][t]]           dW[k][v] = scale * sum over t with tok[k][t] = v of dY[k][t]
// for K workers, each with a table and tokens of its own. Sums are fp32, in the order of the positions, the same on every run.
#include "lordo_embed.h"
#include "lordo_kernels.h"

namespace lordo {
namespace {

constexpr int kSortThreads = 1024, kSortWarps = 32, kMaxDigit = 256;

struct SortArgs {
  const void* tokens;
  int is64, K, bits, passes;
  long long T, cap, V;
  int2 *buf0, *buf1, *segs;
  int* valid;
  int per_warp;  // consecutive positions of a warp, a multiple of 32
};

__device__ __forceinline__ void cluster_sync_all() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ int cluster_load(const int* mine, unsigned rank) {  // the same shared variable of another CTA of the cluster
  unsigned a = (unsigned)__cvta_generic_to_shared(mine), b;
  int v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(b) : "r"(a), "r"(rank));
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(b) : "memory");
  return v;
}

// Radix sort of one worker's (token, position) pairs by a cluster of CTAs, `bits` bits of the token a pass. Every warp owns consecutive
// positions, so the order of equal digits is that of (CTA, warp, batch, lane): stable. Tokens outside [0, V) sort as V, behind all others.
__global__ void __launch_bounds__(kSortThreads) sort_tokens_kernel(SortArgs a) {
  __shared__ int cnt[kSortWarps][kMaxDigit];
  __shared__ int tot[kMaxDigit], base[kMaxDigit], wsum[8];
  const int t = threadIdx.x, lane = t & 31, w = t >> 5;
  unsigned c, C;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(c));
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(C));
  const int k = blockIdx.x / C;
  dep_begin();
  if (a.T == 0 && c == 0 && t == 0) a.valid[k] = 0;
  int2* segs = a.segs + (long long)k * a.V;
  for (long long v = c * kSortThreads + t; v < a.V; v += (long long)C * kSortThreads) segs[v] = make_int2(0, 0);
  const long long begin = ((long long)c * kSortWarps + w) * a.per_warp;
  const long long end = begin + a.per_warp < a.T ? begin + a.per_warp : a.T;
  const int R = 1 << a.bits;
  const int2* src = nullptr;
  int2* dst = a.buf0 + (long long)k * a.cap;
  int2* other = a.buf1 + (long long)k * a.cap;
  auto fetch = [&](long long i) {
    if (src) return __ldcg(src + i);
    const long long at = (long long)k * a.T + i;
    const long long v = a.is64 ? reinterpret_cast<const long long*>(a.tokens)[at] : (long long)reinterpret_cast<const int*>(a.tokens)[at];
    return make_int2(v >= 0 && v < a.V ? (int)v : (int)a.V, (int)i);
  };
  for (int p = 0; p < a.passes; ++p) {
    const int shift = p * a.bits;
    for (int i = t; i < kSortWarps * R; i += kSortThreads) cnt[i / R][i % R] = 0;
    __syncthreads();
    for (long long b = begin; b < end; b += 32) {
      const bool in = b + lane < end;
      const int digit = in ? (fetch(b + lane).x >> shift) & (R - 1) : -1;
      const unsigned same = __match_any_sync(0xffffffffu, digit);
      if (in && lane == __ffs(same) - 1) cnt[w][digit] += __popc(same);
      __syncwarp();
    }
    __syncthreads();
    if (t < R) {  // counts of a digit become the places of its warps
      int run = 0;
#pragma unroll 8
      for (int x = 0; x < kSortWarps; ++x) {
        const int n = cnt[x][t];
        cnt[x][t] = run;
        run += n;
      }
      tot[t] = run;
    }
    cluster_sync_all();
    int all = 0, before = 0;
    if (t < R) {
      for (unsigned r = 0; r < C; ++r) {
        const int n = cluster_load(tot + t, r);
        all += n;
        if (r < c) before += n;
      }
    }
    int scan = all;
    if (t < kMaxDigit) {
      for (int o = 1; o < 32; o <<= 1) {
        const int up = __shfl_up_sync(0xffffffffu, scan, o);
        if (lane >= o) scan += up;
      }
      if (lane == 31) wsum[w] = scan;
    }
    __syncthreads();
    if (t < R) {
      int first = scan - all + before;
      for (int x = 0; x < w; ++x) first += wsum[x];
      base[t] = first;
    }
    __syncthreads();
    for (long long b = begin; b < end; b += 32) {
      const bool in = b + lane < end;
      const int2 e = in ? fetch(b + lane) : make_int2(0, 0);
      const int digit = in ? (e.x >> shift) & (R - 1) : -1;
      const unsigned same = __match_any_sync(0xffffffffu, digit);
      int at = 0;
      if (in) at = base[digit] + cnt[w][digit] + __popc(same & ((1u << lane) - 1u));
      __syncwarp();
      if (in && lane == __ffs(same) - 1) cnt[w][digit] += __popc(same);
      __syncwarp();
      if (in) dst[at] = e;
    }
    cluster_sync_all();  // the order of this pass is complete, and every CTA has read the totals
    src = dst;
    dst = other;
    other = const_cast<int2*>(src);
  }
  for (long long i = (long long)c * kSortThreads + t; i < a.T; i += (long long)C * kSortThreads) {
    const int v = __ldcg(src + i).x;
    const int prev = i > 0 ? __ldcg(src + i - 1).x : -1;
    const int next = i + 1 < a.T ? __ldcg(src + i + 1).x : -1;
    if (v < a.V) {
      if (prev != v) segs[v].x = (int)i;
      if (next != v) segs[v].y = (int)i + 1;
      if (next < 0 || next >= a.V) a.valid[k] = (int)i + 1;
    } else if (i == 0) {
      a.valid[k] = 0;
    }
  }
}

// ---------------------------------------------------------------------------------------------
// Sums. A warp works on 32 * VEC columns of one token's rows.
// ---------------------------------------------------------------------------------------------
template <int DT, int VEC>
__device__ __forceinline__ void add_row(const void* base, long long at, float (&acc)[VEC]) {
  if constexpr (VEC == 1) {
    acc[0] += load1(base, DT, at);
  } else if constexpr (DT == LORDO_F32) {
    const float4 x = __ldcs(reinterpret_cast<const float4*>(reinterpret_cast<const float*>(base) + at));
    acc[0] += x.x; acc[1] += x.y; acc[2] += x.z; acc[3] += x.w;
  } else {
    const uint4 x = __ldcs(reinterpret_cast<const uint4*>(reinterpret_cast<const unsigned short*>(base) + at));
    const unsigned r[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      acc[2 * j] += __uint_as_float(r[j] << 16);
      acc[2 * j + 1] += __uint_as_float(r[j] & 0xFFFF0000u);
    }
  }
}

struct SumArgs {
  const void* dY;
  const int2* order;   // [K][cap]
  const int2* segs;    // [K][V]
  const int* valid;
  float* chunks;       // [K][cap / 32][d]
  long long V, T, cap, d;
  int groups;          // column groups of a row
  float scale;
  void* out;
  double* sq;          // [K][gridDim.x]
  int* count;          // gridDim.x
  long long out_cap;   // rows of a worker in `out` (sums in rows of their own)
};

// Sum of sorted entries [s, e) of worker k, columns from `col` on. Every lane is here; `on`: it has columns.
template <int DT, int VEC>
__device__ __forceinline__ void sum_entries(const SumArgs& a, int k, int s, int e, long long col, bool on, int lane, float (&acc)[VEC]) {
  const int2* order = a.order + (long long)k * a.cap;
  const long long first = (long long)k * a.T * a.d + col;
  for (int b = s; b < e; b += 32) {
    const int mine = b + lane < e ? __ldcg(order + b + lane).y : 0;
    const int n = e - b < 32 ? e - b : 32;
    int j = 0;
    for (; j + 4 <= n; j += 4) {
      long long at[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) at[x] = first + (long long)__shfl_sync(0xffffffffu, mine, j + x) * a.d;
      if (on) {
#pragma unroll
        for (int x = 0; x < 4; ++x) add_row<DT, VEC>(a.dY, at[x], acc);
      }
    }
    for (; j < n; ++j) {
      const long long at = first + (long long)__shfl_sync(0xffffffffu, mine, j) * a.d;
      if (on) add_row<DT, VEC>(a.dY, at, acc);
    }
  }
}

// Sum of one token's entries: the ends one by one, the whole chunks between them from tok_chunks.
template <int DT, int VEC>
__device__ __forceinline__ void sum_segment(const SumArgs& a, int k, int s, int e, long long col, bool on, int lane, float (&acc)[VEC]) {
  const int c0 = (s + kTokChunk - 1) / kTokChunk, c1 = e / kTokChunk;
  if (c1 <= c0) {
    sum_entries<DT, VEC>(a, k, s, e, col, on, lane, acc);
    return;
  }
  sum_entries<DT, VEC>(a, k, s, c0 * kTokChunk, col, on, lane, acc);
  if (on) {
    const float* p = a.chunks + ((long long)k * (a.cap / kTokChunk) + c0) * a.d + col;
    for (int c = c0; c < c1; ++c, p += a.d)
#pragma unroll
      for (int j = 0; j < VEC; ++j) acc[j] += __ldcg(p + j);
  }
  sum_entries<DT, VEC>(a, k, c1 * kTokChunk, e, col, on, lane, acc);
}

template <int DT, int VEC>
__global__ void __launch_bounds__(256) chunk_sums_kernel(SumArgs a) {
  const int lane = threadIdx.x & 31, k = blockIdx.y;
  dep_begin();
  const long long item = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  const long long c = item / a.groups;
  const int s = (int)(c * kTokChunk);
  if (s + kTokChunk > a.valid[k]) return;
  const int2* order = a.order + (long long)k * a.cap;
  if (__ldcg(order + s).x != __ldcg(order + s + kTokChunk - 1).x) return;
  const long long col = ((item - c * a.groups) * 32 + lane) * VEC;
  const bool on = col < a.d;
  float acc[VEC] = {};
  sum_entries<DT, VEC>(a, k, s, s + kTokChunk, col, on, lane, acc);
  if (on) {
    float* p = a.chunks + ((long long)k * (a.cap / kTokChunk) + c) * a.d + col;
#pragma unroll
    for (int j = 0; j < VEC; ++j) p[j] = acc[j];
  }
}

template <int VEC>
__device__ __forceinline__ void put(void* base, int dt, long long at, const float (&x)[VEC]) {
  if constexpr (VEC == 1) {
    store1(base, dt, at, x[0]);
  } else {
#pragma unroll
    for (int j = 0; j < VEC; j += 4) store4(base, dt, at + j, make_float4(x[j], x[j + 1], x[j + 2], x[j + 3]));
  }
}

constexpr int kSumItems = 4;  // items a warp works on one after another
enum SumMode { SUM_DENSE = 0, SUM_ADD = 1, SUM_ROWS = 2 };

// DENSE: an item is a row of the table (rows without a token become zero). ADD, ROWS: an item is a sorted entry, and works where a
// token's entries begin.
template <int DT, int VEC, int MODE>
__global__ void __launch_bounds__(256) token_sums_kernel(SumArgs a, int out_dt) {
  __shared__ double red[8];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, k = blockIdx.y;
  dep_begin();
  const long long rows = MODE == SUM_DENSE ? a.V : a.valid[k];
  const long long items = rows * a.groups;
  float sq = 0.f;
  for (int x = 0; x < kSumItems; ++x) {
    const long long item = ((long long)blockIdx.x * kSumItems + x) * 8 + warp;
    if (item >= items) break;
    const long long row = item / a.groups;
    const long long col = ((item - row * a.groups) * 32 + lane) * VEC;
    const bool on = col < a.d;
    float acc[VEC] = {};
    int2 seg;
    long long v = row;
    if (MODE == SUM_DENSE) {
      seg = __ldcg(a.segs + (long long)k * a.V + row);
    } else {
      const int2* order = a.order + (long long)k * a.cap;
      v = __ldcg(order + row).x;
      if (row > 0 && __ldcg(order + row - 1).x == v) continue;
      seg = __ldcg(a.segs + (long long)k * a.V + v);
    }
    sum_segment<DT, VEC>(a, k, seg.x, seg.y, col, on, lane, acc);
    if (!on) continue;
#pragma unroll
    for (int j = 0; j < VEC; ++j) acc[j] *= a.scale;
    if (MODE == SUM_ROWS) {
      put<VEC>(a.out, LORDO_F32, ((long long)k * a.out_cap + row) * a.d + col, acc);
#pragma unroll
      for (int j = 0; j < VEC; ++j) sq += acc[j] * acc[j];
    } else {
      const long long at = ((long long)k * a.V + v) * a.d + col;
      if (MODE == SUM_ADD) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) acc[j] += load1(a.out, out_dt, at + j);
      }
      put<VEC>(a.out, out_dt, at, acc);
    }
  }
  if (MODE == SUM_ROWS) {
    double s = (double)sq;
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (lane == 0) red[warp] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
      s = 0.0;
      for (int x = 0; x < 8; ++x) s += red[x];
      a.sq[(long long)k * gridDim.x + blockIdx.x] = s;
      if (k == 0 && blockIdx.x == 0) *a.count = (int)gridDim.x;
    }
  }
}

// ---------------------------------------------------------------------------------------------
// Lookup
// ---------------------------------------------------------------------------------------------
template <int DT, int VEC>
__global__ void __launch_bounds__(256) lookup_kernel(const void* __restrict__ W, const void* __restrict__ tokens, int is64, long long V, long long d,
                                                     long long T, long long pieces, float scale, void* __restrict__ out, int out_dt) {
  dep_begin();
  const long long per_row = (d + VEC - 1) / VEC;
  const long long p = (long long)blockIdx.x * 256 + threadIdx.x;
  if (p >= pieces) return;
  const long long row = p / per_row, col = (p - row * per_row) * VEC;
  const long long v = is64 ? reinterpret_cast<const long long*>(tokens)[row] : (long long)reinterpret_cast<const int*>(tokens)[row];
  const long long k = row / T;
  float x[VEC] = {};
  if (v >= 0 && v < V) {
    add_row<DT, VEC>(W, (k * V + v) * d + col, x);
#pragma unroll
    for (int j = 0; j < VEC; ++j) x[j] *= scale;
  }
  put<VEC>(out, out_dt, row * d + col, x);
}

int token_bits(long long V) {  // of the largest key, V
  int b = 1;
  while ((V >> b) != 0) ++b;
  return b;
}

bool wide(const void* p, long long d, int dt) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && d % (dt == LORDO_F32 ? 4 : 8) == 0; }

SumArgs sum_args(const TokProblem& p, const TokScratch& s, int which, int vec) {
  SumArgs a = {};
  a.dY = p.dY; a.order = s.buf[which]; a.segs = s.segs; a.valid = s.valid; a.chunks = s.chunks;
  a.V = p.V; a.T = p.T; a.d = p.d; a.scale = p.scale;
  a.cap = p.T;
  a.groups = (int)((p.d + 32 * vec - 1) / (32 * vec));
  return a;
}

template <int MODE>
void run_sums(SumArgs a, const TokProblem& p, int out_dt, unsigned blocks, int vec, cudaStream_t st) {
  const dim3 grid(blocks, p.K);
  if (p.y_dt == LORDO_F32) {
    if (vec == 4) launch_dep(token_sums_kernel<LORDO_F32, 4, MODE>, grid, 256, 0, st, a, out_dt);
    else launch_dep(token_sums_kernel<LORDO_F32, 1, MODE>, grid, 256, 0, st, a, out_dt);
  } else {
    if (vec == 8) launch_dep(token_sums_kernel<LORDO_BF16, 8, MODE>, grid, 256, 0, st, a, out_dt);
    else launch_dep(token_sums_kernel<LORDO_BF16, 1, MODE>, grid, 256, 0, st, a, out_dt);
  }
}

// Columns of a lane: 16 bytes of dY where rows and arrays allow it.
int sum_vec(const TokProblem& p, const void* out, int out_dt) {
  const int vec = p.y_dt == LORDO_F32 ? 4 : 8;
  return p.d % vec == 0 && wide(p.dY, p.d, p.y_dt) && (reinterpret_cast<uintptr_t>(out) & 15u) == 0 ? vec : 1;
}

unsigned sum_blocks(long long rows, long long d, int vec) {
  const long long items = rows * ((d + 32 * vec - 1) / (32 * vec));
  return items > 0 ? (unsigned)((items + 8 * kSumItems - 1) / (8 * kSumItems)) : 1u;
}

}  // namespace

TokScratch tok_scratch(char* base, int K, long long V, long long d, long long cap) {
  TokScratch s = {};
  long long off = 0;
  auto take = [&](long long bytes) {
    char* p = base + off;
    off += (bytes + 255) / 256 * 256;
    return p;
  };
  s.buf[0] = reinterpret_cast<int2*>(take(8ll * K * cap));
  s.buf[1] = reinterpret_cast<int2*>(take(8ll * K * cap));
  s.segs = reinterpret_cast<int2*>(take(8ll * K * V));
  s.valid = reinterpret_cast<int*>(take(4ll * K));
  s.chunks = reinterpret_cast<float*>(take(4ll * K * (cap / kTokChunk) * d));
  s.bytes = off;
  return s;
}

int tok_sort(const TokProblem& p, const TokScratch& s, cudaStream_t st) {
  const int bits = token_bits(p.V);
  SortArgs a = {};
  a.tokens = p.tokens; a.is64 = p.is64; a.K = p.K; a.T = p.T; a.cap = p.T; a.V = p.V;
  a.passes = (bits + 7) / 8;
  a.bits = (bits + a.passes - 1) / a.passes;
  a.buf0 = s.buf[0]; a.buf1 = s.buf[1]; a.segs = s.segs; a.valid = s.valid;
  int C = 1;
  while (C < 8 && p.T > 2048ll * C) C *= 2;
  const long long warps = (long long)C * kSortWarps;
  a.per_warp = (int)(((p.T + warps - 1) / warps + 31) / 32 * 32);
  cudaLaunchConfig_t lc = {};
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = C; at[1].val.clusterDim.y = 1; at[1].val.clusterDim.z = 1;
  lc.gridDim = dim3(C * p.K); lc.blockDim = dim3(kSortThreads); lc.stream = st;
  lc.attrs = at; lc.numAttrs = 2;
  cudaLaunchKernelEx(&lc, sort_tokens_kernel, a);
  return (a.passes - 1) & 1;
}

void tok_chunks(const TokProblem& p, const TokScratch& s, int which, cudaStream_t st) {
  if (p.T < kTokChunk) return;
  const int vec = sum_vec(p, s.chunks, LORDO_F32);
  const SumArgs a = sum_args(p, s, which, vec);
  const dim3 grid((unsigned)((p.T / kTokChunk * a.groups + 7) / 8), p.K);
  if (p.y_dt == LORDO_F32) {
    if (vec == 4) launch_dep(chunk_sums_kernel<LORDO_F32, 4>, grid, 256, 0, st, a);
    else launch_dep(chunk_sums_kernel<LORDO_F32, 1>, grid, 256, 0, st, a);
  } else {
    if (vec == 8) launch_dep(chunk_sums_kernel<LORDO_BF16, 8>, grid, 256, 0, st, a);
    else launch_dep(chunk_sums_kernel<LORDO_BF16, 1>, grid, 256, 0, st, a);
  }
}

void tok_dense(const TokProblem& p, const TokScratch& s, int which, void* dW, int w_dt, int accumulate, cudaStream_t st) {
  const int vec = sum_vec(p, dW, w_dt);
  SumArgs a = sum_args(p, s, which, vec);
  a.out = dW;
  if (accumulate) run_sums<SUM_ADD>(a, p, w_dt, sum_blocks(p.T, p.d, vec), vec, st);
  else run_sums<SUM_DENSE>(a, p, w_dt, sum_blocks(p.V, p.d, vec), vec, st);
}

long long tok_row_blocks_max(long long cap, long long d) { return sum_blocks(cap, d, 1); }

void tok_rows(const TokProblem& p, const TokScratch& s, int which, const TokRows& r, cudaStream_t st) {
  const int vec = sum_vec(p, r.rows, LORDO_F32);
  SumArgs a = sum_args(p, s, which, vec);
  a.out = r.rows; a.sq = r.sq; a.count = r.count; a.out_cap = r.cap;
  run_sums<SUM_ROWS>(a, p, LORDO_F32, sum_blocks(p.T, p.d, vec), vec, st);
}

}  // namespace lordo

// =============================================================================================
// C ABI
// =============================================================================================
using namespace lordo;

namespace lordo {

int check_tokens(int K, int64_t V, int64_t d, int64_t T, int index) {
  if (K < 1 || K > 64 || V < 1 || d < 1 || T < 0) return LORDO_ERR_INVALID_ARG;
  if (index != LORDO_I32 && index != LORDO_I64) return LORDO_ERR_INVALID_ARG;
  if (V > (1ll << 30) || d > (1ll << 24) || T > (1ll << 30)) return LORDO_ERR_UNSUPPORTED;
  if (((V > T ? V : T) * ((d + 31) / 32)) > (1ll << 34)) return LORDO_ERR_UNSUPPORTED;
  return LORDO_OK;
}

}  // namespace lordo

namespace {
bool known(int dt) { return dt == LORDO_F32 || dt == LORDO_BF16; }
}  // namespace

extern "C" {

int lordo_embedding(const void* W, int w_dtype, int K, int64_t V, int64_t d, const void* tokens, int index, int64_t T, float scale, void* out,
                    int out_dtype, void* stream) {
  int rc = check_tokens(K, V, d, T, index);
  if (rc != LORDO_OK) return rc;
  if (!known(w_dtype) || !known(out_dtype)) return LORDO_ERR_INVALID_ARG;
  if (T == 0) return LORDO_OK;
  if (!W || !tokens || !out) return LORDO_ERR_INVALID_ARG;
  if (misaligned(W, w_dtype) || misaligned(out, out_dtype) || misaligned_tokens(tokens, index)) return LORDO_ERR_ALIGN;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  if (cudaPeekAtLastError() != cudaSuccess) return LORDO_ERR_CUDA;
  const int full = w_dtype == LORDO_F32 ? 4 : 8;
  const int vec = wide(W, d, w_dtype) && (reinterpret_cast<uintptr_t>(out) & 15u) == 0 ? full : 1;
  const long long pieces = (long long)K * T * ((d + vec - 1) / vec);
  if ((pieces + 255) / 256 > 0x7fffffffll) return LORDO_ERR_UNSUPPORTED;
  const dim3 grid((unsigned)((pieces + 255) / 256));
  const int is64 = index == LORDO_I64;
#define LORDO_LOOKUP(DT, VEC)                                                                                                                \
  launch_dep(lookup_kernel<DT, VEC>, grid, 256, 0, st, W, tokens, is64, (long long)V, (long long)d, (long long)T, pieces, scale, out, out_dtype)
  if (w_dtype == LORDO_F32) { if (vec > 1) LORDO_LOOKUP(LORDO_F32, 4); else LORDO_LOOKUP(LORDO_F32, 1); }
  else { if (vec > 1) LORDO_LOOKUP(LORDO_BF16, 8); else LORDO_LOOKUP(LORDO_BF16, 1); }
#undef LORDO_LOOKUP
  return cudaPeekAtLastError() == cudaSuccess ? LORDO_OK : LORDO_ERR_CUDA;
}

int lordo_embedding_grad_query_workspace(int K, int64_t V, int64_t d, int64_t T, size_t* bytes) {
  const int rc = check_tokens(K, V, d, T, LORDO_I32);
  if (rc != LORDO_OK) return rc;
  if (!bytes) return LORDO_ERR_INVALID_ARG;
  *bytes = (size_t)tok_scratch(nullptr, K, V, d, T).bytes;
  return LORDO_OK;
}

int lordo_embedding_grad(const void* dY, int y_dtype, const void* tokens, int index, int K, int64_t V, int64_t d, int64_t T, float scale, void* dW,
                         int w_dtype, int accumulate, void* workspace, size_t workspace_bytes, void* stream) {
  int rc = check_tokens(K, V, d, T, index);
  if (rc != LORDO_OK) return rc;
  if (!known(y_dtype) || !known(w_dtype) || !dW || (accumulate != 0 && accumulate != 1)) return LORDO_ERR_INVALID_ARG;
  if (misaligned(dW, w_dtype)) return LORDO_ERR_ALIGN;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  if (T == 0) {
    if (accumulate) return LORDO_OK;
    return cudaMemsetAsync(dW, 0, (size_t)K * V * d * (w_dtype == LORDO_F32 ? 4 : 2), st) == cudaSuccess ? LORDO_OK : LORDO_ERR_CUDA;
  }
  if (!dY || !tokens || !workspace) return LORDO_ERR_INVALID_ARG;
  if (misaligned(dY, y_dtype) || misaligned_tokens(tokens, index)) return LORDO_ERR_ALIGN;
  if ((reinterpret_cast<uintptr_t>(workspace) & 255u) != 0) return LORDO_ERR_ALIGN;
  const TokScratch s = tok_scratch(reinterpret_cast<char*>(workspace), K, V, d, T);
  if ((size_t)s.bytes > workspace_bytes) return LORDO_ERR_NOMEM;
  if (cudaPeekAtLastError() != cudaSuccess) return LORDO_ERR_CUDA;
  TokProblem p = {tokens, index == LORDO_I64, K, V, T, d, dY, y_dtype, scale};
  const int which = tok_sort(p, s, st);
  tok_chunks(p, s, which, st);
  tok_dense(p, s, which, dW, w_dtype, accumulate, st);
  return cudaPeekAtLastError() == cudaSuccess ? LORDO_OK : LORDO_ERR_CUDA;
}

}  // extern "C"
