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
template <int DT, int VEC>  // VEC consecutive elements as they are stored: 16 bytes, or one
struct Piece {
  uint4 r;
  __device__ __forceinline__ void load(const void* base, long long at) {
    if constexpr (VEC == 1) r.x = __float_as_uint(load1(base, DT, at));
    else r = __ldcs(reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(base) + at * (DT == LORDO_F32 ? 4 : 2)));
  }
  __device__ __forceinline__ void add_to(float (&acc)[VEC]) const {
    const unsigned w[4] = {r.x, r.y, r.z, r.w};
    if constexpr (VEC == 1 || DT == LORDO_F32) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) acc[j] += __uint_as_float(w[j & 3]);
    } else {
#pragma unroll
      for (int j = 0; j < VEC / 2; ++j) {
        acc[2 * j] += __uint_as_float(w[j & 3] << 16);
        acc[2 * j + 1] += __uint_as_float(w[j & 3] & 0xFFFF0000u);
      }
    }
  }
};

template <int VEC>
__device__ __forceinline__ void put(void* base, int dt, long long at, const float (&x)[VEC]) {
  if constexpr (VEC == 1) {
    store1(base, dt, at, x[0]);
  } else if (VEC == 8 && dt == LORDO_BF16) {
    uint4 a;
    a.x = pack_bf16x2(x[0], x[1]); a.y = pack_bf16x2(x[2], x[3]); a.z = pack_bf16x2(x[4 % VEC], x[5 % VEC]); a.w = pack_bf16x2(x[6 % VEC], x[7 % VEC]);
    *reinterpret_cast<uint4*>(reinterpret_cast<unsigned short*>(base) + at) = a;
  } else {
#pragma unroll
    for (int j = 0; j < VEC; j += 4) store4(base, dt, at + j, make_float4(x[j], x[j + 1], x[j + 2], x[j + 3]));
  }
}

enum SumMode { SUM_DENSE = 0, SUM_ADD = 1, SUM_ROWS = 2 };

struct SumArgs {
  const void* dY;
  const int2* order;    // [K][T]
  const int2* segs;     // [K][V]
  const int* valid;
  float* parts;         // [K][windows][2][d]: of the token that came in from the window before, of the one that goes on into the next
  long long V, T, d;
  int groups, windows;  // column groups of a row, windows of a worker
  float scale;
  void* out;
  int out_dt;
  double* sq;           // [K][2 * gridDim.x]
  int* count;           // 2 * gridDim.x
  long long out_cap;    // rows of a worker in `out` (sums in rows of their own)
  unsigned sum_blocks;  // blocks that form sums; the rest write the zeros of rows without a token
};

// The sum of token v, whose first sorted entry is `start`.
template <int VEC, int MODE>
__device__ __forceinline__ void emit(const SumArgs& a, int k, int v, int start, long long col, float (&acc)[VEC], float& sq) {
#pragma unroll
  for (int j = 0; j < VEC; ++j) acc[j] *= a.scale;
  if (MODE == SUM_ROWS) {
    put<VEC>(a.out, LORDO_F32, ((long long)k * a.out_cap + start) * a.d + col, acc);
#pragma unroll
    for (int j = 0; j < VEC; ++j) sq += acc[j] * acc[j];
  } else {
    const long long at = ((long long)k * a.V + v) * a.d + col;
    if (MODE == SUM_ADD) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) acc[j] += load1(a.out, a.out_dt, at + j);
    }
    put<VEC>(a.out, a.out_dt, at, acc);
  }
}

// Sums of squares of a block: sq[k][which * gridDim.x + block].
__device__ __forceinline__ void block_squares(const SumArgs& a, int k, int which, float x) {
  __shared__ double red[8];
  double s = (double)x;
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    s = 0.0;
    for (int w = 0; w < 8; ++w) s += red[w];
    a.sq[(long long)k * 2 * gridDim.x + which * gridDim.x + blockIdx.x] = s;
    if (k == 0 && blockIdx.x == 0) *a.count = 2 * (int)gridDim.x;
  }
}

// A warp walks a window of W sorted entries, 32 * VEC columns of each row of dY, eight rows under way at a time. Tokens whose entries all lie in
// the window are done; the first part of one that goes on and the last of one that came in are left for join_sums_kernel.
constexpr int kAhead = 8;
template <int DT, int VEC, int MODE, int W>
__device__ __forceinline__ void window_sums(const SumArgs& a, int k, int w, long long col, int lane, float& sq) {
  const int valid = a.valid[k], s = w * W;
  if (s >= valid) return;
  const int n = valid - s < W ? valid - s : W;
  const int2* order = a.order + (long long)k * a.T + s;
  const int2 mine = lane < n ? __ldcg(order + lane) : make_int2(-1, 0);
  const int before = s > 0 ? __ldcg(order - 1).x : -1, behind = s + n < valid ? __ldcg(order + n).x : -1;
  int next = __shfl_down_sync(0xffffffffu, mine.x, 1);
  if (lane == n - 1) next = behind;
  const unsigned ends = __ballot_sync(0xffffffffu, lane < n && next != mine.x);
  const bool on = col < a.d;
  bool came_in = before == __shfl_sync(0xffffffffu, mine.x, 0);
  int start = s;
  float acc[VEC] = {};
  float* part = a.parts + ((long long)k * a.windows + w) * 2 * a.d + col;
  const long long first = (long long)k * a.T * a.d + (on ? col : 0);
  for (int b = 0; b < n; b += kAhead) {
    Piece<DT, VEC> x[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int pos = __shfl_sync(0xffffffffu, mine.y, (b + j) & 31);
      if (b + j < n && on) x[j].load(a.dY, first + (long long)pos * a.d);
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (b + j >= n) break;
      if (on) x[j].add_to(acc);
      if ((ends >> (b + j)) & 1u) {
        const int v = __shfl_sync(0xffffffffu, mine.x, b + j);
        if (on) {
          if (came_in) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) part[i] = acc[i];
          } else {
            emit<VEC, MODE>(a, k, v, start, col, acc, sq);
          }
        }
#pragma unroll
        for (int i = 0; i < VEC; ++i) acc[i] = 0.f;
        came_in = false;
        start = s + b + j + 1;
      }
    }
  }
  if (!((ends >> (n - 1)) & 1u) && on) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) part[(came_in ? 0 : a.d) + i] = acc[i];
  }
}

template <int DT, int VEC, int MODE, int W>
__global__ void __launch_bounds__(256) window_sums_kernel(SumArgs a) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, k = blockIdx.y;
  dep_begin();
  if (MODE == SUM_DENSE && blockIdx.x >= a.sum_blocks) {  // 32 rows a warp
    const long long v0 = ((long long)(blockIdx.x - a.sum_blocks) * 8 + warp) * 32;
    if (v0 >= a.V) return;
    const int2 seg = v0 + lane < a.V ? __ldcg(a.segs + (long long)k * a.V + v0 + lane) : make_int2(0, 1);
    unsigned empty = __ballot_sync(0xffffffffu, seg.x >= seg.y);
    const float zero[VEC] = {};
    while (empty) {
      const int r = __ffs(empty) - 1;
      empty &= empty - 1;
      for (long long col = lane * VEC; col < a.d; col += 32 * VEC) put<VEC>(a.out, a.out_dt, ((long long)k * a.V + v0 + r) * a.d + col, zero);
    }
    return;
  }
  const long long item = (long long)blockIdx.x * 8 + warp;
  const long long w = item / a.groups;
  float sq = 0.f;
  if (w < a.windows) window_sums<DT, VEC, MODE, W>(a, k, (int)w, ((item - w * a.groups) * 32 + lane) * VEC, lane, sq);
  if (MODE == SUM_ROWS) block_squares(a, k, 0, sq);
}

// Tokens whose entries begin in one window and go on in others: their parts in the order of the windows.
template <int VEC, int MODE, int W>
__global__ void __launch_bounds__(256) join_sums_kernel(SumArgs a) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, k = blockIdx.y;
  dep_begin();
  const long long item = (long long)blockIdx.x * 8 + warp;
  const int w = (int)(item / a.groups);
  const long long col = ((item - (long long)w * a.groups) * 32 + lane) * VEC;
  const int valid = a.valid[k], last = (w + 1) * W - 1;
  float sq = 0.f;
  if (w < a.windows && last + 1 < valid) {
    const int2* order = a.order + (long long)k * a.T;
    const int v = __ldcg(order + last).x;
    if (v == __ldcg(order + last + 1).x) {
      const int2 seg = __ldcg(a.segs + (long long)k * a.V + v);
      if (seg.x >= w * W && col < a.d) {  // it begins here
        const float* p = a.parts + ((long long)k * a.windows + w) * 2 * a.d + a.d + col;
        float acc[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) acc[i] = __ldcg(p + i);
        const int end = (seg.y - 1) / W;
        p += a.d;
#pragma unroll 4
        for (int x = w + 1; x <= end; ++x, p += 2 * a.d) {
#pragma unroll
          for (int i = 0; i < VEC; ++i) acc[i] += __ldcg(p + i);
        }
        emit<VEC, MODE>(a, k, v, seg.x, col, acc, sq);
      }
    }
  }
  if (MODE == SUM_ROWS) block_squares(a, k, 1, sq);
}

// ---------------------------------------------------------------------------------------------
// Lookup
// ---------------------------------------------------------------------------------------------
template <int DT, int VEC>
__global__ void __launch_bounds__(256) lookup_kernel(const void* __restrict__ W, const void* __restrict__ tokens, int is64, long long V, long long d,
                                                     long long T, long long pieces, float scale, void* __restrict__ out, int out_dt) {
  dep_begin();
  const long long per_row = (d + VEC - 1) / VEC;
  const long long at = (long long)blockIdx.x * 256 + threadIdx.x;
  if (at >= pieces) return;
  const long long row = at / per_row, col = (at - row * per_row) * VEC;
  const long long v = is64 ? reinterpret_cast<const long long*>(tokens)[row] : (long long)reinterpret_cast<const int*>(tokens)[row];
  const long long k = row / T;
  float x[VEC] = {};
  if (v >= 0 && v < V) {
    Piece<DT, VEC> p;
    p.load(W, (k * V + v) * d + col);
    p.add_to(x);
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

// Columns of a lane: 16 bytes of dY where rows and arrays allow it.
int sum_vec(const TokProblem& p, const void* out) {
  const int vec = p.y_dt == LORDO_F32 ? 4 : 8;
  return p.d % vec == 0 && wide(p.dY, p.d, p.y_dt) && (reinterpret_cast<uintptr_t>(out) & 15u) == 0 ? vec : 1;
}

// Sorted entries of a window.
constexpr int kWindow = 32;
int windows_of(long long T) { return (int)((T + kWindow - 1) / kWindow); }

unsigned sum_blocks(long long T, long long d, int vec) {
  const long long items = windows_of(T) * ((d + 32 * vec - 1) / (32 * vec));
  return items > 0 ? (unsigned)((items + 7) / 8) : 1u;
}

template <int MODE>
int run_sums(const TokProblem& p, const TokScratch& s, int which, void* out, int out_dt, const TokRows* r, cudaStream_t st) {
  const int vec = sum_vec(p, out);
  SumArgs a = {};
  a.dY = p.dY; a.order = s.buf[which]; a.segs = s.segs; a.valid = s.valid; a.parts = s.parts;
  a.V = p.V; a.T = p.T; a.d = p.d; a.scale = p.scale;
  a.groups = (int)((p.d + 32 * vec - 1) / (32 * vec));
  a.windows = windows_of(p.T);
  a.out = out; a.out_dt = out_dt;
  if (r) { a.sq = r->sq; a.count = r->count; a.out_cap = r->cap; }
  a.sum_blocks = sum_blocks(p.T, p.d, vec);
  const unsigned zeros = MODE == SUM_DENSE ? (unsigned)((p.V + 255) / 256) : 0u;
  const dim3 grid(a.sum_blocks + zeros, p.K), join(a.sum_blocks, p.K);
  if (p.y_dt == LORDO_F32) {
    if (vec == 4) launch_dep(window_sums_kernel<LORDO_F32, 4, MODE, kWindow>, grid, 256, 0, st, a);
    else launch_dep(window_sums_kernel<LORDO_F32, 1, MODE, kWindow>, grid, 256, 0, st, a);
  } else {
    if (vec == 8) launch_dep(window_sums_kernel<LORDO_BF16, 8, MODE, kWindow>, grid, 256, 0, st, a);
    else launch_dep(window_sums_kernel<LORDO_BF16, 1, MODE, kWindow>, grid, 256, 0, st, a);
  }
  if (vec == 8) launch_dep(join_sums_kernel<8, MODE, kWindow>, join, 256, 0, st, a);
  else if (vec == 4) launch_dep(join_sums_kernel<4, MODE, kWindow>, join, 256, 0, st, a);
  else launch_dep(join_sums_kernel<1, MODE, kWindow>, join, 256, 0, st, a);
  return 2;
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
  s.parts = reinterpret_cast<float*>(take(8ll * K * windows_of(cap) * d));
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

int tok_dense(const TokProblem& p, const TokScratch& s, int which, void* dW, int w_dt, int accumulate, cudaStream_t st) {
  return accumulate ? run_sums<SUM_ADD>(p, s, which, dW, w_dt, nullptr, st) : run_sums<SUM_DENSE>(p, s, which, dW, w_dt, nullptr, st);
}

long long tok_row_blocks_max(long long cap, long long d) { return 2ll * sum_blocks(cap, d, 1); }

int tok_rows(const TokProblem& p, const TokScratch& s, int which, const TokRows& r, cudaStream_t st) {
  return run_sums<SUM_ROWS>(p, s, which, r.rows, LORDO_F32, &r, st);
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
  tok_dense(p, s, which, dW, w_dtype, accumulate, st);
  return cudaPeekAtLastError() == cudaSuccess ? LORDO_OK : LORDO_ERR_CUDA;
}

}  // extern "C"
