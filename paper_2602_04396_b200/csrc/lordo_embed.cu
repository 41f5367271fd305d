// Embedding lookup, and the table's gradient by sorted tokens:
//   out[k][t] = scale * W[k][tok[k][t]]           dW[k][v] = scale * sum over t with tok[k][t] = v of dY[k][t]
// for K workers, each with a table and tokens of its own. Sums are fp32, in the order of the positions, the same on every run.
#include "lordo_embed.h"

#include <algorithm>

#include "lordo_kernels.h"

namespace lordo {
namespace {

constexpr int kSortThreads = 1024, kSortWarps = 32, kMaxDigit = 256;

// Rows [first, last) of every worker's table, for the zeros of rows without a token.
struct Zeros {
  void* W;
  long long V, d, first, last;
  int dt;
};

struct SortArgs {
  const void* tokens;
  int is64, K, bits, passes;
  long long T, V;
  int2 *buf0, *buf1, *segs;
  int* valid;
  int per_warp;       // consecutive positions of a warp, a multiple of 32
  unsigned clusters;  // of the sort; the blocks behind them write zeros
  Zeros zeros;        // rows that are zeroed whether they have a token or not, before any sum is written
};

// One of `blocks` blocks writes its share of the rows, whole.
__device__ __forceinline__ void fill_zeros(const Zeros& z, int K, unsigned block, unsigned blocks) {
  const long long bytes = z.dt == LORDO_F32 ? 4 : 2, per = (z.last - z.first) * z.d * bytes, stride = z.V * z.d * bytes;
  char* base = reinterpret_cast<char*>(z.W) + z.first * z.d * bytes;
  const bool wide = ((reinterpret_cast<unsigned long long>(base) | per | stride) & 15) == 0;
  const long long unit = wide ? 16 : bytes, units = per / unit;
  for (int k = 0; k < K; ++k) {
    char* p = base + k * stride;
    for (long long x = (long long)block * blockDim.x + threadIdx.x; x < units; x += (long long)blocks * blockDim.x) {
      if (wide) reinterpret_cast<uint4*>(p)[x] = make_uint4(0u, 0u, 0u, 0u);
      else if (bytes == 4) reinterpret_cast<unsigned*>(p)[x] = 0u;
      else reinterpret_cast<unsigned short*>(p)[x] = 0;
    }
  }
}

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
  if (blockIdx.x >= a.clusters * C) {
    fill_zeros(a.zeros, a.K, blockIdx.x - a.clusters * C, gridDim.x - a.clusters * C);
    return;
  }
  if (a.T == 0 && c == 0 && t == 0) a.valid[k] = 0;
  int2* segs = a.segs + (long long)k * a.V;
  for (long long v = c * kSortThreads + t; v < a.V; v += (long long)C * kSortThreads) segs[v] = make_int2(0, 0);
  const long long begin = ((long long)c * kSortWarps + w) * a.per_warp;
  const long long end = begin + a.per_warp < a.T ? begin + a.per_warp : a.T;
  const int R = 1 << a.bits;
  const int2* src = nullptr;
  int2* dst = a.buf0 + (long long)k * a.T;
  int2* other = a.buf1 + (long long)k * a.T;
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
      int n[8];
#pragma unroll
      for (unsigned r = 0; r < 8; ++r) n[r] = r < C ? cluster_load(tot + t, r) : 0;
#pragma unroll
      for (unsigned r = 0; r < 8; ++r) {
        all += n[r];
        if (r < c) before += n[r];
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

// The same where a CTA has at most 1024 * NB positions: a thread keeps its NB pairs in registers, a pass hands them to the thread that owns their place
// by way of that CTA's shared memory, and only the last one writes to global memory. Counts of a digit lie warp by warp, a warp scans eight
// digits. Bound by latency (16384 tokens for each of eight workers, two passes, 21 us from a cold start). With it in place of the kernel above, and the
// joining's loads under way together, the gradient of two workers' 5001 tokens went from 31.0 to 27.2 us.
template <int NB>
__global__ void __launch_bounds__(kSortThreads) sort_small_kernel(SortArgs a) {
  __shared__ unsigned short cnt[kMaxDigit][kSortWarps + 2];
  __shared__ int tot[kMaxDigit], base[kMaxDigit], wsum[8];
  __shared__ int2 buf[kSortThreads * NB];
  constexpr int L = kSortThreads * NB;
  const int t = threadIdx.x, lane = t & 31, w = t >> 5;
  unsigned c, C;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(c));
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(C));
  const int k = blockIdx.x / C;
  dep_begin();
  if (blockIdx.x >= a.clusters * C) {  // a whole cluster
    fill_zeros(a.zeros, a.K, blockIdx.x - a.clusters * C, gridDim.x - a.clusters * C);
    return;
  }
  const int T = (int)a.T, V = (int)a.V, begin = (int)c * L + w * (32 * NB) + lane;
  int2 e[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    const int i = begin + 32 * b;
    e[b] = make_int2(-1, i);
    if (i < T) {
      const long long at = (long long)k * T + i;
      const long long v = a.is64 ? reinterpret_cast<const long long*>(a.tokens)[at] : (long long)reinterpret_cast<const int*>(a.tokens)[at];
      e[b].x = v >= 0 && v < V ? (int)v : V;
    }
  }
  int2* segs = a.segs + (long long)k * V;
  for (int v = (int)c * kSortThreads + t; v < V; v += (int)C * kSortThreads) segs[v] = make_int2(0, 0);
  const int R = 1 << a.bits;
  int2* out = ((a.passes - 1) & 1 ? a.buf1 : a.buf0) + (long long)k * T;
  for (int p = 0; p < a.passes; ++p) {
    const int shift = p * a.bits;
    for (int i = t; i < R * (kSortWarps + 2) / 2; i += kSortThreads) reinterpret_cast<unsigned*>(cnt)[i] = 0u;
    __syncthreads();
    int rank[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const bool in = begin + 32 * b < T;
      const int digit = in ? (e[b].x >> shift) & (R - 1) : -1;
      const unsigned same = __match_any_sync(0xffffffffu, digit);
      rank[b] = in ? cnt[digit][w] + __popc(same & ((1u << lane) - 1u)) : 0;
      __syncwarp();
      if (in && lane == __ffs(same) - 1) cnt[digit][w] += (unsigned short)__popc(same);
      __syncwarp();
    }
    __syncthreads();
    // a warp scans eight digits at a time, side by side
    for (int x0 = 8 * w; x0 < R; x0 += 8 * kSortWarps) {
      int n[8], sum[8];
#pragma unroll
      for (int x = 0; x < 8; ++x) sum[x] = n[x] = x0 + x < R ? cnt[x0 + x][lane] : 0;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
#pragma unroll
        for (int x = 0; x < 8; ++x) {
          const int up = __shfl_up_sync(0xffffffffu, sum[x], o);
          if (lane >= o) sum[x] += up;
        }
      }
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        if (x0 + x >= R) break;
        cnt[x0 + x][lane] = (unsigned short)(sum[x] - n[x]);
        if (lane == 31) tot[x0 + x] = sum[x];
      }
    }
    if (C > 1) cluster_sync_all(); else __syncthreads();
    int all = 0, before = 0;
    if (t < R) {
      int n[8];
#pragma unroll
      for (unsigned r = 0; r < 8; ++r) n[r] = r < C ? cluster_load(tot + t, r) : 0;
#pragma unroll
      for (unsigned r = 0; r < 8; ++r) {
        all += n[r];
        if (r < c) before += n[r];
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
    const bool last = p + 1 == a.passes;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      if (begin + 32 * b >= T) continue;
      const int digit = (e[b].x >> shift) & (R - 1);
      const int at = base[digit] + cnt[digit][w] + rank[b];
      unsigned to = (unsigned)__cvta_generic_to_shared(buf + at % L);
      asm volatile("mapa.shared::cluster.u32 %0, %0, %1;" : "+r"(to) : "r"(at / L));
      asm volatile("st.shared::cluster.v2.u32 [%0], {%1, %2};" ::"r"(to), "r"(e[b].x), "r"(e[b].y) : "memory");
      if (last) out[at] = e[b];
    }
    if (C > 1) cluster_sync_all(); else __syncthreads();  // all pairs are in place, and every CTA has read the totals
#pragma unroll
    for (int b = 0; b < NB; ++b)
      if (begin + 32 * b < T) e[b] = buf[w * (32 * NB) + lane + 32 * b];
  }
  auto token_at = [&](int i) {  // of the order, in whichever CTA's shared memory
    return i < 0 || i >= T ? -1 : i / L == (int)c ? buf[i % L].x : cluster_load(&buf[i % L].x, (unsigned)(i / L));
  };
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    const int i = begin + 32 * b;
    if (i >= T) continue;
    const int v = e[b].x, prev = token_at(i - 1), next = token_at(i + 1);
    if (v < V) {
      if (prev != v) segs[v].x = i;
      if (next != v) segs[v].y = i + 1;
      if (next < 0 || next >= V) a.valid[k] = i + 1;
    } else if (i == 0) {
      a.valid[k] = 0;
    }
  }
  if (T == 0 && c == 0 && t == 0) a.valid[k] = 0;
  if (C > 1) cluster_sync_all();  // the others may still read this CTA's shared memory
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
  int* count;           // of sums of squares: 2 * gridDim.x, or gridDim.x where nothing is joined
  long long out_cap;    // rows of a worker in `out` (sums in rows of their own)
  unsigned sum_blocks;  // blocks that form sums; the rest write the zeros of rows without a token,
  long long zero0, zero1, zero2;  // [zero0, zero1) beside the windows, [zero1, zero2) beside the joining
};

// What a row of the table holds before it is added to.
template <int ODT, int VEC>
struct Old {
  unsigned r[ODT == LORDO_F32 ? VEC : (VEC + 1) / 2];
  __device__ __forceinline__ void load(const void* base, long long at) {
    if constexpr (VEC == 1) {
      r[0] = ODT == LORDO_F32 ? reinterpret_cast<const unsigned*>(base)[at] : reinterpret_cast<const unsigned short*>(base)[at];
    } else {
      constexpr int kWords = ODT == LORDO_F32 ? VEC : VEC / 2;
      const char* p = reinterpret_cast<const char*>(base) + at * (ODT == LORDO_F32 ? 4 : 2);
#pragma unroll
      for (int j = 0; j < kWords; j += 2) {
        const uint2 x = reinterpret_cast<const uint2*>(p)[j / 2];
        r[j] = x.x; r[j + 1] = x.y;
      }
    }
  }
  __device__ __forceinline__ float value(int j) const {
    return ODT == LORDO_F32 ? __uint_as_float(r[j]) : __uint_as_float(j & 1 ? r[j / 2] & 0xFFFF0000u : r[j / 2] << 16);
  }
};

// The sum of token v, whose first sorted entry is `start`; old: the row it is added to; sq: squares of a row's VEC columns in fp32, of rows in fp64.
template <int VEC, int MODE, int ODT>
__device__ __forceinline__ void emit(const SumArgs& a, int k, int v, int start, long long col, float (&acc)[VEC], const Old<ODT, VEC>& old, double& sq) {
#pragma unroll
  for (int j = 0; j < VEC; ++j) acc[j] *= a.scale;
  if (MODE == SUM_ROWS) {
    put<VEC>(a.out, LORDO_F32, ((long long)k * a.out_cap + start) * a.d + col, acc);
    float squares = 0.f;
#pragma unroll
    for (int j = 0; j < VEC; ++j) squares += acc[j] * acc[j];
    if (squares < INFINITY) {
      sq += (double)squares;
    } else {  // fp32 does not hold them, though it may each sum
#pragma unroll
      for (int j = 0; j < VEC; ++j) sq += (double)acc[j] * (double)acc[j];
    }
  } else {
    if (MODE == SUM_ADD) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) acc[j] += old.value(j);
    }
    put<VEC>(a.out, ODT, ((long long)k * a.V + v) * a.d + col, acc);
  }
}

// Sums of squares of a block: sq[k][which * gridDim.x + block].
__device__ __forceinline__ void block_squares(const SumArgs& a, int k, int which, double s) {
  __shared__ double red[8];
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    s = 0.0;
    for (int w = 0; w < 8; ++w) s += red[w];
    a.sq[((long long)k * (a.windows > 1 ? 2 : 1) + which) * gridDim.x + blockIdx.x] = s;
    if (k == 0 && blockIdx.x == 0) *a.count = (a.windows > 1 ? 2 : 1) * (int)gridDim.x;
  }
}

// A warp walks a window of W sorted entries, 32 * VEC columns of each row of dY, eight rows under way at a time. Tokens whose entries all lie in
// the window are done; the first part of one that goes on and the last of one that came in are left for join_sums_kernel.
constexpr int kAhead = 8;
template <int DT, int VEC, int MODE, int W, int ODT>
__device__ __forceinline__ void window_sums(const SumArgs& a, int k, int w, long long col, int lane, double& sq) {
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
  Piece<DT, VEC> x[kAhead];
  Old<ODT, VEC> old[kAhead];
  auto fetch = [&](int i, Piece<DT, VEC>& row, Old<ODT, VEC>& was) {  // entry i of the window; every lane is here
    const int pos = __shfl_sync(0xffffffffu, mine.y, i & 31);
    if (i < n && on) row.load(a.dY, first + (long long)pos * a.d);
    if (MODE == SUM_ADD) {
      const int v = __shfl_sync(0xffffffffu, mine.x, i & 31);
      if (i < n && on && ((ends >> (i & 31)) & 1u)) was.load(a.out, ((long long)k * a.V + v) * a.d + col);
    }
  };
#pragma unroll
  for (int j = 0; j < kAhead; ++j) fetch(j, x[j], old[j]);
  for (int b = 0; b < n; b += kAhead) {
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
            emit<VEC, MODE, ODT>(a, k, v, start, col, acc, old[j], sq);
          }
        }
#pragma unroll
        for (int i = 0; i < VEC; ++i) acc[i] = 0.f;
        came_in = false;
        start = s + b + j + 1;
      }
      fetch(b + j + kAhead, x[j], old[j]);
    }
  }
  if (!((ends >> (n - 1)) & 1u) && on) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) part[(came_in ? 0 : a.d) + i] = acc[i];
  }
}

// Zeros of those rows from v0 to v1 that have no token, 32 rows a warp.
template <int VEC>
__device__ __forceinline__ void empty_rows(const SumArgs& a, int k, long long v0, long long v1, int lane) {
  if (v0 >= v1) return;
  const int2 seg = v0 + lane < v1 ? __ldcg(a.segs + (long long)k * a.V + v0 + lane) : make_int2(0, 1);
  unsigned empty = __ballot_sync(0xffffffffu, seg.x >= seg.y);
  const float zero[VEC] = {};
  while (empty) {
    const int r = __ffs(empty) - 1;
    empty &= empty - 1;
    for (long long col = lane * VEC; col < a.d; col += 32 * VEC) put<VEC>(a.out, a.out_dt, ((long long)k * a.V + v0 + r) * a.d + col, zero);
  }
}

template <int DT, int VEC, int MODE, int W, int ODT>
__global__ void __launch_bounds__(256) window_sums_kernel(SumArgs a) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, k = blockIdx.y;
  dep_begin();
  if (MODE == SUM_DENSE && blockIdx.x >= a.sum_blocks) {
    empty_rows<VEC>(a, k, a.zero0 + ((long long)(blockIdx.x - a.sum_blocks) * 8 + warp) * 32, a.zero1, lane);
    return;
  }
  const long long item = (long long)blockIdx.x * 8 + warp;
  const long long w = item / a.groups;
  double sq = 0.0;
  if (w < a.windows) window_sums<DT, VEC, MODE, W, ODT>(a, k, (int)w, ((item - w * a.groups) * 32 + lane) * VEC, lane, sq);
  if (MODE == SUM_ROWS) block_squares(a, k, 0, sq);
}

// Tokens whose entries begin in one window and go on in others: their parts in the order of the windows.
template <int VEC, int MODE, int W, int ODT>
__global__ void __launch_bounds__(256) join_sums_kernel(SumArgs a) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, k = blockIdx.y;
  dep_begin();
  if (MODE == SUM_DENSE && blockIdx.x >= a.sum_blocks) {
    empty_rows<VEC>(a, k, a.zero1 + ((long long)(blockIdx.x - a.sum_blocks) * 8 + warp) * 32, a.zero2, lane);
    return;
  }
  const long long item = (long long)blockIdx.x * 8 + warp;
  const int w = (int)(item / a.groups);
  const long long col = ((item - (long long)w * a.groups) * 32 + lane) * VEC;
  const int valid = a.valid[k], last = (w + 1) * W - 1;
  double sq = 0.0;
  if (w < a.windows && last + 1 < valid) {
    const int2* order = a.order + (long long)k * a.T;
    const int v = __ldcg(order + last).x;
    if (v == __ldcg(order + last + 1).x) {
      const int2 seg = __ldcg(a.segs + (long long)k * a.V + v);
      if (seg.x >= w * W && col < a.d) {  // it begins here
        const float* p = a.parts + ((long long)k * a.windows + w) * 2 * a.d + a.d + col;
        float acc[VEC];
        Old<ODT, VEC> old;
        if (MODE == SUM_ADD) old.load(a.out, ((long long)k * a.V + v) * a.d + col);
#pragma unroll
        for (int i = 0; i < VEC; ++i) acc[i] = __ldcg(p + i);
        const int end = (seg.y - 1) / W;
        p += a.d;
        constexpr int kParts = 64 / VEC < 16 ? 64 / VEC : 16;  // under way together
        for (int x = w + 1; x <= end; x += kParts) {
          float y[kParts][VEC];
#pragma unroll
          for (int j = 0; j < kParts; ++j, p += 2 * a.d)
#pragma unroll
            for (int i = 0; i < VEC; ++i) y[j][i] = x + j <= end ? __ldcg(p + i) : 0.f;
#pragma unroll
          for (int j = 0; j < kParts; ++j)
#pragma unroll
            for (int i = 0; i < VEC; ++i) acc[i] += y[j][i];
        }
        emit<VEC, MODE, ODT>(a, k, v, seg.x, col, acc, old, sq);
      }
    }
  }
  if (MODE == SUM_ROWS) block_squares(a, k, 1, sq);
}

// ---------------------------------------------------------------------------------------------
// Lookup. A warp has kLookRows consecutive rows of the output, 32 * VEC columns of each: their tokens are one load, and the rows of the table
// are under way together.
// ---------------------------------------------------------------------------------------------
constexpr int kLookRows = 8;
template <int DT, int VEC>
__global__ void __launch_bounds__(256) lookup_kernel(const void* __restrict__ W, const void* __restrict__ tokens, int is64, long long V, long long d,
                                                     long long T, long long rows, int groups, float scale, void* __restrict__ out, int out_dt) {
  const int lane = threadIdx.x & 31;
  dep_begin();
  const long long item = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  const long long first = item / groups * kLookRows;
  if (first >= rows) return;
  const int n = rows - first < kLookRows ? (int)(rows - first) : kLookRows;
  long long mine = -1;  // row of all workers' tables, or none
  if (lane < n) {
    const long long at = first + lane;
    const long long v = is64 ? reinterpret_cast<const long long*>(tokens)[at] : (long long)reinterpret_cast<const int*>(tokens)[at];
    if (v >= 0 && v < V) mine = at / T * V + v;
  }
  const long long col = (item % groups * 32 + lane) * VEC;
  const bool on = col < d;
  Piece<DT, VEC> x[kLookRows];
#pragma unroll
  for (int j = 0; j < kLookRows; ++j) {
    const long long row = __shfl_sync(0xffffffffu, mine, j);
    x[j].r = make_uint4(0u, 0u, 0u, 0u);
    if (on && row >= 0) x[j].load(W, row * d + col);
  }
#pragma unroll
  for (int j = 0; j < kLookRows; ++j) {
    if (!on || j >= n) break;
    float y[VEC] = {};
    x[j].add_to(y);
#pragma unroll
    for (int i = 0; i < VEC; ++i) y[i] *= scale;
    put<VEC>(out, out_dt, (first + j) * d + col, y);
  }
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

// Which rows' zeros are written when. While tokens are sorted the memory is idle, so a first part of the table is zeroed then without
// knowing which rows will have a token; as much more as the joining takes is left to it. What is left is written beside the windows. (All of it
// there: 50304 x 768, K = 8, 16384 tokens 187 us, with 64 and 64 MB 179.5, 64 and 128 178.3, 128 and 128 181.3.)
constexpr long long kSortBytes = 64ll << 20, kJoinBytes = 128ll << 20;

int sort(const TokProblem& p, const TokScratch& s, const Zeros& zeros, cudaStream_t st) {
  const int bits = token_bits(p.V);
  SortArgs a = {};
  a.tokens = p.tokens; a.is64 = p.is64; a.K = p.K; a.T = p.T; a.V = p.V;
  a.passes = (bits + 7) / 8;
  a.bits = (bits + a.passes - 1) / a.passes;
  a.buf0 = s.buf[0]; a.buf1 = s.buf[1]; a.segs = s.segs; a.valid = s.valid;
  a.zeros = zeros;
  int C = 1;
  while (C < 8 && p.T > 1024ll * C) C *= 2;
  const long long warps = (long long)C * kSortWarps;
  a.per_warp = (int)(((p.T + warps - 1) / warps + 31) / 32 * 32);
  a.clusters = (unsigned)p.K;
  const unsigned fill = zeros.last > zeros.first ? (unsigned)((80 + C - 1) / C * C) : 0u;
  cudaLaunchConfig_t lc = {};
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = C; at[1].val.clusterDim.y = 1; at[1].val.clusterDim.z = 1;
  lc.gridDim = dim3(C * p.K + fill); lc.blockDim = dim3(kSortThreads); lc.stream = st;
  lc.attrs = at; lc.numAttrs = 2;
  if (a.per_warp <= 32) cudaLaunchKernelEx(&lc, sort_small_kernel<1>, a);
  else if (a.per_warp <= 64) cudaLaunchKernelEx(&lc, sort_small_kernel<2>, a);
  else if (a.per_warp <= 96) cudaLaunchKernelEx(&lc, sort_small_kernel<3>, a);
  else cudaLaunchKernelEx(&lc, sort_tokens_kernel, a);
  return (a.passes - 1) & 1;
}

template <int MODE>
int run_sums(const TokProblem& p, const TokScratch& s, void* out, int out_dt, const TokRows* r, cudaStream_t st) {
  const int vec = sum_vec(p, out);
  SumArgs a = {};
  a.zero0 = a.zero1 = a.zero2 = p.V;
  if (MODE == SUM_DENSE) {
    const long long row = p.K * p.d * (out_dt == LORDO_F32 ? 4 : 2);
    a.zero0 = std::min((long long)p.V, kSortBytes / row);
    a.zero1 = std::max(a.zero0, p.V - kJoinBytes / row);
  }
  const int which = sort(p, s, Zeros{out, p.V, p.d, 0, MODE == SUM_DENSE ? a.zero0 : 0, out_dt}, st);
  a.dY = p.dY; a.order = s.buf[which]; a.segs = s.segs; a.valid = s.valid; a.parts = s.parts;
  a.V = p.V; a.T = p.T; a.d = p.d; a.scale = p.scale;
  a.groups = (int)((p.d + 32 * vec - 1) / (32 * vec));
  a.windows = windows_of(p.T);
  a.out = out; a.out_dt = out_dt;
  if (r) { a.sq = r->sq; a.count = r->count; a.out_cap = r->cap; }
  a.sum_blocks = sum_blocks(p.T, p.d, vec);
  const dim3 grid(a.sum_blocks + (unsigned)((a.zero1 - a.zero0 + 255) / 256), p.K), join(a.sum_blocks + (unsigned)((a.zero2 - a.zero1 + 255) / 256), p.K);
  const bool joins = a.windows > 1 || a.zero2 > a.zero1;  // else no token lies in two windows
#define LORDO_SUMS(DT, VEC, ODT)                                                              \
  launch_dep(window_sums_kernel<DT, VEC, MODE, kWindow, ODT>, grid, 256, 0, st, a);           \
  if (joins) launch_dep(join_sums_kernel<VEC, MODE, kWindow, ODT>, join, 256, 0, st, a)
#define LORDO_SUMS_VEC(DT, FULL, ODT) \
  if (vec > 1) { LORDO_SUMS(DT, FULL, ODT); } else { LORDO_SUMS(DT, 1, ODT); }
  if (out_dt == LORDO_F32) {
    if (p.y_dt == LORDO_F32) { LORDO_SUMS_VEC(LORDO_F32, 4, LORDO_F32) } else { LORDO_SUMS_VEC(LORDO_BF16, 8, LORDO_F32) }
  } else if constexpr (MODE != SUM_ROWS) {
    if (p.y_dt == LORDO_F32) { LORDO_SUMS_VEC(LORDO_F32, 4, LORDO_BF16) } else { LORDO_SUMS_VEC(LORDO_BF16, 8, LORDO_BF16) }
  }
#undef LORDO_SUMS_VEC
#undef LORDO_SUMS
  return joins ? 3 : 2;
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

int tok_dense(const TokProblem& p, const TokScratch& s, void* dW, int w_dt, int accumulate, cudaStream_t st) {
  return accumulate ? run_sums<SUM_ADD>(p, s, dW, w_dt, nullptr, st) : run_sums<SUM_DENSE>(p, s, dW, w_dt, nullptr, st);
}

long long tok_row_blocks_max(long long cap, long long d) { return 2ll * sum_blocks(cap, d, 1); }

int tok_rows(const TokProblem& p, const TokScratch& s, const TokRows& r, cudaStream_t st) {
  return run_sums<SUM_ROWS>(p, s, r.rows, LORDO_F32, &r, st);
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
  const long long rows = (long long)K * T, groups = (d + 32 * vec - 1) / (32 * vec);
  const long long blocks = ((rows + kLookRows - 1) / kLookRows * groups + 7) / 8;
  if (blocks > 0x7fffffffll) return LORDO_ERR_UNSUPPORTED;
  const dim3 grid((unsigned)blocks);
  const int is64 = index == LORDO_I64;
#define LORDO_LOOKUP(DT, VEC)                                                                                                                  \
  launch_dep(lookup_kernel<DT, VEC>, grid, 256, 0, st, W, tokens, is64, (long long)V, (long long)d, (long long)T, rows, (int)groups, scale, out, \
             out_dtype)
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
  tok_dense(p, s, dW, w_dtype, accumulate, st);
  return cudaPeekAtLastError() == cudaSuccess ? LORDO_OK : LORDO_ERR_CUDA;
}

}  // extern "C"
