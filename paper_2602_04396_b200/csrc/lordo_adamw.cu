// AdamW over many tensors at once, K workers' replicas each, with moments in 32 or in 8 bits:
//   g = c_k G; m <- b1 m + (1-b1) g; v <- b2 v + (1-b2) g^2; m^ = m/(1-b1^s), v^ = v/(1-b2^s)
//   W <- W - lr ((w m^ + (1-w) g) / (sqrt(v^) + eps) + wd W)
// and the outer synchronisation of such tensors.
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "lordo_adamw.h"
#include "lordo_kernels.h"

namespace lordo {
namespace {

__device__ __forceinline__ int find_tensor(const unsigned* start, int count, unsigned x) {
  int lo = 0, hi = count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (start[mid] <= x) lo = mid; else hi = mid - 1;
  }
  return lo;
}

template <int DT>
__device__ __forceinline__ void load8(const void* base, long long at, float (&x)[8]) {
  if constexpr (DT == LORDO_F32) {
    const float4* p = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(base) + at);
    const float4 a = p[0], b = p[1];
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  } else {
    const uint4 a = *reinterpret_cast<const uint4*>(reinterpret_cast<const unsigned short*>(base) + at);
    const unsigned r[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[2 * j] = __uint_as_float(r[j] << 16);
      x[2 * j + 1] = __uint_as_float(r[j] & 0xFFFF0000u);
    }
  }
}

template <int DT>
__device__ __forceinline__ void store8(void* base, long long at, const float (&x)[8]) {
  if constexpr (DT == LORDO_F32) {
    float4* p = reinterpret_cast<float4*>(reinterpret_cast<float*>(base) + at);
    p[0] = make_float4(x[0], x[1], x[2], x[3]);
    p[1] = make_float4(x[4], x[5], x[6], x[7]);
  } else {
    uint4 a;
    a.x = pack_bf16x2(x[0], x[1]); a.y = pack_bf16x2(x[2], x[3]); a.z = pack_bf16x2(x[4], x[5]); a.w = pack_bf16x2(x[6], x[7]);
    *reinterpret_cast<uint4*>(reinterpret_cast<unsigned short*>(base) + at) = a;
  }
}

// Gradient of element e of worker k of a table whose rows were summed by token.
__device__ __forceinline__ float row_grad(const AwTensor& T, int k, long long e) {
  const long long v = e / T.d;
  const int2 seg = __ldg(T.segs + (long long)k * (T.n / T.d) + v);
  return seg.x < seg.y ? T.rows[((long long)k * T.cap + seg.x) * T.d + (e - v * T.d)] : 0.f;
}
__device__ __forceinline__ void row_grad8(const AwTensor& T, int k, long long e, float (&g)[8]) {
  if ((T.d & 7) == 0) {
    const long long v = e / T.d;
    const int2 seg = __ldg(T.segs + (long long)k * (T.n / T.d) + v);
    if (seg.x < seg.y) {
      load8<LORDO_F32>(T.rows, ((long long)k * T.cap + seg.x) * T.d + (e - v * T.d), g);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) g[j] = 0.f;
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) g[j] = row_grad(T, k, e + j);
  }
}

// ---------------------------------------------------------------------------------------------
// Clip coefficients: partial sums of squares of chunks, one per block; the last block of a worker (scope 0) or of a tensor of a worker
// (scope 1) adds its partial sums, in a fixed order whichever block it is.
// ---------------------------------------------------------------------------------------------
__device__ __forceinline__ double block_sum(double x, double* red) {
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = x;
  __syncthreads();
  double s = 0.0;
#pragma unroll
  for (int w = 0; w < 8; ++w) s += red[w];
  return s;
}

template <int GDT>
__global__ void __launch_bounds__(256) adamw_norm_kernel(const __grid_constant__ AwTable tab, AwLaunch l, AwClip c) {
  __shared__ double red[2][8];
  __shared__ bool last_s;
  const int t = threadIdx.x;
  const int k = (int)(blockIdx.x / l.units);
  const unsigned q = blockIdx.x - (unsigned)k * l.units;
  const int i = find_tensor(tab.start, l.count, q);
  const AwTensor& T = l.tensors[i];
  const long long n = T.n;
  const int index = T.index;
  const void* G = tab.G[i];
  dep_begin();
  double s = 0.0;
  if (G) {
    const long long e0 = (long long)(q - tab.start[i]) * kAwChunk;
    const long long e1 = e0 + kAwChunk < n ? e0 + kAwChunk : n;
    const long long f0 = (long long)k * n + e0, f1 = (long long)k * n + e1;
    const long long a0 = (f0 + 7) & ~7ll, a1 = f1 & ~7ll;
    for (long long f = a0 + 8 * t; f < a1; f += 2 * 2048) {
      float x[2][8];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        if (f + u * 2048 < a1) {
          load8<GDT>(G, f + u * 2048, x[u]);
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) x[u][j] = 0.f;
        }
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {  // eight squares in fp32, the rest in fp64
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) sum += x[u][j] * x[u][j];
        s += (double)sum;
      }
    }
    const long long edge = t < 8 ? f0 + t : (a1 > a0 ? a1 : a0) + t - 8;  // elements before the first and behind the last vector
    if (t < 16 && edge < f1 && (t >= 8 || edge < a0)) {
      const float x = load1(G, GDT, edge);
      s += (double)x * (double)x;
    }
  } else if (q == tab.start[i]) {  // its first chunk stands for the whole tensor
    const int count = *T.rowsq_count;
    const double* p = T.rowsq + (long long)k * count;
    for (int x = t; x < count; x += 256) s += __ldcg(p + x);
  }
  s = block_sum(s, red[0]);
  const unsigned first = c.scope ? c.at + tab.start[i] : 0u;
  const unsigned many = c.scope ? tab.start[i + 1] - tab.start[i] : c.total;
  if (t == 0) {
    c.partial[(size_t)k * c.total + c.at + q] = s;
    __threadfence();
    unsigned* ticket = c.tickets + (c.scope ? (long long)index * l.K + k : k);
    last_s = atomicInc(ticket, many - 1) == many - 1;  // back to zero with the last block
  }
  __syncthreads();
  if (!last_s) return;
  __threadfence();
  const double* p = c.partial + (size_t)k * c.total + first;
  double a = 0.0;
  for (unsigned x = t; x < many; x += 256) a += __ldcg(p + x);
  const double total = block_sum(a, red[1]);
  if (t == 0 && !isfinite(total)) atomicOr(c.status, LORDO_FLAG_NONFINITE_GRAD);
  const float coef = (float)fmin(1.0, c.rho / (sqrt(total) + 1e-6));
  if (c.scope) {
    if (t == 0) c.coef[(long long)index * l.K + k] = coef;
  } else {
    for (int x = t; x < c.n_tensors; x += 256) c.coef[(long long)x * l.K + k] = coef;
  }
}

// ---------------------------------------------------------------------------------------------
// Step, 32-bit moments
// ---------------------------------------------------------------------------------------------
// The moments' operations are rounded one by one, as written in the definition: what a compiler fuses must not decide how 8-bit codes round.
__device__ __forceinline__ void moments(const AwStep& s, float g, float& m, float& v) {
  m = __fadd_rn(__fmul_rn(s.b1, m), __fmul_rn(s.a1, g));
  v = __fadd_rn(__fmul_rn(s.b2, v), __fmul_rn(__fmul_rn(s.a2, g), g));
}

__device__ __forceinline__ void update(const AwStep& s, float wd, float c, float g, float& m, float& v, float& w) {
  g = __fmul_rn(g, c);
  moments(s, g, m, v);
  const float up = (s.omega * (m * s.inv_bc1) + s.a_omega * g) / (sqrtf(v * s.inv_bc2) + s.eps);
  w -= s.lr * (up + wd * w);
}

template <int WDT, int GDT>
__global__ void __launch_bounds__(256) adamw_step_kernel(const __grid_constant__ AwTable tab, AwLaunch l, const float* __restrict__ coef, int stride, AwStep s) {
  const int t = threadIdx.x;
  const int k = (int)(blockIdx.x / l.units);
  const unsigned q = blockIdx.x - (unsigned)k * l.units;
  const int i = find_tensor(tab.start, l.count, q);
  const AwTensor T = l.tensors[i];
  const void* G = tab.G[i];
  dep_begin();
  const float c = coef ? __ldcg(coef + (long long)T.index * stride + k) : 1.f;
  const long long e0 = (long long)(q - tab.start[i]) * l.piece;
  const long long e1 = e0 + l.piece < T.n ? e0 + l.piece : T.n;
  const long long base = (long long)k * T.n, f0 = base + e0, f1 = base + e1;
  const long long a0 = (f0 + 7) & ~7ll, a1 = f1 & ~7ll;
  float* M = reinterpret_cast<float*>(T.m);
  float* V = reinterpret_cast<float*>(T.v);
  for (long long f = a0 + 8 * t; f < a1; f += 2048) {
    float g[8], w[8], m[8], v[8];
    if (G) load8<GDT>(G, f, g); else row_grad8(T, k, f - base, g);
    load8<WDT>(T.W, f, w);
    load8<LORDO_F32>(M, f, m);
    load8<LORDO_F32>(V, f, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) update(s, T.wd, c, g[j], m[j], v[j], w[j]);
    store8<LORDO_F32>(M, f, m);
    store8<LORDO_F32>(V, f, v);
    store8<WDT>(T.W, f, w);
  }
  const long long edge = t < 8 ? f0 + t : (a1 > a0 ? a1 : a0) + t - 8;
  if (t < 16 && edge < f1 && (t >= 8 || edge < a0)) {
    const float g = G ? load1(G, GDT, edge) : row_grad(T, k, edge - base);
    float w = load1(T.W, WDT, edge), m = M[edge], v = V[edge];
    update(s, T.wd, c, g, m, v, w);
    M[edge] = m;
    V[edge] = v;
    store1(T.W, WDT, edge, w);
  }
}

// ---------------------------------------------------------------------------------------------
// 8-bit moments: E4M3 codes of m and of sqrt(v), a power of two per block of 256 as their scale, rounded up or down at random.
// Rounded to the nearest the averages would stand still: b2 = 0.999 moves v by 0.1 % a step, and codes are 6 to 12 % apart. With powers
// of two for scales a value stays where it is on the grid when the largest of its block changes; an fp32 scale (the largest itself) would
// move all 256 off the grid in every step, and the noise of rounding them again would add up. sqrt(v) has half the range of v.
// ---------------------------------------------------------------------------------------------
// What the generator mixes to 16 random bits for each of four consecutive elements; the next four are kGolden on.
__device__ __forceinline__ unsigned long long counter4(unsigned long long key, long long e) { return key + kGolden * (unsigned long long)((e >> 2) + 1); }

// Exponent byte of the scale that puts `top` (the bits of a magnitude) into [128, 256) times itself.
__device__ __forceinline__ int scale_code(unsigned top) {
  const int e = (int)(top >> 23) - 7;
  return e < 1 ? 1 : e;
}
__device__ __forceinline__ float pow2(int code) { return __int_as_float(code << 23); }  // 2^(code - 127), code in [1, 254]

// E4M3 code of a magnitude t < 256, rounded down after (u + 1/2) / 65536 of a step was added; u16 = 16 u. Below 2^-6 the steps are 2^-9
// wide, as they are for t + 2^-6. Infinities and NaN become NaN.
__device__ __forceinline__ unsigned code8(float t, unsigned u16) {
  const bool sub = t < 0.015625f;
  const unsigned b = __float_as_uint(fabsf(sub ? t + 0.015625f : t));
  const int code = (int)((b + u16 + 8u) >> 20) - (sub ? 968 : 960);
  return (unsigned)(code > 127 ? 127 : code);
}
// The same for finite t in [2^-6, 256), in the top seven bits behind the sign's place.
__device__ __forceinline__ unsigned code8_normal(float t, unsigned u16) { return (__float_as_uint(t) + u16 + (8u - (960u << 20))) << 4; }

// Four values of E4M3 codes.
__device__ __forceinline__ void values8(unsigned c, float* x) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const __half2_raw r = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(c >> (16 * h)), __NV_E4M3);
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&r));
    x[2 * h] = f.x;
    x[2 * h + 1] = f.y;
  }
}

// 16 times the 16 random bits of element j of four, for the first moment and for the second
__device__ __forceinline__ unsigned first16(unsigned long long r, int j) {
  const unsigned w = j < 2 ? (unsigned)r : (unsigned)(r >> 32);
  return (j & 1 ? w >> 12 : w << 4) & 0xFFFF0u;
}
__device__ __forceinline__ unsigned second16(unsigned first) { return (first * 40503u) & 0xFFFF0u; }

constexpr unsigned kInfBits = 0x7F800000u;

__device__ __forceinline__ unsigned top8(const float (&x)[8]) {
  unsigned t = 0u;
#pragma unroll
  for (int j = 0; j < 8; j += 2) t = __vimax3_u32(t, __float_as_uint(x[j]) & 0x7FFFFFFFu, __float_as_uint(x[j + 1]) & 0x7FFFFFFFu);
  return t;
}
__device__ __forceinline__ unsigned low8(const float (&x)[8]) {
  unsigned t = 0xFFFFFFFFu;
#pragma unroll
  for (int j = 0; j < 8; j += 2) t = __vimin3_u32(t, __float_as_uint(x[j]) & 0x7FFFFFFFu, __float_as_uint(x[j + 1]) & 0x7FFFFFFFu);
  return t;
}

// Codes of four elements. NORMAL: every |x| inv lies in [2^-6, 256).
template <bool SECOND, bool NORMAL>
__device__ __forceinline__ unsigned pack8(const float* x, float inv, const unsigned (&u16)[4]) {
  unsigned b[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const unsigned u = SECOND ? second16(u16[j]) : u16[j];
    const unsigned bits = __float_as_uint(x[j]);
    if (NORMAL) {
      b[j] = code8_normal(fabsf(x[j]) * inv, u);
    } else {
      unsigned c = code8(fabsf(x[j]) * inv, u);
      if (SECOND && c == 0u && x[j] > 0.f) c = 1u;
      b[j] = c << 24;
    }
    b[j] = SECOND ? b[j] : (b[j] & 0x7FFFFFFFu) | (bits & 0x80000000u);
  }
  return __byte_perm(__byte_perm(b[0], b[1], 0x0073), __byte_perm(b[2], b[3], 0x0073), 0x5410);  // the top byte of each
}

// sqrt(v) by one of Newton's (Heron's) steps on r^2 = v from r = v rsqrt(v), whose derivative 2 r is 2 / rsqrt(v): of normal numbers off by less than
// a unit in the last place, as a rule rounded to the nearest. The step is not a number for 0 (and below 2^-126), infinity and NaN; the maximum
// then takes v 1e-20, which is 0, infinity and NaN, and below the root of any other v. Seven instructions without a branch; sqrtf has one.
__device__ __forceinline__ float root(float v) {
  float y;
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(v));
  const float r = v * y;
  return fmaxf(fmaf(fmaf(-r, r, v), 0.5f * y, r), v * 1e-20f);
}
__device__ __forceinline__ float reciprocal(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

struct Step8 {  // constants of a step, of its worker and tensor
  float c, b1, a1, b2, a2, keep, lm, lg, root_inv_bc2, eps;
};

// A lane's eight elements of a block of 256 of one worker's tensor: codes in, codes and scales out. The scales are powers of two, so that b1 (m8 S) is
// (b1 S) m8 to the last bit, and b2 (s8 S)^2 is (b2 S^2) s8^2.
__device__ __forceinline__ void step8_lane(const Step8& s, unsigned long long counter, float (&g)[8], float (&w)[8], unsigned (&mc)[2], unsigned (&vc)[2],
                                           int& mcode, int& vcode) {
  const float ms = pow2(mcode), vs = pow2(vcode);
  const float b1 = s.b1 * ms, b2 = s.b2 * (vs * vs);
  float m[8], r[8];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    values8(mc[h], m + 4 * h);
    values8(vc[h], r + 4 * h);
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float x = __fmul_rn(g[j], s.c);
    m[j] = __fadd_rn(__fmul_rn(b1, m[j]), __fmul_rn(s.a1, x));
    r[j] = root(__fadd_rn(__fmul_rn(b2, r[j] * r[j]), __fmul_rn(__fmul_rn(s.a2, x), x)));
    w[j] = fmaf(-(s.lm * m[j] + s.lg * x), reciprocal(fmaf(r[j], s.root_inv_bc2, s.eps)), w[j] * s.keep);
  }
  const unsigned mtop = __reduce_max_sync(0xffffffffu, top8(m)), vtop = __reduce_max_sync(0xffffffffu, top8(r));
  mcode = scale_code(mtop);
  vcode = scale_code(vtop);
  const float mi = pow2(254 - mcode), vi = pow2(254 - vcode);
  // magnitudes below 2^-6 of the grid, which take half as many instructions again, are rare: a block has them or it has not
  const bool low = __uint_as_float(low8(m)) * mi < 0.015625f || __uint_as_float(low8(r)) * vi < 0.015625f;
  const bool slow = __any_sync(0xffffffffu, low) || mtop >= kInfBits || vtop >= kInfBits;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const unsigned long long x = mix64(counter + h * kGolden);
    unsigned u[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) u[j] = first16(x, j);
    if (slow) {
      mc[h] = pack8<false, false>(m + 4 * h, mi, u);
      vc[h] = pack8<true, false>(r + 4 * h, vi, u);
    } else {
      mc[h] = pack8<false, true>(m + 4 * h, mi, u);
      vc[h] = pack8<true, true>(r + 4 * h, vi, u);
    }
  }
}

struct Arrays8 {  // of one worker
  const void* G;
  void* W;
  unsigned char *m, *v, *ms, *vs;
};

template <int BYTES>
__device__ __forceinline__ void copy_async(unsigned to, const void* from) {
  if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(to), "l"(from), "n"(BYTES) : "memory");
}
template <int DT>
__device__ __forceinline__ void copy8(unsigned to, const void* base, long long at) {  // eight elements, 32 lanes' 16 bytes side by side
  const char* p = reinterpret_cast<const char*>(base) + at * (DT == LORDO_F32 ? 4 : 2);
  copy_async<16>(to, p);
  if constexpr (DT == LORDO_F32) copy_async<16>(to + 512, p + 16);
}
template <int DT>
__device__ __forceinline__ void shared8(const char* from, float (&x)[8]) {
  const uint4 a = *reinterpret_cast<const uint4*>(from);
  if constexpr (DT == LORDO_F32) {
    const uint4 b = *reinterpret_cast<const uint4*>(from + 512);
    x[0] = __uint_as_float(a.x); x[1] = __uint_as_float(a.y); x[2] = __uint_as_float(a.z); x[3] = __uint_as_float(a.w);
    x[4] = __uint_as_float(b.x); x[5] = __uint_as_float(b.y); x[6] = __uint_as_float(b.z); x[7] = __uint_as_float(b.w);
  } else {
    const unsigned w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[2 * j] = __uint_as_float(w[j] << 16);
      x[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
    }
  }
}

// Whole blocks b0 + warp, + 8, ... below b1 (at most 32 of a warp), eight elements a lane, all of it aligned. A lane copies what it will use to its
// warp's ring in shared memory, some blocks ahead; no other lane touches that.
constexpr int kRing8 = 48 * 1024;
template <int WDT, int GDT>
__device__ __forceinline__ void step8_blocks(const Arrays8& a, const Step8& s, unsigned long long key, long long b0, long long b1, int lane, int warp, char* ring) {
  constexpr int kW = WDT == LORDO_F32 ? 1024 : 512, kG = GDT == LORDO_F32 ? 1024 : 512, kStage = kW + kG + 512, kStages = kRing8 / 8 / kStage;
  const long long first = b0 + warp;
  if (first >= b1) return;
  const int count = (int)((b1 - first + 7) / 8);
  const int mcodes = lane < count ? a.ms[first + 8 * lane] : 1, vcodes = lane < count ? a.vs[first + 8 * lane] : 1;
  char* mine = ring + warp * (kStages * kStage);
  const unsigned at = (unsigned)__cvta_generic_to_shared(mine);
  const long long e0 = first * kAwBlock + 8 * lane;
  auto fetch = [&](int x, int slot) {
    if (x < count) {
      const long long e = e0 + (long long)x * (8 * kAwBlock);
      const unsigned to = at + slot * kStage;
      copy8<WDT>(to + 16 * lane, a.W, e);
      copy8<GDT>(to + kW + 16 * lane, a.G, e);
      copy_async<8>(to + kW + kG + 8 * lane, a.m + e);
      copy_async<8>(to + kW + kG + 256 + 8 * lane, a.v + e);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int x = 0; x < kStages - 1; ++x) fetch(x, x);
  unsigned long long counter = counter4(key, e0);
  int slot = 0, into = kStages - 1;
  for (int x = 0; x < count; ++x) {
    fetch(x + kStages - 1, into);
    asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
    const char* p = mine + slot * kStage;
    float g[8], w[8];
    shared8<WDT>(p + 16 * lane, w);
    shared8<GDT>(p + kW + 16 * lane, g);
    const uint2 y = *reinterpret_cast<const uint2*>(p + kW + kG + 8 * lane), z = *reinterpret_cast<const uint2*>(p + kW + kG + 256 + 8 * lane);
    unsigned mc[2] = {y.x, y.y}, vc[2] = {z.x, z.y};
    int mcode = __shfl_sync(0xffffffffu, mcodes, x), vcode = __shfl_sync(0xffffffffu, vcodes, x);
    step8_lane(s, counter, g, w, mc, vc, mcode, vcode);
    const long long e = e0 + (long long)x * (8 * kAwBlock);
    store8<WDT>(a.W, e, w);
    *reinterpret_cast<uint2*>(a.m + e) = make_uint2(mc[0], mc[1]);
    *reinterpret_cast<uint2*>(a.v + e) = make_uint2(vc[0], vc[1]);
    if (lane == 0) {
      a.ms[first + 8 * x] = (unsigned char)mcode;
      a.vs[first + 8 * x] = (unsigned char)vcode;
    }
    counter += kGolden * (8 * kAwBlock / 4);
    slot = slot + 1 == kStages ? 0 : slot + 1;
    into = into + 1 == kStages ? 0 : into + 1;
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");
}

template <int WDT, int GDT>
__global__ void __launch_bounds__(256) adamw_step8_kernel(const __grid_constant__ AwTable tab, AwLaunch l, const float* __restrict__ coef, int stride, AwStep a) {
  __shared__ __align__(16) char ring[kRing8];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int k = (int)(blockIdx.x / l.units);
  const unsigned q = blockIdx.x - (unsigned)k * l.units;
  const int i = find_tensor(tab.start, l.count, q);
  const AwTensor T = l.tensors[i];
  const void* G = tab.G[i];
  const unsigned long long key = mix64(a.key + kGolden * ((unsigned long long)T.index * l.K + k + 1));
  Step8 s;
  s.b1 = a.b1; s.a1 = a.a1; s.b2 = a.b2; s.a2 = a.a2; s.root_inv_bc2 = a.root_inv_bc2; s.eps = a.eps;
  s.keep = 1.f - a.lr * T.wd; s.lm = a.lr * a.omega * a.inv_bc1; s.lg = a.lr * a.a_omega;
  dep_begin();
  s.c = coef ? __ldcg(coef + (long long)T.index * stride + k) : 1.f;
  const long long base = (long long)k * T.n;
  Arrays8 x;
  x.G = G ? reinterpret_cast<const char*>(G) + base * (GDT == LORDO_F32 ? 4 : 2) : nullptr;
  x.W = reinterpret_cast<char*>(T.W) + base * (WDT == LORDO_F32 ? 4 : 2);
  x.m = reinterpret_cast<unsigned char*>(T.m) + base;
  x.v = reinterpret_cast<unsigned char*>(T.v) + base;
  x.ms = T.ms + (long long)k * T.nb;
  x.vs = T.vs + (long long)k * T.nb;
  long long b0 = (long long)(q - tab.start[i]) * (l.piece / kAwBlock);
  const long long b1 = b0 + l.piece / kAwBlock < T.nb ? b0 + l.piece / kAwBlock : T.nb;
  if (G && (base & 7) == 0) {
    const long long whole = T.n / kAwBlock < b1 ? T.n / kAwBlock : b1;
    step8_blocks<WDT, GDT>(x, s, key, b0, whole, lane, warp, ring);
    b0 = whole > b0 ? whole : b0;
  }
  // the last block of a worker, workers whose arrays begin at odd addresses, gradients by tokens
  for (long long b = b0 + warp; b < b1; b += 8) {
    const long long e = b * kAwBlock + 8 * lane;
    const bool vec = (base & 7) == 0 && e + 8 <= T.n;
    int mcode = x.ms[b], vcode = x.vs[b];
    float g[8], w[8];
    unsigned mc[2] = {0u, 0u}, vc[2] = {0u, 0u};
    if (vec) {
      if (G) load8<GDT>(x.G, e, g); else row_grad8(T, k, e, g);
      load8<WDT>(x.W, e, w);
      const uint2 y = *reinterpret_cast<const uint2*>(x.m + e), z = *reinterpret_cast<const uint2*>(x.v + e);
      mc[0] = y.x; mc[1] = y.y; vc[0] = z.x; vc[1] = z.y;
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        g[j] = w[j] = 0.f;
        if (e + j < T.n) {
          g[j] = G ? load1(x.G, GDT, e + j) : row_grad(T, k, e + j);
          w[j] = load1(x.W, WDT, e + j);
          mc[j >> 2] |= (unsigned)x.m[e + j] << (8 * (j & 3));
          vc[j >> 2] |= (unsigned)x.v[e + j] << (8 * (j & 3));
        }
      }
    }
    step8_lane(s, counter4(key, e), g, w, mc, vc, mcode, vcode);
    if (vec) {
      store8<WDT>(x.W, e, w);
      *reinterpret_cast<uint2*>(x.m + e) = make_uint2(mc[0], mc[1]);
      *reinterpret_cast<uint2*>(x.v + e) = make_uint2(vc[0], vc[1]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (e + j < T.n) {
          store1(x.W, WDT, e + j, w[j]);
          x.m[e + j] = (unsigned char)(mc[j >> 2] >> (8 * (j & 3)));
          x.v[e + j] = (unsigned char)(vc[j >> 2] >> (8 * (j & 3)));
        }
      }
    }
    if (lane == 0) {  // every lane has read the old scales before the reductions
      x.ms[b] = (unsigned char)mcode;
      x.vs[b] = (unsigned char)vcode;
    }
  }
}

// ---------------------------------------------------------------------------------------------
// Outer synchronisation: moments <- mean over the workers; D = X0 - mean W; average: X0 <- X0 - D; Nesterov: B <- mu B + D,
// X0 <- X0 - eta (D + mu B); every W_k <- X0. Each operation is rounded on its own: with bf16 weights D of the next synchronisation is
// what X0 loses in its cast, and a last bit that depends on what a compiler fuses would become a whole step of bf16 there.
// ---------------------------------------------------------------------------------------------
template <int WDT, int N>  // N consecutive elements of every worker: 4 (a float4's alignment everywhere) or 1
__device__ __forceinline__ void outer_weights(const AwTensor& T, int K, const AwOuter& o, float inv_k, long long e) {
  float s[N] = {}, x0[N], b[N];
#pragma unroll 4
  for (int k = 0; k < K; ++k) {
    if constexpr (N == 4) {
      const float4 w = load4(T.W, WDT, (long long)k * T.n + e);
      s[0] += w.x; s[1] += w.y; s[2] += w.z; s[3] += w.w;
    } else {
      s[0] += load1(T.W, WDT, (long long)k * T.n + e);
    }
  }
#pragma unroll
  for (int j = 0; j < N; ++j) {
    x0[j] = T.X0[e + j];
    const float d = __fsub_rn(x0[j], __fmul_rn(s[j], inv_k));
    if (o.nesterov) {
      b[j] = __fadd_rn(__fmul_rn(o.mu, T.B[e + j]), d);
      x0[j] = __fsub_rn(x0[j], __fmul_rn(o.eta, __fadd_rn(d, __fmul_rn(o.mu, b[j]))));
    } else {
      x0[j] -= d;
    }
  }
#pragma unroll
  for (int j = 0; j < N; ++j) {
    T.X0[e + j] = x0[j];
    if (o.nesterov) T.B[e + j] = b[j];
  }
#pragma unroll 4
  for (int k = 0; k < K; ++k) {
    if constexpr (N == 4) store4(T.W, WDT, (long long)k * T.n + e, make_float4(x0[0], x0[1], x0[2], x0[3]));
    else store1(T.W, WDT, (long long)k * T.n + e, x0[0]);
  }
}

template <int N>
__device__ __forceinline__ void outer_mean(float* p, long long n, int K, float inv_k, long long e) {
  float s[N] = {};
#pragma unroll 4
  for (int k = 0; k < K; ++k) {
    if constexpr (N == 4) {
      const float4 x = *reinterpret_cast<const float4*>(p + (long long)k * n + e);
      s[0] += x.x; s[1] += x.y; s[2] += x.z; s[3] += x.w;
    } else {
      s[0] += p[(long long)k * n + e];
    }
  }
#pragma unroll
  for (int j = 0; j < N; ++j) s[j] *= inv_k;
#pragma unroll 4
  for (int k = 0; k < K; ++k) {
    if constexpr (N == 4) *reinterpret_cast<float4*>(p + (long long)k * n + e) = make_float4(s[0], s[1], s[2], s[3]);
    else p[(long long)k * n + e] = s[0];
  }
}

template <int WDT>
__global__ void __launch_bounds__(256) adamw_outer_kernel(AwLaunch l, const unsigned* __restrict__ start, AwOuter o) {
  const int i = find_tensor(start, l.count, blockIdx.x);
  const AwTensor T = l.tensors[i];
  dep_begin();
  const float inv_k = 1.f / (float)l.K;
  const long long e0 = (long long)(blockIdx.x - start[i]) * kAwOuter;
  const long long e1 = e0 + kAwOuter < T.n ? e0 + kAwOuter : T.n;
  if (T.n % 4 == 0) {
    for (long long e = e0 + 4 * threadIdx.x; e < e1; e += 1024) {
      outer_weights<WDT, 4>(T, l.K, o, inv_k, e);
      if (o.sync_m) outer_mean<4>(reinterpret_cast<float*>(T.m), T.n, l.K, inv_k, e);
      if (o.sync_v) outer_mean<4>(reinterpret_cast<float*>(T.v), T.n, l.K, inv_k, e);
    }
  } else {
    for (long long e = e0 + threadIdx.x; e < e1; e += 256) {
      outer_weights<WDT, 1>(T, l.K, o, inv_k, e);
      if (o.sync_m) outer_mean<1>(reinterpret_cast<float*>(T.m), T.n, l.K, inv_k, e);
      if (o.sync_v) outer_mean<1>(reinterpret_cast<float*>(T.v), T.n, l.K, inv_k, e);
    }
  }
}

// Mean over the workers of one array of 8-bit moments, one block of 256 of every worker: a lane has eight elements.
template <bool SECOND>
__device__ __forceinline__ void outer_mean8(const AwTensor& T, int K, float inv_k, unsigned long long key, long long b, long long e, int left, int lane) {
  unsigned char* C = reinterpret_cast<unsigned char*>(SECOND ? T.v : T.m);
  unsigned char* S = SECOND ? T.vs : T.ms;
  const bool vec = left == 8 && (T.n & 7) == 0;
  float a[8] = {};
  for (int k = 0; k < K; ++k) {
    const float scale = pow2(S[(long long)k * T.nb + b]);
    const unsigned char* p = C + (long long)k * T.n + e;
    unsigned c[2] = {0u, 0u};
    if (vec) {
      const uint2 x = *reinterpret_cast<const uint2*>(p);
      c[0] = x.x; c[1] = x.y;
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j < left) c[j >> 2] |= (unsigned)p[j] << (8 * (j & 3));
    }
    float x[8];
    values8(c[0], x);
    values8(c[1], x + 4);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      x[j] *= scale;
      a[j] += SECOND ? x[j] * x[j] : x[j];
    }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    a[j] *= inv_k;
    if (SECOND) a[j] = root(a[j]);
  }
  const int code = scale_code(__reduce_max_sync(0xffffffffu, top8(a)));
  const float inv = pow2(254 - code);
  unsigned c[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const unsigned long long r = mix64(counter4(key, e) + h * kGolden);
    const unsigned u[4] = {first16(r, 0), first16(r, 1), first16(r, 2), first16(r, 3)};
    c[h] = pack8<SECOND, false>(a + 4 * h, inv, u);
  }
  for (int k = 0; k < K; ++k) {
    unsigned char* p = C + (long long)k * T.n + e;
    if (vec) {
      *reinterpret_cast<uint2*>(p) = make_uint2(c[0], c[1]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j < left) p[j] = (unsigned char)(c[j >> 2] >> (8 * (j & 3)));
    }
  }
  __syncwarp();  // every lane has read the scales
  for (int k = lane; k < K; k += 32) S[(long long)k * T.nb + b] = (unsigned char)code;
}

template <int WDT>
__global__ void __launch_bounds__(256) adamw_outer8_kernel(AwLaunch l, const unsigned* __restrict__ start, AwOuter o) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int i = find_tensor(start, l.count, blockIdx.x);
  const AwTensor T = l.tensors[i];
  const unsigned long long key = mix64(o.key + kGolden * ((unsigned long long)T.index + 1));
  dep_begin();
  const float inv_k = 1.f / (float)l.K;
  const long long b0 = (long long)(blockIdx.x - start[i]) * (kAwOuter / kAwBlock);
  for (int x = warp; x < kAwOuter / kAwBlock; x += 8) {
    const long long b = b0 + x;
    if (b >= T.nb) break;
    const long long at = b * kAwBlock, e = at + 8 * lane;
    const int left = e >= T.n ? 0 : T.n - e < 8 ? (int)(T.n - e) : 8;
    if (T.n % 4 == 0) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
        if (at + 128 * h + 4 * lane < T.n) outer_weights<WDT, 4>(T, l.K, o, inv_k, at + 128 * h + 4 * lane);
    } else {
      for (int j = lane; j < kAwBlock && at + j < T.n; j += 32) outer_weights<WDT, 1>(T, l.K, o, inv_k, at + j);
    }
    if (o.sync_m) outer_mean8<false>(T, l.K, inv_k, key, b, e, left, lane);
    if (o.sync_v) outer_mean8<true>(T, l.K, inv_k, key, b, e, left, lane);
  }
}

__global__ void __launch_bounds__(256) adamw_init_kernel(AwLaunch l, const unsigned* __restrict__ start) {
  const int i = find_tensor(start, l.count, blockIdx.x);
  const AwTensor T = l.tensors[i];
  const long long e0 = (long long)(blockIdx.x - start[i]) * kAwOuter;
  const long long e1 = e0 + kAwOuter < T.n ? e0 + kAwOuter : T.n;
  for (long long e = e0 + threadIdx.x; e < e1; e += 256) {
    const float w = load1(T.W, l.w_dt, e);
    if (T.X0) T.X0[e] = w;
    if (T.B) T.B[e] = 0.f;
    for (int k = 0; k < l.K; ++k) {
      const long long f = (long long)k * T.n + e;
      if (k) store1(T.W, l.w_dt, f, w);
      if (l.small) {
        reinterpret_cast<unsigned char*>(T.m)[f] = 0;
        reinterpret_cast<unsigned char*>(T.v)[f] = 0;
        if (e % kAwBlock == 0) T.ms[(long long)k * T.nb + e / kAwBlock] = T.vs[(long long)k * T.nb + e / kAwBlock] = 1;
      } else {
        reinterpret_cast<float*>(T.m)[f] = 0.f;
        reinterpret_cast<float*>(T.v)[f] = 0.f;
      }
    }
  }
}

}  // namespace

void launch_aw_norm(const AwLaunch& l, const AwTable& t, const AwClip& c, cudaStream_t st) {
  const dim3 grid(l.units * (unsigned)l.K);
  if (l.g_dt == LORDO_F32) launch_dep(adamw_norm_kernel<LORDO_F32>, grid, 256, 0, st, t, l, c);
  else launch_dep(adamw_norm_kernel<LORDO_BF16>, grid, 256, 0, st, t, l, c);
}

void launch_aw_step(const AwLaunch& l, const AwTable& t, const float* coef, int stride, const AwStep& s, cudaStream_t st) {
  const dim3 grid(l.units * (unsigned)l.K);
#define LORDO_AW(W, G)                                                                              \
  if (l.small) launch_dep(adamw_step8_kernel<W, G>, grid, 256, 0, st, t, l, coef, stride, s);       \
  else launch_dep(adamw_step_kernel<W, G>, grid, 256, 0, st, t, l, coef, stride, s)
  if (l.w_dt == LORDO_F32) {
    if (l.g_dt == LORDO_F32) { LORDO_AW(LORDO_F32, LORDO_F32); } else { LORDO_AW(LORDO_F32, LORDO_BF16); }
  } else {
    if (l.g_dt == LORDO_F32) { LORDO_AW(LORDO_BF16, LORDO_F32); } else { LORDO_AW(LORDO_BF16, LORDO_BF16); }
  }
#undef LORDO_AW
}

void launch_aw_outer(const AwLaunch& l, const unsigned* start, const AwOuter& o, cudaStream_t st) {
  const dim3 grid(l.units);
  if (l.small) {
    if (l.w_dt == LORDO_F32) launch_dep(adamw_outer8_kernel<LORDO_F32>, grid, 256, 0, st, l, start, o);
    else launch_dep(adamw_outer8_kernel<LORDO_BF16>, grid, 256, 0, st, l, start, o);
  } else {
    if (l.w_dt == LORDO_F32) launch_dep(adamw_outer_kernel<LORDO_F32>, grid, 256, 0, st, l, start, o);
    else launch_dep(adamw_outer_kernel<LORDO_BF16>, grid, 256, 0, st, l, start, o);
  }
}

void launch_aw_init(const AwLaunch& l, const unsigned* start, cudaStream_t st) {
  adamw_init_kernel<<<l.units, 256, 0, st>>>(l, start);
}

}  // namespace lordo
