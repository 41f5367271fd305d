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
// Row of element e, a multiple of 8, of such a table, whose rows are whole eighths.
__device__ __forceinline__ unsigned row_of(const AwTensor& T, long long e) {
  return (unsigned)(((unsigned long long)(unsigned)(e >> 3) * T.row_mul) >> (31 + T.row_shift));
}
__device__ __forceinline__ void row_grad8(const AwTensor& T, int k, long long e, float (&g)[8]) {
  if (T.row_mul) {
    const long long v = row_of(T, e);
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
    const long long e0 = (long long)(q - tab.start[i]) * c.chunk;
    const long long e1 = e0 + c.chunk < n ? e0 + c.chunk : n;
    const long long f0 = (long long)k * n + e0, f1 = (long long)k * n + e1;
    const long long a0 = (f0 + 7) & ~7ll, a1 = f1 & ~7ll;
    double part[2] = {0.0, 0.0};
    for (long long f = a0 + 8 * t; f < a1; f += 4 * 2048) {
      uint4 x[4][GDT == LORDO_F32 ? 2 : 1];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const uint4* p = reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(G) + (f + u * 2048) * (GDT == LORDO_F32 ? 4 : 2));
#pragma unroll
        for (int h = 0; h < (GDT == LORDO_F32 ? 2 : 1); ++h) x[u][h] = f + u * 2048 < a1 ? p[h] : make_uint4(0u, 0u, 0u, 0u);
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {  // eight squares in fp32, the rest in fp64
        float sum = 0.f;
#pragma unroll
        for (int h = 0; h < (GDT == LORDO_F32 ? 2 : 1); ++h) {
          const unsigned w[4] = {x[u][h].x, x[u][h].y, x[u][h].z, x[u][h].w};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if (GDT == LORDO_F32) {
              sum += __uint_as_float(w[j]) * __uint_as_float(w[j]);
            } else {
              const float lo = __uint_as_float(w[j] << 16), hi = __uint_as_float(w[j] & 0xFFFF0000u);
              sum += lo * lo + hi * hi;
            }
          }
        }
        part[u & 1] += (double)sum;
      }
    }
    s = part[0] + part[1];
    if (!(s < INFINITY)) {  // fp32 does not hold the squares of gradients above 6e18: the thread's once more, all in fp64
      s = 0.0;
      for (long long f = a0 + 8 * t; f < a1; f += 2048) {
        float g[8];
        load8<GDT>(G, f, g);
#pragma unroll
        for (int j = 0; j < 8; ++j) s += (double)g[j] * (double)g[j];
      }
    }
    const long long edge = t < 8 ? f0 + t : (a1 > a0 ? a1 : a0) + t - 8;  // elements before the first and behind the last vector
    if (t < 16 && edge < f1 && (t >= 8 || edge < a0)) {
      const float x = load1(G, GDT, edge);
      s += (double)x * (double)x;
    }
  } else {  // one chunk stands for the whole tensor
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
  const double ratio = c.rho / (sqrt(total) + 1e-6);
  const float coef = ratio >= 1.0 ? 1.f : (float)ratio;  // NaN stays what it is: fmin's 1 would leave the rest of a gradient that holds one unclipped
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

// E4M3 code of a magnitude t < 256, rounded down after (u + 1/2) / 65536 of a step was added; u256 = 256 u + 128. A float's own bits are that code
// once t is scaled by 2^-120: the exponent's bias becomes E4M3's, floats below 2^-126 are its subnormal codes, and three bits of the mantissa stand
// above 20 that are dropped. Infinities and NaN become NaN.
__device__ __forceinline__ unsigned code8(float t, unsigned u256) {
  const unsigned c = (__float_as_uint(fabsf(t) * 0x1p-120f) + (u256 >> 4)) >> 20;
  return c > 127u ? 127u : c;
}

// Four values of E4M3 codes.
__device__ __forceinline__ void values8(unsigned c, float2 (&x)[2]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const __half2_raw r = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(c >> (16 * h)), __NV_E4M3);
    x[h] = __half22float2(*reinterpret_cast<const __half2*>(&r));
  }
}

// 256 u + 128 of element j of four, u its 16 random bits: one byte permutation; the same for the second moment.
__device__ __forceinline__ unsigned first16(unsigned long long r, int j) {
  return __byte_perm(j < 2 ? (unsigned)r : (unsigned)(r >> 32), 0x00000080u, j & 1 ? 0x7324 : 0x7104);
}
__device__ __forceinline__ unsigned second16(unsigned first) { return (((first - 128u) * 40503u) & 0xFFFF00u) | 128u; }

// Bits of the largest magnitude of a lane's eight values, of either sign and of none below 0; of the least of the latter.
__device__ __forceinline__ unsigned top_signed(const float2 (&x)[4]) {
  int up = 0;
  unsigned down = 0u;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    up = __vimax3_s32(up, __float_as_int(x[j].x), __float_as_int(x[j].y));
    down = __vimax3_u32(down, __float_as_uint(x[j].x), __float_as_uint(x[j].y));
  }
  const unsigned low = down & 0x7FFFFFFFu;  // of the negative ones where there are any
  return (unsigned)up > low ? (unsigned)up : low;
}
__device__ __forceinline__ unsigned top_positive(const float2 (&x)[4]) {
  unsigned t = 0u;
#pragma unroll
  for (int j = 0; j < 4; ++j) t = __vimax3_u32(t, __float_as_uint(x[j].x), __float_as_uint(x[j].y));
  return t;
}
__device__ __forceinline__ unsigned low_positive(const float2 (&x)[4]) {
  unsigned t = 0xFFFFFFFFu;
#pragma unroll
  for (int j = 0; j < 4; ++j) t = __vimin3_u32(t, __float_as_uint(x[j].x), __float_as_uint(x[j].y));
  return t;
}

// Bits of the largest finite magnitude of a lane's eight values. A scale is formed of these where a block holds an infinity or NaN: those are lost in
// any case, and a scale that followed them (2^121) would take the block's other 255 moments along.
constexpr unsigned kInfinity = 0x7F800000u;
__device__ __forceinline__ unsigned top_finite(const float2 (&x)[4]) {
  unsigned t = 0u;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const unsigned b = __float_as_uint(j & 1 ? x[j >> 1].y : x[j >> 1].x) & 0x7FFFFFFFu;
    if (b < kInfinity && b > t) t = b;
  }
  return t;
}

// 16 x + y. Written out: as a shift by four, nvcc 12.9 lost it where x came from one half of a packed product and the result's top byte was taken.
__device__ __forceinline__ unsigned mad16(unsigned x, unsigned y) {
  unsigned r;
  asm("mad.lo.u32 %0, %1, 16, %2;" : "=r"(r) : "r"(x), "r"(y));
  return r;
}

enum Pack8 { PACK_SIGNED, PACK_POSITIVE, PACK_ANY };
// Codes of four values. inv is 2^-120 times the reciprocal of the scale for all but ANY, where it is that itself: there a value may be anything, and
// positive ones do not become zero with SECOND (the smallest code instead). u256: first16 of the four.
template <int KIND, bool SECOND>
__device__ __forceinline__ unsigned pack8(const float2 (&x)[2], float inv, const unsigned (&u256)[4]) {
  unsigned b[4];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const float2 t = KIND == PACK_ANY ? x[h] : __fmul2_rn(x[h], make_float2(inv, inv));
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const float y = j ? t.y : t.x;
      const unsigned u = SECOND ? second16(u256[2 * h + j]) : u256[2 * h + j];
      if (KIND == PACK_ANY) {
        unsigned c = code8(y * inv, u);
        if (SECOND && c == 0u && y > 0.f) c = 1u;
        b[2 * h + j] = (c << 24) | (SECOND ? 0u : __float_as_uint(y) & 0x80000000u);
      } else {
        const unsigned c = mad16(__float_as_uint(y), u);  // the code in bits 24 to 30
        b[2 * h + j] = KIND == PACK_SIGNED ? (c & 0x7FFFFFFFu) | (__float_as_uint(y) & 0x80000000u) : c;
      }
    }
  }
  return __byte_perm(__byte_perm(b[0], b[1], 0x0073), __byte_perm(b[2], b[3], 0x0073), 0x5410);  // the top byte of each
}

// sqrt(v) by one of Newton's (Heron's) steps on r^2 = v from r = v rsqrt(v), whose derivative 2 r is 2 / rsqrt(v): of normal numbers off by less than
// a unit in the last place, as a rule rounded to the nearest. The step is not a number for 0 (and below 2^-126), infinity and NaN; there, unless
// all are NORMAL, the maximum takes v 1e-20, which is 0, infinity and NaN, and below the root of any other v. No branch; sqrtf has one.
template <bool NORMAL>
__device__ __forceinline__ float2 root(float2 v) {
  float2 y;
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y.x) : "f"(v.x));
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y.y) : "f"(v.y));
  const float2 r = __fmul2_rn(v, y), minus = __fmul2_rn(v, make_float2(-y.x, -y.y));
  const float2 x = __ffma2_rn(__ffma2_rn(minus, r, v), __fmul2_rn(y, make_float2(0.5f, 0.5f)), r);
  if (NORMAL) return x;
  const float2 least = __fmul2_rn(v, make_float2(1e-20f, 1e-20f));
  return make_float2(fmaxf(x.x, least.x), fmaxf(x.y, least.y));
}
__device__ __forceinline__ float reciprocal(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

struct Step8 {  // constants of a step, of its worker and tensor
  float one, c, b1, a1, b2, a2, lw, lm, lg, root_inv_bc2, eps;
};

__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }

// What follows the moments: roots, weights, codes of a lane's eight elements. The change of a weight is formed apart and added once: a factor 1 - lr wd is
// rounded to 2^-24, a bias of every element and step that is larger than the decay itself where lr wd is small, and w times it is a second rounding of
// w (it takes half an instruction an element less, 1 % of the time of a step). v becomes its codes in vc. NORMAL: every v is a normal number whose root
// is at least the smallest code, and scales are below 2^7.
template <bool NORMAL, bool QHM>
__device__ __forceinline__ void finish8(const Step8& s, unsigned long long counter, const float2 (&g)[4], const float2 (&m)[4], const float2 (&v)[4],
                                        float2 (&w)[4], unsigned (&mc)[2], unsigned (&vc)[2], float mi, float vi) {
  const float2 lm = both(-s.lm), lg = both(-s.lg * s.c), lw = both(-s.lw), q = both(s.root_inv_bc2), eps = both(s.eps);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const unsigned long long x = mix64(counter + h * kGolden);
    unsigned u[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) u[j] = first16(x, j);
    const float2 mh[2] = {m[2 * h], m[2 * h + 1]}, rh[2] = {root<NORMAL>(v[2 * h]), root<NORMAL>(v[2 * h + 1])};
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int at = 2 * h + j;
      const float2 d = __ffma2_rn(rh[j], q, eps);
      float2 up = __fmul2_rn(lm, mh[j]);
      if (QHM) up = __ffma2_rn(lg, g[at], up);
      w[at] = __fadd2_rn(w[at], __ffma2_rn(up, make_float2(reciprocal(d.x), reciprocal(d.y)), __fmul2_rn(w[at], lw)));
    }
    mc[h] = NORMAL ? pack8<PACK_SIGNED, false>(mh, mi * 0x1p-120f, u) : pack8<PACK_ANY, false>(mh, mi, u);
    vc[h] = NORMAL ? pack8<PACK_POSITIVE, true>(rh, vi * 0x1p-120f, u) : pack8<PACK_ANY, true>(rh, vi, u);
  }
}

// A lane's eight elements of a block of 256 of one worker's tensor: codes in, codes and scales out. Arithmetic goes by pairs of elements in one
// instruction each (the issue slots are what a step is short of), every product and sum of the moments rounded on its own: a sum is p times one
// plus q, because nvcc 12.9 fuses a packed product with a packed sum that takes it, mul.rn.f32x2 with add.rn.f32x2 too. The scales are powers of two, so that
// b1 (m8 S) is (b1 S) m8 to the last bit, and b2 (s8 S)^2 is (b2 S^2) s8^2. The weights' quotient is good to two units in the last place.
template <bool QHM>
__device__ __forceinline__ void step8_lane(const Step8& s, unsigned long long counter, const float2 (&g)[4], float2 (&w)[4], unsigned (&mc)[2],
                                           unsigned (&vc)[2], int& mcode, int& vcode) {
  const float ms = pow2(mcode), vs = pow2(vcode);
  const float2 b1 = both(s.b1 * ms), b2 = both(s.b2 * (vs * vs)), c = both(s.c), a1 = both(s.a1), a2 = both(s.a2), one = both(s.one);
  float2 m[4], v[4];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float2 x[2], y[2];
    values8(mc[h], x);
    values8(vc[h], y);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int at = 2 * h + j;
      const float2 z = __fmul2_rn(g[at], c);
      m[at] = __ffma2_rn(__fmul2_rn(b1, x[j]), one, __fmul2_rn(a1, z));
      v[at] = __ffma2_rn(__fmul2_rn(b2, __fmul2_rn(y[j], y[j])), one, __fmul2_rn(__fmul2_rn(a2, z), z));
    }
  }
  unsigned mtop = __reduce_max_sync(0xffffffffu, top_signed(m)), vtop = __reduce_max_sync(0xffffffffu, top_positive(v));
  const bool lost = (mtop > vtop ? mtop : vtop) >= kInfinity;
  if (lost) {
    mtop = __reduce_max_sync(0xffffffffu, top_finite(m));
    vtop = __reduce_max_sync(0xffffffffu, top_finite(v));
  }
  const float rtop = root<false>(both(__uint_as_float(vtop))).x;
  mcode = scale_code(mtop);
  vcode = scale_code(__float_as_uint(rtop));
  const float mi = pow2(254 - mcode), vi = pow2(254 - vcode);
  // scales above 2^6 (their reciprocal's 2^-120 would not be a normal number), infinities, NaN; v whose root is below the smallest code, or not normal
  constexpr unsigned kLarge = (127u + 14u) << 23;
  const float least = fmaxf(0x1p-18f * (pow2(vcode) * pow2(vcode)), 0x1p-126f);
  const bool slow = lost || mtop >= kLarge || __float_as_uint(rtop) >= kLarge || __any_sync(0xffffffffu, __uint_as_float(low_positive(v)) < least);
  if (!slow) {
    finish8<true, QHM>(s, counter, g, m, v, w, mc, vc, mi, vi);
  } else if (lost || (mtop | vtop)) {
    finish8<false, QHM>(s, counter, g, m, v, w, mc, vc, mi, vi);
  } else {  // a block that never had a gradient
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = __ffma2_rn(w[j], both(-s.lw), w[j]);
    mc[0] = mc[1] = vc[0] = vc[1] = 0u;
  }
}

struct Arrays8 {  // of one worker
  const void* G;
  void* W;
  unsigned char *m, *v, *ms, *vs;
  const int2* segs;   // with a gradient by tokens
  const float* rows;
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
__device__ __forceinline__ void widen8(const uint4& a, const uint4& b, float2 (&x)[4]) {  // b: fp32 only
  if constexpr (DT == LORDO_F32) {
    x[0] = make_float2(__uint_as_float(a.x), __uint_as_float(a.y)); x[1] = make_float2(__uint_as_float(a.z), __uint_as_float(a.w));
    x[2] = make_float2(__uint_as_float(b.x), __uint_as_float(b.y)); x[3] = make_float2(__uint_as_float(b.z), __uint_as_float(b.w));
  } else {
    const unsigned w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = make_float2(__uint_as_float(w[j] << 16), __uint_as_float(w[j] & 0xFFFF0000u));
  }
}
template <int DT>
__device__ __forceinline__ void shared8(const char* from, float2 (&x)[4]) {
  widen8<DT>(*reinterpret_cast<const uint4*>(from), DT == LORDO_F32 ? *reinterpret_cast<const uint4*>(from + 512) : uint4{}, x);
}
template <int DT>
__device__ __forceinline__ void put8(char* to, const float2 (&x)[4]) {
  if constexpr (DT == LORDO_F32) {
    reinterpret_cast<float4*>(to)[0] = make_float4(x[0].x, x[0].y, x[1].x, x[1].y);
    reinterpret_cast<float4*>(to)[1] = make_float4(x[2].x, x[2].y, x[3].x, x[3].y);
  } else {
    *reinterpret_cast<uint4*>(to) = make_uint4(pack_bf16x2(x[0].x, x[0].y), pack_bf16x2(x[1].x, x[1].y), pack_bf16x2(x[2].x, x[2].y), pack_bf16x2(x[3].x, x[3].y));
  }
}

// Whole blocks b0 + warp, + 8, ... below b1 (at most 32 of a warp), eight elements a lane, all of it aligned. A lane copies what it will use to its
// warp's ring in shared memory, some blocks ahead; no other lane touches that.
// ROWS: the gradient is in rows that were summed by token (fp32); which row a lane wants of a block is looked up a block ahead of the copies.
constexpr int kRing8 = 48 * 1024;
template <int WDT, int GDT, bool ROWS, bool QHM>
__device__ __forceinline__ void step8_blocks(const AwTensor& T, const Arrays8& a, const Step8& s, unsigned long long key, long long b0, long long b1, int lane, int warp, char* ring) {
  constexpr int kWb = WDT == LORDO_F32 ? 4 : 2, kGb = GDT == LORDO_F32 ? 4 : 2, kStep = 8 * kAwBlock;  // elements from block to block
  constexpr int kM = 256 * (kWb + kGb), kStage = kM + 512, kStages = kRing8 / 8 / kStage;
  const long long first = b0 + warp;
  if (first >= b1) return;
  const int count = (int)((b1 - first + 7) / 8);
  int mcodes = lane < count ? a.ms[first + 8 * lane] : 1, vcodes = lane < count ? a.vs[first + 8 * lane] : 1;
  const long long e0 = first * kAwBlock + 8 * lane;
  char* mine = ring + warp * (kStages * kStage) + 16 * lane;  // of W and G; codes 8 * lane in
  const unsigned at = (unsigned)__cvta_generic_to_shared(mine);
  char* pw = reinterpret_cast<char*>(a.W) + e0 * kWb;
  const char* pg = reinterpret_cast<const char*>(a.G) + e0 * kGb;
  unsigned char *pm = a.m + e0, *pv = a.v + e0;
  const float* row = nullptr;  // of the next block that is fetched, or null: no token
  auto look_up = [&](unsigned x) {
    if (ROWS && x < count) {
      const long long e = e0 + x * kStep;
      const unsigned v = row_of(T, e);
      const int2 seg = __ldg(a.segs + v);
      row = seg.x < seg.y ? a.rows + (long long)seg.x * T.d + (e - (long long)v * T.d) : nullptr;
    }
  };
  auto fetch = [&](unsigned slot) {
    copy8<WDT>(at + slot, pw, 0);
    if (!ROWS) {
      copy8<GDT>(at + slot + 256 * kWb, pg, 0);
    } else if (row) {
      copy8<GDT>(at + slot + 256 * kWb, row, 0);
    } else {
      float4* p = reinterpret_cast<float4*>(mine + slot + 256 * kWb);
      p[0] = p[32] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    copy_async<8>(at + slot + kM - 8 * lane, pm);
    copy_async<8>(at + slot + kM + 256 - 8 * lane, pv);
  };
  auto advance = [&]() {
    pw += kStep * kWb;
    pg += kStep * kGb;
    pm += kStep;
    pv += kStep;
  };
  look_up(0);
#pragma unroll
  for (int x = 0; x < kStages - 1; ++x) {
    if (x < count) fetch(x * kStage);
    look_up(x + 1);
    asm volatile("cp.async.commit_group;" ::: "memory");
    advance();
  }
  unsigned long long counter = counter4(key, e0);
  unsigned slot = 0, into = (kStages - 1) * kStage;
  for (int x = 0; x < count; ++x) {
    if (x + kStages - 1 < count) fetch(into);
    look_up(x + kStages);
    asm volatile("cp.async.commit_group;\ncp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
    const char* p = mine + slot;
    float2 g[4], w[4];
    shared8<WDT>(p, w);
    shared8<GDT>(p + 256 * kWb, g);
    const uint2 y = *reinterpret_cast<const uint2*>(p + kM - 8 * lane), z = *reinterpret_cast<const uint2*>(p + kM + 256 - 8 * lane);
    unsigned mc[2] = {y.x, y.y}, vc[2] = {z.x, z.y};
    int mcode = __shfl_sync(0xffffffffu, mcodes, x), vcode = __shfl_sync(0xffffffffu, vcodes, x);
    step8_lane<QHM>(s, counter, g, w, mc, vc, mcode, vcode);
    constexpr int kBack = (kStages - 1) * kStep;
    put8<WDT>(pw - kBack * kWb, w);
    *reinterpret_cast<uint2*>(pm - kBack) = make_uint2(mc[0], mc[1]);
    *reinterpret_cast<uint2*>(pv - kBack) = make_uint2(vc[0], vc[1]);
    if (lane == x) {
      mcodes = mcode;
      vcodes = vcode;
    }
    advance();
    counter += kGolden * (kStep / 4);
    into = slot;
    slot = slot + kStage == kStages * kStage ? 0u : slot + kStage;
  }
  if (lane < count) {
    a.ms[first + 8 * lane] = (unsigned char)mcodes;
    a.vs[first + 8 * lane] = (unsigned char)vcodes;
  }
}

template <int WDT, int GDT, bool QHM>
__global__ void __launch_bounds__(256, 4) adamw_step8_kernel(const __grid_constant__ AwTable tab, AwLaunch l, const float* __restrict__ coef, int stride, AwStep a) {
  __shared__ __align__(16) char ring[kRing8];
  const int lane = threadIdx.x & 31, warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0);  // the compiler sees that a warp has one
  const int k = (int)(blockIdx.x / l.units);
  const unsigned q = blockIdx.x - (unsigned)k * l.units;
  const int i = find_tensor(tab.start, l.count, q);
  const AwTensor T = l.tensors[i];
  const void* G = tab.G[i];
  const unsigned long long key = mix64(a.key + kGolden * ((unsigned long long)T.index * l.K + k + 1));
  Step8 s;
  s.one = a.one; s.b1 = a.b1; s.a1 = a.a1; s.b2 = a.b2; s.a2 = a.a2; s.root_inv_bc2 = a.root_inv_bc2; s.eps = a.eps;
  s.lw = a.lr * T.wd; s.lm = a.lr * a.omega * a.inv_bc1; s.lg = a.lr * a.a_omega;
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
  x.segs = T.segs + (G || !T.d ? 0 : (long long)k * (T.n / T.d));
  x.rows = T.rows + (long long)k * T.cap * T.d;
  if ((base & 7) == 0 && (G || T.row_mul)) {
    const long long whole = T.n / kAwBlock < b1 ? T.n / kAwBlock : b1;
    if (G) step8_blocks<WDT, GDT, false, QHM>(T, x, s, key, b0, whole, lane, warp, ring);
    else step8_blocks<WDT, LORDO_F32, true, QHM>(T, x, s, key, b0, whole, lane, warp, ring);
    b0 = whole > b0 ? whole : b0;
  }
  // the last block of a worker, workers whose arrays begin at odd addresses, gradients by tokens
  for (long long b = b0 + warp; b < b1; b += 8) {
    const long long e = b * kAwBlock + 8 * lane;
    const bool vec = (base & 7) == 0 && e + 8 <= T.n;
    int mcode = x.ms[b], vcode = x.vs[b];
    float ge[8], we[8];
    unsigned mc[2] = {0u, 0u}, vc[2] = {0u, 0u};
    if (vec) {
      if (G) load8<GDT>(x.G, e, ge); else row_grad8(T, k, e, ge);
      load8<WDT>(x.W, e, we);
      const uint2 y = *reinterpret_cast<const uint2*>(x.m + e), z = *reinterpret_cast<const uint2*>(x.v + e);
      mc[0] = y.x; mc[1] = y.y; vc[0] = z.x; vc[1] = z.y;
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        ge[j] = we[j] = 0.f;
        if (e + j < T.n) {
          ge[j] = G ? load1(x.G, GDT, e + j) : row_grad(T, k, e + j);
          we[j] = load1(x.W, WDT, e + j);
          mc[j >> 2] |= (unsigned)x.m[e + j] << (8 * (j & 3));
          vc[j >> 2] |= (unsigned)x.v[e + j] << (8 * (j & 3));
        }
      }
    }
    float2 g[4], w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      g[j] = make_float2(ge[2 * j], ge[2 * j + 1]);
      w[j] = make_float2(we[2 * j], we[2 * j + 1]);
    }
    step8_lane<QHM>(s, counter4(key, e), g, w, mc, vc, mcode, vcode);
    if (vec) {
      put8<WDT>(reinterpret_cast<char*>(x.W) + e * (WDT == LORDO_F32 ? 4 : 2), w);
      *reinterpret_cast<uint2*>(x.m + e) = make_uint2(mc[0], mc[1]);
      *reinterpret_cast<uint2*>(x.v + e) = make_uint2(vc[0], vc[1]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (e + j < T.n) {
          store1(x.W, WDT, e + j, j & 1 ? w[j >> 1].y : w[j >> 1].x);
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
// The three arrays of a tensor (weights, first, second moments) are blocks of their own, blockIdx.y, of 2048 elements of all workers. What counts is
// how many loads an SM has under way: 50304 x 768, K = 8, fp32 moments 1032 us with eight blocks an SM (32 registers), 1064 with six, 1074 with
// four, 1117 with one block of 4096 for all three arrays; 8-bit moments 610, with eight blocks (spilling) 645, with four 657.
constexpr int kOuterItems = 2;  // per thread, at a distance of a block's threads: all their loads of a worker are under way together

template <int WDT, int N>  // N consecutive elements of every worker: 4 (a float4's alignment everywhere) or 1
__device__ __forceinline__ void outer_weights(const AwTensor& T, int K, const AwOuter& o, float inv_k, long long e0, long long e1) {
  float s[kOuterItems][N] = {};
  for (int k = 0; k < K; ++k) {
#pragma unroll
    for (int x = 0; x < kOuterItems; ++x) {
      const long long e = e0 + x * 256 * N;
      if (e >= e1) break;
      if constexpr (N == 4) {
        const float4 w = load4(T.W, WDT, (long long)k * T.n + e);
        s[x][0] += w.x; s[x][1] += w.y; s[x][2] += w.z; s[x][3] += w.w;
      } else {
        s[x][0] += load1(T.W, WDT, (long long)k * T.n + e);
      }
    }
  }
#pragma unroll
  for (int x = 0; x < kOuterItems; ++x) {
    const long long e = e0 + x * 256 * N;
    if (e >= e1) break;
    float x0[N], b[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
      x0[j] = T.X0[e + j];
      const float d = __fsub_rn(x0[j], __fmul_rn(s[x][j], inv_k));
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
      s[x][j] = x0[j];
    }
  }
  for (int k = 0; k < K; ++k) {
#pragma unroll
    for (int x = 0; x < kOuterItems; ++x) {
      const long long e = e0 + x * 256 * N;
      if (e >= e1) break;
      if constexpr (N == 4) store4(T.W, WDT, (long long)k * T.n + e, make_float4(s[x][0], s[x][1 % N], s[x][2 % N], s[x][3 % N]));
      else store1(T.W, WDT, (long long)k * T.n + e, s[x][0]);
    }
  }
}

template <int N>
__device__ __forceinline__ void outer_mean(float* p, long long n, int K, float inv_k, long long e0, long long e1) {
  float s[kOuterItems][N] = {};
  for (int k = 0; k < K; ++k) {
#pragma unroll
    for (int x = 0; x < kOuterItems; ++x) {
      const long long e = e0 + x * 256 * N;
      if (e >= e1) break;
      if constexpr (N == 4) {
        const float4 v = *reinterpret_cast<const float4*>(p + (long long)k * n + e);
        s[x][0] += v.x; s[x][1] += v.y; s[x][2] += v.z; s[x][3] += v.w;
      } else {
        s[x][0] += p[(long long)k * n + e];
      }
    }
  }
#pragma unroll
  for (int x = 0; x < kOuterItems; ++x)
#pragma unroll
    for (int j = 0; j < N; ++j) s[x][j] *= inv_k;
  for (int k = 0; k < K; ++k) {
#pragma unroll
    for (int x = 0; x < kOuterItems; ++x) {
      const long long e = e0 + x * 256 * N;
      if (e >= e1) break;
      if constexpr (N == 4) *reinterpret_cast<float4*>(p + (long long)k * n + e) = make_float4(s[x][0], s[x][1 % N], s[x][2 % N], s[x][3 % N]);
      else p[(long long)k * n + e] = s[x][0];
    }
  }
}

// Eight codes of a lane, at p; WHOLE: of a whole block at an address that is a multiple of 8, else `left` of them.
template <bool WHOLE>
__device__ __forceinline__ uint2 load_codes(const unsigned char* p, int left) {
  if constexpr (WHOLE) {
    return *reinterpret_cast<const uint2*>(p);
  } else {
    unsigned c[2] = {0u, 0u};
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < left) c[j >> 2] |= (unsigned)p[j] << (8 * (j & 3));
    return make_uint2(c[0], c[1]);
  }
}
template <bool WHOLE>
__device__ __forceinline__ void store_codes(unsigned char* p, int left, const unsigned (&c)[2]) {
  if constexpr (WHOLE) {
    *reinterpret_cast<uint2*>(p) = make_uint2(c[0], c[1]);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < left) p[j] = (unsigned char)(c[j >> 2] >> (8 * (j & 3)));
  }
}

// Mean over the workers of a block of 256 of 8-bit moments: a lane has eight elements; four workers' codes are under way together.
template <bool SECOND, bool WHOLE>
__device__ __forceinline__ void outer_mean8(const AwTensor& T, int K, float inv_k, unsigned long long key, long long b, int lane) {
  const long long e = b * kAwBlock + 8 * lane;
  unsigned char* C = reinterpret_cast<unsigned char*>(SECOND ? T.v : T.m) + e;
  unsigned char* S = (SECOND ? T.vs : T.ms) + b;
  const int left = e >= T.n ? 0 : T.n - e < 8 ? (int)(T.n - e) : 8;
  float2 a[4] = {};
  auto add = [&](uint2 c, int scale) {
    const float2 s = both(pow2(scale));
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float2 z[2];
      values8(h ? c.y : c.x, z);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float2 y = __fmul2_rn(z[j], s);
        a[2 * h + j] = SECOND ? __ffma2_rn(y, y, a[2 * h + j]) : __fadd2_rn(a[2 * h + j], y);
      }
    }
  };
  int k = 0;
  for (; k + 4 <= K; k += 4) {
    uint2 c[4];
    int scale[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      c[x] = load_codes<WHOLE>(C + (long long)(k + x) * T.n, left);
      scale[x] = S[(long long)(k + x) * T.nb];
    }
#pragma unroll
    for (int x = 0; x < 4; ++x) add(c[x], scale[x]);
  }
  for (; k < K; ++k) add(load_codes<WHOLE>(C + (long long)k * T.n, left), S[(long long)k * T.nb]);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    a[j] = __fmul2_rn(a[j], both(inv_k));
    if (SECOND) a[j] = root<false>(a[j]);
  }
  unsigned top = __reduce_max_sync(0xffffffffu, SECOND ? top_positive(a) : top_signed(a));
  if (top >= kInfinity) top = __reduce_max_sync(0xffffffffu, top_finite(a));
  const int code = scale_code(top);
  const float inv = pow2(254 - code);
  unsigned c[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const unsigned long long r = mix64(counter4(key, e) + h * kGolden);
    const unsigned u[4] = {first16(r, 0), first16(r, 1), first16(r, 2), first16(r, 3)};
    const float2 x[2] = {a[2 * h], a[2 * h + 1]};
    c[h] = pack8<PACK_ANY, SECOND>(x, inv, u);
  }
  for (k = 0; k < K; ++k) store_codes<WHOLE>(C + (long long)k * T.n, left, c);
  __syncwarp();  // every lane has read the scales
  for (k = lane; k < K; k += 32) S[(long long)k * T.nb] = (unsigned char)code;
}

template <int WDT, bool SMALL>
__global__ void __launch_bounds__(256, SMALL ? 6 : 8) adamw_outer_kernel(AwLaunch l, const unsigned* __restrict__ start, AwOuter o) {
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5, array = blockIdx.y;
  const int i = find_tensor(start, l.count, blockIdx.x);
  const AwTensor T = l.tensors[i];
  const unsigned long long key = mix64(o.key + kGolden * ((unsigned long long)T.index + 1));
  dep_begin();
  if ((array == 1 && !o.sync_m) || (array == 2 && !o.sync_v)) return;
  const float inv_k = 1.f / (float)l.K;
  const long long e0 = (long long)(blockIdx.x - start[i]) * l.piece;
  const long long e1 = e0 + l.piece < T.n ? e0 + l.piece : T.n;
  const bool four = T.n % 4 == 0;
  if (array && SMALL) {
    for (long long b = e0 / kAwBlock + warp; b * kAwBlock < e1; b += 8) {
      const bool whole = (T.n & 7) == 0 && (b + 1) * kAwBlock <= T.n;
      if (array == 1) {
        if (whole) outer_mean8<false, true>(T, l.K, inv_k, key, b, lane); else outer_mean8<false, false>(T, l.K, inv_k, key, b, lane);
      } else {
        if (whole) outer_mean8<true, true>(T, l.K, inv_k, key, b, lane); else outer_mean8<true, false>(T, l.K, inv_k, key, b, lane);
      }
    }
    return;
  }
  float* p = reinterpret_cast<float*>(array == 1 ? T.m : T.v);
  for (long long e = e0 + (four ? 4 * t : t); e < e1; e += kOuterItems * 256 * (four ? 4 : 1)) {
    if (four) {
      if (array == 0) outer_weights<WDT, 4>(T, l.K, o, inv_k, e, e1); else outer_mean<4>(p, T.n, l.K, inv_k, e, e1);
    } else {
      if (array == 0) outer_weights<WDT, 1>(T, l.K, o, inv_k, e, e1); else outer_mean<1>(p, T.n, l.K, inv_k, e, e1);
    }
  }
}

__global__ void __launch_bounds__(256) adamw_init_kernel(AwLaunch l, const unsigned* __restrict__ start) {
  const int i = find_tensor(start, l.count, blockIdx.x);
  const AwTensor T = l.tensors[i];
  const long long e0 = (long long)(blockIdx.x - start[i]) * l.piece;
  const long long e1 = e0 + l.piece < T.n ? e0 + l.piece : T.n;
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
  if (l.small && s.a_omega != 0.f) launch_dep(adamw_step8_kernel<W, G, true>, grid, 256, 0, st, t, l, coef, stride, s);  \
  else if (l.small) launch_dep(adamw_step8_kernel<W, G, false>, grid, 256, 0, st, t, l, coef, stride, s);                \
  else launch_dep(adamw_step_kernel<W, G>, grid, 256, 0, st, t, l, coef, stride, s)
  if (l.w_dt == LORDO_F32) {
    if (l.g_dt == LORDO_F32) { LORDO_AW(LORDO_F32, LORDO_F32); } else { LORDO_AW(LORDO_F32, LORDO_BF16); }
  } else {
    if (l.g_dt == LORDO_F32) { LORDO_AW(LORDO_BF16, LORDO_F32); } else { LORDO_AW(LORDO_BF16, LORDO_BF16); }
  }
#undef LORDO_AW
}

void launch_aw_outer(const AwLaunch& l, const unsigned* start, const AwOuter& o, cudaStream_t st) {
  const dim3 grid(l.units, 3);
  if (l.small) {
    if (l.w_dt == LORDO_F32) launch_dep(adamw_outer_kernel<LORDO_F32, true>, grid, 256, 0, st, l, start, o);
    else launch_dep(adamw_outer_kernel<LORDO_BF16, true>, grid, 256, 0, st, l, start, o);
  } else {
    if (l.w_dt == LORDO_F32) launch_dep(adamw_outer_kernel<LORDO_F32, false>, grid, 256, 0, st, l, start, o);
    else launch_dep(adamw_outer_kernel<LORDO_BF16, false>, grid, 256, 0, st, l, start, o);
  }
}

void launch_aw_init(const AwLaunch& l, const unsigned* start, cudaStream_t st) {
  adamw_init_kernel<<<l.units, 256, 0, st>>>(l, start);
}

}  // namespace lordo
