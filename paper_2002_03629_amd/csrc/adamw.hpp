// AdamW over many tensors (gfx950 only).
//
// Every element is read and written once and nothing is shared but an 8-bit block's scale: the step is bound by memory, 28
// bytes an element with fp32 weights, gradients and moments, 16 with moments in 8 bits.  What a call can lose is launches: a
// launch takes as many tensors as its arguments hold, cut into chunks that the workgroups find by a search over the
// chunks' counts, so that many small tensors cost one launch and no table in device memory.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/jacobi_adamw.h"

namespace jm {

typedef __attribute__((ext_vector_type(2))) uint32_t aw_u32x2;
typedef __attribute__((ext_vector_type(4))) uint32_t aw_u32x4;
typedef uint16_t aw_bf16;

constexpr int AW_TENSORS = 52;           // of a launch: 3.6 KB of arguments
constexpr int AW_THREADS = 256;
constexpr int AW_ITEMS = 4;              // quads of elements a thread takes, all requested before the first is used
constexpr int AW_CHUNK = AW_THREADS * 4 * AW_ITEMS;

struct AdamwTensor {
  void* p;
  const void* g;
  void* m;
  void* v;
  float* ms;
  float* vs;
  void* copy;
  long long n;
};

struct AdamwArgs {
  AdamwTensor t[AW_TENSORS];
  unsigned first[AW_TENSORS + 1];        // chunks of the tensors before
  int count;
  double lr, b1, b2, c1, c2, eps, wd, gs;
  const double* scalars;                 // {lr, c1, c2, gs} or NULL
};

// Tensor of chunk `id`: the last one whose first chunk is not behind it.
__device__ __forceinline__ int aw_find(const AdamwArgs& a, unsigned id) {
  int lo = 0, hi = a.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.first[mid] <= id) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// ---- four elements from `i` on, those below n; `whole`: the quad is aligned and complete
__device__ __forceinline__ void aw_load(const float* p, long long i, long long n, bool whole, float (&x)[4]) {
  if (whole) {
    const float4 f = *(const float4*)(p + i);
    x[0] = f.x; x[1] = f.y; x[2] = f.z; x[3] = f.w;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = i + e < n ? p[i + e] : 0.0f;
  }
}
__device__ __forceinline__ void aw_load(const aw_bf16* p, long long i, long long n, bool whole, float (&x)[4]) {
  if (whole) {
    const uint2 f = *(const uint2*)(p + i);
    x[0] = __uint_as_float(f.x << 16); x[1] = __uint_as_float(f.x & 0xffff0000u);
    x[2] = __uint_as_float(f.y << 16); x[3] = __uint_as_float(f.y & 0xffff0000u);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = i + e < n ? __uint_as_float((uint32_t)p[i + e] << 16) : 0.0f;
  }
}
__device__ __forceinline__ uint32_t aw_load(const uint8_t* p, long long i, long long n, bool whole) {
  if (whole) return *(const uint32_t*)(p + i);
  uint32_t x = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) x |= i + e < n ? (uint32_t)p[i + e] << 8 * e : 0u;
  return x;
}
__device__ __forceinline__ void aw_store(float* p, long long i, long long n, bool whole, const float (&x)[4]) {
  if (whole) {
    *(float4*)(p + i) = make_float4(x[0], x[1], x[2], x[3]);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (i + e < n) p[i + e] = x[e];
  }
}
__device__ __forceinline__ void aw_store(aw_bf16* p, long long i, long long n, bool whole, const float (&x)[4]) {
  typedef __attribute__((ext_vector_type(4))) __bf16 quad;
  const quad h = {(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3]};
  const uint2 w = __builtin_bit_cast(uint2, h);
  if (whole) {
    *(uint2*)(p + i) = w;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (i + e < n) p[i + e] = (aw_bf16)((e < 2 ? w.x : w.y) >> 16 * (e & 1));
  }
}
__device__ __forceinline__ void aw_store(uint8_t* p, long long i, long long n, bool whole, uint32_t x) {
  if (whole) {
    *(uint32_t*)(p + i) = x;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (i + e < n) p[i + e] = (uint8_t)(x >> 8 * e);
  }
}

// ---- 8-bit moments
constexpr double AW_M = 127.0 * 127.0, AW_V = 255.0 * 255.0 * 255.0 * 255.0;

// (the largest code's value is the scale itself: 127^2 and 255^4 times their rounded reciprocals are 1)
__device__ __forceinline__ double aw_value_m(int c, double scale) { return scale * ((double)(c * abs(c)) * (1.0 / AW_M)); }
__device__ __forceinline__ double aw_value_v(int c, double scale) {
  const double q = (double)(c * c);
  return scale * (q * q * (1.0 / AW_V));
}
static_assert(AW_M * (1.0 / AW_M) == 1.0 && AW_V * (1.0 / AW_V) == 1.0, "");

// b v + o x, every operation rounded by itself: moments that are decimal fractions of their scale meet ties of fp32, where a
// fused product would decide otherwise than the definition.
__device__ __forceinline__ double aw_average(double b, double v, double o, double x) {
#pragma clang fp contract(off)
  const double old = b * v, now = o * x;
  return old + now;
}

// The largest of a wave's values, none negative, by their bits: a NaN is above infinity and stays.
__device__ __forceinline__ float aw_wave_max(float x) {
  uint32_t b = __float_as_uint(x);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) b = max(b, (uint32_t)__shfl_xor((int)b, d));
  return __uint_as_float(b);
}

// The code of x = |moment| / scale (0 .. 1): floor(top * root(x) + 1/2).  The root is taken in fp32; where that lies within
// 2^-9 of the border to the next code (its error is below 2^-12 steps) the border itself decides, in 64 bits.
template <bool SECOND>
__device__ __forceinline__ int aw_code(double x) {
  const float f = (float)x;
  const float r = SECOND ? 255.0f * sqrtf(sqrtf(f)) : 127.0f * sqrtf(f);
  const float s = r + 0.5f, c = floorf(s), d = s - c;
  int code = (int)c;
  if (d < 0x1p-9f || d > 1.0f - 0x1p-9f) {
    // candidates: the code whose lower border is nearest
    const int k = (int)floorf(s + 0x1p-8f);                      // (the border is (k - 1/2) / top)
    const double b = (double)(2 * k - 1);
    const double border = SECOND ? b * b * (b * b) : b * b;
    const double y = SECOND ? x * (16.0 * AW_V) : x * (4.0 * AW_M);
    code = k > 0 && y < border ? k - 1 : k;
  }
  return min(code, SECOND ? 255 : 127);
}

struct AdamwNumbers {
  double b1, b2, one_b1, one_b2, gs;
  float lr_c1, c2, eps, keep;            // keep = 1 - lr wd
};

__device__ __forceinline__ AdamwNumbers aw_numbers(const AdamwArgs& a) {
  double lr = a.lr, c1 = a.c1, c2 = a.c2, gs = a.gs;
  if (a.scalars) {
    lr = a.scalars[0];
    c1 = a.scalars[1];
    c2 = a.scalars[2];
    gs = a.scalars[3];
  }
  AdamwNumbers k;
  k.b1 = a.b1;
  k.b2 = a.b2;
  k.one_b1 = 1.0 - a.b1;
  k.one_b2 = 1.0 - a.b2;
  k.gs = gs;
  k.lr_c1 = (float)(lr * c1);
  k.c2 = (float)c2;
  k.eps = (float)a.eps;
  k.keep = (float)(1.0 - lr * a.wd);
  return k;
}

__device__ __forceinline__ float aw_new(float p, float m, float v, const AdamwNumbers& k) {
  return p * k.keep - k.lr_c1 * m / (sqrtf(v * k.c2) + k.eps);
}

template <typename P, typename G>
__global__ __launch_bounds__(AW_THREADS) void adamw_kernel(AdamwArgs a) {
  const int which = aw_find(a, blockIdx.x);
  const AdamwTensor& t = a.t[which];
  const long long n = t.n, base = (long long)(blockIdx.x - a.first[which]) * AW_CHUNK;
  P* p = (P*)t.p;
  const G* g = (const G*)t.g;
  float *m = (float*)t.m, *v = (float*)t.v;
  aw_bf16* copy = (aw_bf16*)t.copy;
  const AdamwNumbers k = aw_numbers(a);
  const float b1 = (float)k.b1, b2 = (float)k.b2, o1 = (float)k.one_b1, o2 = (float)k.one_b2, gs = (float)k.gs;
  const bool whole = (((uintptr_t)m | (uintptr_t)v) & 15) == 0 && ((uintptr_t)p & (4 * sizeof(P) - 1)) == 0 &&
                     ((uintptr_t)g & (4 * sizeof(G) - 1)) == 0 && ((uintptr_t)copy & 7) == 0 && base + AW_CHUNK <= n;
  float pv[AW_ITEMS][4], gv[AW_ITEMS][4], mv[AW_ITEMS][4], vv[AW_ITEMS][4];
#pragma unroll
  for (int i = 0; i < AW_ITEMS; ++i) {
    const long long at = base + (long long)(i * AW_THREADS + threadIdx.x) * 4;
    aw_load(p, at, n, whole, pv[i]);
    aw_load(g, at, n, whole, gv[i]);
    aw_load(m, at, n, whole, mv[i]);
    aw_load(v, at, n, whole, vv[i]);
  }
#pragma unroll
  for (int i = 0; i < AW_ITEMS; ++i) {
    const long long at = base + (long long)(i * AW_THREADS + threadIdx.x) * 4;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float x = gv[i][e] * gs;
      mv[i][e] = b1 * mv[i][e] + o1 * x;
      vv[i][e] = b2 * vv[i][e] + o2 * (x * x);
      pv[i][e] = aw_new(pv[i][e], mv[i][e], vv[i][e], k);
    }
    aw_store(m, at, n, whole, mv[i]);
    aw_store(v, at, n, whole, vv[i]);
    aw_store(p, at, n, whole, pv[i]);
    if (copy) aw_store(copy, at, n, whole, pv[i]);
  }
}

// Moments in 8 bits: a wave takes whole blocks, four elements a lane, and agrees on the scale by exchange among its lanes.
// Moments are formed in 64 bits (this device's rate for them is that of 32): a code then does not hang on how an fp32 sum
// next to the border of two codes was rounded.
template <typename P, typename G>
__global__ __launch_bounds__(AW_THREADS) void adamw_8bit_kernel(AdamwArgs a) {
  const int which = aw_find(a, blockIdx.x);
  const AdamwTensor& t = a.t[which];
  const long long n = t.n, base = (long long)(blockIdx.x - a.first[which]) * AW_CHUNK;
  P* p = (P*)t.p;
  const G* g = (const G*)t.g;
  uint8_t *m = (uint8_t*)t.m, *v = (uint8_t*)t.v;
  aw_bf16* copy = (aw_bf16*)t.copy;
  const AdamwNumbers k = aw_numbers(a);
  const bool whole = (((uintptr_t)m | (uintptr_t)v) & 3) == 0 && ((uintptr_t)p & (4 * sizeof(P) - 1)) == 0 &&
                     ((uintptr_t)g & (4 * sizeof(G) - 1)) == 0 && ((uintptr_t)copy & 7) == 0 && base + AW_CHUNK <= n;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  float pv[AW_ITEMS][4], gv[AW_ITEMS][4], ms[AW_ITEMS], vs[AW_ITEMS];
  uint32_t mc[AW_ITEMS], vc[AW_ITEMS];
#pragma unroll
  for (int i = 0; i < AW_ITEMS; ++i) {
    const long long block = base / ADAMW_BLOCK + i * (AW_THREADS / 64) + wave, at = block * ADAMW_BLOCK + 4 * lane;
    const bool there = block * ADAMW_BLOCK < n;
    ms[i] = there ? t.ms[block] : 0.0f;
    vs[i] = there ? t.vs[block] : 0.0f;
    mc[i] = aw_load(m, at, n, whole);
    vc[i] = aw_load(v, at, n, whole);
    aw_load(p, at, n, whole, pv[i]);
    aw_load(g, at, n, whole, gv[i]);
  }
#pragma unroll
  for (int i = 0; i < AW_ITEMS; ++i) {
    const long long block = base / ADAMW_BLOCK + i * (AW_THREADS / 64) + wave, at = block * ADAMW_BLOCK + 4 * lane;
    if (block * ADAMW_BLOCK >= n) break;                             // (the wave's: elements behind n are zeros below)
    double md[4], vd[4];
    float mm = 0.0f, vm = 0.0f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const double x = (double)gv[i][e] * k.gs;
      md[e] = aw_average(k.b1, aw_value_m((int)(int8_t)(mc[i] >> 8 * e), ms[i]), k.one_b1, x);
      vd[e] = aw_average(k.b2, aw_value_v((int)(vc[i] >> 8 * e & 255), vs[i]), k.one_b2 * x, x);
      if (at + e >= n) md[e] = vd[e] = 0.0;
      const float mf = (float)md[e], vf = (float)vd[e];
      pv[i][e] = aw_new(pv[i][e], mf, vf, k);
      mm = __uint_as_float(max(__float_as_uint(mm), __float_as_uint(fabsf(mf))));
      vm = __uint_as_float(max(__float_as_uint(vm), __float_as_uint(vf)));
    }
    mm = aw_wave_max(mm);
    vm = aw_wave_max(vm);
    const double mi = mm > 0.0f ? 1.0 / (double)mm : 0.0, vi = vm > 0.0f ? 1.0 / (double)vm : 0.0;
    uint32_t mo = 0, vo = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int c = aw_code<false>(fabs(md[e]) * mi);
      int d = aw_code<true>(vd[e] * vi);
      d = vd[e] > 0.0 ? max(d, 1) : d;
      mo |= ((uint32_t)(md[e] < 0.0 ? -c : c) & 255u) << 8 * e;
      vo |= ((uint32_t)d & 255u) << 8 * e;
    }
    aw_store(m, at, n, whole, mo);
    aw_store(v, at, n, whole, vo);
    aw_store(p, at, n, whole, pv[i]);
    if (copy) aw_store(copy, at, n, whole, pv[i]);
    if (lane == 0) {
      t.ms[block] = mm + (mm - mm);          // (NaN also where the largest is infinite)
      t.vs[block] = vm + (vm - vm);
    }
  }
}

// Values of 8-bit moments: p is the output of m, copy that of v.
__global__ __launch_bounds__(AW_THREADS) void adamw_unpack_kernel(AdamwArgs a) {
  const int which = aw_find(a, blockIdx.x);
  const AdamwTensor& t = a.t[which];
  const long long n = t.n, base = (long long)(blockIdx.x - a.first[which]) * AW_CHUNK;
  const uint8_t *m = (const uint8_t*)t.m, *v = (const uint8_t*)t.v;
  float *mo = (float*)t.p, *vo = (float*)t.copy;
  const bool whole = (((uintptr_t)m | (uintptr_t)v) & 3) == 0 && (((uintptr_t)mo | (uintptr_t)vo) & 15) == 0 && base + AW_CHUNK <= n;
  uint32_t mc[AW_ITEMS], vc[AW_ITEMS];
  float ms[AW_ITEMS], vs[AW_ITEMS];
#pragma unroll
  for (int i = 0; i < AW_ITEMS; ++i) {
    const long long at = base + (long long)(i * AW_THREADS + threadIdx.x) * 4;
    ms[i] = at < n ? t.ms[at / ADAMW_BLOCK] : 0.0f;
    vs[i] = at < n ? t.vs[at / ADAMW_BLOCK] : 0.0f;
    mc[i] = aw_load(m, at, n, whole);
    vc[i] = aw_load(v, at, n, whole);
  }
#pragma unroll
  for (int i = 0; i < AW_ITEMS; ++i) {
    const long long at = base + (long long)(i * AW_THREADS + threadIdx.x) * 4;
    float x[4], y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[e] = (float)aw_value_m((int)(int8_t)(mc[i] >> 8 * e), ms[i]);
      y[e] = (float)aw_value_v((int)(vc[i] >> 8 * e & 255), vs[i]);
    }
    aw_store(mo, at, n, whole, x);
    aw_store(vo, at, n, whole, y);
  }
}

}  // namespace jm
