// Host side of the optimiser's entry points (include/jacobi_adamw.h).
#include <cfloat>
#include <cmath>
#include <cstring>

#include "adamw.hpp"
#include "entry.hpp"

using namespace jm;

namespace {

typedef void (*AdamwKernel)(AdamwArgs);

constexpr unsigned long long MAX_CHUNKS = 0xffffffffULL / AW_THREADS;      // of a launch: fewer than 2^32 threads

// Launches `kernel` over the tensors, as many at a time as a launch's arguments hold.
template <typename Fill>
int launch_tensors(AdamwKernel kernel, AdamwArgs& a, int32_t n, const int64_t* sizes, hipStream_t s, Fill fill) {
  a.count = 0;
  unsigned long long chunks = 0;
  for (int32_t i = 0; i <= n; ++i) {
    const unsigned long long mine = i < n ? ((unsigned long long)sizes[i] + AW_CHUNK - 1) / AW_CHUNK : 0;
    if (a.count > 0 && (i == n || a.count == AW_TENSORS || chunks + mine > MAX_CHUNKS)) {
      a.first[a.count] = (unsigned)chunks;
      hipLaunchKernelGGL(kernel, dim3((unsigned)chunks), dim3(AW_THREADS), 0, s, a);
      HIP_TRY(hipGetLastError());
      a.count = 0;
      chunks = 0;
    }
    if (mine == 0) continue;
    a.first[a.count] = (unsigned)chunks;
    a.t[a.count].n = sizes[i];
    fill(a.t[a.count], i);
    ++a.count;
    chunks += mine;
  }
  return MADE_OK;
}

int check_sizes(const char* who, int32_t n, const int64_t* sizes) {
  if (n < 0) return fail(MADE_ERR_ARG, "%s: n=%d", who, n);
  if (n > 0 && !sizes) return fail(MADE_ERR_ARG, "%s: NULL argument", who);
  for (int32_t i = 0; i < n; ++i)
    if (sizes[i] < 0 || (unsigned long long)sizes[i] > MAX_CHUNKS * AW_CHUNK) return fail(MADE_ERR_ARG, "%s: tensor %d has %lld elements", who, i, (long long)sizes[i]);
  return MADE_OK;
}

}  // namespace

extern "C" int adamw_step(const adamw_config* cfg, int32_t n, const int64_t* sizes, void* const* params, const void* const* grads,
                          void* const* m, void* const* v, float* const* m_scale, float* const* v_scale, void* const* copies,
                          const double* scalars, void* stream) {
  const char* who = "adamw_step";
  if (!cfg) return fail(MADE_ERR_ARG, "%s: NULL config", who);
  const adamw_config& c = *cfg;
  if (!(c.beta1 >= 0 && c.beta1 < 1 && c.beta2 >= 0 && c.beta2 < 1)) return fail(MADE_ERR_ARG, "%s: beta1=%g, beta2=%g must be in [0, 1)", who, c.beta1, c.beta2);
  if (!(c.eps == 0 || (c.eps >= FLT_MIN && c.eps <= FLT_MAX)) || !std::isfinite(c.weight_decay)) return fail(MADE_ERR_ARG, "%s: eps=%g, weight_decay=%g", who, c.eps, c.weight_decay);
  if (!scalars && (!std::isfinite(c.lr) || !std::isfinite(c.grad_scale) || c.step < 1))
    return fail(MADE_ERR_ARG, "%s: lr=%g, grad_scale=%g, step=%d", who, c.lr, c.grad_scale, c.step);
  const bool p16 = c.param_dtype == MADE_BF16, g16 = c.grad_dtype == MADE_BF16;
  if ((!p16 && c.param_dtype != MADE_F32) || (!g16 && c.grad_dtype != MADE_F32))
    return fail(MADE_ERR_ARG, "%s: param_dtype=%d, grad_dtype=%d are not MADE_F32 or MADE_BF16", who, c.param_dtype, c.grad_dtype);
  if (c.moment_bits != 8 && c.moment_bits != 32) return fail(MADE_ERR_ARG, "%s: moment_bits=%d is neither 8 nor 32", who, c.moment_bits);
  if (copies && p16) return fail(MADE_ERR_ARG, "%s: copies go with fp32 weights", who);
  TRY(check_sizes(who, n, sizes));
  if (n == 0) return MADE_OK;
  const bool eight = c.moment_bits == 8;
  if (!params || !grads || !m || !v || (eight && (!m_scale || !v_scale))) return fail(MADE_ERR_ARG, "%s: NULL argument", who);
  for (int32_t i = 0; i < n; ++i)
    if (sizes[i] > 0 && (!params[i] || !grads[i] || !m[i] || !v[i] || (eight && (!m_scale[i] || !v_scale[i])) || (copies && !copies[i])))
      return fail(MADE_ERR_ARG, "%s: tensor %d has a NULL pointer", who, i);
  AdamwArgs a;
  memset(&a, 0, sizeof a);
  a.lr = c.lr;
  a.b1 = c.beta1;
  a.b2 = c.beta2;
  a.eps = c.eps;
  a.wd = c.weight_decay;
  a.gs = c.grad_scale;
  if (!scalars) {
    a.c1 = 1.0 / (1.0 - std::pow(c.beta1, (double)c.step));
    a.c2 = 1.0 / (1.0 - std::pow(c.beta2, (double)c.step));
  }
  a.scalars = scalars;
  AdamwKernel kernel;
  if (eight) kernel = p16 ? (g16 ? adamw_8bit_kernel<aw_bf16, aw_bf16> : adamw_8bit_kernel<aw_bf16, float>)
                          : (g16 ? adamw_8bit_kernel<float, aw_bf16> : adamw_8bit_kernel<float, float>);
  else kernel = p16 ? (g16 ? adamw_kernel<aw_bf16, aw_bf16> : adamw_kernel<aw_bf16, float>)
                    : (g16 ? adamw_kernel<float, aw_bf16> : adamw_kernel<float, float>);
  return launch_tensors(kernel, a, n, sizes, (hipStream_t)stream, [&](AdamwTensor& t, int32_t i) {
    t.p = params[i];
    t.g = grads[i];
    t.m = m[i];
    t.v = v[i];
    t.ms = eight ? m_scale[i] : nullptr;
    t.vs = eight ? v_scale[i] : nullptr;
    t.copy = copies ? copies[i] : nullptr;
  });
}

extern "C" int adamw_unpack(int32_t n, const int64_t* sizes, const void* const* m, const void* const* v, const float* const* m_scale,
                            const float* const* v_scale, float* const* m_out, float* const* v_out, void* stream) {
  const char* who = "adamw_unpack";
  TRY(check_sizes(who, n, sizes));
  if (n == 0) return MADE_OK;
  if (!m || !v || !m_scale || !v_scale || !m_out || !v_out) return fail(MADE_ERR_ARG, "%s: NULL argument", who);
  for (int32_t i = 0; i < n; ++i)
    if (sizes[i] > 0 && (!m[i] || !v[i] || !m_scale[i] || !v_scale[i] || !m_out[i] || !v_out[i]))
      return fail(MADE_ERR_ARG, "%s: tensor %d has a NULL pointer", who, i);
  AdamwArgs a;
  memset(&a, 0, sizeof a);
  return launch_tensors(adamw_unpack_kernel, a, n, sizes, (hipStream_t)stream, [&](AdamwTensor& t, int32_t i) {
    t.m = const_cast<void*>(m[i]);
    t.v = const_cast<void*>(v[i]);
    t.ms = const_cast<float*>(m_scale[i]);
    t.vs = const_cast<float*>(v_scale[i]);
    t.p = m_out[i];
    t.copy = v_out[i];
  });
}
