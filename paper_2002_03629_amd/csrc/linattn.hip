// Host side of the linear-attention entry points (include/jacobi_linattn.h).
#include "../../include/jacobi_linattn.h"

#include <algorithm>
#include <cmath>
#include <cstring>
#include <initializer_list>

#include "entry.hpp"
#include "linattn.hpp"

using namespace jm;

namespace {

constexpr int UNITS = 256;      // compute units of the device
constexpr int MAX_T = 1 << 30;                    // positions and the ends of segments behind them stay below 2^31
constexpr long long MAX_THREADS = 0xffffffffLL;   // of a launch
constexpr int MAX_GRID = 65535;                   // workgroups along a launch's second and third axis

int block_rows(const linattn_config& c) { return c.dtype == MADE_BF16 ? LA_BF16_ROWS : LA_F32_ROWS; }

int check(const char* who, const linattn_config* c, bool step) {
  if (!c) return fail(MADE_ERR_ARG, "%s: NULL config", who);
  if (c->B < 0 || (!step && (c->T < 0 || c->T > MAX_T))) return fail(MADE_ERR_ARG, "%s: B=%d, T=%d out of range", who, c->B, c->T);
  if (c->Dk < 1 || c->Dv < 1 || c->Dk > LA_MAX_D || c->Dv > LA_MAX_D)
    return fail(MADE_ERR_ARG, "%s: Dk=%d, Dv=%d, widths of 1 to %d are supported", who, c->Dk, c->Dv, LA_MAX_D);
  if (c->kv_heads < 1 || c->heads < 1 || c->heads % c->kv_heads != 0)
    return fail(MADE_ERR_ARG, "%s: heads=%d must be a positive multiple of kv_heads=%d", who, c->heads, c->kv_heads);
  if (c->dtype != MADE_F32 && c->dtype != MADE_BF16) return fail(MADE_ERR_ARG, "%s: dtype=%d is neither MADE_F32 nor MADE_BF16", who, c->dtype);
  const int64_t need[4] = {(int64_t)c->heads * c->Dk, (int64_t)c->kv_heads * c->Dk, (int64_t)c->kv_heads * c->Dv, (int64_t)c->heads * c->Dv};
  const int64_t ld[4] = {c->ld_q, c->ld_k, c->ld_v, c->ld_o};
  for (int i = 0; i < 4; ++i) {
    if (std::max(ld[i], need[i]) > LA_MAX_LD)
      return fail(MADE_ERR_ARG, "%s: rows of %c are %lld elements apart, at most %d are supported", who, "qkvo"[i],
                  (long long)std::max(ld[i], need[i]), LA_MAX_LD);
    if (ld[i] != 0 && ld[i] < need[i])
      return fail(MADE_ERR_ARG, "%s: row stride %lld of %c is shorter than a row (%lld)", who, (long long)ld[i], "qkvo"[i], (long long)need[i]);
  }
  if (!std::isfinite(c->scale)) return fail(MADE_ERR_ARG, "%s: scale is not finite", who);
  return MADE_OK;
}

// How a call's sequences are cut.  rows: of a segment; slots: segments in all; q_split: workgroups that share a state's query heads.
struct Split {
  int rows, slots;
  bool on;
  int q_split;
};

int tiles(int d) { return d <= 32 ? 1 : d <= 64 ? 2 : 4; }

// Whether a walk's workgroups have fewer than 2^32 threads together.
bool walk_fits(const linattn_config& c, long long slots, int q_split, int roles) {
  const long long units = slots * c.kv_heads * q_split + 7;
  return units * roles <= MAX_THREADS / ((c.dtype == MADE_BF16 ? 128 : 64) * tiles(std::max(c.Dk, c.Dv)));
}

// One workgroup for each head of a sequence, unless those fill less than the device: then the sequences are cut into
// segments, whose sums and entering states take a second pass over keys and values and two more launches.  The number of
// blocks to a segment is the one with the least time by what was measured (us, widths of 128, bf16 / fp32): a block of the
// walk 4.4 / 6.8 on a compute unit of its own and 3.2 / 5 more for each further head that shares the state, 1.7 times that
// where two workgroups share the unit; a block of the pass for the sums 1.9 / 2.9; 4 and 2 to begin; the states in memory
// three times; 8 for the launches.  32768 steps of 32 heads: whole 2260 us, cut in 16 405; 16 x 1024 of 16: 77 and 110.
Split choose(const linattn_config& c, bool backward) {
  const int C = block_rows(c);
  const long long blocks = ((long long)c.T + C - 1) / C;     // of the longest sequence there may be
  const int whole_rows = (int)(std::max<long long>(blocks, 1) * C);
  Split best = {whole_rows, c.B, false, 1};
  const int group = c.heads / c.kv_heads;
  const double size = (c.dtype == MADE_BF16 ? 1.0 : 1.55) * (0.55 + 0.45 * tiles(c.Dk) * tiles(c.Dv) / 16.0);
  const double sums = size * 1.9 * (backward ? 0.5 * (1 + group) : 1.0), heads = (double)c.kv_heads;
  auto turns = [](double n) { return n <= UNITS ? 1.0 : 1.7 * std::ceil(n / (2 * UNITS)); };
  double least = 1e300;
  // (numbers of segments about an eighth apart; the heads of a group may be shared out, each part then walks the state again,
  // but not among more workgroups than run at once)
  for (long long m = 1, last = 0; m <= std::max<long long>(blocks, 1) && m <= 1 << 20; m += std::max<long long>(1, m / 8)) {
    const long long L = std::max<long long>(1, (blocks + m - 1) / m);
    if (L == last) continue;
    last = L;
    const bool cut = L < blocks;
    if (cut && c.kv_heads > MAX_GRID) continue;              // (of the join)
    const double slots = !cut ? c.B : c.offsets ? (double)(blocks / L + c.B) : (double)((blocks + L - 1) / L) * c.B;
    const double states = slots * heads * c.Dk * c.Dv * 4.0 * (backward ? 2 : 1);
    const double extra = !cut ? 0.0 : turns(slots * heads * (backward ? 2 : 1)) * (sums * (double)L + 2.0) + states * 3.0 / 5e6 + 8.0;
    for (int q = 1; q <= (backward ? 1 : group) && (q == 1 || slots * heads * q <= 2 * UNITS); ++q) {
      if (group % q != 0) continue;
      const double walk = size * (4.4 + 3.2 * (group / q - 1));
      const double cost = turns(slots * heads * q * (backward ? 3 : 1)) * (walk * (double)L + 4.0) + extra;
      if (cost < least && slots < 1e9 && walk_fits(c, (long long)slots, q, backward ? 3 : 1)) {
        least = cost;
        best.rows = cut ? (int)(L * C) : whole_rows;
        best.slots = (int)slots;
        best.on = cut;
        best.q_split = q;
      }
    }
  }
  return best;
}

long long state_floats(const linattn_config& c, const Split& s) { return s.on ? (long long)s.slots * c.kv_heads * c.Dk * c.Dv : 0; }

LinattnView view(const void* p, int64_t ld, int heads, int dim) {
  LinattnView v;
  v.p = const_cast<void*>(p);
  v.ld = ld ? ld : (int64_t)heads * dim;
  v.dim = dim;
  return v;
}

// Rows of 16-byte pieces: the base, the row stride and the width are multiples of 16 bytes.
bool pieces(const LinattnView& v, int dtype) {
  const int size = dtype == MADE_BF16 ? 2 : 4;
  return !v.p || ((uintptr_t)v.p % 16 == 0 && v.ld * size % 16 == 0 && v.dim * size % 16 == 0);
}

template <bool OUT, bool VEC>
void launch_walk(int dtype, int n, const LinattnArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)(((long long)a.slots * a.kv_heads * a.q_split + 7) / 8 * 8 * a.roles));
#define JM_WALK(N)                                                                                              \
  if (dtype == MADE_BF16) hipLaunchKernelGGL((linattn_walk_bf16_kernel<N, OUT, VEC>), grid, dim3(128 * N), 0, s, a); \
  else hipLaunchKernelGGL((linattn_walk_f32_kernel<N, OUT, VEC>), grid, dim3(64 * N), 0, s, a)
  switch (n) {
    case 1: JM_WALK(1); break;
    case 2: JM_WALK(2); break;
    default: JM_WALK(4); break;
  }
#undef JM_WALK
}

void launch_walk(int dtype, const LinattnArgs& a, bool out, hipStream_t s) {
  bool vec = true;
  for (int i = 0; i < a.roles; ++i) {
    const LinattnRole& r = a.role[i];
    vec = vec && pieces(r.k, dtype) && pieces(r.v, dtype) && (!out || (pieces(r.q, dtype) && pieces(r.o, dtype)));
  }
  const int n = tiles(std::max(a.role[0].dk, a.role[0].dv));      // (the roles of a call have the same two widths)
  if (out) vec ? launch_walk<true, true>(dtype, n, a, s) : launch_walk<true, false>(dtype, n, a, s);
  else vec ? launch_walk<false, true>(dtype, n, a, s) : launch_walk<false, false>(dtype, n, a, s);
}

// As many launches as the sequences of all roles need (one up to 65535 of them, unless there are very many heads).
void launch_join(LinattnArgs& a, hipStream_t s) {
  const int x = (a.role[0].dk * a.role[0].dv + 255) / 256;
  const long long all = (long long)a.B * a.roles, most = std::min<long long>(MAX_GRID, MAX_THREADS / (256LL * x * a.kv_heads));
  for (a.join0 = 0; a.join0 < all; a.join0 += most)
    hipLaunchKernelGGL(linattn_join_kernel, dim3(x, a.kv_heads, (unsigned)std::min(most, all - a.join0)), dim3(256), 0, s, a);
}

LinattnArgs common(const linattn_config& c, const float* log_decay, const Split& s) {
  LinattnArgs a;
  memset(&a, 0, sizeof a);
  a.log_decay = log_decay;
  a.offsets = c.offsets;
  a.B = c.B;
  a.T = c.T;
  a.kv_heads = c.kv_heads;
  a.q_split = 1;
  a.seg_rows = s.rows;
  a.slots = s.slots;
  return a;
}

// A workspace that is too small is none; `split` becomes the uncut call then.
int take_workspace(const char* who, const linattn_config& c, void* workspace, int64_t bytes, int sets, Split& split) {
  if (workspace && (uintptr_t)workspace % 256 != 0) return fail(MADE_ERR_ARG, "%s: the workspace is not 256-byte aligned", who);
  const long long need = state_floats(c, split) * 4 * sets;
  if (split.on && (!workspace || bytes < need)) {
    const int C = block_rows(c);
    split.rows = (int)(((long long)c.T + C - 1) / C * C);
    split.slots = c.B;
    split.on = false;
  }
  return MADE_OK;
}

int check_grid(const char* who, const linattn_config& c, const Split& s, int roles) {
  if (!walk_fits(c, s.slots, s.q_split, roles)) return fail(MADE_ERR_ARG, "%s: B=%d, heads=%d are more than one launch takes", who, c.B, c.kv_heads);
  return MADE_OK;
}

// Arrays that a call writes are none of those that it reads, and no two of them are one (by their addresses; NULL: absent).
int check_apart(const char* who, const char* written, std::initializer_list<const void*> out, std::initializer_list<const void*> in) {
  for (const void* const* x = out.begin(); x != out.end(); ++x) {
    for (const void* y : in)
      if (*x && *x == y) return fail(MADE_ERR_ARG, "%s: %s is one of the inputs", who, written);
    for (const void* const* y = x + 1; y != out.end(); ++y)
      if (*x && *x == *y) return fail(MADE_ERR_ARG, "%s: two gradients, outputs or workspaces are one array", who);
  }
  return MADE_OK;
}

}  // namespace

extern "C" int linattn_workspace_bytes(const linattn_config* cfg, int32_t backward, int64_t* bytes) {
  if (!bytes) return fail(MADE_ERR_ARG, "linattn_workspace_bytes: NULL argument");
  TRY(check("linattn_workspace_bytes", cfg, false));
  *bytes = state_floats(*cfg, choose(*cfg, backward != 0)) * 4 * (backward ? 2 : 1);
  return MADE_OK;
}

extern "C" int linattn_forward(const linattn_config* cfg, const void* q, const void* k, const void* v, const float* log_decay,
                               const float* state_in, void* o, float* state_out, void* workspace, int64_t workspace_bytes,
                               void* stream) {
  const char* who = "linattn_forward";
  TRY(check(who, cfg, false));
  const linattn_config& c = *cfg;
  if (c.B == 0) return MADE_OK;
  if (!log_decay || (c.T > 0 && (!q || !k || !v || !o))) return fail(MADE_ERR_ARG, "%s: NULL argument", who);
  const void* ws = workspace_bytes > 0 ? workspace : nullptr;
  TRY(check_apart(who, "an output", {o, ws}, {q, k, v, log_decay, state_in, c.offsets}));
  TRY(check_apart(who, "state_out", {state_out, o, ws}, {q, k, v, log_decay, c.offsets}));      // (it may be state_in)
  Split split = choose(c, false);
  TRY(take_workspace(who, c, workspace, workspace_bytes, 1, split));
  TRY(check_grid(who, c, split, 1));
  hipStream_t s = (hipStream_t)stream;
  LinattnArgs a = common(c, log_decay, split);
  a.roles = 1;
  LinattnRole& r = a.role[0];
  r.q = view(q, c.ld_q, c.heads, c.Dk);
  r.k = view(k, c.ld_k, c.kv_heads, c.Dk);
  r.v = view(v, c.ld_v, c.kv_heads, c.Dv);
  r.o = view(o, c.ld_o, c.heads, c.Dv);
  r.start = state_in;
  r.end = state_out;
  r.seg = split.on ? (float*)workspace : nullptr;
  r.dk = c.Dk;
  r.dv = c.Dv;
  r.st_r = c.Dv;
  r.st_c = 1;
  r.gq = c.heads / c.kv_heads;
  r.gk = 1;
  r.parts = state_out ? 3 : 2;
  r.p_scale = r.i_scale = c.scale;
  r.s_scale = 1.0f;
  if (split.on) launch_walk(c.dtype, a, false, s);
  // (without a workspace for its copy, a state replaced in place is read by one workgroup alone: the one that writes it)
  if (split.on || !state_out || state_out != state_in) a.q_split = split.q_split;
  if (split.on) launch_join(a, s);
  launch_walk(c.dtype, a, true, s);
  HIP_TRY(hipGetLastError());
  return MADE_OK;
}

extern "C" int linattn_backward(const linattn_config* cfg, const void* q, const void* k, const void* v, const float* log_decay,
                                const float* state_in, const void* d_o, const float* d_state_out, void* dq, void* dk, void* dv,
                                float* d_state_in, void* workspace, int64_t workspace_bytes, void* stream) {
  const char* who = "linattn_backward";
  TRY(check(who, cfg, false));
  const linattn_config& c = *cfg;
  if (c.B == 0) return MADE_OK;
  if (!log_decay || (c.T > 0 && (!q || !k || !v || !d_o || !dq || !dk || !dv))) return fail(MADE_ERR_ARG, "%s: NULL argument", who);
  if (d_state_in && d_state_in == d_state_out) return fail(MADE_ERR_ARG, "%s: d_state_in is d_state_out", who);
  TRY(check_apart(who, "a gradient or the workspace", {dq, dk, dv, d_state_in, workspace_bytes > 0 ? workspace : nullptr},
                  {q, k, v, d_o, log_decay, state_in, d_state_out, c.offsets}));
  Split split = choose(c, true);
  TRY(take_workspace(who, c, workspace, workspace_bytes, 2, split));
  TRY(check_grid(who, c, split, 3));
  hipStream_t s = (hipStream_t)stream;
  const int G = c.heads / c.kv_heads;
  const LinattnView vq = view(q, c.ld_q, c.heads, c.Dk), vk = view(k, c.ld_k, c.kv_heads, c.Dk),
                    vv = view(v, c.ld_v, c.kv_heads, c.Dv), vdo = view(d_o, c.ld_o, c.heads, c.Dv);
  float* seg_s = split.on ? (float*)workspace : nullptr;
  float* seg_r = split.on ? seg_s + state_floats(c, split) : nullptr;
  LinattnRole S, R;                                   // the states forward, and their gradients back in time
  memset(&S, 0, sizeof S);
  S.k = vk;
  S.v = vv;
  S.start = state_in;
  S.seg = seg_s;
  S.dk = c.Dk;
  S.dv = c.Dv;
  S.st_r = c.Dv;
  S.st_c = 1;
  S.gq = S.gk = 1;
  S.parts = 2;
  S.p_scale = S.i_scale = c.scale;
  S.s_scale = 1.0f;
  R = S;
  R.q = vk;                                           // (as the role of dv)
  R.k = vq;
  R.v = vdo;
  R.o = view(dv, c.ld_v, c.kv_heads, c.Dv);
  R.start = d_state_out;
  R.end = d_state_in;
  R.seg = seg_r;
  R.gk = G;
  R.back = 1;
  R.parts = d_state_in ? 3 : 2;
  R.i_scale = 1.0f;
  R.s_scale = c.scale;
  LinattnArgs a = common(c, log_decay, split);
  if (split.on) {
    a.roles = 2;
    a.role[0] = S;
    a.role[1] = R;
    launch_walk(c.dtype, a, false, s);
    launch_join(a, s);
  }
  LinattnRole Q = S, K = R;                           // dq: the states forward, transposed; dk: their gradients, transposed
  Q.q = vdo;
  Q.k = vv;
  Q.v = vk;
  Q.o = view(dq, c.ld_q, c.heads, c.Dk);
  Q.gq = G;
  K.q = vv;
  K.k = vdo;
  K.v = vq;
  K.o = view(dk, c.ld_k, c.kv_heads, c.Dk);
  K.end = nullptr;
  K.parts = 2;
  Q.dk = K.dk = c.Dv;
  Q.dv = K.dv = c.Dk;
  Q.st_r = K.st_r = 1;
  Q.st_c = K.st_c = c.Dv;
  a.role[0] = Q;
  a.role[1] = K;
  a.role[2] = R;
  a.roles = 3;
  launch_walk(c.dtype, a, true, s);
  HIP_TRY(hipGetLastError());
  return MADE_OK;
}

extern "C" int linattn_step(const linattn_config* cfg, const void* q, const void* k, const void* v, const float* log_decay,
                            float* state, int32_t n_slots, const int32_t* slots, void* o, void* stream) {
  const char* who = "linattn_step";
  TRY(check(who, cfg, true));
  const linattn_config& c = *cfg;
  if (n_slots < 0 || (!slots && n_slots < c.B)) return fail(MADE_ERR_ARG, "%s: n_slots=%d, B=%d", who, n_slots, c.B);
  if (c.B == 0) return MADE_OK;
  if (!q || !k || !v || !log_decay || !state || !o) return fail(MADE_ERR_ARG, "%s: NULL argument", who);
  TRY(check_apart(who, "o or the state", {o, state}, {q, k, v, log_decay, slots}));
  LinattnStepArgs a;
  a.q = view(q, c.ld_q, c.heads, c.Dk);
  a.k = view(k, c.ld_k, c.kv_heads, c.Dk);
  a.v = view(v, c.ld_v, c.kv_heads, c.Dv);
  a.o = view(o, c.ld_o, c.heads, c.Dv);
  a.log_decay = log_decay;
  a.state = state;
  a.slots = slots;
  a.n_slots = n_slots;
  a.B = c.B;
  a.kv_heads = c.kv_heads;
  a.group = c.heads / c.kv_heads;
  a.dk = c.Dk;
  a.dv = c.Dv;
  a.scale = c.scale;
  a.vec = (uintptr_t)state % 16 == 0 && c.Dv % 4 == 0;
  const long long units = (long long)c.B * c.kv_heads;
  // whole rows of the state (512 bytes) in one workgroup where there are enough of them to fill the device (250 rows of 8
  // states of 128 x 128: 128 columns 49.6 us, 32 columns 51.6; one row of 8 states of that size: 8.9 and 5.8)
  const bool wide = units >= 2 * UNITS && c.Dv > 64;
  const long long grid = units * (wide ? (c.Dv + 127) / 128 : (c.Dv + 31) / 32);
  if (grid > MAX_THREADS / 256) return fail(MADE_ERR_ARG, "%s: B=%d, heads=%d are more than one launch takes", who, c.B, c.kv_heads);
  hipStream_t s = (hipStream_t)stream;
#define JM_STEP(T, COLS) hipLaunchKernelGGL((linattn_step_kernel<T, COLS>), dim3((unsigned)grid), dim3(256), 0, s, a)
  if (c.dtype == MADE_BF16) {
    if (wide) JM_STEP(la_bf16, 128);
    else JM_STEP(la_bf16, 32);
  } else {
    if (wide) JM_STEP(float, 128);
    else JM_STEP(float, 32);
  }
#undef JM_STEP
  HIP_TRY(hipGetLastError());
  return MADE_OK;
}
