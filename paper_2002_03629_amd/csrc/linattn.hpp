// Linear attention with a decay for each head (gfx950 only).
//
//     S_t = lambda S_{t-1} + k_t v_t^T,    o_t = scale S_t^T q_t
//
// The recurrence over C steps at once, from the state S that enters them (i, j = 0 .. C-1):
//     o_i = scale ( lambda^(i+1) S^T q_i + sum_{j <= i} lambda^(i-j) (q_i . k_j) v_j )
//     S  <- lambda^C S + sum_j lambda^(C-1-j) k_j v_j^T
// which is four matrix products.  One workgroup owns the state of one head for a run of steps (a segment) and walks its
// blocks of C steps: the state stays in accumulator registers, divided among the waves by value columns, the block's q, k, v
// pass through LDS, the next block's are requested before the products of this one.
//
// What it costs (one sequence of 32768 steps, 32 heads, widths of 128, bf16, 16 segments to a head: 410 us in all with calls in
// a row, 1.07 GB of q, k, v and o take 172 at the 6.26 TB/s that an elementwise product of 8 GiB reaches): the walk 287 us, 4.5 us
// of a compute unit for a block's 64 KB (2.7 at that rate); by the counters the SIMDs issue vector instructions 55 % and run
// MFMAs 34 % of the time (issue cycles and busy cycles over those of the shader engines), LDS is read or written 40 %.  Vector and matrix time added up in every variant timed, so fewer
// instructions is what has paid.  The pass for the sums 140 us, 2.2 us a block's 32 KB (1.3), 52 % and 25 %.
//
// The gradients are the same recurrence with the arrays in other roles, so the same kernel computes them:
//     dq: queries do, keys v, values k, forward in time, the states of the forward pass (transposed)
//     dk: queries v, keys do, values q, back in time;     dv: queries k, keys q, values do, back in time
// Back in time the state R_t = dL/dS_t enters the first step of a block undecayed (`late` below), and a state has the keys
// and values of all its query heads.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace jm {

typedef uint16_t la_bf16;
typedef __attribute__((ext_vector_type(4))) uint32_t la_u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t la_u32x2;
typedef __attribute__((ext_vector_type(4))) float la_f32x4;
typedef __attribute__((ext_vector_type(8))) __bf16 la_bf16x8;
typedef __attribute__((ext_vector_type(8))) float la_f32x8;
typedef __attribute__((ext_vector_type(16))) float la_f32x16;

constexpr int LA_MAX_D = 128;
constexpr int LA_MAX_LD = 1 << 23;     // elements from row to row: a block's offsets fit 32 bits

// One operand array in a kernel's role: element (row, head, d) at p + row * ld + head * dim + d.
struct LinattnView {
  void* p;
  long long ld;
  int dim;
};

struct LinattnRole {
  LinattnView q, k, v, o;
  const float* start;   // states that enter the sequences [B, kv_heads, Dk, Dv], or NULL
  float* end;           // states that leave them, or NULL
  float* seg;           // workspace [slot, kv_heads, Dk, Dv]: sums of the segments, then the states that enter them; NULL: none
  int dk, dv;           // width of the role's keys and values
  int st_r, st_c;       // state element (key r, value c) at r * st_r + c * st_c (dq and dk hold it transposed)
  int gq, gk;           // query heads / key heads per state (one of them is 1)
  int back;             // 1: steps are taken from the last to the first
  int parts;            // bf16: parts the decayed values are split into for the state (2, or 3 for states that leave in fp32)
  float p_scale, s_scale, i_scale;   // factors of the scores, of what enters the state, of what is read from it
};

struct LinattnArgs {
  LinattnRole role[3];
  const float* log_decay;
  const int* offsets;   // [B + 1] or NULL
  int B, T, kv_heads;
  int roles;
  int q_split;          // workgroups that share the query heads of a state (each walks the state; roles with gq > 1)
  int seg_rows;         // rows of a segment (a multiple of the block)
  int slots;            // segments in all (packed: an upper bound)
  long long join0;      // the join: (role, sequence) pairs of the launches before
};

// lambda^n, g2 = log2 lambda (the hardware's exponential is within 1 ulp; below 2^-126 it is zero)
__device__ __forceinline__ float la_pow(float g2, int n) {
  const float x = __builtin_amdgcn_exp2f(g2 * (float)n);
  return n == 0 ? 1.0f : x;
}

// The same value in every lane, as a scalar.
__device__ __forceinline__ float la_uniform(float x) {
  return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x)));
}

// ------------------------------------------------------------------------------------------------------------------
// segments
// ------------------------------------------------------------------------------------------------------------------
struct LinattnSegment {
  int b, index, count;   // sequence, the segment's place in it, segments of the sequence
  int row0, len;         // the sequence's rows
};

__device__ __forceinline__ void la_rows(const LinattnArgs& a, int b, int& row0, int& len) {
  const int lo = min(max(a.offsets[b], 0), a.T);
  row0 = lo;
  len = min(max(a.offsets[b + 1], lo), a.T) - lo;
}

__host__ __device__ __forceinline__ int la_count(const LinattnArgs& a, int len) { return len <= a.seg_rows ? 1 : (len + a.seg_rows - 1) / a.seg_rows; }

// Number of the first segment of sequence b, whose rows begin at row0.  Cut packed sequences (R rows to a segment): none has
// more segments than floor(row0 / R) + b grows by to the next one (ceil(n / R) <= floor((row0 + n) / R) - floor(row0 / R) + 1),
// so that no sum over those before is needed; numbers between are no segment's.
__host__ __device__ __forceinline__ int la_first_slot(const LinattnArgs& a, int b, int row0) {
  return !a.offsets ? b * la_count(a, a.T) : a.seg_rows < a.T ? row0 / a.seg_rows + b : b;
}

// The segment with number `slot` (false: there is none).  Cut packed sequences: the last one whose first segment is not behind
// `slot`, searched by every wave, 64 candidates at a time, then 64 among those up to the next (a sum of the counts before
// took 260 ms in all for 65536 sequences of 8 rows).
__device__ __forceinline__ bool la_find(const LinattnArgs& a, int slot, LinattnSegment& s) {
  if (!a.offsets) {
    s.count = la_count(a, a.T);
    s.b = slot / s.count;
    s.index = slot - s.b * s.count;
    s.row0 = 0;              // (b T may pass 32 bits: the caller forms it)
    s.len = a.T;
    return s.b < a.B;
  }
  const int lane = threadIdx.x & 63;
  const bool cut = a.seg_rows < a.T;
  int lo = cut ? 0 : slot, n = cut ? a.B : 1;
  while (true) {
    const int step = (n + 63) / 64;
    int row0 = 0, len = 0;
    bool here = false;
    if (lane * step < n) {
      la_rows(a, lo + lane * step, row0, len);
      here = la_first_slot(a, lo + lane * step, row0) <= slot;
    }
    const unsigned long long hit = __ballot(here);
    if (!hit) return false;
    const int f = 63 - __clzll((long long)hit);
    lo += f * step;
    n = min(step, n - f * step);
    if (step > 1) continue;
    s.b = lo;
    s.row0 = __builtin_amdgcn_readfirstlane(__shfl(row0, f));
    s.len = __builtin_amdgcn_readfirstlane(__shfl(len, f));
    s.count = la_count(a, s.len);
    s.index = slot - la_first_slot(a, lo, s.row0);
    return s.index < s.count;
  }
}

// ------------------------------------------------------------------------------------------------------------------
// the walk
// ------------------------------------------------------------------------------------------------------------------
constexpr int LA_BF16_ROWS = 64, LA_F32_ROWS = 32;      // steps of a block

// Memory is reached through buffer descriptors: a lane whose element does not exist gets an offset past the end, reads zero
// and writes nothing, without a branch.  An offset is a lane's part, below 2^30 bytes or LA_NOWHERE, and a scalar part.
constexpr unsigned LA_NOWHERE = 0x80000000u;

__device__ __forceinline__ __amdgpu_buffer_rsrc_t la_buffer(const void* p, int bytes = 0x7fffffff) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, bytes, 0x00027000);
}

// n rows of an operand from the row of position 0 (`first`) on, in the order of the walk.  The descriptor begins at their
// lowest row and ends behind their highest; position p is la_lane + at0 bytes from its begin: what lies behind the n rows
// falls out of it, forward above its end, back below zero.
template <typename T>
struct LaBlock {
  __amdgpu_buffer_rsrc_t buf;
  int ld;                   // bytes from row to row (at most 2^25: the host checks), negative back in time
  unsigned at0;             // of position 0
};
template <typename T>
__device__ __forceinline__ LaBlock<T> la_block(const LinattnView& x, long long first, int back, int n, int head) {
  LaBlock<T> b;
  const T* base = (const T*)x.p + (back ? first - (n - 1) : first) * x.ld + (long long)head * x.dim;
  const int ld = (int)x.ld * (int)sizeof(T);
  b.buf = la_buffer(base, __builtin_amdgcn_readfirstlane(n * ld));
  b.ld = back ? -ld : ld;
  b.at0 = back ? (unsigned)((n - 1) * ld) : 0u;
  return b;
}
// A lane's part of an offset: position p, element d of the head; LA_NOWHERE for elements that do not exist.
template <typename T>
__device__ __forceinline__ unsigned la_lane(const LinattnView& x, int back, int p, int d) {
  const int ld = (int)x.ld * (int)sizeof(T);
  return d < x.dim ? (unsigned)((back ? -p : p) * ld + d * (int)sizeof(T)) : LA_NOWHERE;
}

// E consecutive rows x 1 piece of 16 bytes; `lane` is the first row's la_lane.
template <typename T, int E>
__device__ __forceinline__ void la_load_group(la_u32x4 (&r)[E], const LaBlock<T>& b, unsigned lane) {
#pragma unroll
  for (int e = 0; e < E; ++e) r[e] = __builtin_amdgcn_raw_buffer_load_b128(b.buf, lane + b.at0 + (unsigned)(e * b.ld), 0, 0);
}

// Where an operand's rows are not made of 16-byte pieces its elements are fetched one by one when LDS is filled.
template <typename T>
__device__ __forceinline__ T la_element(const LinattnView& x, long long first, int back, int n, int head, int pos, int d) {
  return pos < n && d < x.dim ? ((const T*)x.p)[(back ? first - pos : first + pos) * x.ld + (long long)head * x.dim + d] : (T)0;
}

// What a walk knows of its place.
struct LinattnPlace {
  LinattnSegment s;
  int which, head, p0, p1;       // role, state head, positions in the order of the walk
  int q0, gq;                    // first of this workgroup's query heads, their number
  long long first;               // row of position 0
  long long state_at, seg_at;    // the sequence's state, the segment's place in the workspace (elements)
  float g2;                      // log2 lambda
};

// The roles of a unit (segment, head) read the same arrays: their workgroups have numbers that are equal modulo 8, so that
// one XCD's L2 sees all of them.
__device__ __forceinline__ bool la_place(const LinattnArgs& a, bool out, LinattnPlace& w) {
  const int id = blockIdx.x, pack = 8 * a.roles;
  const int part = id / pack * 8 + id % 8, unit = part / a.q_split;
  w.which = id % pack / 8;
  if (unit >= a.slots * a.kv_heads) return false;
  w.head = unit % a.kv_heads;
  w.gq = a.role[w.which].gq / a.q_split;
  w.q0 = w.head * a.role[w.which].gq + part % a.q_split * w.gq;
  const int slot = unit / a.kv_heads;
  LinattnSegment s;
  if (!la_find(a, slot, s)) return false;
  // (the same in every lane: they form addresses that are scalars)
  s.b = __builtin_amdgcn_readfirstlane(s.b);
  s.index = __builtin_amdgcn_readfirstlane(s.index);
  s.count = __builtin_amdgcn_readfirstlane(s.count);
  s.row0 = __builtin_amdgcn_readfirstlane(s.row0);
  s.len = __builtin_amdgcn_readfirstlane(s.len);
  w.s = s;
  if (!out && s.index == s.count - 1) return false;    // (nothing follows the last segment)
  const LinattnRole& R = a.role[w.which];
  w.p0 = s.index * a.seg_rows;
  w.p1 = min(w.p0 + a.seg_rows, s.len);
  const long long row = a.offsets ? (long long)s.row0 : (long long)s.b * a.T;
  w.first = R.back ? row + s.len - 1 : row;
  w.state_at = ((long long)s.b * a.kv_heads + w.head) * R.dk * R.dv;
  w.seg_at = ((long long)slot * a.kv_heads + w.head) * R.dk * R.dv;
  w.g2 = la_uniform(a.log_decay[w.head] * 1.44269504088896340736f);
  return true;
}

// Workgroups that share a state's query heads each read the state that enters, one of them writes the one that leaves, and
// nothing orders the two: where a call replaces states in place, a sequence of one segment is read from a copy too, which
// the join makes (q_split > 1 has at most 512 states and parts: a copy is a few us).
__host__ __device__ __forceinline__ bool la_copied(const LinattnArgs& a, const LinattnRole& R) { return a.q_split > 1 && R.end && R.end == R.start; }
__host__ __device__ __forceinline__ const float* la_state_in(const LinattnArgs& a, const LinattnRole& R, const LinattnPlace& w) {
  return R.seg && (w.s.count > 1 || la_copied(a, R)) ? R.seg + w.seg_at : R.start ? R.start + w.state_at : nullptr;
}
__device__ __forceinline__ float* la_state_out(const LinattnRole& R, const LinattnPlace& w, bool out) {
  return !out ? R.seg + w.seg_at : R.end && w.s.index == w.s.count - 1 && w.q0 == w.head * R.gq ? R.end + w.state_at : nullptr;
}

// The lane's number, formed anew: what is made of it need not be kept from one use to the next.
__device__ __forceinline__ int la_lane_id() {
  int x;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(x));
  return x;
}

__device__ __forceinline__ la_bf16x8 la_operand(la_u32x4 x) { return __builtin_bit_cast(la_bf16x8, x); }
// fp32 values as two bf16 parts, x = hi + lo + O(2^-18 x)
__device__ __forceinline__ la_u32x4 la_round(la_f32x8 x) { return __builtin_bit_cast(la_u32x4, __builtin_convertvector(x, la_bf16x8)); }
__device__ __forceinline__ la_f32x8 la_widen(la_u32x4 x) {
  la_f32x8 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    r[2 * i] = __uint_as_float(x[i] << 16);
    r[2 * i + 1] = __uint_as_float(x[i] & 0xffff0000u);
  }
  return r;
}
__device__ __forceinline__ la_u32x4 la_rest(la_f32x8 x, la_u32x4 hi) { return la_round(x - la_widen(hi)); }

// ---- bf16: blocks of 64 steps, 16 x 16 x 32 MFMA.  Two waves to 32 value columns: with 16 columns each a wave's state is 32
// registers (keys of 128), so that 4 waves of a SIMD cover each other's waits.
//
// An accumulator's element e of lane l is (row 4 (l / 16) + e, column l % 16); an operand's lane holds 8 values of its row,
// k = 8 (l / 16) ..  Two accumulators above each other are so an operand with 32 values of k in the order of quads
// 0 4 1 5 2 6 3 7: the state and the scores become operands as they lie, and what they are multiplied with is laid out in
// that order: q and k by rows (dims), k and v by columns (steps).
constexpr int LA_FADE = 32;     // place of the factor lambda^0 in the table

template <int KT, bool OUT>
struct LaLds {
  // 16-byte units of a row and of a column are exchanged (la_row_swizzle, la_swizzle) so that the 16 rows or columns an
  // operand is read from lie in different banks
  __align__(16) unsigned char q[OUT ? 64 * KT * 64 : 16];
  __align__(16) unsigned char k[OUT ? 64 * KT * 64 : 16];
  __align__(16) unsigned char kt[KT * 32 * 128];
  __align__(16) unsigned char vt[KT * 32 * 128];
  __align__(16) unsigned char p[OUT ? 6 : 1][2][64 * 16];        // scores as operands: pair of tiles, part, lane
  __align__(16) float fade[OUT ? LA_FADE + 64 : 4];              // p_scale lambda^m at LA_FADE + m, zeros before
  __align__(16) float weight[64];                                // lambda^(n-1+late-j): what the block's end keeps of step j
};

__device__ __forceinline__ int la_swizzle(int d) { return ((d >> 1) ^ (d >> 4)) & 7; }
template <int KT>
__device__ __forceinline__ int la_row_swizzle(int row) {
  return KT == 4 ? row & 15 : KT == 2 ? row >> 1 & 7 : row >> 2 & 3;
}
// The group of rows a lane takes: neighbours take both halves of a column's unit.
__device__ __forceinline__ int la_group(int m) { return (m & 8) | (m & 1) << 2 | (m >> 1 & 3); }

__device__ __forceinline__ uint32_t la_pack(float x, float y) {
  typedef __attribute__((ext_vector_type(2))) __bf16 pair;
  const pair h = {(__bf16)x, (__bf16)y};
  return __builtin_bit_cast(uint32_t, h);
}

// place of the scores of queries 16 it .. and steps 32 kb ..
__device__ __forceinline__ constexpr int la_pair(int it, int kb) { return it < 2 ? it : 2 * it - 2 + kb; }

// row p, piece u: its two quads are the same halves of two neighbouring units
template <int KT>
__device__ __forceinline__ void la_put_row(la_u32x4 r, unsigned char* dst, int p, int u) {
  unsigned char* row = dst + p * (KT * 64) + (u >> 1 & 1) * 8;
  const int unit = ((u >> 2) * 4 + (u & 1) * 2) ^ la_row_swizzle<KT>(p);
  *(la_u32x2*)(row + unit * 16) = la_u32x2{r[0], r[1]};
  *(la_u32x2*)(row + (unit ^ 1) * 16) = la_u32x2{r[2], r[3]};
}

// rows 4 tg .. 4 tg + 3, piece u, turned over
__device__ __forceinline__ void la_put_columns(const la_u32x4 (&r)[4], unsigned char* dst, int tg, int u) {
  // (la_swizzle(8 u + dd) = la_swizzle(8 u) ^ dd / 2: four addresses and fixed distances from them)
  unsigned char* column = dst + 8 * u * 128 + (tg >> 2 & 1) * 8;
  const int unit = (4 * (tg >> 3) + (tg & 3)) ^ la_swizzle(8 * u);
#pragma unroll
  for (int dd = 0; dd < 8; ++dd) {
    const uint32_t sel = dd & 1 ? 0x07060302u : 0x05040100u;
    la_u32x2 o;
    o[0] = __builtin_amdgcn_perm(r[1][dd / 2], r[0][dd / 2], sel);
    o[1] = __builtin_amdgcn_perm(r[3][dd / 2], r[2][dd / 2], sel);
    *(la_u32x2*)(column + ((unit ^ (dd / 2)) * 16) + dd * 128) = o;
  }
}

template <int TILES, int NT>
__device__ __forceinline__ void la_fetch_rows(const LinattnView& x, long long first, int back, int n, int head, unsigned char* dst) {
#pragma unroll 4
  for (int i = threadIdx.x; i < 64 * 32 * TILES; i += NT) {
    const int pos = i / (32 * TILES), d = i % (32 * TILES);
    *(la_bf16*)(dst + pos * (TILES * 64) + (((d >> 5) * 4 + (d >> 2 & 3)) ^ la_row_swizzle<TILES>(pos)) * 16 + (d >> 4 & 1) * 8 + (d & 3) * 2) =
        la_element<la_bf16>(x, first, back, n, head, pos, d);
  }
}

template <int TILES, int NT>
__device__ __forceinline__ void la_fetch_columns(const LinattnView& x, long long first, int back, int n, int head, unsigned char* dst) {
#pragma unroll 4
  for (int i = threadIdx.x; i < 64 * 32 * TILES; i += NT) {
    const int pos = i / (32 * TILES), d = i % (32 * TILES), tg = pos >> 2;
    *(la_bf16*)(dst + d * 128 + ((4 * (tg >> 3) + (tg & 3)) ^ la_swizzle(d)) * 16 + (tg >> 2 & 1) * 8 + (pos & 3) * 2) =
        la_element<la_bf16>(x, first, back, n, head, pos, d);
  }
}

__device__ __forceinline__ la_f32x4 la_mfma16(la_u32x4 x, la_u32x4 y, la_f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(la_operand(x), la_operand(y), c, 0, 0, 0);
}

// OUT = true: the walk with outputs.  OUT = false: only the state a segment adds, from zero, into the workspace.
// VEC: every operand's rows come in 16-byte pieces (else none is taken to).
// The second half of the keys, and waves of values, that a role does not have are passed over, so that one kernel of N x 32
// keys and values serves the roles of a gradient together.
template <int N, bool OUT, bool VEC>
__global__ __launch_bounds__(128 * N, N == 4 ? 4 : 2) void linattn_walk_bf16_kernel(LinattnArgs a) {
  constexpr int C = LA_BF16_ROWS, KT = N, VT = N, NT = 128 * VT, NW = 2 * VT;
  __shared__ LaLds<N, OUT> lds;
  LinattnPlace w;
  if (!la_place(a, OUT, w)) return;
  const LinattnRole& R = a.role[w.which];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int cl = lane & 15, g = lane >> 4;
  const int late = R.back, head = w.head, gq = w.gq, gk = R.gk;
  const int dk = R.dk, dv = R.dv, st_r = R.st_r, parts = R.parts;
  const float g2 = w.g2;

  // ---- state: element e of tile t is (key 16 t + 4 g + e, value 16 wave + cl)
  la_f32x4 S[2 * KT];
  const int col = 16 * wave + cl;
  const unsigned state_off = (unsigned)(4 * g * R.st_r + col * R.st_c) * 4;
  if (OUT) {
    const float* src = la_state_in(a, R, w);
    const __amdgpu_buffer_rsrc_t buf = la_buffer(src);
#pragma unroll
    for (int t = 0; t < 2 * KT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int key = 16 * t + e;
        const bool there = (src != nullptr) & (key + 4 * g < dk) & (col < dv);
        S[t][e] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(buf, there ? state_off : LA_NOWHERE, key * st_r * 4, 0));
      }
  } else {
#pragma unroll
    for (int t = 0; t < 2 * KT; ++t) S[t] = la_f32x4{};
  }

  if (OUT) {
    for (int i = threadIdx.x; i < LA_FADE + 64; i += NT) lds.fade[i] = i < LA_FADE ? 0.0f : R.p_scale * la_pow(g2, i - LA_FADE);
  }

  const bool mine = 16 * wave < dv;            // this wave has values
  const int stages = gq > gk ? gq : gk;
  const auto q_head = [&](int st) { return w.q0 + (gq > 1 ? st : 0); };
  const auto k_head = [&](int st) { return head * gk + (gk > 1 ? st : 0); };
  // The next block's pieces, always into the same registers: what a stage does not need is asked for from nowhere (a branch
  // around the loads would have their results moved, and so waited for, where it ends).  Groups of 4 rows of k, then of v:
  // 64 to a wave, so that a wave's are all of one array.
  constexpr int PER = (KT + VT + NW - 1) / NW, PERQ = (KT + VT - 1) / VT;
  la_u32x4 kv[PER][4], qs[PERQ][2];
  unsigned kv_lane[PER], q_lane[PERQ];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int part = wave + i * NW;                                          // of KT + VT parts of 64 groups
    const bool keys = part < KT;
    const int at = (keys ? part : part - KT) * 64 + lane, U = keys ? 4 * KT : 4 * VT;
    const LinattnView x = keys ? R.k : R.v;
    kv_lane[i] = part < KT + VT ? la_lane<la_bf16>(x, R.back, la_group(at / U) * 4, at % U * 8) : LA_NOWHERE;
  }
#pragma unroll
  for (int i = 0; i < PERQ; ++i) {
    const int at = threadIdx.x + i * NT;
    q_lane[i] = at < 128 * KT ? la_lane<la_bf16>(R.q, R.back, at / (4 * KT) * 2, at % (4 * KT) * 8) : LA_NOWHERE;
  }
  auto request = [&](int p, int st) {
    const long long row = R.back ? w.first - p : w.first + p;
    const int n = max(0, min(C, w.p1 - p));                                  // (none behind the last block)
    const int nk = gk > 1 || st == 0 ? n : 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const LinattnView x = wave + i * NW < KT ? R.k : R.v;
      la_load_group(kv[i], la_block<la_bf16>(x, row, R.back, nk, k_head(st)), kv_lane[i]);
    }
    if (OUT) {
      const LaBlock<la_bf16> q = la_block<la_bf16>(R.q, row, R.back, gq > 1 || st == 0 ? n : 0, q_head(st));
#pragma unroll
      for (int i = 0; i < PERQ; ++i) la_load_group(qs[i], q, q_lane[i]);
    }
  };
  if (VEC) request(w.p0, 0);

  // The state in the registers is the state divided by `frame`: a block's decay goes into `frame` and only where that leaves
  // 2^-10 .. 2^10 into the 2 KT x 4 registers (fp32's range is shorter by as much; multiplying every block
  // would be 32 instructions a wave).
  float frame = 1.0f;

  la_f32x4 O[4];
  for (int p = w.p0; p < w.p1; p += C) {
    const int n = min(C, w.p1 - p);
    const float factor = la_uniform(frame * la_pow(g2, n));
    const bool rescale = __builtin_amdgcn_readfirstlane(!(factor >= 0x1p-10f && factor <= 0x1p10f));
    const float next = la_uniform(rescale ? 1.0f : factor);
    const long long row = R.back ? w.first - p : w.first + p;
    for (int st = 0; st < stages; ++st) {
      const bool new_q = gq > 1 || st == 0, new_kv = gk > 1 || st == 0, last = st == stages - 1;
      __syncthreads();                       // every wave has read the block before
      if (VEC) {
        const int lane = la_lane_id();
        if (OUT && new_q) {
#pragma unroll
          for (int i = 0; i < PERQ; ++i) {
            const int at = 64 * wave + lane + i * NT;
            if (at < 128 * KT) {
#pragma unroll
              for (int e = 0; e < 2; ++e) la_put_row<KT>(qs[i][e], lds.q, at / (4 * KT) * 2 + e, at % (4 * KT));
            }
          }
        }
        if (new_kv) {
#pragma unroll
          for (int i = 0; i < PER; ++i) {
            const int part = wave + i * NW;
            if (part < KT) {
              const int at = part * 64 + lane, tg = la_group(at / (4 * KT)), u = at % (4 * KT);
              if (OUT) {
#pragma unroll
                for (int e = 0; e < 4; ++e) la_put_row<KT>(kv[i][e], lds.k, 4 * tg + e, u);
              }
              la_put_columns(kv[i], lds.kt, tg, u);
            } else if (part < KT + VT) {
              const int at = (part - KT) * 64 + lane;
              la_put_columns(kv[i], lds.vt, la_group(at / (4 * VT)), at % (4 * VT));
            }
          }
        }
      } else {
        if (OUT && new_q) la_fetch_rows<KT, NT>(R.q, row, R.back, n, q_head(st), lds.q);
        if (new_kv) {
          if (OUT) la_fetch_rows<KT, NT>(R.k, row, R.back, n, k_head(st), lds.k);
          la_fetch_columns<KT, NT>(R.k, row, R.back, n, k_head(st), lds.kt);
          la_fetch_columns<VT, NT>(R.v, row, R.back, n, k_head(st), lds.vt);
        }
      }
      if (new_kv && wave == 0) {
        const int j = la_lane_id();
        lds.weight[j] = R.s_scale / next * la_pow(g2, max(0, n - 1 + late - j));
      }
      if (VEC) request(last ? p + C : p, last ? 0 : st + 1);
      __syncthreads();

      // (what a lane's number makes of addresses is formed again for every product: kept, it would take the registers that
      // let four waves share a SIMD)
      if (OUT) {
        // Scores of the 6 pairs of tiles with steps <= queries, transposed, divided among the waves: every wave needs them all,
        // as operands in two parts, and gets them through LDS while its product with the state runs.
        for (int pair = wave; pair < 6; pair += NW) {
          const int it = pair < 2 ? pair : pair / 2 + 1, kb0 = pair == 3 || pair == 5;
          const int lane = la_lane_id(), cl = lane & 15, g = lane >> 4;
          const int sw = la_row_swizzle<KT>(cl);
          const unsigned char* q_ = lds.q + (16 * it + cl) * (KT * 64);
          const unsigned char* k_ = lds.k + (32 * kb0 + cl) * (KT * 64);
          la_u32x4 qf[KT], kf[2][KT];
#pragma unroll
          for (int kb = 0; kb < KT; ++kb) {
            const int unit = ((4 * kb + g) ^ sw) * 16;
            qf[kb] = *(const la_u32x4*)(q_ + unit);
            kf[0][kb] = *(const la_u32x4*)(k_ + unit);
            kf[1][kb] = *(const la_u32x4*)(k_ + unit + 16 * KT * 64);
          }
          __builtin_amdgcn_sched_barrier(0);      // (all requested before the first is waited for)
          la_f32x4 P[2] = {};
#pragma unroll
          for (int kb = 0; kb < KT; ++kb)
#pragma unroll
            for (int t = 0; t < 2; ++t) P[t] = la_mfma16(kf[t][kb], qf[kb], P[t]);
          const float* f = lds.fade + LA_FADE + 16 * (it - 2 * kb0) + cl - 4 * g;
          la_f32x8 x;
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = P[e / 4][e % 4] * f[-(16 * (e / 4) + e % 4)];
          const la_u32x4 hi = la_round(x);
          *(la_u32x4*)&lds.p[pair][0][lane * 16] = hi;
          *(la_u32x4*)&lds.p[pair][1][lane * 16] = la_rest(x, hi);
        }
        if (new_q && mine) {
          const int lane = la_lane_id();
          // (la_row_swizzle(16 it + c) = la_row_swizzle(c))
          const int qat = (lane & 15) * (KT * 64) + ((lane >> 4) ^ la_row_swizzle<KT>(lane & 15)) * 16;
          auto q_frag = [&](int it, int kb) { return *(const la_u32x4*)(lds.q + (qat ^ 64 * kb) + it * 16 * KT * 64); };
          // O^T = S^T Q^T: the accumulator of the state is an operand as it lies
          la_u32x4 qf[2][4];
#pragma unroll
          for (int it = 0; it < 4; ++it) qf[0][it] = q_frag(it, 0);
#pragma unroll
          for (int kb = 0; kb < KT; ++kb) {
            if (2 * kb == KT && 32 * kb >= dk) break;
            // (the next operands are on their way while these are multiplied; equal accumulators lie four MFMAs apart)
            if (kb + 1 < KT) {
#pragma unroll
              for (int it = 0; it < 4; ++it) qf[(kb + 1) & 1][it] = q_frag(it, kb + 1);
            }
            const la_f32x8 x = __builtin_shufflevector(S[2 * kb], S[2 * kb + 1], 0, 1, 2, 3, 4, 5, 6, 7);
            const la_u32x4 hi = la_round(x), lo = la_rest(x, hi);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int it = 0; it < 4; ++it) O[it] = la_mfma16(hi, qf[kb & 1][it], kb == 0 ? la_f32x4{} : O[it]);
#pragma unroll
            for (int it = 0; it < 4; ++it) O[it] = la_mfma16(lo, qf[kb & 1][it], O[it]);
          }
          float f = R.i_scale * frame * la_pow(g2, (lane & 15) + 1 - late);
          const float to16 = la_pow(g2, 16);
#pragma unroll
          for (int it = 0; it < 4; ++it) {
#pragma unroll
            for (int e = 0; e < 4; ++e) O[it][e] *= f;
            f *= to16;
          }
        }
        __syncthreads();
      }
      if (!mine) continue;
      const int lane = la_lane_id(), cl = lane & 15, g = lane >> 4;
      // (la_swizzle(16 t + c) = la_swizzle(c) ^ t for c < 16; a column is 128 bytes: exchanging units changes its low bits alone)
      const int kat = cl * 128 + (g ^ la_swizzle(cl)) * 16, vat = (16 * wave + cl) * 128 + (g ^ la_swizzle(16 * wave + cl)) * 16;
      auto v_frag = [&](int kb) { return *(const la_u32x4*)(lds.vt + (vat ^ 64 * kb)); };
      auto kt_frag = [&](int t, int kb) { return *(const la_u32x4*)(lds.kt + (kat ^ 16 * (4 * kb ^ (t & 7))) + t * 16 * 128); };
      if (OUT) {
        // O^T += V^T P^T
        la_u32x4 pf[2][6], vf[2];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) vf[kb] = v_frag(kb);
#pragma unroll
        for (int part = 0; part < 2; ++part) {
#pragma unroll
          for (int i = 0; i < 6; ++i) pf[part][i] = *(const la_u32x4*)&lds.p[i][part][lane * 16];
          if (part == 0) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int it = 0; it < 4; ++it) O[it] = la_mfma16(vf[0], pf[part][la_pair(it, 0)], O[it]);
#pragma unroll
          for (int it = 2; it < 4; ++it) O[it] = la_mfma16(vf[1], pf[part][la_pair(it, 1)], O[it]);
        }
      }
      if (OUT && (gq > 1 || last)) {
        // element e of tile it is (value 16 wave + 4 g + e, step 16 it + cl)
        const LaBlock<la_bf16> o = la_block<la_bf16>(R.o, row, R.back, n, q_head(st));
#pragma unroll
        for (int it = 0; it < 4; ++it) {
          const unsigned at = la_lane<la_bf16>(R.o, R.back, cl, 16 * wave + 4 * g) + o.at0 + (unsigned)(16 * it * o.ld);
          const la_u32x2 y = {la_pack(O[it][0], O[it][1]), la_pack(O[it][2], O[it][3])};
          if (VEC) {
            __builtin_amdgcn_raw_buffer_store_b64(y, o.buf, at, 0, 0);
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
              __builtin_amdgcn_raw_buffer_store_b16((short)(y[i / 2] >> 16 * (i & 1)), o.buf, 16 * wave + 4 * g + i < dv ? at + 2 * i : LA_NOWHERE, 0, 0);
          }
        }
      }
      // S = lambda^n S + K^T V', the decayed values V' in two parts (one would lose as much as the outputs' own rounding) or three
      if (rescale && (gk > 1 ? st == 0 : last)) {
#pragma unroll
        for (int t = 0; t < 2 * KT; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) S[t][e] *= factor;
      }
      if (gk > 1 || last) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
          const la_f32x4 w0 = *(const la_f32x4*)&lds.weight[32 * kb + 4 * g], w1 = *(const la_f32x4*)&lds.weight[32 * kb + 16 + 4 * g];
          const la_f32x8 x = la_widen(v_frag(kb)) * __builtin_shufflevector(w0, w1, 0, 1, 2, 3, 4, 5, 6, 7);
          const la_u32x4 h0 = la_round(x), h1 = la_rest(x, h0);
#pragma unroll
          for (int t = 0; t < 2 * KT; ++t) {
            if (t == KT && 16 * t >= dk) break;
            const la_u32x4 kf = kt_frag(t, kb);
            S[t] = la_mfma16(kf, h0, S[t]);
            S[t] = la_mfma16(kf, h1, S[t]);
          }
          if (parts > 2) {
            asm volatile("" ::: "memory");      // (k is read again, not kept)
            const la_u32x4 h2 = la_rest(x - la_widen(h0), h1);
#pragma unroll
            for (int t = 0; t < 2 * KT; ++t) {
              if (t == KT && 16 * t >= dk) break;
              S[t] = la_mfma16(kt_frag(t, kb), h2, S[t]);
            }
          }
        }
      }
    }
    frame = next;
  }

  float* dst = la_state_out(R, w, OUT);
  if (dst) {
    const __amdgpu_buffer_rsrc_t buf = la_buffer(dst);
    const int lane = la_lane_id(), key0 = 4 * (lane >> 4), col0 = 16 * wave + (lane & 15);      // (not kept from the loads)
    const unsigned state_off = (unsigned)(key0 * st_r + col0 * R.st_c) * 4;
#pragma unroll
    for (int t = 0; t < 2 * KT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int key = 16 * t + e;
        __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(S[t][e] * frame), buf, ((key + key0 < dk) & (col0 < dv)) ? state_off : LA_NOWHERE,
                                              key * st_r * 4, 0);
      }
  }
}

// ---- fp32: blocks of 32 steps, 32 x 32 x 2 MFMA (an accumulator's rows are operand values as they lie, so nothing is turned
// over).  Wave w holds the value columns 32 w .. 32 w + 31.
//
// Bound by the chain of a block's products, not by memory: 3 x 1777 steps of 6 heads, widths 72 and 100, one workgroup to a
// unit, one wave to a SIMD: the walk 36 us (MFMAs 42 %, vector issue 11 % of the time), the pass for the sums 18, the join 5;
// the 45 MB take 7.2 at 6.26 TB/s.
template <int KT, bool OUT>
struct LaLdsF32 {
  static constexpr int PITCH = KT * 32 + 4, VPITCH = PITCH;
  __align__(16) float q[OUT ? 32 * PITCH : 4];
  __align__(16) float k[32 * PITCH];
  __align__(16) float v[32 * VPITCH];
  __align__(16) float weight[32];
  __align__(16) float fade[64];
  la_f32x4 p[OUT ? KT : 1][4][64];     // each wave's share of the scores' sums: quad of rows, lane
};

template <int TILES, int NT>
__device__ __forceinline__ void la_fetch_rows(const LinattnView& x, long long first, int back, int n, int head, float* dst, int pitch) {
#pragma unroll 4
  for (int i = threadIdx.x; i < 32 * 32 * TILES; i += NT) {
    const int pos = i / (32 * TILES), d = i % (32 * TILES);
    dst[pos * pitch + d] = la_element<float>(x, first, back, n, head, pos, d);
  }
}

// groups of 4 rows x 16 bytes
template <int TILES, int PER, int NT>
__device__ __forceinline__ void la_put_rows(const la_u32x4 (&r)[PER][4], float* dst, int pitch) {
  constexpr int U = TILES * 8;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int at = threadIdx.x + i * NT;
    if (at < 8 * U) {
#pragma unroll
      for (int e = 0; e < 4; ++e) *(la_u32x4*)(dst + (at / U * 4 + e) * pitch + 4 * (at % U)) = r[i][e];
    }
  }
}

template <int N, bool OUT, bool VEC>
__global__ __launch_bounds__(64 * N, 2) void linattn_walk_f32_kernel(LinattnArgs a) {
  constexpr int C = LA_F32_ROWS, KT = N, VT = N, NT = 64 * VT;
  __shared__ LaLdsF32<N, OUT> lds;
  LinattnPlace w;
  if (!la_place(a, OUT, w)) return;
  const LinattnRole& R = a.role[w.which];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int cl = lane & 31, hh = lane >> 5;
  const int late = R.back, head = w.head, gq = w.gq, gk = R.gk;
  const int dk = R.dk, dv = R.dv, st_r = R.st_r;
  const float g2 = w.g2;

  // ---- state: element e = 4 jj + i of tile kt is (key 32 kt + 8 jj + 4 hh + i, value 32 wave + cl)
  la_f32x16 S[KT];
  const int col = 32 * wave + cl;
  unsigned state_off = (unsigned)(4 * hh * R.st_r + col * R.st_c) * 4;
  if (OUT) {
    const float* src = la_state_in(a, R, w);
    const __amdgpu_buffer_rsrc_t buf = la_buffer(src);
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int key = 32 * kt + 8 * (e / 4) + e % 4;
        const bool there = (src != nullptr) & (key + 4 * hh < dk) & (col < dv);
        S[kt][e] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(buf, there ? state_off : LA_NOWHERE, key * st_r * 4, 0));
      }
  } else {
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) S[kt] = la_f32x16{};
  }

  float row_in = 0.0f;
  if (OUT) {
    for (int i = threadIdx.x; i < 64; i += NT) lds.fade[i] = i < 31 ? 0.0f : R.p_scale * la_pow(g2, i - 31);
    row_in = R.i_scale * la_pow(g2, cl + 1 - late);
  }

  const bool mine = 32 * wave < dv;            // this wave has values
  const int stages = gq > gk ? gq : gk;
  const auto q_head = [&](int st) { return w.q0 + (gq > 1 ? st : 0); };
  const auto k_head = [&](int st) { return head * gk + (gk > 1 ? st : 0); };
  constexpr int PERK = (KT + VT - 1) / VT;
  la_u32x4 qs[PERK][4], ks[PERK][4], vs[1][4];
  unsigned q_lane[PERK], k_lane[PERK];
#pragma unroll
  for (int i = 0; i < PERK; ++i) {
    const int at = threadIdx.x + i * NT, p4 = at / (8 * KT) * 4, d = at % (8 * KT) * 4;
    q_lane[i] = OUT && at < 64 * KT ? la_lane<float>(R.q, R.back, p4, d) : LA_NOWHERE;
    k_lane[i] = at < 64 * KT ? la_lane<float>(R.k, R.back, p4, d) : LA_NOWHERE;
  }
  const unsigned v_lane = la_lane<float>(R.v, R.back, (int)threadIdx.x / (8 * VT) * 4, (int)threadIdx.x % (8 * VT) * 4);
  auto request = [&](int p, int st) {           // (as in the bf16 walk: always into the same registers)
    const long long row = R.back ? w.first - p : w.first + p;
    const int n = max(0, min(C, w.p1 - p)), nk = gk > 1 || st == 0 ? n : 0;
    const LaBlock<float> k = la_block<float>(R.k, row, R.back, nk, k_head(st));
    if (OUT) {
      const LaBlock<float> q = la_block<float>(R.q, row, R.back, gq > 1 || st == 0 ? n : 0, q_head(st));
#pragma unroll
      for (int i = 0; i < PERK; ++i) la_load_group(qs[i], q, q_lane[i]);
    }
#pragma unroll
    for (int i = 0; i < PERK; ++i) la_load_group(ks[i], k, k_lane[i]);
    la_load_group(vs[0], la_block<float>(R.v, row, R.back, nk, k_head(st)), v_lane);
  };
  if (VEC) request(w.p0, 0);

  la_f32x16 O;
  for (int p = w.p0; p < w.p1; p += C) {
    const int n = min(C, w.p1 - p);
    const float keep = la_pow(g2, n);
    const long long row = R.back ? w.first - p : w.first + p;
    for (int st = 0; st < stages; ++st) {
      const bool new_q = gq > 1 || st == 0, new_kv = gk > 1 || st == 0, last = st == stages - 1;
      __syncthreads();                       // every wave has read the block before
      if (OUT && new_q) {
        if (VEC) la_put_rows<KT, PERK, NT>(qs, lds.q, lds.PITCH);
        else la_fetch_rows<KT, NT>(R.q, row, R.back, n, q_head(st), lds.q, lds.PITCH);
      }
      if (new_kv) {
        if (VEC) {
          la_put_rows<KT, PERK, NT>(ks, lds.k, lds.PITCH);
          la_put_rows<VT, 1, NT>(vs, lds.v, lds.VPITCH);
        } else {
          la_fetch_rows<KT, NT>(R.k, row, R.back, n, k_head(st), lds.k, lds.PITCH);
          la_fetch_rows<VT, NT>(R.v, row, R.back, n, k_head(st), lds.v, lds.VPITCH);
        }
        if (threadIdx.x < C) lds.weight[threadIdx.x] = R.s_scale * la_pow(g2, max(0, n - 1 + late - (int)threadIdx.x));
      }
      if (VEC) request(last ? p + C : p, last ? 0 : st + 1);
      __syncthreads();

      const float* v_ = lds.v + 4 * hh * lds.VPITCH + 32 * wave + cl;
      if (OUT) {
        const float* q_ = lds.q + cl * lds.PITCH + 4 * hh;
        const float* k_ = lds.k + cl * lds.PITCH + 4 * hh;
        // each wave takes its share of the scores' sum over the keys' width
        la_f32x16 P = {};
#pragma unroll
        for (int i = 0; i < 4 * KT / VT; ++i) {
          const int m = wave + i * VT;
          if (8 * m >= dk) break;
          const float4 k4 = *(const float4*)(k_ + 8 * m), q4 = *(const float4*)(q_ + 8 * m);
          P = __builtin_amdgcn_mfma_f32_32x32x2f32(k4.x, q4.x, P, 0, 0, 0);
          P = __builtin_amdgcn_mfma_f32_32x32x2f32(k4.y, q4.y, P, 0, 0, 0);
          P = __builtin_amdgcn_mfma_f32_32x32x2f32(k4.z, q4.z, P, 0, 0, 0);
          P = __builtin_amdgcn_mfma_f32_32x32x2f32(k4.w, q4.w, P, 0, 0, 0);
        }
#pragma unroll
        for (int jj = 0; jj < 4; ++jj) lds.p[wave][jj][lane] = la_f32x4{P[4 * jj], P[4 * jj + 1], P[4 * jj + 2], P[4 * jj + 3]};
        if (new_q && mine) {
          O = la_f32x16{};
#pragma unroll
          for (int kt = 0; kt < KT; ++kt) {
            if (kt > 0 && 32 * kt >= dk) break;
#pragma unroll
            for (int jj = 0; jj < 4; ++jj) {
              const float4 q4 = *(const float4*)(q_ + 32 * kt + 8 * jj);
              O = __builtin_amdgcn_mfma_f32_32x32x2f32(S[kt][4 * jj], q4.x, O, 0, 0, 0);
              O = __builtin_amdgcn_mfma_f32_32x32x2f32(S[kt][4 * jj + 1], q4.y, O, 0, 0, 0);
              O = __builtin_amdgcn_mfma_f32_32x32x2f32(S[kt][4 * jj + 2], q4.z, O, 0, 0, 0);
              O = __builtin_amdgcn_mfma_f32_32x32x2f32(S[kt][4 * jj + 3], q4.w, O, 0, 0, 0);
            }
          }
#pragma unroll
          for (int e = 0; e < 16; ++e) O[e] *= row_in;
        }
        __syncthreads();
        if (!mine) continue;
        const float* f = lds.fade + 31 + cl - 4 * hh;
#pragma unroll
        for (int jj = 0; jj < 4; ++jj) {
          la_f32x4 x = lds.p[0][jj][lane];
#pragma unroll
          for (int w = 1; w < VT; ++w) x += lds.p[w][jj][lane];
#pragma unroll
          for (int i = 0; i < 4; ++i) P[4 * jj + i] = x[i] * f[-(8 * jj + i)];
        }
#pragma unroll
        for (int e = 0; e < 16; ++e)
          O = __builtin_amdgcn_mfma_f32_32x32x2f32(v_[(8 * (e / 4) + e % 4) * lds.VPITCH], P[e], O, 0, 0, 0);
      }
      if (!mine) continue;
      if (gk > 1 ? st == 0 : last) {
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) S[kt] *= keep;
      }
      if (gk > 1 || last) {
        const float* k_ = lds.k + 4 * hh * lds.PITCH + cl;
        la_f32x16 x;
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = v_[(8 * (e / 4) + e % 4) * lds.VPITCH] * lds.weight[8 * (e / 4) + e % 4 + 4 * hh];
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
          if (kt > 0 && 32 * kt >= dk) break;
#pragma unroll
          for (int e = 0; e < 16; ++e)
            S[kt] = __builtin_amdgcn_mfma_f32_32x32x2f32(k_[(8 * (e / 4) + e % 4) * lds.PITCH + 32 * kt], x[e], S[kt], 0, 0, 0);
        }
      }

      if (OUT && (gq > 1 || last)) {
        // element e = 4 jj + i is (value 32 wave + 8 jj + 4 hh + i, step cl)
        const LaBlock<float> o = la_block<float>(R.o, row, R.back, n, q_head(st));
        const unsigned at = la_lane<float>(R.o, R.back, cl, 0) + o.at0;
#pragma unroll
        for (int jj = 0; jj < 4; ++jj) {
          const int c0 = 32 * wave + 8 * jj + 4 * hh;
          if (VEC) {
            const la_f32x4 y = {O[4 * jj], O[4 * jj + 1], O[4 * jj + 2], O[4 * jj + 3]};
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(la_u32x4, y), o.buf, c0 < dv ? at + 4 * c0 : LA_NOWHERE, 0, 0);
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
              __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(O[4 * jj + i]), o.buf, c0 + i < dv ? at + 4 * (c0 + i) : LA_NOWHERE, 0, 0);
          }
        }
      }
    }
  }

  float* dst = la_state_out(R, w, OUT);
  if (dst) {
    const __amdgpu_buffer_rsrc_t buf = la_buffer(dst);
    int key0 = 4 * hh, col0 = col;
    asm volatile("" : "+v"(state_off), "+v"(key0), "+v"(col0));      // (formed again, not kept from the loads)
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int key = 32 * kt + 8 * (e / 4) + e % 4;
        __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(S[kt][e]), buf, ((key + key0 < dk) & (col0 < dv)) ? state_off : LA_NOWHERE,
                                              key * st_r * 4, 0);
      }
  }
}

// The states that enter the segments, from what each segment adds: start[0] = the sequence's first state,
// start[m + 1] = lambda^rows start[m] + sum[m], in place (of one segment: its copy, see la_copied).  One thread an element, grid
// (elements, kv heads, roles x sequences).
// Bound by memory: 32 heads' 16 segments of 128 x 128 (2 x 33.5 MB) 15 us, 24 packed sequences' 128 segments of 8 heads 31 us.
__global__ __launch_bounds__(256) void linattn_join_kernel(LinattnArgs a) {
  const long long at = a.join0 + blockIdx.z;
  const int b = (int)(at % a.B), head = blockIdx.y;
  const LinattnRole& R = a.role[at / a.B];
  const int n = R.dk * R.dv, i = blockIdx.x * 256 + threadIdx.x;
  int row0 = 0, len = a.T;
  if (a.offsets) la_rows(a, b, row0, len);
  const int slot = la_first_slot(a, b, row0), count = min(la_count(a, len), a.slots - slot);
  if (i >= n || count < (la_copied(a, R) ? 1 : 2)) return;
  const float f = la_pow(a.log_decay[head] * 1.44269504088896340736f, a.seg_rows);
  float* p = R.seg + ((long long)slot * a.kv_heads + head) * n + i;
  const long long stride = (long long)a.kv_heads * n;
  float run = R.start ? R.start[((long long)b * a.kv_heads + head) * n + i] : 0.0f;
  // (eight sums are asked for at once: one after the other they would cost a memory's latency each)
  for (int m0 = 0; m0 < count; m0 += 8) {
    float sum[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] = m0 + e < count - 1 ? p[e * stride] : 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (m0 + e < count) p[e * stride] = run;
      run = f * run + sum[e];
    }
    p += 8 * stride;
  }
}

// ------------------------------------------------------------------------------------------------------------------
// single steps
// ------------------------------------------------------------------------------------------------------------------
struct LinattnStepArgs {
  LinattnView q, k, v, o;
  const float* log_decay;
  float* state;
  const int* slots;     // [B] or NULL
  int n_slots, B, kv_heads, group;
  int dk, dv;
  float scale;
  int vec;              // state rows are read in 16-byte pieces
};

__device__ __forceinline__ float la_value(float x) { return x; }
__device__ __forceinline__ float la_value(la_bf16 x) { return __uint_as_float((uint32_t)x << 16); }
__device__ __forceinline__ void la_store(float* p, float x) { *p = x; }
__device__ __forceinline__ void la_store(la_bf16* p, float x) { *(__bf16*)p = (__bf16)x; }

constexpr int LA_STEP_GROUP = 8;   // query heads whose sums are taken at once

// One workgroup takes COLS value columns of one row's state: every element is read and written once, which is all the time
// there is to it.  A thread holds 4 columns of every (1024 / COLS)-th key; the sums over keys of q * S meet through lanes
// and LDS.  States pass by the caches (non-temporal): between two steps of a layer those of the others come.  250 rows (some
// without a place) of 8 states of 128 x 128, 237 MB in and out: 52.4 us with states last used long ago, 49.6 used by the call
// before (with ordinary loads and stores 68.2 and 49.5; multiplying as many floats in place takes 47.5 and 37.1); one row
// of 8 states of 64 x 64: 4.9 us, a launch's time.
template <typename T, int COLS>
__global__ __launch_bounds__(256) void linattn_step_kernel(LinattnStepArgs a) {
  constexpr int CW = COLS / 4, RG = 256 / CW, PER = LA_MAX_D / RG;
  __shared__ float key_s[LA_MAX_D], query_s[LA_STEP_GROUP][LA_MAX_D];
  __shared__ float sum_s[4][LA_STEP_GROUP][COLS];
  __shared__ int next_s;
  const int slices = (a.dv + COLS - 1) / COLS;
  const int slice = blockIdx.x % slices, unit = blockIdx.x / slices, head = unit % a.kv_heads;
  int row = unit / a.kv_heads;
  const int slot = a.slots ? a.slots[row] : row;
  if (slot < 0 || slot >= a.n_slots) return;
  const int cg = threadIdx.x % CW, rg = threadIdx.x / CW, wave = threadIdx.x >> 6;
  const int c0 = slice * COLS + 4 * cg;
  float* base = a.state + ((long long)slot * a.kv_heads + head) * a.dk * a.dv + c0;
  float x[PER][4];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int r = rg + i * RG;
#pragma unroll
    for (int c = 0; c < 4; ++c) x[i][c] = 0.0f;
    if (r < a.dk) {
      if (a.vec) {
        if (c0 < a.dv) {
          const la_f32x4 y = __builtin_nontemporal_load((const la_f32x4*)(base + (long long)r * a.dv));
#pragma unroll
          for (int c = 0; c < 4; ++c) x[i][c] = y[c];
        }
      } else {
#pragma unroll
        for (int c = 0; c < 4; ++c)
          if (c0 + c < a.dv) x[i][c] = base[(long long)r * a.dv + c];
      }
    }
  }
  // rows that name this slot: the first one's workgroup takes them all, in their order
  int more = 0;
  if (a.slots) {
    int before = 0, after = 0;
    for (int i = threadIdx.x; i < a.B; i += 256) {
      const int same = a.slots[i] == slot;
      before |= same && i < row;
      after |= same && i > row;
    }
    if (__syncthreads_or(before)) return;
    more = __syncthreads_or(after);
  }
  const float lam = expf(a.log_decay[head]);
  while (true) {
    const T* k = (const T*)a.k.p + row * a.k.ld + (long long)head * a.dk;
    const T* v = (const T*)a.v.p + row * a.v.ld + (long long)head * a.dv;
    if (threadIdx.x < a.dk) key_s[threadIdx.x] = la_value(k[threadIdx.x]);
    float val[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) val[c] = c0 + c < a.dv ? la_value(v[c0 + c]) : 0.0f;
    for (int g0 = 0; g0 < a.group; g0 += LA_STEP_GROUP) {
      const int ng = min(LA_STEP_GROUP, a.group - g0);
      const T* q = (const T*)a.q.p + row * a.q.ld + ((long long)head * a.group + g0) * a.dk;
      for (int i = threadIdx.x; i < ng * a.dk; i += 256) query_s[i / a.dk][i % a.dk] = la_value(q[i]);
      __syncthreads();
      if (g0 == 0) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          const int r = rg + i * RG;
          if (r < a.dk) {
#pragma unroll
            for (int c = 0; c < 4; ++c) x[i][c] = lam * x[i][c] + key_s[r] * val[c];
          }
        }
      }
      for (int g = 0; g < ng; ++g) {
        float acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          const int r = rg + i * RG;
          if (r < a.dk) {
#pragma unroll
            for (int c = 0; c < 4; ++c) acc[c] += query_s[g][r] * x[i][c];
          }
        }
#pragma unroll
        for (int d = CW; d < 64; d <<= 1) {
#pragma unroll
          for (int c = 0; c < 4; ++c) acc[c] += __shfl_xor(acc[c], d);
        }
        if ((threadIdx.x & 63) < CW) *(float4*)&sum_s[wave][g][4 * cg] = make_float4(acc[0], acc[1], acc[2], acc[3]);
      }
      __syncthreads();
      for (int i = threadIdx.x; i < ng * COLS; i += 256) {
        const int g = i / COLS, c = i % COLS;
        if (slice * COLS + c < a.dv)
          la_store((T*)a.o.p + row * a.o.ld + ((long long)head * a.group + g0 + g) * a.dv + slice * COLS + c,
                   a.scale * (sum_s[0][g][c] + sum_s[1][g][c] + sum_s[2][g][c] + sum_s[3][g][c]));
      }
    }
    if (!more) break;
    if (threadIdx.x == 0) next_s = a.B;
    __syncthreads();
    for (int i = row + 1 + threadIdx.x; i < a.B; i += 256)
      if (a.slots[i] == slot) {
        atomicMin(&next_s, i);
        break;
      }
    __syncthreads();
    if (next_s >= a.B) break;
    row = next_s;
    __syncthreads();       // (next_s, key_s and query_s are written again)
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int r = rg + i * RG;
    if (r < a.dk) {
      if (a.vec) {
        if (c0 < a.dv)
          __builtin_nontemporal_store(la_f32x4{x[i][0], x[i][1], x[i][2], x[i][3]}, (la_f32x4*)(base + (long long)r * a.dv));
      } else {
#pragma unroll
        for (int c = 0; c < 4; ++c)
          if (c0 + c < a.dv) base[(long long)r * a.dv + c] = x[i][c];
      }
    }
  }
}

}  // namespace jm
