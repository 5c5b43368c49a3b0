// Linear attention with a decay for each head (gfx950 only).
//
//     S_t = lambda S_{t-1} + k_t v_t^T,    o_t = scale S_t^T q_t
//
// The recurrence over C steps at once, from the state S that enters them (i, j = 0 .. C-1):
//     o_i = scale ( lambda^(i+1) S^T q_i + sum_{j <= i} lambda^(i-j) (q_i . k_j) v_j )
//     S  <- lambda^C S + sum_j lambda^(C-1-j) k_j v_j^T
// which is four matrix products.  One workgroup owns the state of one head for a run of steps (a segment) and walks its
// blocks of C steps: the state stays in accumulator registers, wave w holds its value columns 32 w .. 32 w + 31, the
// block's q, k, v pass through LDS, the next block's are requested before the products of this one.
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
typedef __attribute__((ext_vector_type(4))) __bf16 la_bf16x4;
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
  int parts;            // bf16: parts the decayed values are split into for the state (1: rounded; 3: exact to fp32)
  float p_scale, s_scale, i_scale;   // factors of the scores, of what enters the state, of what is read from it
};

struct LinattnArgs {
  LinattnRole role[3];
  const float* log_decay;
  const int* offsets;   // [B + 1] or NULL
  int B, T, kv_heads;
  int roles;
  int seg_rows;         // rows of a segment (a multiple of the block)
  int slots;            // segments in all (packed: an upper bound)
};

// lambda^n, g2 = log2 lambda (the hardware's exponential is within 1 ulp; below 2^-126 it is zero)
__device__ __forceinline__ float la_pow(float g2, int n) {
  const float x = __builtin_amdgcn_exp2f(g2 * (float)n);
  return n == 0 ? 1.0f : x;
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

__device__ __forceinline__ int la_count(const LinattnArgs& a, int len) { return max(1, (len + a.seg_rows - 1) / a.seg_rows); }

// The segment with number `slot` (false: there are fewer).  Packed sequences: every wave adds up the counts of 64
// sequences at a time.
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
  int base = 0;
  for (int b0 = 0; b0 < a.B; b0 += 64) {
    int row0 = 0, len = 0, n = 0;
    if (b0 + lane < a.B) {
      la_rows(a, b0 + lane, row0, len);
      n = la_count(a, len);
    }
    int incl = n;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int up = __shfl_up(incl, d);
      if (lane >= d) incl += up;
    }
    const unsigned long long hit = __ballot(slot < base + incl);
    if (hit) {
      const int f = __ffsll((long long)hit) - 1;
      s.b = b0 + f;
      s.count = __builtin_amdgcn_readfirstlane(__shfl(n, f));
      s.index = slot - base - (__builtin_amdgcn_readfirstlane(__shfl(incl, f)) - s.count);
      s.row0 = __builtin_amdgcn_readfirstlane(__shfl(row0, f));
      s.len = __builtin_amdgcn_readfirstlane(__shfl(len, f));
      return true;
    }
    base += __builtin_amdgcn_readfirstlane(__shfl(incl, 63));
  }
  return false;
}

// Number of the first segment of sequence b, and its rows.
__device__ __forceinline__ int la_first_slot(const LinattnArgs& a, int b, int& len) {
  if (!a.offsets) {
    len = a.T;
    return b * la_count(a, a.T);
  }
  const int lane = threadIdx.x & 63;
  int n = 0, row0 = 0;
  for (int i = lane; i < b; i += 64) {
    la_rows(a, i, row0, len);
    n += la_count(a, len);
  }
#pragma unroll
  for (int d = 32; d; d >>= 1) n += __shfl_xor(n, d);
  la_rows(a, b, row0, len);
  return n;
}

// ------------------------------------------------------------------------------------------------------------------
// the walk
// ------------------------------------------------------------------------------------------------------------------
template <typename T>
struct LaShape;
template <>
struct LaShape<la_bf16> {
  static constexpr int C = 64;
};
template <>
struct LaShape<float> {
  static constexpr int C = 32;
};

// Memory is reached through buffer descriptors: a lane whose element does not exist gets an offset past the end, reads zero
// and writes nothing, without a branch.  An offset is a lane's part, below 2^30 bytes or LA_NOWHERE, and a scalar part.
constexpr unsigned LA_NOWHERE = 0x80000000u;

__device__ __forceinline__ __amdgpu_buffer_rsrc_t la_buffer(const void* p) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, 0x7fffffff, 0x00027000);
}

// The C rows of a block as they lie in memory: position p of the walk is row p (forward) or C - 1 - p (back) from `base`.
template <typename T>
__device__ __forceinline__ const T* la_block(const LinattnView& x, long long first, int back, int head) {
  return (const T*)x.p + (back ? first - (LaShape<T>::C - 1) : first) * x.ld + (long long)head * x.dim;
}

// A thread's share of a block of an operand whose rows come in 16-byte pieces: groups of 4 consecutive rows x 1 piece,
// group tid + i NT.
template <typename T, int TILES, int NT>
struct LaStage {
  static constexpr int C = LaShape<T>::C;
  static constexpr int PIECE = 16 / sizeof(T);
  static constexpr int U = TILES * 32 / PIECE;                // pieces of a row
  static constexpr int N = (C / 4) * U;                       // groups
  static constexpr int PER = (N + NT - 1) / NT;
  static constexpr int NTG = NT / U;                          // groups of rows the threads hold at a time
  la_u32x4 r[PER][4];

  static __device__ __forceinline__ int piece() { return threadIdx.x % U; }
  static __device__ __forceinline__ int group() { return threadIdx.x / U; }

  // rows at positions 0 .. n-1 of the block; beyond n and dim: zeros
  __device__ __forceinline__ void load(const LinattnView& x, long long first, int back, int n, int head) {
    const __amdgpu_buffer_rsrc_t buf = la_buffer(la_block<T>(x, first, back, head));
    const unsigned ld = (unsigned)x.ld * (unsigned)sizeof(T);                // (at most 2^25 bytes: the host checks)
    const int t0 = group(), t0_row = back ? C / 4 - 1 - (PER - 1) * NTG - t0 : t0;
    const unsigned off = (unsigned)(4 * t0_row) * ld + piece() * 16;
    const bool in_row = piece() * PIECE < x.dim;
#pragma unroll
    for (int i = 0; i < PER; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const unsigned rows = back ? 4 * (PER - 1 - i) * NTG + 3 - e : 4 * i * NTG + e;
        const bool there = in_row && 4 * (t0 + i * NTG) + e < n;
        r[i][e] = __builtin_amdgcn_raw_buffer_load_b128(buf, there ? off : LA_NOWHERE, __builtin_amdgcn_readfirstlane(rows * ld), 0);
      }
  }
};

// Where an operand's rows are not made of 16-byte pieces its elements are fetched one by one when LDS is filled.
template <typename T>
__device__ __forceinline__ T la_element(const LinattnView& x, long long first, int back, int n, int head, int pos, int d) {
  return pos < n && d < x.dim ? ((const T*)x.p)[(back ? first - pos : first + pos) * x.ld + (long long)head * x.dim + d] : (T)0;
}

template <typename T, int KT, int VT, bool OUT>
struct LaLds;
// bf16: q and k by rows (two quads of every 16 exchanged: the order an accumulator's rows have as an operand), k and v by
// columns, steps in the same order, 16-byte units of a column exchanged among each other so that neither the writes by rows
// nor the reads by columns meet in a bank
template <int KT, int VT, bool OUT>
struct LaLds<la_bf16, KT, VT, OUT> {
  static constexpr int PITCH = KT * 32 * 2 + 16;
  __align__(16) unsigned char q[OUT ? 64 * PITCH : 16];
  __align__(16) unsigned char k[OUT ? 64 * PITCH : 16];
  __align__(16) unsigned char kt[KT * 32 * 128];
  __align__(16) unsigned char vt[VT * 32 * 128];
  __align__(16) float weight[64];      // lambda^(n-1+late-j) of step j of the block: what the block's end keeps of it
  __align__(16) float fade[96];        // p_scale lambda^m at 31 + m, zeros before: the factor of a pair of steps m apart
  __align__(16) unsigned char p[OUT ? 3 : 1][2][2][64 * 16];   // scores as operands: tile, half of its steps, part, lane
};
template <int KT, int VT, bool OUT>
struct LaLds<float, KT, VT, OUT> {
  static constexpr int PITCH = KT * 32 + 4, VPITCH = VT * 32 + 4;
  __align__(16) float q[OUT ? 32 * PITCH : 4];
  __align__(16) float k[32 * PITCH];
  __align__(16) float v[32 * VPITCH];
  __align__(16) float weight[32];
  __align__(16) float fade[64];
  la_f32x4 p[OUT ? VT : 1][4][64];     // each wave's share of the scores' sums: quad of rows, lane
};

__device__ __forceinline__ int la_swizzle(int d) { return ((d >> 1) ^ (d >> 4)) & 7; }

// place of step `pos` (of the block) in a column, in bf16 elements: unit of 8, quad and element of the quad
__device__ __forceinline__ int la_unit(int tg) { return 2 * (tg >> 2) + (tg & 1); }       // tg = pos / 4
__device__ __forceinline__ int la_half(int tg) { return (tg >> 1) & 1; }

template <int TILES, int NT>
__device__ __forceinline__ void la_put_rows(const LaStage<la_bf16, TILES, NT>& st, unsigned char* dst, int pitch) {
  typedef LaStage<la_bf16, TILES, NT> S;
  const int u = S::piece(), t0 = S::group();
#pragma unroll
  for (int i = 0; i < S::PER; ++i) {
    const int tg = t0 + i * S::NTG;
    if (tg < 16) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        unsigned char* p = dst + (4 * tg + e) * pitch + (u >> 1) * 32 + (u & 1) * 8;
        *(uint2*)p = make_uint2(st.r[i][e][0], st.r[i][e][1]);
        *(uint2*)(p + 16) = make_uint2(st.r[i][e][2], st.r[i][e][3]);
      }
    }
  }
}

template <int TILES, int NT>
__device__ __forceinline__ void la_put_columns(const LaStage<la_bf16, TILES, NT>& st, unsigned char* dst) {
  typedef LaStage<la_bf16, TILES, NT> S;
  const int u = S::piece(), t0 = S::group();
#pragma unroll
  for (int i = 0; i < S::PER; ++i) {
    const int tg = t0 + i * S::NTG;
    if (tg < 16) {
      // (la_swizzle(8 u + dd) = la_swizzle(8 u) ^ dd / 2: four addresses and fixed distances from them)
      unsigned char* column = dst + 8 * u * 128 + la_half(tg) * 8;
      const int unit = la_unit(tg) ^ la_swizzle(8 * u);
#pragma unroll
      for (int dd = 0; dd < 8; ++dd) {
        const uint32_t sel = dd & 1 ? 0x07060302u : 0x05040100u;
        uint2 o;
        o.x = __builtin_amdgcn_perm(st.r[i][1][dd / 2], st.r[i][0][dd / 2], sel);
        o.y = __builtin_amdgcn_perm(st.r[i][3][dd / 2], st.r[i][2][dd / 2], sel);
        *(uint2*)(column + ((unit ^ (dd / 2)) * 16) + dd * 128) = o;
      }
    }
  }
}

template <int TILES, int NT>
__device__ __forceinline__ void la_put_rows(const LaStage<float, TILES, NT>& st, float* dst, int pitch) {
  typedef LaStage<float, TILES, NT> S;
  const int u = S::piece(), t0 = S::group();
#pragma unroll
  for (int i = 0; i < S::PER; ++i) {
    const int tg = t0 + i * S::NTG;
    if (tg < 8) {
#pragma unroll
      for (int e = 0; e < 4; ++e) *(la_u32x4*)(dst + (4 * tg + e) * pitch + 4 * u) = st.r[i][e];
    }
  }
}

// the same from memory, element by element
template <int TILES, int NT>
__device__ __forceinline__ void la_fetch_rows(const LinattnView& x, long long first, int back, int n, int head, unsigned char* dst, int pitch) {
#pragma unroll 4
  for (int i = threadIdx.x; i < 64 * 32 * TILES; i += NT) {
    const int pos = i / (32 * TILES), d = i % (32 * TILES);
    // quads 1 and 2 of every 16 elements are exchanged
    const int at = (d & ~12) | (d & 4) << 1 | (d & 8) >> 1;
    *(la_bf16*)(dst + pos * pitch + 2 * at) = la_element<la_bf16>(x, first, back, n, head, pos, d);
  }
}

template <int TILES, int NT>
__device__ __forceinline__ void la_fetch_columns(const LinattnView& x, long long first, int back, int n, int head, unsigned char* dst) {
#pragma unroll 4
  for (int i = threadIdx.x; i < 64 * 32 * TILES; i += NT) {
    const int pos = i / (32 * TILES), d = i % (32 * TILES), tg = pos / 4;
    *(la_bf16*)(dst + d * 128 + (la_unit(tg) ^ la_swizzle(d)) * 16 + la_half(tg) * 8 + (pos & 3) * 2) =
        la_element<la_bf16>(x, first, back, n, head, pos, d);
  }
}

template <int TILES, int NT>
__device__ __forceinline__ void la_fetch_rows(const LinattnView& x, long long first, int back, int n, int head, float* dst, int pitch) {
#pragma unroll 4
  for (int i = threadIdx.x; i < 32 * 32 * TILES; i += NT) {
    const int pos = i / (32 * TILES), d = i % (32 * TILES);
    dst[pos * pitch + d] = la_element<float>(x, first, back, n, head, pos, d);
  }
}

// fp32 values as two bf16 parts, x = hi + lo + O(2^-17 x)
__device__ __forceinline__ la_bf16x8 la_round(la_f32x8 x) { return __builtin_convertvector(x, la_bf16x8); }
__device__ __forceinline__ la_bf16x8 la_rest(la_f32x8 x, la_bf16x8 hi) { return la_round(x - __builtin_convertvector(hi, la_f32x8)); }

// OUT = true: the walk with outputs.  OUT = false: only the state a segment adds, from zero, into the workspace.
// VEC: every operand's rows come in 16-byte pieces (else none is taken to).
template <typename T, int KT, int VT, bool OUT, bool VEC>
__global__ __launch_bounds__(64 * VT, KT > VT ? 1 : 2) void linattn_walk_kernel(LinattnArgs a) {
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int C = LaShape<T>::C, IT = C / 32, NT = 64 * VT;
  __shared__ LaLds<T, KT, VT, OUT> lds;

  // the roles of a unit (segment, head) read the same arrays: their workgroups have numbers that are equal modulo 8, so
  // that one XCD's L2 sees all of them
  const int id = blockIdx.x, pack = 8 * a.roles;
  const int unit = id / pack * 8 + id % 8, which = id % pack / 8;
  if (unit >= a.slots * a.kv_heads) return;
  const LinattnRole& R = a.role[which];
  const int head = unit % a.kv_heads;
  LinattnSegment s;
  if (!la_find(a, unit / a.kv_heads, s)) return;
  // (the same in every lane: they form addresses that are scalars)
  s.b = __builtin_amdgcn_readfirstlane(s.b);
  s.index = __builtin_amdgcn_readfirstlane(s.index);
  s.count = __builtin_amdgcn_readfirstlane(s.count);
  s.row0 = __builtin_amdgcn_readfirstlane(s.row0);
  s.len = __builtin_amdgcn_readfirstlane(s.len);
  if (!OUT && s.index == s.count - 1) return;    // (nothing follows the last segment)

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int cl = lane & 31, hh = lane >> 5;
  const float g2 = a.log_decay[head] * 1.44269504088896340736f;
  const int late = R.back;
  const int p0 = s.index * a.seg_rows, p1 = min(p0 + a.seg_rows, s.len);    // positions in the order of the walk
  const long long seq_row = a.offsets ? (long long)s.row0 : (long long)s.b * a.T;
  const long long first = R.back ? seq_row + s.len - 1 : seq_row;           // row of position 0
  const long long state_at = ((long long)s.b * a.kv_heads + head) * R.dk * R.dv;

  // ---- state: element e = 4 jj + i of tile kt is (key 32 kt + 8 jj + 4 hh + i, value 32 wave + cl)
  la_f32x16 S[KT];
  const int col = 32 * wave + cl;
  unsigned state_off = (unsigned)(4 * hh * R.st_r + col * R.st_c) * 4;
  const long long seg_at = ((long long)(unit / a.kv_heads) * a.kv_heads + head) * R.dk * R.dv;
  {
    const float* src = !OUT ? nullptr : R.seg && s.count > 1 ? R.seg + seg_at : R.start ? R.start + state_at : nullptr;
    const __amdgpu_buffer_rsrc_t buf = la_buffer(src);
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int key = 32 * kt + 8 * (e / 4) + e % 4;
        const bool there = src && key + 4 * hh < R.dk && col < R.dv;
        S[kt][e] = OUT ? __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(buf, there ? state_off : LA_NOWHERE, key * R.st_r * 4, 0)) : 0.0f;
      }
  }

  float row_in[IT];
  if (OUT) {
    for (int i = threadIdx.x; i < C + 32; i += NT) lds.fade[i] = i < 31 ? 0.0f : R.p_scale * la_pow(g2, i - 31);
#pragma unroll
    for (int it = 0; it < IT; ++it) row_in[it] = R.i_scale * la_pow(g2, 32 * it + cl + 1 - late);
  }

  LaStage<T, KT, NT> qs, ks;
  LaStage<T, VT, NT> vs;
  const int stages = R.gq > R.gk ? R.gq : R.gk;
  const auto q_head = [&](int st) { return head * R.gq + (R.gq > 1 ? st : 0); };
  const auto k_head = [&](int st) { return head * R.gk + (R.gk > 1 ? st : 0); };
  // The next block's pieces, always into the same registers: what a stage does not need is asked for from nowhere (a branch
  // around the loads would have their results moved, and so waited for, where it ends).
  auto request = [&](int p, int st) {
    const long long row = R.back ? first - p : first + p;
    const int n = min(C, p1 - p);                                          // (none behind the last block)
    if (OUT && VEC) qs.load(R.q, row, R.back, R.gq > 1 || st == 0 ? n : 0, q_head(st));
    if (VEC) {
      const int nk = R.gk > 1 || st == 0 ? n : 0;
      ks.load(R.k, row, R.back, nk, k_head(st));
      vs.load(R.v, row, R.back, nk, k_head(st));
    }
  };
  request(p0, 0);

  la_f32x16 O[IT];
  for (int p = p0; p < p1; p += C) {
    const int n = min(C, p1 - p);
    const float keep = la_pow(g2, n);
    for (int st = 0; st < stages; ++st) {
      const bool new_q = R.gq > 1 || st == 0, new_kv = R.gk > 1 || st == 0, last = st == stages - 1;
      __syncthreads();                       // every wave has read the block before
      const long long row = R.back ? first - p : first + p;
      if (OUT && new_q) {
        if (VEC) la_put_rows(qs, lds.q, lds.PITCH);
        else la_fetch_rows<KT, NT>(R.q, row, R.back, n, q_head(st), lds.q, lds.PITCH);
      }
      if (new_kv) {
        if constexpr (F32) {
          if (VEC) la_put_rows(ks, lds.k, lds.PITCH);
          else la_fetch_rows<KT, NT>(R.k, row, R.back, n, k_head(st), lds.k, lds.PITCH);
          if (VEC) la_put_rows(vs, lds.v, lds.VPITCH);
          else la_fetch_rows<VT, NT>(R.v, row, R.back, n, k_head(st), lds.v, lds.VPITCH);
        } else {
          if (VEC) {
            if (OUT) la_put_rows(ks, lds.k, lds.PITCH);
            la_put_columns(ks, lds.kt);
          } else {
            if (OUT) la_fetch_rows<KT, NT>(R.k, row, R.back, n, k_head(st), lds.k, lds.PITCH);
            la_fetch_columns<KT, NT>(R.k, row, R.back, n, k_head(st), lds.kt);
          }
          if (VEC) la_put_columns(vs, lds.vt);
          else la_fetch_columns<VT, NT>(R.v, row, R.back, n, k_head(st), lds.vt);
        }
        if (threadIdx.x < C) lds.weight[threadIdx.x] = R.s_scale * la_pow(g2, max(0, n - 1 + late - (int)threadIdx.x));
      }
      request(last ? p + C : p, last ? 0 : st + 1);
      __syncthreads();

      if constexpr (!F32) {
        // (la_swizzle(32 n + c) = la_swizzle(c) ^ 2 n: unit 2 mb + hh of column 32 kt + cl lies where mb ^ kt says)
        const unsigned char* kt_ = lds.kt + cl * 128;
        const unsigned char* vt_ = lds.vt + (32 * wave + cl) * 128;
        const int ksw = (hh ^ la_swizzle(cl)) * 16, vsw = (hh ^ la_swizzle(32 * wave + cl)) * 16;
        auto v_frag = [&](int mb) { return __builtin_bit_cast(la_bf16x8, *(const uint4*)(vt_ + (vsw ^ 32 * mb))); };
        auto kt_frag = [&](int kt, int mb) {
          return __builtin_bit_cast(la_bf16x8, *(const uint4*)(kt_ + (ksw ^ 32 * (mb ^ kt)) + kt * 32 * 128));
        };
        if (OUT) {
          const unsigned char* q_ = lds.q + cl * lds.PITCH + hh * 16;
          const unsigned char* k_ = lds.k + cl * lds.PITCH + hh * 16;
          auto q_frag = [&](int it, int m) { return __builtin_bit_cast(la_bf16x8, *(const uint4*)(q_ + it * 32 * lds.PITCH + m * 32)); };
          auto k_frag = [&](int jt, int m) { return __builtin_bit_cast(la_bf16x8, *(const uint4*)(k_ + jt * 32 * lds.PITCH + m * 32)); };
          // Scores of the tiles (steps jt, queries it), transposed, a tile to a wave: every wave needs them all, as operands
          // in two parts, and gets them through LDS while its product with the state runs.
#pragma unroll
          for (int t = 0; t < 3; ++t) {
            if (t % VT != wave) continue;
            const int jt = t >> 1, it = (t + 1) >> 1;
            la_f32x16 P = {};
#pragma unroll
            for (int m = 0; m < 2 * KT; ++m) P = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k_frag(jt, m), q_frag(it, m), P, 0, 0, 0);
            const float* f = lds.fade + 31 + 32 * (it - jt) + cl - 4 * hh;
#pragma unroll
            for (int mm = 0; mm < 2; ++mm) {
              la_f32x8 x;
#pragma unroll
              for (int e = 0; e < 8; ++e) x[e] = P[8 * mm + e] * f[-(16 * mm + 8 * (e / 4) + e % 4)];
              const la_bf16x8 hi = la_round(x);
              *(la_bf16x8*)&lds.p[t][mm][0][lane * 16] = hi;
              *(la_bf16x8*)&lds.p[t][mm][1][lane * 16] = la_rest(x, hi);
            }
          }
          if (new_q) {
            // O^T = S^T Q^T: the accumulator of the state is an operand as it lies
#pragma unroll
            for (int it = 0; it < IT; ++it) O[it] = la_f32x16{};
#pragma unroll
            for (int kt = 0; kt < KT; ++kt)
#pragma unroll
              for (int mm = 0; mm < 2; ++mm) {
                la_f32x8 x;
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = S[kt][8 * mm + e];
                const la_bf16x8 hi = la_round(x), lo = la_rest(x, hi);
#pragma unroll
                for (int it = 0; it < IT; ++it) {
                  const la_bf16x8 qf = q_frag(it, 2 * kt + mm);
                  O[it] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(hi, qf, O[it], 0, 0, 0);
                  O[it] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lo, qf, O[it], 0, 0, 0);
                }
              }
#pragma unroll
            for (int it = 0; it < IT; ++it)
#pragma unroll
              for (int e = 0; e < 16; ++e) O[it][e] *= row_in[it];
          }
          __syncthreads();
          // O^T += V^T P^T
#pragma unroll
          for (int t = 0; t < 3; ++t) {
            const int jt = t >> 1, it = (t + 1) >> 1;
#pragma unroll
            for (int mm = 0; mm < 2; ++mm) {
              const la_bf16x8 vf = v_frag(2 * jt + mm);
              O[it] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, *(const la_bf16x8*)&lds.p[t][mm][0][lane * 16], O[it], 0, 0, 0);
              O[it] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, *(const la_bf16x8*)&lds.p[t][mm][1][lane * 16], O[it], 0, 0, 0);
            }
          }
        }
        // S = lambda^n S + K^T V'
        if (R.gk > 1 ? st == 0 : last) {
#pragma unroll
          for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int e = 0; e < 16; ++e) S[kt][e] *= keep;
        }
        if (R.gk > 1 || last) {
#pragma unroll
          for (int mb = 0; mb < 4; ++mb) {
            const la_f32x8 v8 = __builtin_convertvector(v_frag(mb), la_f32x8);
            const float4 w0 = *(const float4*)&lds.weight[16 * mb + 4 * hh], w1 = *(const float4*)&lds.weight[16 * mb + 8 + 4 * hh];
            la_f32x8 x = {v8[0] * w0.x, v8[1] * w0.y, v8[2] * w0.z, v8[3] * w0.w, v8[4] * w1.x, v8[5] * w1.y, v8[6] * w1.z, v8[7] * w1.w};
            for (int part = 0; part < R.parts; ++part) {
              const la_bf16x8 h = la_round(x);
#pragma unroll
              for (int kt = 0; kt < KT; ++kt) {
                S[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kt_frag(kt, mb), h, S[kt], 0, 0, 0);
              }
              x -= __builtin_convertvector(h, la_f32x8);
            }
          }
        }
      } else {
        const float* v_ = lds.v + 4 * hh * lds.VPITCH + 32 * wave + cl;
        if (OUT) {
          const float* q_ = lds.q + cl * lds.PITCH + 4 * hh;
          const float* k_ = lds.k + cl * lds.PITCH + 4 * hh;
          // each wave takes its share of the scores' sum over the keys' width
          la_f32x16 P = {};
#pragma unroll
          for (int i = 0; i < 4 * KT / VT; ++i) {
            const int m = wave + i * VT;
            const float4 k4 = *(const float4*)(k_ + 8 * m), q4 = *(const float4*)(q_ + 8 * m);
            P = __builtin_amdgcn_mfma_f32_32x32x2f32(k4.x, q4.x, P, 0, 0, 0);
            P = __builtin_amdgcn_mfma_f32_32x32x2f32(k4.y, q4.y, P, 0, 0, 0);
            P = __builtin_amdgcn_mfma_f32_32x32x2f32(k4.z, q4.z, P, 0, 0, 0);
            P = __builtin_amdgcn_mfma_f32_32x32x2f32(k4.w, q4.w, P, 0, 0, 0);
          }
#pragma unroll
          for (int jj = 0; jj < 4; ++jj) lds.p[wave][jj][lane] = la_f32x4{P[4 * jj], P[4 * jj + 1], P[4 * jj + 2], P[4 * jj + 3]};
          if (new_q) {
            O[0] = la_f32x16{};
#pragma unroll
            for (int kt = 0; kt < KT; ++kt)
#pragma unroll
              for (int jj = 0; jj < 4; ++jj) {
                const float4 q4 = *(const float4*)(q_ + 32 * kt + 8 * jj);
                O[0] = __builtin_amdgcn_mfma_f32_32x32x2f32(S[kt][4 * jj], q4.x, O[0], 0, 0, 0);
                O[0] = __builtin_amdgcn_mfma_f32_32x32x2f32(S[kt][4 * jj + 1], q4.y, O[0], 0, 0, 0);
                O[0] = __builtin_amdgcn_mfma_f32_32x32x2f32(S[kt][4 * jj + 2], q4.z, O[0], 0, 0, 0);
                O[0] = __builtin_amdgcn_mfma_f32_32x32x2f32(S[kt][4 * jj + 3], q4.w, O[0], 0, 0, 0);
              }
#pragma unroll
            for (int e = 0; e < 16; ++e) O[0][e] *= row_in[0];
          }
          __syncthreads();
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
            O[0] = __builtin_amdgcn_mfma_f32_32x32x2f32(v_[(8 * (e / 4) + e % 4) * lds.VPITCH], P[e], O[0], 0, 0, 0);
        }
        if (R.gk > 1 ? st == 0 : last) {
#pragma unroll
          for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int e = 0; e < 16; ++e) S[kt][e] *= keep;
        }
        if (R.gk > 1 || last) {
          const float* k_ = lds.k + 4 * hh * lds.PITCH + cl;
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int j = 8 * (e / 4) + e % 4;
            const float x = v_[j * lds.VPITCH] * lds.weight[j + 4 * hh];
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) S[kt] = __builtin_amdgcn_mfma_f32_32x32x2f32(k_[j * lds.PITCH + 32 * kt], x, S[kt], 0, 0, 0);
          }
        }
      }

      if (OUT && (R.gq > 1 || last)) {
        // element e = 4 jj + i of tile it is (value 32 wave + 8 jj + 4 hh + i, step 32 it + cl)
        const __amdgpu_buffer_rsrc_t buf = la_buffer(la_block<T>(R.o, row, R.back, q_head(st)));
        const unsigned ld = (unsigned)R.o.ld;
#pragma unroll
        for (int it = 0; it < IT; ++it) {
          const int pos = 32 * it + cl;
          const unsigned off = ((unsigned)(R.back ? C - 1 - pos : pos) * ld + 32 * wave + 4 * hh) * (unsigned)sizeof(T);
#pragma unroll
          for (int jj = 0; jj < 4; ++jj) {
            const int c0 = 32 * wave + 8 * jj + 4 * hh;
            const la_f32x4 y = {O[it][4 * jj], O[it][4 * jj + 1], O[it][4 * jj + 2], O[it][4 * jj + 3]};
            if (VEC) {
              const unsigned at = pos < n && c0 < R.dv ? off : LA_NOWHERE;
              if constexpr (F32) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(la_u32x4, y), buf, at, 32 * jj, 0);
              else __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(la_u32x2, __builtin_convertvector(y, la_bf16x4)), buf, at, 16 * jj, 0);
            } else {
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const unsigned at = pos < n && c0 + i < R.dv ? off : LA_NOWHERE;
                if constexpr (F32) __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(y[i]), buf, at, 32 * jj + 4 * i, 0);
                else __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(short, (__bf16)y[i]), buf, at, 16 * jj + 2 * i, 0);
              }
            }
          }
        }
      }
    }
  }

  float* dst = !OUT ? R.seg + seg_at : R.end && s.index == s.count - 1 ? R.end + state_at : nullptr;
  if (dst) {
    const __amdgpu_buffer_rsrc_t buf = la_buffer(dst);
    int key0 = 4 * hh, col0 = col;
    asm volatile("" : "+v"(state_off), "+v"(key0), "+v"(col0));      // (formed again, not kept from the loads)
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int key = 32 * kt + 8 * (e / 4) + e % 4;
        __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(S[kt][e]), buf, key + key0 < R.dk && col0 < R.dv ? state_off : LA_NOWHERE,
                                              key * R.st_r * 4, 0);
      }
  }
}

// The states that enter the segments, from what each segment adds: start[0] = the sequence's first state,
// start[m + 1] = lambda^rows start[m] + sum[m], in place.  One thread an element, grid (elements, kv heads, sequences x roles).
__global__ __launch_bounds__(256) void linattn_join_kernel(LinattnArgs a) {
  const int b = blockIdx.z % a.B, head = blockIdx.y;
  const LinattnRole& R = a.role[blockIdx.z / a.B];
  const int n = R.dk * R.dv, i = blockIdx.x * 256 + threadIdx.x;
  int len;
  const int slot = la_first_slot(a, b, len), count = min(la_count(a, len), a.slots - slot);
  if (i >= n || count < 2) return;
  const float f = la_pow(a.log_decay[head] * 1.44269504088896340736f, a.seg_rows);
  float* p = R.seg + ((long long)slot * a.kv_heads + head) * n + i;
  const long long stride = (long long)a.kv_heads * n;
  float run = R.start ? R.start[((long long)b * a.kv_heads + head) * n + i] : 0.0f;
  float sum = p[0];
  for (int m = 0; m < count - 1; ++m) {
    const float next = m + 1 < count - 1 ? p[stride] : 0.0f;
    *p = run;
    run = f * run + sum;
    sum = next;
    p += stride;
  }
  *p = run;
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
// and LDS.
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
        if (c0 < a.dv) *(float4*)x[i] = *(const float4*)(base + (long long)r * a.dv);
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
        if (c0 < a.dv) *(float4*)(base + (long long)r * a.dv) = *(const float4*)x[i];
      } else {
#pragma unroll
        for (int c = 0; c < 4; ++c)
          if (c0 + c < a.dv) base[(long long)r * a.dv + c] = x[i][c];
      }
    }
  }
}

}  // namespace jm
