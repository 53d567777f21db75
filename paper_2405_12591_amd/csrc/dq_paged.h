// Shared pieces of the paged 8-bit cache's kernels: types, argument checks, norm and rotation of a row's
// piece, codes to and from 32-bit values.
#pragma once
#include "dq_common.h"

namespace dq {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kPagedTile = 64;        // tokens of a work tile and of a run of the value layout
constexpr int kPagedThreads = 256;
constexpr int kMaxAxes = 8;
constexpr long kMostTokens = (1l << 31) - 256;   // of a sequence: token indexes, and a tile's behind them, stay in 32 bits
constexpr long kMaxThreads = 1l << 32;   // a launch has fewer (along x)
constexpr float kSmallestAmax = 0x1p-100f;   // a block below it is held as zeros (its inverse step would leave fp32)

// ---- argument checks (host) ----
inline bool heads_ok(const dq_heads* x, bool batched) {
  return x && x->data && !((uintptr_t)x->data & 15) && x->heads > 0 && x->token_stride >= 0 && x->head_stride >= 0 &&
         !(x->token_stride & 7) && !(x->head_stride & 7) && (!batched || (x->batch_stride >= 0 && !(x->batch_stride & 7)));
}

inline bool norm_ok(const dq_head_norm* n) { return !n || (n->eps >= 0.f && !(((uintptr_t)n->q_weight | (uintptr_t)n->k_weight) & 15)); }

inline bool rotary_ok(const dq_rotary* r, int head_dim, long rows, bool positions_needed) {
  if (!r) return true;
  if (!r->inv_freq || r->rot_dim <= 0 || r->rot_dim % 16 || r->rot_dim > head_dim) return false;
  if (r->axes < 1 || r->axes > kMaxAxes || (r->interleaved != 0 && r->interleaved != 1)) return false;
  if (r->axes > 1 && (!r->axis_of_pair || !r->positions || r->position_stride < rows)) return false;
  if (positions_needed && !r->positions) return false;
  return true;
}

inline bool paged_cache_ok(const dq_paged_cache* c) {
  if (!c || !c->k_codes || !c->k_scales || !c->v_codes || !c->v_scales || !c->k_tail || !c->v_tail) return false;
  if (((uintptr_t)c->k_codes | (uintptr_t)c->v_codes | (uintptr_t)c->k_tail | (uintptr_t)c->v_tail) & 15) return false;
  if (((uintptr_t)c->k_scales | (uintptr_t)c->v_scales) & 3) return false;
  if (c->head_dim != 64 && c->head_dim != 128) return false;
  if (c->page_tokens != 64 && c->page_tokens != 128) return false;
  if (c->dtype != DQ_F16 && c->dtype != DQ_BF16) return false;
  if (c->codes != DQ_CODES_INT8 && c->codes != DQ_CODES_E4M3) return false;
  if (c->pages <= 0 || c->kv_heads <= 0 || c->slots <= 0) return false;
  const long runs = (long)c->kv_heads * (c->page_tokens / kPagedTile);
  return c->pages * runs < (1l << 31) && c->slots * runs < (1l << 31);
}

inline bool paged_batch_ok(const dq_paged_batch* b, const dq_paged_cache* c, bool uses_starts) {
  if (!b || !b->seq_lens || !b->page_table || b->batch <= 0 || b->rows < 0) return false;
  if (b->table_width <= 0 || b->table_stride < b->table_width) return false;
  if ((long)b->table_width * c->page_tokens >= kMostTokens) return false;
  if (uses_starts && !b->starts && b->rows != b->batch) return false;
  if (!b->tail_slots && b->batch > c->slots) return false;
  return true;
}

// ---- the batch (device) ----
// A sequence's rows and lengths, brought into the bounds of the call.
struct Sequence {
  int row0, n;      // its rows
  int old;          // tokens before them: row i is token old + i, which may lie before 0 or past `len`
  int len;          // tokens it can have here: seq_lens, or what the page table holds if that is less
};
__device__ __forceinline__ Sequence sequence_of(const dq_paged_batch& bt, int page_tokens, int b) {
  Sequence s;
  const int lo = bt.starts ? bt.starts[b] : b, hi = bt.starts ? bt.starts[b + 1] : b + 1;
  s.row0 = min(max(lo, 0), bt.rows);
  s.n = min(max(hi, s.row0), bt.rows) - s.row0;
  const int len = min(max(bt.seq_lens[b], 0), (int)kMostTokens);
  s.old = len - s.n;
  s.len = min(len, bt.table_width * page_tokens);
  return s;
}

// The same where the whole wave asks for one sequence: in scalar registers, so that loops over its tokens are scalar too (as
// vector values they made every conditional load a divergent branch, and the wait behind it one for all loads).
__device__ __forceinline__ Sequence sequence_of_wave(const dq_paged_batch& bt, int page_tokens, int b) {
  Sequence s = sequence_of(bt, page_tokens, b);
  s.row0 = __builtin_amdgcn_readfirstlane(s.row0);
  s.n = __builtin_amdgcn_readfirstlane(s.n);
  s.old = __builtin_amdgcn_readfirstlane(s.old);
  s.len = __builtin_amdgcn_readfirstlane(s.len);
  return s;
}

// Work items dealt to sequences without a scan: with `at` the rows before sequence b's, its items start at first(b) =
// at * mul / unit + per_seq * b, which leaves it at least rows * mul / unit + per_seq - 1 of them.
__device__ __forceinline__ int item_first(const int32_t* starts, int rows, int b, int mul, int unit, int per_seq) {
  const long at = starts ? min(max(starts[b], 0), rows) - min(max(starts[0], 0), rows) : b;
  return (int)(at * mul / unit) + per_seq * b;
}
// The sequence an item belongs to.  All 64 lanes look at once, so that a batch of up to 64 sequences takes one round trip
// (bisection took four or more, 2 us of an appended token).
__device__ __forceinline__ int item_owner(const int32_t* starts, int rows, int batch, int item, int mul, int unit, int per_seq) {
  int lo = 0, n = batch;                                  // the owner is in [lo, lo + n)
  while (n > 1) {
    const int step = (n + 63) / 64, b = lo + (int)(threadIdx.x & 63) * step;
    const bool begun = b < lo + n && item_first(starts, rows, b, mul, unit, per_seq) <= item;
    const int last = max(__popcll(__ballot(begun)) - 1, 0);
    n = min(step, n - last * step);
    lo += last * step;
  }
  return lo;
}

// ---- 16-bit values ----
template <typename T> struct Pair;
template <> struct Pair<_Float16> { typedef f16x2 type; };
template <> struct Pair<__bf16> { typedef bf16x2 type; };

template <typename T>
__device__ __forceinline__ void unpack2(uint32_t w, float& a, float& b) {
  if constexpr (__is_same(T, __bf16)) {
    a = __builtin_bit_cast(float, w << 16);
    b = __builtin_bit_cast(float, w & 0xFFFF0000u);
  } else {
    const f16x2 h = __builtin_bit_cast(f16x2, w);
    a = (float)h.x;
    b = (float)h.y;
  }
}
template <typename T>
__device__ __forceinline__ uint32_t pack2(float a, float b) {   // to nearest even
  typename Pair<T>::type h;
  h.x = (T)a;
  h.y = (T)b;
  return __builtin_bit_cast(uint32_t, h);
}
template <typename T>
__device__ __forceinline__ void unpack8(const u32x4& w, float* x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) unpack2<T>(w[i], x[2 * i], x[2 * i + 1]);
}
template <typename T>
__device__ __forceinline__ u32x4 pack8(const float* x) {
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = pack2<T>(x[2 * i], x[2 * i + 1]);
  return w;
}

// Sum / maximum over the 2, 4, 8 or 16 lanes that share a row (aligned groups of neighbours).
template <int CTRL>
__device__ __forceinline__ float lane_move(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xF, 0xF, true));
}
template <int LANES, typename Op>
__device__ __forceinline__ float row_reduce(float x, Op op) {
  if constexpr (LANES >= 2) x = op(x, lane_move<0xB1>(x));    // neighbour
  if constexpr (LANES >= 4) x = op(x, lane_move<0x4E>(x));    // other pair of four
  if constexpr (LANES >= 8) x = op(x, lane_move<0x141>(x));   // other four of eight (mirrored)
  if constexpr (LANES >= 16) x = op(x, lane_move<0x140>(x));  // other eight of sixteen (mirrored)
  return x;
}

// ---- norm and rotation ----
// A row of D channels is shared by D / 16 lanes ("units"), two pieces of 8 channels each, laid so that a lane
// holds both channels of every pair it turns: the pieces at 8u and rot/2 + 8u of the rotated channels (pairs
// 8u .. 8u+7), or 16 neighbours (neighbouring pairs, and the channels that are not rotated).
struct RowLayout {
  int at0, at1;     // first channels of the unit's two pieces
  int pair0;        // first of its eight pairs, or -1
};
__device__ __forceinline__ RowLayout row_layout(int unit, int rot_dim, int interleaved) {
  RowLayout l;
  const bool turned = 16 * unit < rot_dim;
  const bool halves = turned && !interleaved;
  l.at0 = halves ? 8 * unit : 16 * unit;
  l.at1 = halves ? rot_dim / 2 + 8 * unit : 16 * unit + 8;
  l.pair0 = turned ? 8 * unit : -1;
  return l;
}

// Cosine and sine of t quarter turns (|t| < 2^51).  t + 1.5 2^52 has the quarters nearest to t in its last bits; what is left of t,
// in [-1/2, 1/2], comes in fp64 (the largest position, 2^31, keeps 2^-24 turns) and is rounded once, as an angle x, |x| <= pi / 4.
// The Taylor polynomials of degree 9 and 10 are cut off at 2e-9 and 5e-10, below fp32's rounding, and end in one rounding of
// 1 - .. or x - ..: sine and cosine are off by about one unit of 2^-24.  (The hardware's are off by 2^-20 or so, which turned ten times as
// many 16-bit roundings; an angle rounded three times a quarter more: 1.8e-4 of fp16 results instead of 1.5e-4.)
__device__ __forceinline__ void turn(double t, float* cs, float* sn) {
  const double whole = 6755399441055744.0, k = t + whole;
  const int quarter = (int)(uint32_t)__builtin_bit_cast(uint64_t, k);
  const float x = (float)((t - (k - whole)) * 1.57079632679489662), z = x * x;
  float s = __builtin_fmaf(z, 1.0f / 362880, -1.0f / 5040), c = __builtin_fmaf(z, -1.0f / 3628800, 1.0f / 40320);
  s = __builtin_fmaf(z, s, 1.0f / 120);
  c = __builtin_fmaf(z, c, -1.0f / 720);
  s = __builtin_fmaf(z, s, -1.0f / 6);
  c = __builtin_fmaf(z, c, 1.0f / 24);
  s = __builtin_fmaf(z * x, s, x);
  c = __builtin_fmaf(z, c, -0.5f);
  c = __builtin_fmaf(z, c, 1.0f);
  const float a = (quarter & 1) ? s : c, b = (quarter & 1) ? c : s;
  *cs = ((quarter + 1) & 2) ? -a : a;
  *sn = (quarter & 2) ? -b : b;
}

// What the angles of a unit's eight pairs are made of, asked for ahead of the rows' own loads.
struct UnitTurns {
  int p[8];
  double f[8];
};
__device__ __forceinline__ void load_turns(const dq_rotary& r, const RowLayout& l, long column, int own_place, UnitTurns& t) {
  if (l.pair0 < 0) return;
#pragma unroll
  for (int i = 0; i < 8; ++i) t.f[i] = r.inv_freq[l.pair0 + i];
  if (r.axes > 1) {
    const uint8_t* axis = r.axis_of_pair + l.pair0;
    int at[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) at[i] = min((int)axis[i], r.axes - 1);
#pragma unroll
    for (int i = 0; i < 8; ++i) t.p[i] = r.positions[at[i] * r.position_stride + column];
  } else {
    const int p = r.positions ? r.positions[column] : own_place;
#pragma unroll
    for (int i = 0; i < 8; ++i) t.p[i] = p;
  }
}
__device__ __forceinline__ void make_turns(const RowLayout& l, const UnitTurns& t, float* cs, float* sn) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    cs[i] = 1.f;
    sn[i] = 0.f;
  }
  if (l.pair0 < 0) return;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    turn((double)t.p[i] * (t.f[i] * 0.63661977236758134308), cs + i, sn + i);
    if (i & 1) __builtin_amdgcn_sched_barrier(0);         // two pairs at a time: eight in a row hold 60 registers more
  }
}

// x: the unit's 16 channels in fp32, normed and rotated in place.  w: its weights.  LANES lanes share the row.
template <int LANES>
__device__ __forceinline__ void norm_unit(float* x, const float* w, float eps, float inv_dim) {
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) s = __builtin_fmaf(x[i], x[i], s);
  s = row_reduce<LANES>(s, [](float a, float b) { return a + b; });
  const float r = 1.0f / sqrtf(s * inv_dim + eps);
#pragma unroll
  for (int i = 0; i < 16; ++i) x[i] *= r * w[i];
}
template <bool INTERLEAVED>   // (a template: as a test at run time it became 28 selects a unit)
__device__ __forceinline__ void turn_unit(float* x, const float* cs, const float* sn) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int f = INTERLEAVED ? 2 * i : i, g = INTERLEAVED ? 2 * i + 1 : 8 + i;
    const float a = x[f], b = x[g];
    x[f] = a * cs[i] - b * sn[i];
    x[g] = a * sn[i] + b * cs[i];
  }
}

// A unit's 16 channels: norm (w: the weights, packed; they stay so from head to head: 8 registers, not 16), rotation, one rounding.
template <typename T, int LANES, bool INTERLEAVED>
__device__ __forceinline__ void ready_unit(u32x4 (&v)[2], u32x4 (&w)[2], bool normed, bool turned, float eps, float inv_dim, const float* cs,
                                           const float* sn) {
  float x[16];
  unpack8<T>(v[0], x);
  unpack8<T>(v[1], x + 8);
  if (normed) {                                           // (the lanes of a row are in this branch together)
    float y[16];
    asm volatile("" : "+v"(w[0]), "+v"(w[1]));
    unpack8<T>(w[0], y);
    unpack8<T>(w[1], y + 8);
    norm_unit<LANES>(x, y, eps, inv_dim);
  }
  if (turned) turn_unit<INTERLEAVED>(x, cs, sn);
  v[0] = pack8<T>(x);
  v[1] = pack8<T>(x + 8);
}

__device__ __forceinline__ void load_unit(u32x4 (&v)[2], const uint16_t* p, const RowLayout& l) {
  v[0] = *reinterpret_cast<const u32x4*>(p + l.at0);
  v[1] = *reinterpret_cast<const u32x4*>(p + l.at1);
}
__device__ __forceinline__ void store_unit(uint16_t* p, const RowLayout& l, const u32x4 (&v)[2]) {   // rows that this kernel does not read again
  __builtin_nontemporal_store(v[0], reinterpret_cast<u32x4*>(p + l.at0));
  __builtin_nontemporal_store(v[1], reinterpret_cast<u32x4*>(p + l.at1));
}

// Heads [h0, h1) of one token's row: the thread is the row's unit of LANES.  v: the first head's pieces, asked for ahead.
template <typename T, int LANES, bool INTERLEAVED>
__device__ __forceinline__ void rotate_row(u32x4 (&v)[2], const uint16_t* in, uint16_t* out, long in_head, long out_head, int h0, int h1, bool live,
                                           const RowLayout& l, const uint16_t* weight, float eps, float inv_dim, const float* cs, const float* sn) {
  u32x4 w[2] = {};
  if (weight && live) load_unit(w, weight, l);
  for (int h = h0; h < h1; ++h) {
    u32x4 y[2] = {v[0], v[1]};
    if (live && h + 1 < h1) load_unit(v, in + (h + 1) * in_head, l);   // the next head's pieces are on their way meanwhile
    ready_unit<T, LANES, INTERLEAVED>(y, w, weight != nullptr, l.pair0 >= 0, eps, inv_dim, cs, sn);
    if (live) store_unit(out + h * out_head, l, y);
  }
}

// ---- codes ----
template <bool FP8> constexpr float kQmax = FP8 ? 448.f : 127.f;

// Inverse step of a block: 12 significant bits, so that the product with a 16-bit value is exact in fp32.
template <bool FP8>
__device__ __forceinline__ float inverse_step(float amax) {
  return amax < kSmallestAmax ? 0.f : __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, kQmax<FP8> / amax) & ~0xFFFu);
}
// Four codes of four exact products.
template <bool FP8>
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
  if constexpr (FP8) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
  } else {
    const uint32_t x = (uint32_t)(int)__builtin_rintf(a) & 255u, y = (uint32_t)(int)__builtin_rintf(b) & 255u;
    const uint32_t z = (uint32_t)(int)__builtin_rintf(c) & 255u, w = (uint32_t)(int)__builtin_rintf(d);
    return x | y << 8 | z << 16 | w << 24;
  }
}
// The values of four codes.
template <bool FP8>
__device__ __forceinline__ void values4(uint32_t w, float* x) {
  if constexpr (FP8) {
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    x[0] = lo.x; x[1] = lo.y; x[2] = hi.x; x[3] = hi.y;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = (float)(int8_t)(w >> (8 * i));
  }
}

}  // namespace dq
