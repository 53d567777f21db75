// Shared pieces of attention over latents and of drafted trees: argument checks, and how a launch's workgroups share the tiles
// of a ragged batch.
#pragma once
#include "dq_paged_attn.h"

namespace dq {

inline bool latent_cache_ok(const dq_latent_cache* c) {
  if (!c || !c->rows || ((uintptr_t)c->rows & 15) || c->pages <= 0) return false;
  if (c->page_tokens != 64 && c->page_tokens != 128) return false;
  if (!(c->latent_dim == 512 && c->rot_dim == 64) && !(c->latent_dim == 256 && c->rot_dim == 32)) return false;
  return c->dtype == DQ_F16 || c->dtype == DQ_BF16;
}
inline bool latent_batch_ok(const dq_paged_batch* b, const dq_latent_cache* c, bool uses_starts) {
  if (!b || !b->seq_lens || !b->page_table || b->batch <= 0 || b->rows < 0) return false;
  if (b->table_width <= 0 || b->table_stride < b->table_width) return false;
  if ((long)b->table_width * c->page_tokens >= kMostTokens) return false;
  return !uses_starts || b->starts || b->rows == b->batch;
}

inline bool scale_ok(float scale) { return scale * 1.44269504088896340736f < INFINITY; }

// Whether rows of heads that are read and rows of heads that are written may have channels in common.  Slices of one buffer do not: other columns
// of its rows, or other channels of its heads.  Exact where both have the same strides (a stride over one entry says nothing), on the safe side elsewhere.
inline bool heads_meet(const dq_heads* a, long a_rows, int a_dim, const dq_heads* b, long b_rows, int b_dim) {
  typedef __int128 wide;
  if (a_rows <= 0 || b_rows <= 0) return false;
  auto reach = [](const dq_heads* h, long rows, int dim) {   // elements from the first channel to behind the last one
    return (wide)(rows - 1) * h->token_stride + (wide)(h->heads - 1) * h->head_stride + dim;
  };
  const wide apart = ((wide)(intptr_t)b->data - (wide)(intptr_t)a->data) / 2;
  if (apart >= reach(a, a_rows, a_dim) || -apart >= reach(b, b_rows, b_dim)) return false;
  auto common = [](bool any_a, int64_t x, bool any_b, int64_t y) -> int64_t { return !any_a ? y : !any_b || x == y ? x : -1; };
  const int64_t token = common(a_rows > 1, a->token_stride, b_rows > 1, b->token_stride), head = common(a->heads > 1, a->head_stride, b->heads > 1, b->head_stride);
  if (token > 0) {                                        // the rows' columns, none of them past the next row
    const wide in = (apart % token + token) % token;
    if (in >= reach(a, 1, a_dim) && in + reach(b, 1, b_dim) <= token) return false;
  }
  if (token < 0 || head < 0) return true;
  // A row D further on and a head E further on lie at x = apart + D token + E head: they meet if -b_dim < x < a_dim.
  struct Steps { wide stride, from, to; } far = {token, 1 - a_rows, b_rows - 1}, near = {head, 1 - a->heads, b->heads - 1};
  if (far.stride < near.stride) { const Steps x = far; far = near; near = x; }
  auto up = [](wide n, wide d) { return n >= 0 ? (n + d - 1) / d : -(-n / d); };   // n / d, rounded up
  auto near_meets = [&](wide x) {                         // with near's steps from x
    wide n = near.stride ? up(1 - b_dim - x, near.stride) : 0;
    n = n < near.from ? near.from : n;
    return n <= near.to && x + n * near.stride > -b_dim && x + n * near.stride < a_dim;
  };
  if (far.stride == 0) return near_meets(apart);
  wide n = up(1 - b_dim - near.to * near.stride - apart, far.stride);
  n = n < far.from ? far.from : n;
  for (int tries = 0; n <= far.to && apart + n * far.stride < a_dim - near.from * near.stride; ++n)
    if (++tries > 8 || near_meets(apart + n * far.stride)) return true;   // (three at the most where rows and heads do not cross)
  return false;
}

// Whether b may be written while a is read, each head by the threads that read it: the same rows of heads, or none that meet.
inline bool heads_in_place(const dq_heads* a, const dq_heads* b, long rows, int dim) {
  return (a->data == b->data && (rows <= 1 || a->token_stride == b->token_stride) && (a->heads <= 1 || a->head_stride == b->head_stride)) ||
         !heads_meet(a, rows, dim, b, rows, dim);
}

// ---- memory to LDS, past the registers ----
typedef __attribute__((address_space(3))) char* LdsBytes;
typedef __attribute__((address_space(3))) const u32x4* LdsPieces;
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4* LdsQuads;

// An address that all lanes have in common, in scalar registers (an asm operand's "s" is no more than a wish without it).
__device__ __forceinline__ uint64_t in_scalars(const void* p) {
  return (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)((uint64_t)p >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint64_t)p);
}

// 64 pieces of 16 bytes, one behind the other from `lds` on: a lane's piece is at base + offset, or at `from`.  As instructions of
// their own: the compiler waits for all such copies ahead of every LDS read, the ones for later tiles too.  Kernels count
// them themselves (no register is written; a wait that counts too many of them waits longer).
// once: past the caches' order (rows that one workgroup reads: a cache of 378 MB in 80 us, 89 without).
// (m0 is declared as written, so that the compiler carries no setting of its own across.  Its warning, that m0 is not preserved, is meant so.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
template <bool once = false> __device__ __forceinline__ void copy_to_lds(const uint16_t* base, uint32_t offset, uint32_t lds) {
  if constexpr (once) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" ::"s"(__builtin_amdgcn_readfirstlane(lds)), "v"(offset), "s"(in_scalars(base)) : "m0", "memory");
    return;
  }
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(__builtin_amdgcn_readfirstlane(lds)), "v"(offset), "s"(in_scalars(base)) : "m0", "memory");
}
__device__ __forceinline__ void copy_to_lds(const uint16_t* from, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(__builtin_amdgcn_readfirstlane(lds)), "v"(from) : "m0", "memory");
}
#pragma clang diagnostic pop
// Waits for all of the wave's copies but the newest N; for the workgroup's other waves.  As instructions that no LDS read passes (the
// compiler moves reads across the barrier builtin), its result no less: what was read may be copied over from then on.
template <int N> __device__ __forceinline__ void wait_copies() { asm volatile("s_waitcnt vmcnt(%0)" ::"i"(N) : "memory"); }
__device__ __forceinline__ void barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
__device__ __forceinline__ uint32_t lds_of(const void* p) { return (uint32_t)(uintptr_t)(LdsBytes)p; }

// Eight 16-bit values: the left operand of a product with rows as they lie (token by token) as channels.  Of each 16 lanes, four read
// 8 bytes each of one token's 16 channels, and lane i gets channel i of four tokens; `a` and `b` are the first and last four tokens.
template <typename V> __device__ __forceinline__ V turned_rows(LdsBytes a, LdsBytes b) {
  struct { s16x4 a, b; } const both = {__builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsQuads)a), __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsQuads)b)};
  return __builtin_bit_cast(V, both);
}

// sum + the eight values of v, in fp32, two at a time.
__device__ __forceinline__ float add_eight(float sum, f16x8 v) {
#pragma unroll
  for (int i = 0; i < 8; i += 2) sum = __builtin_amdgcn_fdot2(f16x2{v[i], v[i + 1]}, f16x2{(_Float16)1.f, (_Float16)1.f}, sum, false);
  return sum;
}
__device__ __forceinline__ float add_eight(float sum, bf16x8 v) {
#pragma unroll
  for (int i = 0; i < 8; i += 2) sum = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{v[i], v[i + 1]}, bf16x2{(__bf16)1.f, (__bf16)1.f}, sum, false);
  return sum;
}

// What a token that is not there has: zeros (nothing sees it, but 0 * NaN of what lies there would not be 0).
__device__ const u32x4 g_blank[1] = {{0, 0, 0, 0}};

constexpr u32x4 kNanPiece = {0x7FFF7FFFu, 0x7FFF7FFFu, 0x7FFF7FFFu, 0x7FFF7FFFu};   // eight NaN of either type

// A ragged batch's tiles in one line: sequence after sequence, in a sequence unit after unit (a tile of query columns, a kv head), in a
// unit from its first token tile on.  Workgroup w takes tiles [w quota, (w + 1) quota) of the line, whatever units they belong
// to, so that all end together however lengths differ.  A unit that one workgroup takes whole is written out; pieces of the others
// are left in the workspace, two at most for a workgroup (slot 2 w: a piece that does not begin its unit; 2 w + 1: one that does
// and does not end it), and joined by a second launch, over the columns, which finds them by the same counting.  (One
// workgroup alone joining a unit of 128 columns of 512 channels in 16 pieces would read 4 MB.)
struct Line {
  int workgroups;
  int min_quota;           // tiles that are worth a workgroup of their own
};
struct Weight {
  int units, tiles;        // of a sequence
};

__device__ __forceinline__ long wave_sum(long x) {
  for (int o = 1; o < 64; o *= 2) x += __shfl_xor(x, o);
  return x;
}
__device__ __forceinline__ long wave_uniform(long x) {
  return (long)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)x));
}

// weight_of(b): a sequence's Weight.  Every lane of a wave calls it with other sequences.
template <typename F> __device__ __forceinline__ long line_total(int batch, F weight_of) {
  long mine = 0;
  for (int b = threadIdx.x & 63; b < batch; b += 64) {
    const Weight w = weight_of(b);
    mine += (long)w.units * w.tiles;
  }
  return wave_uniform(wave_sum(mine));
}
// a / b, neither negative: in 32 bits where they do (b positive).
__device__ __forceinline__ long over(long a, long b) { return (a | b) >> 32 ? a / b : (long)((uint32_t)a / (uint32_t)b); }
__device__ __forceinline__ long line_quota(const Line& l, long total) { return max(over(total + l.workgroups - 1, l.workgroups), (long)l.min_quota); }

// The sequence that holds place `at` of the line (at < total), and the place at which it begins.
template <typename F> __device__ __forceinline__ int line_owner(int batch, long at, F weight_of, long& begin) {
  const int lane = threadIdx.x & 63;
  long before = 0;
  for (int b0 = 0; b0 < batch; b0 += 64) {
    long mine = 0;
    if (b0 + lane < batch) {
      const Weight w = weight_of(b0 + lane);
      mine = (long)w.units * w.tiles;
    }
    long upto = mine;
    for (int o = 1; o < 64; o *= 2) {
      const long x = __shfl_up(upto, o);
      if (lane >= o) upto += x;
    }
    const uint64_t owner = __ballot(at < before + upto && at >= before + upto - mine);
    if (owner) {
      const int l = __builtin_ctzll(owner);
      begin = wave_uniform(before + __shfl(upto - mine, l));
      return b0 + l;
    }
    before += wave_uniform(__shfl(upto, 63));
  }
  begin = before;
  return batch;
}

// A sequence a lane and 31 bits of places, as nearly always: each one's places and their running sum, looked at once.  false: the line is longer.
template <typename F> __device__ __forceinline__ bool short_line(int batch, F weight_of, int& mine, int& upto) {
  if (batch > 64) return false;
  const int lane = threadIdx.x & 63;
  const Weight w = lane < batch ? weight_of(lane) : Weight{0, 0};
  const long places = (long)w.units * w.tiles;
  if (__any(places >= 1l << 24)) return false;
  mine = upto = (int)places;
  for (int o = 1; o < 64; o *= 2) {
    const int x = __shfl_up(upto, o);
    if (lane >= o) upto += x;
  }
  return true;
}

// A workgroup's places of the line, [at, end), and the sequence that holds the first of them, which begins at place `begin`; false: it has none.
struct LineStart {
  long at, end, begin;
  int b;
};
template <typename F> __device__ __forceinline__ bool line_start(const Line& l, int batch, F weight_of, LineStart& s) {
  int mine, upto;
  if (short_line(batch, weight_of, mine, upto)) {
    const uint32_t total = (uint32_t)__builtin_amdgcn_readlane(upto, 63), quota = (uint32_t)line_quota(l, total), at = blockIdx.x * quota;
    if (at >= total) return false;
    s.at = at;
    s.end = min(at + quota, total);
    s.b = __builtin_ctzll(__ballot((uint32_t)upto > at));
    s.begin = (uint32_t)__builtin_amdgcn_readlane(upto - mine, s.b);
    return true;
  }
  const long total = line_total(batch, weight_of), quota = line_quota(l, total);
  s.at = (long)blockIdx.x * quota;
  s.end = min(s.at + quota, total);
  if (s.at >= s.end) return false;
  s.b = line_owner(batch, s.at, weight_of, s.begin);
  return true;
}

// The line's length, and its places before sequence b.
struct LineSums {
  long total, before;
};
template <typename F> __device__ __forceinline__ LineSums line_sums(int batch, int b, F weight_of) {
  int mine, upto;
  if (short_line(batch, weight_of, mine, upto)) return {__builtin_amdgcn_readlane(upto, 63), __builtin_amdgcn_readlane(upto - mine, __builtin_amdgcn_readfirstlane(b))};
  long all = 0, lower = 0;
  for (int i = threadIdx.x & 63; i < batch; i += 64) {
    const Weight w = weight_of(i);
    const long n = (long)w.units * w.tiles;
    all += n;
    if (i < b) lower += n;
  }
  return {wave_uniform(wave_sum(all)), wave_uniform(wave_sum(lower))};
}

// Pieces of a unit whose tiles are places [begin, begin + tiles) of the line: the workgroups first .. last, one piece each.
struct Pieces {
  long first, last;
};
__device__ __forceinline__ Pieces pieces_of(long begin, int tiles, long quota) { return {over(begin, quota), over(begin + tiles - 1, quota)}; }
__device__ __forceinline__ long slot_of(const Pieces& p, long w) { return w == p.first ? 2 * w + 1 : 2 * w; }

// Joins the pieces of kJoinColumns<D> columns (those below `valid`): a wave a column, or as many as 16-byte loads of a piece let it, where there are few
// pieces, four waves, which take every fourth piece, where there are many.  o: [slot, column, D] floats, ml: [slot, column, 2]; eight
// pieces are asked for at once.  (A workgroup a column spent most of its time on finding its unit: 39 us where this takes 9, 64 columns of 128
// units in 4 or 5 pieces.)
template <int D> constexpr int kJoinColumns = D >= 256 ? 4 : 16;   // (512 channels: 16 us, 21 with sixteen; 128 channels 9.4, 10.0 with eight, 9.7 with 32; 64 channels 6.8, 8.1 with 32)
template <typename T, int D, typename Slot, typename Out>
__device__ __forceinline__ void join_columns(int count, Slot slot_of_piece, const float* o, const float* ml, int columns, int column0, int valid, Out out_of) {
  constexpr int PER = D >= 256 ? D / 64 : 4, LANES = D / PER, AT_ONCE = 64 / LANES, AHEAD = 8;   // channels of a lane, lanes of a column, columns of a wave
  __shared__ __align__(16) float s_o[4][64 * PER];
  __shared__ float s_m[4][AT_ONCE], s_l[4][AT_ONCE];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), in = lane % LANES, sub = lane / LANES;
  const int end = min(column0 + kJoinColumns<D>, valid);
  struct Sum { float m, l; f32x4 x[PER / 4]; };
  auto add = [&](int c, int from, int step) {
    const int column = min(c, end - 1);
    Sum r = {-INFINITY, 0.f, {}};
    for (int i0 = from; i0 < count; i0 += step * AHEAD) {
      f32x4 y[AHEAD][PER / 4];
      float pm[AHEAD], pl[AHEAD];
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) {                   // (behind the last piece: that one again, with no weight)
        const long at = slot_of_piece(min(i0 + step * k, count - 1)) * columns + column;
        const f32x2 v = *reinterpret_cast<const f32x2*>(ml + 2 * at);
        pm[k] = i0 + step * k < count ? v.x : -INFINITY;
        pl[k] = v.y;
#pragma unroll
        for (int e = 0; e < PER / 4; ++e) y[k][e] = *reinterpret_cast<const f32x4*>(o + at * D + PER * in + 4 * e);
      }
      float top = r.m;
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) top = fmaxf(top, pm[k]);
      const float at = top == -INFINITY ? 0.f : top, back = __builtin_amdgcn_exp2f(r.m - at);
      r.m = top;
      r.l *= back;
#pragma unroll
      for (int e = 0; e < PER / 4; ++e) r.x[e] *= back;
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) {
        const float w = __builtin_amdgcn_exp2f(pm[k] - at);
        r.l = __builtin_fmaf(pl[k], w, r.l);
#pragma unroll
        for (int e = 0; e < PER; ++e) r.x[e / 4][e % 4] = __builtin_fmaf(y[k][e / 4][e % 4], w, r.x[e / 4][e % 4]);
      }
    }
    return r;
  };
  auto store = [&](int c, const f32x4 (&x)[PER / 4], float l) {
    if (c >= end) return;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    uint16_t* const out = out_of(c) + PER * in;
#pragma unroll
    for (int e = 0; e < PER / 4; ++e)
      *reinterpret_cast<u32x2*>(out + 4 * e) = u32x2{pack2<T>(x[e][0] * inv, x[e][1] * inv), pack2<T>(x[e][2] * inv, x[e][3] * inv)};
  };
  if (count <= 4 * AHEAD) {
    for (int c = column0 + wave * AT_ONCE; c < end; c += 4 * AT_ONCE) {
      const Sum r = add(c + sub, 0, 1);
      store(c + sub, r.x, r.l);
    }
    return;
  }
  int turn = 0;
  for (int c = column0; c < end; c += AT_ONCE, ++turn) {
    const Sum r = add(c + sub, wave, 4);
    __syncthreads();                                      // the last columns' results have been read
#pragma unroll
    for (int e = 0; e < PER / 4; ++e) *reinterpret_cast<f32x4*>(&s_o[wave][PER * lane + 4 * e]) = r.x[e];
    if (in == 0) { s_m[wave][sub] = r.m; s_l[wave][sub] = r.l; }
    __syncthreads();
    if (wave != (turn & 3)) continue;
    const float top = fmaxf(fmaxf(s_m[0][sub], s_m[1][sub]), fmaxf(s_m[2][sub], s_m[3][sub])), at = top == -INFINITY ? 0.f : top;
    f32x4 x[PER / 4] = {};
    float l = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = __builtin_amdgcn_exp2f(s_m[w][sub] - at);
      l = __builtin_fmaf(s_l[w][sub], f, l);
#pragma unroll
      for (int e = 0; e < PER; ++e) x[e / 4][e % 4] = __builtin_fmaf(s_o[w][PER * lane + e], f, x[e / 4][e % 4]);
    }
    store(c + sub, x, l);
  }
}

}  // namespace dq
