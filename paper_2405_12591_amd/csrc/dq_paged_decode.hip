// Attention of a few query rows per sequence (a generated token, drafted ones) over the paged 8-bit cache.
#include "dq_paged_attn.h"

namespace dq {

constexpr int kCols = 16;   // (row, query head) columns of a workgroup: one matrix instruction's

// The sequence and split a slot works on: a slot is a share of a sequence's tiles, the same for all kv heads.  `shares` slots are
// meant to get as many tiles each, t = all tiles / shares; a sequence has tiles / t of them, rounded, at least one, at most
// decode_cap().  With one length a sequence each that is an even split; in a batch of one long and many short sequences the long one
// gets nearly all slots: 16 sequences of 8 heads, one of 32768 tokens and 15 of 500, 26 us, 220 with a slot each; 4 x 40 heads of 9384 to
// 16384 tokens 93 us (98 split evenly).  Where there is one share a sequence, what is over a share gets another slot (32 x 8
// heads of 64 to 8192 tokens 64 us, 77 rounded).  Up to 64 sequences, one a lane; more of them are split evenly.
struct Share {
  int b, split, splits;    // splits == 0: an empty slot
  int first_slot;          // of the sequence
  Sequence s;
};
__device__ __forceinline__ int first_tile_of(const Sequence& s, int window) { return window_start(s.old, window) / kPagedTile; }

__device__ __forceinline__ Share share_of(const PagedAttnArgs& a, int slot) {
  Share r;
  const int P = a.c.page_tokens, batch = a.bt.batch;
  if (batch > 64 || a.shares == 0) {
    r.splits = a.shares ? a.shares / batch : 1;
    r.b = slot / r.splits;
    r.split = slot % r.splits;
    r.first_slot = slot - r.split;
    r.s = sequence_of_wave(a.bt, P, r.b);
    if (r.s.n == 0) r.splits = 0;
    return r;
  }
  const int lane = threadIdx.x & 63;
  Sequence s = {0, 0, 0, 0};
  if (lane < batch) s = sequence_of(a.bt, P, lane);
  const int tiles = s.n ? max((s.len + kPagedTile - 1) / kPagedTile - first_tile_of(s, a.window), 0) : 0;
  int total = tiles;                                      // (lanes of no sequence need not know it)
  for (int o = 1; o < batch; o *= 2) total += __shfl_xor(total, o);
  const float per = fmaxf((float)total / (float)a.shares, 1.f), round = a.shares == batch ? 0.99f : 0.5f;
  const int cap = decode_cap(tiles, a.c.head_dim, a.max_rows * a.group);
  const int mine = s.n ? max(min((int)((float)tiles / per + round), min(cap, kMaxSplits)), 1) : 0;
  int upto = mine;                                        // slots of the sequences up to this one
  for (int o = 1; o < batch; o *= 2) {
    const int x = __shfl_up(upto, o);
    if (lane >= o) upto += x;
  }
  const uint64_t owner = __ballot(slot < upto && slot >= upto - mine);
  if (owner == 0) {
    r.splits = 0;
    return r;
  }
  r.b = __builtin_ctzll(owner);
  r.splits = __builtin_amdgcn_readlane(mine, r.b);
  r.first_slot = __builtin_amdgcn_readlane(upto, r.b) - r.splits;
  r.split = slot - r.first_slot;
  r.s.row0 = __builtin_amdgcn_readlane(s.row0, r.b);
  r.s.n = __builtin_amdgcn_readlane(s.n, r.b);
  r.s.old = __builtin_amdgcn_readlane(s.old, r.b);
  r.s.len = __builtin_amdgcn_readlane(s.len, r.b);
  return r;
}

// One workgroup of four or eight waves per (slot, kv head); its columns are the (row, query head) pairs that read the kv head.  Every
// wave works tiles of 64 tokens on its own, dealt round-robin over the waves of all splits, and keeps a running maximum, sum
// and output; waves are joined through LDS, splits through memory.
//
// Scores are formed transposed, S^T = K Q^T, token rows against query columns.  Row r of the four 16-row products stands
// for token 16 (r / 4) + 4 t4 + r % 4, so a lane ends up with the scores of 16 neighbouring tokens of its column:
// exactly the right operand that O^T += V^T P^T wants, with the value codes of those tokens in one 16-byte load.
// Nothing moves between lanes but the maximum, and that only when it grew.
//
// The values' scale rides in the exponent: u = s + log2(scale_v), p = 2^(u - m), O += p c, l += (sum p) / scale_v; the
// products see codes and p only, and p is largest (2^8 at most) where the contribution to the output is.
//
// Bound by memory where caches are long: two bytes a token and channel, 16 x 8 heads of 32768 tokens of 128 channels 1074 MB, 163 us,
// 6.6 TB/s as a plain read of that size; four sequences of 9384 to 16384 tokens, 40 heads, 530 MB, 91 us, 5.8 TB/s.  By latency where
// they are short: one tile a wave 5.0 us, launch, lengths, page, codes and joins after one another; 64 units of 64 tiles of 64
// channels (33 MB) 13.1 us.  Tiles requested two or three ahead made no launch faster and short ones slower.
template <typename T, int D, bool FP8, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void paged_decode_kernel(PagedAttnArgs a) {
  constexpr int NC = D / 64, NCT = D / 16, THREADS = 64 * WAVES;
  typedef typename Vec8<T>::type tx8;
  __shared__ float s_o[WAVES][kCols][D + 1];
  __shared__ float s_m[WAVES][kCols], s_l[WAVES][kCols];
  __shared__ JoinSpace s_join;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, G = lane >> 4;
  const int H = a.c.kv_heads, P = a.c.page_tokens, slot = (int)blockIdx.x / H, h = (int)blockIdx.x % H;
  const Share sh = share_of(a, slot);
  if (sh.splits == 0) return;
  const Sequence& s = sh.s;
  const int b = sh.b, splits = sh.splits, unit = b * H + h;
  const int n = min(s.n, a.max_rows), len = s.len, before = s.old;
  const int cols = n * a.group;
  const int qi = min(col / a.group, n - 1), hq = h * a.group + col % a.group;
  const bool live = col < cols;
  // tokens [see_lo, see_hi) of this column, and what every column sees
  const int place = before + qi;
  const int see_hi = a.causal ? min(place + 1, len) : len, see_lo = window_start(place, a.window);
  const int all_hi = a.causal ? min(before + 1, len) : len, all_lo = window_start(before + n - 1, a.window);
  const int first_tile = first_tile_of(s, a.window);
  const int runs = P / kPagedTile, code_tiles = len / P * runs, tiles = (len + kPagedTile - 1) / kPagedTile;

  // ---- queries: 8 channels 64 c + 16 G + 8 half of the column, in f16 ----
  const uint16_t* const q_row = a.q.data + (long)(s.row0 + qi) * a.q.token_stride + (long)(live ? hq : h * a.group) * a.q.head_stride;
  f16x8 q[NC][2];
  float sc = a.scale_log2;
  {
    float x[NC][2][8], amax = 0.f;
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        unpack8<T>(*reinterpret_cast<const u32x4*>(q_row + 64 * c + 16 * G + 8 * hf), x[c][hf]);
#pragma unroll
        for (int j = 0; j < 8; ++j) amax = fmaxf(amax, fabsf(x[c][hf][j]));
      }
    int shift = 0;
    if constexpr (__is_same(T, __bf16)) {
      amax = fmaxf(amax, __shfl_xor(amax, 16));
      amax = fmaxf(amax, __shfl_xor(amax, 32));
      shift = fit_shift(amax);
      sc = __builtin_ldexpf(sc, -shift);
    }
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int hf = 0; hf < 2; ++hf)
#pragma unroll
        for (int j = 0; j < 8; ++j) q[c][hf][j] = (_Float16)(__is_same(T, __bf16) ? __builtin_ldexpf(x[c][hf][j], shift) : x[c][hf][j]);
  }

  f32x4 o[NCT];
#pragma unroll
  for (int ct = 0; ct < NCT; ++ct) o[ct] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;

  // Softmax of a tile's 16 products of this lane (tokens 64 tile + 16 G + ..), in place: u -> p = 2^(u f + add - m).
  auto softmax = [&](float (&u)[16], int tile, float f, float add, float inv_sv, auto mask) __attribute__((always_inline)) {
    if constexpr (decltype(mask)::value) {
      const float poison = f - f;                         // NaN where the block is: for those who see it, not through a masked -inf
      f = f == f ? f : 1.f;
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const int t = tile * kPagedTile + 16 * G + j;
        u[j] = t < see_lo || t >= see_hi ? -INFINITY : u[j] + poison;
      }
    }
    float top = u[0];
#pragma unroll
    for (int j = 1; j < 16; ++j) top = fmaxf(top, u[j]);
    top = __builtin_fmaf(top, f, add);
    if (__any(top > m + kLazy)) {
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float m_new = fmaxf(m, top);
      const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - m_new);
      m = m_new;
      l *= alpha;
#pragma unroll
      for (int ct = 0; ct < NCT; ++ct) o[ct] *= alpha;
    }
    const float base = m == -INFINITY ? add : add - m;
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      u[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(u[j], f, base));
      sum += u[j];
    }
    l = __builtin_fmaf(sum, inv_sv, l);
  };

  // ---- full pages ----
  const int stride = splits * WAVES, mine = first_tile + sh.split * WAVES + wave;
  const int k_row = 16 * ((lane & 15) >> 2) + (lane & 3);   // + 4 t4: the token of this lane's row
  for (int batch0 = mine; batch0 < code_tiles; batch0 += 64 * stride) {
    // the next 64 tiles' blocks and scales, one per lane
    const int t_l = batch0 + lane * stride;
    int blk = -1;
    float sk = 0.f, lsv = 0.f, isv = 0.f;
    if (t_l < code_tiles) {
      const int page = a.bt.page_table[(long)b * a.bt.table_stride + t_l / runs];
      const bool ok = page >= 0 && page < a.c.pages;
      const long block = (long)(ok ? page : 0) * H + h;
      blk = ok ? (int)(block * runs) + t_l % runs : -1;
      sk = ok ? a.c.k_scales[block] : __builtin_nanf("");
      const float sv = ok ? a.c.v_scales[block] : 1.f;
      lsv = __builtin_amdgcn_logf(sv);
      isv = 1.f / sv;
    }
    place_zero_blocks<D, FP8>(a.c.v_codes, blk, blk >= 0, lsv, isv);
    const int count = min(64, (code_tiles - batch0 + stride - 1) / stride);
    u32x4 kb[4][NC], vb[NCT];
    auto load_k = [&](int i) __attribute__((always_inline)) {
      const GlobalBytes p = codes_of(a.c.k_codes, __builtin_amdgcn_readlane(blk, i), kPagedTile * D) + k_row * D + 16 * G;
#pragma unroll
      for (int t4 = 0; t4 < 4; ++t4)
#pragma unroll
        for (int c = 0; c < NC; ++c) kb[t4][c] = __builtin_nontemporal_load((GlobalPieces)(p + 4 * t4 * D + 64 * c));
    };
    auto load_v = [&](int i) __attribute__((always_inline)) {
      const GlobalBytes p = codes_of(a.c.v_codes, __builtin_amdgcn_readlane(blk, i), kPagedTile * D) + (lane & 15) * kPagedTile + 16 * G;
#pragma unroll
      for (int ct = 0; ct < NCT; ++ct) vb[ct] = __builtin_nontemporal_load((GlobalPieces)(p + ct * 16 * kPagedTile));
    };
    load_k(0);
    load_v(0);
    for (int i = 0; i < count; ++i) {
      const float f = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, sk), i));
      const float add = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, lsv), i));
      const float inv_sv = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, isv), i));
      float u[16];
#pragma unroll
      for (int t4 = 0; t4 < 4; ++t4) {
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          acc = mma16(codes_f16<FP8>(kb[t4][c].x, kb[t4][c].y), q[c][0], acc);
          acc = mma16(codes_f16<FP8>(kb[t4][c].z, kb[t4][c].w), q[c][1], acc);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) u[4 * t4 + j] = acc[j];
      }
      if (i + 1 < count) load_k(i + 1);
      const int tile = batch0 + i * stride;
      if (tile * kPagedTile < all_lo || tile * kPagedTile + kPagedTile > all_hi) softmax(u, tile, keep_sign(f * sc), add, inv_sv, Masked{});
      else softmax(u, tile, keep_sign(f * sc), add, inv_sv, Whole{});
      // 11 bits, as the codes' products want them (the sum keeps fp32): the error of one more fp16 rounding a token
      f16x8 p0, p1;
#pragma unroll
      for (int j = 0; j < 8; ++j) { p0[j] = (_Float16)u[j]; p1[j] = (_Float16)u[8 + j]; }
#pragma unroll
      for (int ct = 0; ct < NCT; ++ct) {
        o[ct] = mma16(codes_f16<FP8>(vb[ct].x, vb[ct].y), p0, o[ct]);
        o[ct] = mma16(codes_f16<FP8>(vb[ct].z, vb[ct].w), p1, o[ct]);
      }
      if (i + 1 < count) load_v(i + 1);
    }
  }

  // ---- the page being filled: 16-bit rows, products in their own type ----
  const int tail_first = max(code_tiles, first_tile);
  for (int tile = tail_first; tile < tiles; ++tile) {
    if ((tile - first_tile) % stride != sh.split * WAVES + wave) continue;
    const int at_slot = a.bt.tail_slots ? a.bt.tail_slots[b] : b;
    const bool ok = at_slot >= 0 && at_slot < a.c.slots;
    const int run = tile - code_tiles, left = ok ? len - tile * kPagedTile : 0;   // tokens of the tile
    const long at = (((long)(ok ? at_slot : 0) * H + h) * runs + run) * kPagedTile * D;
    const uint16_t* const kt = a.c.k_tail + at + k_row * D + 16 * G;
    const uint16_t* const vt = a.c.v_tail + at + (lane & 15) * kPagedTile + 16 * G;
    const float f = ok ? keep_sign(a.scale_log2) : __builtin_nanf("");
    float u[16];
    tx8 qt[NC][2];
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) qt[c][hf] = __builtin_bit_cast(tx8, *reinterpret_cast<const u32x4*>(q_row + 64 * c + 16 * G + 8 * hf));
#pragma unroll
    for (int t4 = 0; t4 < 4; ++t4) {
      f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int hf = 0; hf < 2; ++hf)
          acc = mma16(__builtin_bit_cast(tx8, *reinterpret_cast<const u32x4*>(kt + 4 * t4 * D + 64 * c + 8 * hf)), qt[c][hf], acc);
#pragma unroll
      for (int j = 0; j < 4; ++j) u[4 * t4 + j] = acc[j];
    }
    softmax(u, tile, f, 0.f, 1.f, Masked{});
    uint32_t keep[8];                                     // rows behind the last token may hold anything: 0 * NaN is not 0
#pragma unroll
    for (int j = 0; j < 8; ++j) keep[j] = keep_tokens(~0u, left - 16 * G - 2 * j);
    // in the rows' type, which their products need: 8 bits with bf16 rows, one more such rounding for each of the page's tokens
    u32x4 p0, p1;
#pragma unroll
    for (int j = 0; j < 4; ++j) { p0[j] = pack2<T>(u[2 * j], u[2 * j + 1]); p1[j] = pack2<T>(u[8 + 2 * j], u[8 + 2 * j + 1]); }
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct) {
      u32x4 v0 = *reinterpret_cast<const u32x4*>(vt + ct * 16 * kPagedTile), v1 = *reinterpret_cast<const u32x4*>(vt + ct * 16 * kPagedTile + 8);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v0[j] &= keep[j];
        v1[j] &= keep[4 + j];
      }
      o[ct] = mma16(__builtin_bit_cast(tx8, v0), __builtin_bit_cast(tx8, p0), o[ct]);
      o[ct] = mma16(__builtin_bit_cast(tx8, v1), __builtin_bit_cast(tx8, p1), o[ct]);
    }
  }

  // ---- waves, then splits ----
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
#pragma unroll
  for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
    for (int j = 0; j < 4; ++j) s_o[wave][col][16 * ct + 4 * G + j] = o[ct][j];
  if (G == 0) { s_m[wave][col] = m; s_l[wave][col] = l; }
  __syncthreads();
  auto out_of = [&](int c) { return a.out.data + (long)(s.row0 + c / a.group) * a.out.token_stride + (long)(h * a.group + c % a.group) * a.out.head_stride; };
  const long part_step = (long)H * kCols * (D + 2);        // from split to split
  float* const parts = a.partials + ((long)sh.first_slot * H + h) * kCols * (D + 2);
  float* const part = parts + sh.split * part_step;
  for (int idx = 2 * tid; idx < cols * D; idx += 2 * THREADS) {
    const int cc = idx / D, ch = idx % D;
    float M = s_m[0][cc];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) M = fmaxf(M, s_m[w][cc]);
    const float base = M == -INFINITY ? 0.f : M;
    float x = 0.f, y = 0.f, ll = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const float f = __builtin_amdgcn_exp2f(s_m[w][cc] - base);
      x = __builtin_fmaf(s_o[w][cc][ch], f, x);
      y = __builtin_fmaf(s_o[w][cc][ch + 1], f, y);
      ll = __builtin_fmaf(s_l[w][cc], f, ll);
    }
    if (splits == 1) {
      const float inv = ll == 0.f ? 0.f : 1.f / ll;
      *reinterpret_cast<uint32_t*>(out_of(cc) + ch) = pack2<T>(x * inv, y * inv);
    } else {
      float* const p = part + (long)cc * (D + 2);
      store_pair(p + ch, x, y);
      if (ch == 0) store_pair(p + D, M, ll);
    }
  }
  if (splits > 1) join_splits<T, D>(a.counters + unit, splits, parts, part_step, cols, s_join, out_of);
}

template <typename T, int D, int WAVES>
static void launch_decode_waves(const PagedAttnArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)((long)(a.shares ? a.bt.batch > 64 ? a.shares : a.shares + a.bt.batch : a.bt.batch) * a.c.kv_heads));
  if (a.c.codes == DQ_CODES_E4M3) hipLaunchKernelGGL((paged_decode_kernel<T, D, true, WAVES>), grid, dim3(64 * WAVES), 0, st, a);
  else hipLaunchKernelGGL((paged_decode_kernel<T, D, false, WAVES>), grid, dim3(64 * WAVES), 0, st, a);
}

// Eight waves a workgroup where tiles are small (64 channels) and units few: waves are joined through LDS for less than splits through
// memory.  5 tiles of one unit 5.0 us (5.6 with four waves), 64 units of 64 tiles of 16 columns 13.4 (15.0), 32 of 512 tiles 25.4 (27.6);
// but 512 units of 8 tiles 10.4 (7.8), and 128 channels, which leave room for one such workgroup a compute unit, 2 to 15 % more.
template <typename T, int D>
static void launch_decode(const PagedAttnArgs& a, hipStream_t st) {
  if constexpr (D == 64)
    if (a.units < 128) return launch_decode_waves<T, D, 8>(a, st);
  launch_decode_waves<T, D, 4>(a, st);
}

int32_t launch_paged_decode(const PagedAttnArgs& a, hipStream_t st) {
  if (a.c.dtype == DQ_BF16) { if (a.c.head_dim == 128) launch_decode<__bf16, 128>(a, st); else launch_decode<__bf16, 64>(a, st); }
  else { if (a.c.head_dim == 128) launch_decode<_Float16, 128>(a, st); else launch_decode<_Float16, 64>(a, st); }
  DQ_HIP_CHECK(hipGetLastError());
  return DQ_OK;
}

}  // namespace dq
