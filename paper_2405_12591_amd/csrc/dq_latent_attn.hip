// Attention over latents in the absorbed form: one key and one value for all heads, a paged cache of 16-bit rows.
#include "dq_latent.h"

namespace dq {

struct LatentArgs {
  dq_latent_cache c;
  dq_paged_batch bt;
  dq_heads q, out;
  const uint64_t* seen;    // of the sequence's own rows, the ones a row sees; null: up to its place
  int max_rows, causal;
  float scale_log2;
  Line line;
  float *o, *ml;           // pieces: [slot, column, R], [slot, column, 2]
};

constexpr int kLatentTile = 32;   // tokens
// Tiles that are a place of the line: one, which all waves work on, or, where each wave works on tiles of its own, one for each (pieces cut
// between them leave waves idle, twice in a workgroup: 64 sequences of 5056 tokens, 16 columns, 90 us where this takes 81).
template <int M> constexpr int kLatentRound = M == 16 ? 4 : 1;

template <int M>
__device__ __forceinline__ Weight latent_weight(const LatentArgs& a, int b) {
  const Sequence s = sequence_of(a.bt, a.c.page_tokens, b);
  const int n = min(s.n, a.max_rows);
  constexpr int PLACE = kLatentTile * kLatentRound<M>;
  return {n ? (int)(((long)n * a.q.heads + M - 1) / M) : 0, max((int)((s.len + (long)PLACE - 1) / PLACE), 1)};
}

template <typename T, int R, int CB>
struct LatentShape {
  static constexpr int ROT = R == 512 ? 64 : 32, W = R + ROT;
  static constexpr int CH = CB == 4 ? 2 : 4;              // waves that share a block of 32 columns, each with a part of the channels
  static constexpr int WAVES = CB * CH, M = 32 * CB;
  static constexpr int BUFFERS = 3;
};

// The first n of 32 tokens, as bits; 32 tokens' bits from place `at` on (there are 64, from 0).
__device__ __forceinline__ uint32_t low_bits(int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1; }
__device__ __forceinline__ uint32_t bits_from(uint64_t bits, int at) {
  const uint64_t w = at >= 0 ? bits >> (at & 63) : bits << (-at & 63);
  return at > -32 && at < 64 ? (uint32_t)w : 0u;
}

// A workgroup takes 32 CB (row, head) columns over its tiles of 32 tokens, which are copied to LDS past the registers and are keys and values
// both.  CH waves share a block of 32 columns: each multiplies its part of the channels, S^T = [c | k_rot] q^T, hands its sums to the
// others through LDS, and then holds its part of O^T += c^T P^T, whose left operand comes from the same rows by transposing reads.  (So a
// wave's queries and results fit 256 registers and two waves a SIMD hide each other's latencies: with all channels' queries in one wave,
// alone on its SIMD, 16 sequences of 14 thousand tokens with 128 heads took 178 us where this takes 104.)  Key rows are taken in the order that
// leaves a lane the probabilities of 8 neighbouring tokens twice, the right operand of the second product.  Bound by matrix instructions: those
// 64 GFLOP are 47 us at the rate of a large product; 16 us go into the pieces' writing (67 MB), 16 more into their join.
template <typename T, int R, int CB>
__global__ __launch_bounds__((64 * LatentShape<T, R, CB>::WAVES), (LatentShape<T, R, CB>::WAVES / 4)) void latent_attn_kernel(LatentArgs a) {
  typedef LatentShape<T, R, CB> Shape;
  constexpr int ROT = Shape::ROT, W = Shape::W, CH = Shape::CH, M = Shape::M, NB = Shape::BUFFERS, WAVES = Shape::WAVES;
  constexpr int TT = kLatentTile, NK = R / 16 / CH, NR = ROT / 16 >= CH ? ROT / 16 / CH : 1, NCT = R / 32 / CH;   // a wave's steps and channel tiles
  constexpr int ROWS = TT / WAVES, LOADS = ROWS * R * 2 / 1024 + 1;   // rows that a wave copies of a tile, and its copies
  typedef typename Vec8<T>::type tx8;
  __shared__ __align__(1024) char s_c[NB][TT * R * 2], s_r[NB][TT * ROT * 2];
  __shared__ __align__(16) f32x4 s_sums[WAVES][4][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r32 = lane & 31, hl = lane >> 5;
  const int cb = wave / CH, chs = wave % CH, H = a.q.heads, P = a.c.page_tokens;
  const auto weight_of = [&](int b) { return latent_weight<M>(a, b); };
  LineStart here;
  if (!line_start(a.line, a.bt.batch, weight_of, here)) return;
  const long end = here.end;
  long at = here.at, begin = here.begin;
  int b = here.b;

  // ---- places in LDS ----
  // A row's 16-byte pieces are exchanged within runs of 16 by bits of the token, so that the 16 lanes that read one piece of 16 tokens'
  // rows (keys), and those that read four pieces of four (values), touch all banks.
  auto swap_of = [](int token) { return (token & 3) << 2 | (token >> 2 & 3); };
  auto rot_swap_of = [](int token) { return ROT == 64 ? token >> 1 & 7 : token >> 2 & 3; };
  // A lane's places are formed with every tile: held over the loop they, and what comes of them, would not fit beside queries and results.
  auto this_lane = []() __attribute__((always_inline)) {
    int l = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
    asm volatile("" : "+v"(l));
    return l;
  };
  struct KeyPlace { int c, rot; };                        // ^ 32 (k % 8), + 256 (k / 8); ^ 32 k
  auto key_place = [&]() __attribute__((always_inline)) {
    const int l = this_lane(), token = (l & 19) | (l & 4) << 1 | (l & 8) >> 1, half = l >> 5;
    return KeyPlace{token * R * 2 + ((half ^ swap_of(token)) << 4), token * ROT * 2 + ((half ^ rot_swap_of(token)) << 4)};
  };
  struct ValuePlace { int a, b; };                        // tokens 8 half + (lane % 16) / 4, and 4 more; ^ 64 (c % 4), + 256 (c / 4)
  auto value_place = [&]() __attribute__((always_inline)) {
    const int l = this_lane(), token = (l >> 5 << 3) + (l >> 2 & 3), piece = (l >> 4 & 1) << 1 | (l >> 1 & 1);
    return ValuePlace{token * R * 2 + ((piece ^ swap_of(token)) << 4) + (l & 1) * 8, (token + 4) * R * 2 + ((piece ^ swap_of(token + 4)) << 4) + (l & 1) * 8};
  };

  for (; at < end;) {
    const Sequence s = sequence_of_wave(a.bt, P, b);
    const Weight wt = weight_of(b);
    const int n = min(s.n, a.max_rows), len = s.len, before = s.old;
    const int unit = __builtin_amdgcn_readfirstlane((int)over(at - begin, wt.tiles)), tiles = __builtin_amdgcn_readfirstlane(wt.tiles);
    const int t0 = __builtin_amdgcn_readfirstlane((int)(at - begin - (long)unit * tiles)), t1 = (int)min((long)tiles, t0 + (end - at));
    const int pairs = n * H, first = unit * M;
    const int rows_lo = first / H, rows_hi = min(first + M - 1, pairs - 1) / H;

    // ---- queries ----
    const int my_pair = min(first + cb * 32 + r32, pairs - 1), my_row = my_pair / H;
    const uint16_t* const q_row = a.q.data + (long)(s.row0 + my_row) * a.q.token_stride + (long)(my_pair % H) * a.q.head_stride + 8 * hl;
    tx8 q[NK + NR];
#pragma unroll
    for (int k = 0; k < NK; ++k) q[k] = __builtin_bit_cast(tx8, *reinterpret_cast<const u32x4*>(q_row + 16 * (chs * NK + k)));
    const bool turns = ROT / 16 >= CH || chs < ROT / 16;    // (four waves, two steps of shared channels)
#pragma unroll
    for (int k = 0; k < NR; ++k) q[NK + k] = __builtin_bit_cast(tx8, turns ? *reinterpret_cast<const u32x4*>(q_row + R + 16 * (chs * NR + k)) : u32x4{0, 0, 0, 0});
    const int all_hi = a.seen ? min(before, len) : a.causal ? min(before + rows_lo + 1, len) : len;   // what every column, any column sees
    const int any_hi = !a.seen && a.causal ? min(before + rows_hi + 1, len) : len;
    const int t_end = min(t1, (max(any_hi, 0) + TT - 1) / TT);

    f32x16 o[NCT];
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[ct][e] = 0.f;
    float m = -INFINITY, l = 0.f;

    int pages = 0, pages_from = t0;                       // of 64 tiles from pages_from on, one a lane
    auto load_pages = [&](int from) __attribute__((always_inline)) {
      pages_from = from;
      const int t = from + this_lane();
      const int page = t < tiles && (long)t * TT < len ? a.bt.page_table[(long)b * a.bt.table_stride + t * TT / P] : -1;
      pages = page >= 0 && page < a.c.pages ? page : -1;
    };
    // Tile t's copies: begin_tile(t), then copy(i) for every i < LOADS.  A tile lies in one page, whose rows are all there to be copied; what
    // is not to be seen of it, or of a page that does not exist, is replaced in LDS (mend_tile).  Copy i has rows EACH (wave + WAVES i) and on.
    constexpr int EACH = 1024 / (R * 2);
    const uint16_t* copy_from = nullptr;
    uint32_t copy_to = 0, copy_rot_to = 0, missing = 0;   // missing: bit t % NB
    auto begin_tile = [&](int t) __attribute__((always_inline)) {
      if (t - pages_from >= 64) load_pages(t);
      const int page = __builtin_amdgcn_readlane(pages, t - pages_from);
      missing = (missing & ~(1u << t % NB)) | (page < 0 ? 1u << t % NB : 0u);
      copy_from = a.c.rows + ((long)max(page, 0) * P + t * TT % P) * W;
      copy_to = lds_of(s_c[t % NB]) + 1024 * wave;
      copy_rot_to = lds_of(s_r[t % NB]) + ROWS * wave * ROT * 2;
    };
    auto load_tile = [&](int t) __attribute__((always_inline)) {
      begin_tile(t);
      const int l = this_lane(), row = R == 512 ? 0 : l >> 5, rot_row = l / (ROT / 8);
      const uint32_t piece = ((R == 512 ? l : l & 31) ^ swap_of(EACH * wave + row)) << 4;
#pragma unroll
      for (int i = 0; i < LOADS - 1; ++i)
        copy_to_lds(copy_from + EACH * (wave + WAVES * i) * W, row * W * 2 + (piece ^ swap_of(WAVES * EACH * i) << 4), copy_to + 1024 * WAVES * i);
      if (rot_row < ROWS)
        copy_to_lds(copy_from + ROWS * wave * W + R, rot_row * W * 2 + ((l % (ROT / 8) ^ rot_swap_of(ROWS * wave + rot_row)) << 4), copy_rot_to);
    };
    // Behind the wave's copies of tile t, ahead of the barrier: values behind the last token become zeros (0 * NaN is not 0), a page that does not
    // exist rows of zeros with keys of NaN.
    auto mend_tile = [&](int t) __attribute__((always_inline)) {
      const int left = missing >> t % NB & 1 ? 0 : len - t * TT;
      if (left >= TT) return;
      const int l = this_lane(), copy_row = R == 512 ? 0 : l >> 5, rot_row = l / (ROT / 8);
#pragma unroll 1
      for (int i = 0; i < LOADS - 1; ++i)
        if (EACH * (wave + WAVES * i) + copy_row >= left) *reinterpret_cast<u32x4*>(s_c[t % NB] + 1024 * (wave + WAVES * i) + 16 * l) = u32x4{0, 0, 0, 0};
      if ((missing >> t % NB & 1) && rot_row < ROWS) *reinterpret_cast<u32x4*>(s_r[t % NB] + ROWS * wave * ROT * 2 + 16 * l) = kNanPiece;
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    };

    // ---- tile by tile ----
    constexpr int KS = NK + NR, AHEAD = CB == 4 ? 3 : KS < 8 ? KS : 8, V_AHEAD = CB == 4 ? 2 : 4;   // LDS reads on their way ahead of the products that take them
    KeyPlace kp;
    ValuePlace vp;
    auto key = [&](int t, int k) __attribute__((always_inline)) {
      if (k < NK) {
        const int step = chs * NK + k;
        return __builtin_bit_cast(tx8, *(LdsPieces)((LdsBytes)s_c[t % NB] + (kp.c ^ 32 * (step % 8)) + 256 * (step / 8)));
      }
      return __builtin_bit_cast(tx8, *(LdsPieces)((LdsBytes)s_r[t % NB] + (kp.rot ^ 32 * (turns ? chs * NR + k - NK : 0))));
    };
    auto value = [&](int t, int i) __attribute__((always_inline)) {
      const int c = chs * NCT + i % NCT;
      const LdsBytes from = (LdsBytes)s_c[t % NB] + 16 * (i / NCT) * R * 2 + 256 * (c / 4);
      return turned_rows<tx8>(from + (vp.a ^ 64 * (c % 4)), from + (vp.b ^ 64 * (c % 4)));
    };
    load_pages(t0);
    __syncthreads();                                      // buffers have been read
    // A tile's two halves: the wave's sums, handed over; then, behind a barrier, the whole scores, their softmax and the product with the values.
    auto hand_over = [&](int t) __attribute__((always_inline)) {
      kp = key_place();
      f32x16 u;
#pragma unroll
      for (int e = 0; e < 16; ++e) u[e] = 0.f;
      tx8 kf[AHEAD];
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) kf[k] = key(t, k);
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        u = mma32(kf[k % AHEAD], q[k], u);
        if (k + AHEAD < KS) kf[k % AHEAD] = key(t, k + AHEAD);
        __builtin_amdgcn_sched_barrier(0);
      }
      const int l_sums = this_lane();
#pragma unroll
      for (int i = 0; i < 4; ++i) s_sums[wave][i][l_sums] = f32x4{u[4 * i], u[4 * i + 1], u[4 * i + 2], u[4 * i + 3]};
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    };
    auto finish = [&](int t) __attribute__((always_inline)) {
      // in an order that gives all of them the same bits: the waves must agree on maxima
      f32x16 u;
      const int l_sums = this_lane();
      auto sums_of = [&](int w, f32x16& to, bool add) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const f32x4 x = s_sums[cb * CH + w][i][l_sums];
#pragma unroll
          for (int e = 0; e < 4; ++e) to[4 * i + e] = add ? to[4 * i + e] + x[e] : x[e];
          if (CB == 4 && add && i % 2) __builtin_amdgcn_sched_barrier(0);
        }
      };
      sums_of(0, u, false);
#pragma unroll
      for (int w = 1; w < CH; ++w) {
        __builtin_amdgcn_sched_barrier(0);
        sums_of(w, u, true);
      }
      if (t * TT + TT > all_hi) {
        // what a column sees is looked up here, in the few tiles that ask for it: held over the loop it would take registers
        const int lane_now = this_lane(), from = t * TT + 8 * (lane_now >> 5);
        const int row = min(first + cb * 32 + (lane_now & 31), pairs - 1) / H;
        uint32_t seen = low_bits((a.seen ? all_hi : a.causal ? min(before + row + 1, len) : len) - from);
        if (a.seen) {
          uint64_t bits = a.seen[s.row0 + row];
          if (s.n < 64) bits &= (1ull << s.n) - 1;
          seen |= bits_from(bits, from - before) & low_bits(len - from);
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) u[e] = seen >> (16 * (e >> 3) + (e & 7)) & 1 ? u[e] : -INFINITY;
      }
      float top = u[0];
#pragma unroll
      for (int e = 1; e < 16; ++e) top = fmaxf(top, u[e]);
      top *= a.scale_log2;
      if (__any(top > m + kLazy)) {
        top = fmaxf(top, __shfl_xor(top, 32));
        const float m_new = fmaxf(m, top), alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - m_new);
        m = m_new;
        l *= alpha;
#pragma unroll
        for (int ct = 0; ct < NCT; ++ct) o[ct] *= alpha;
      }
      // probabilities in the rows' type, which their product with c needs; the sum, in fp32, is of what they were rounded to
      const float base = m == -INFINITY ? 0.f : -m;
      tx8 p[2];
#pragma unroll
      for (int e = 0; e < 16; ++e) p[e >> 3][e & 7] = to_element<tx8>(__builtin_amdgcn_exp2f(__builtin_fmaf(u[e], a.scale_log2, base)));
      l = add_eight(add_eight(l, p[0]), p[1]);
      vp = value_place();
      tx8 vf[V_AHEAD];
#pragma unroll
      for (int i = 0; i < V_AHEAD; ++i) vf[i] = value(t, i);
#pragma unroll
      for (int i = 0; i < 2 * NCT; ++i) {
        o[i % NCT] = mma32(vf[i % V_AHEAD], p[i / NCT], o[i % NCT]);
        if (i + V_AHEAD < 2 * NCT) vf[i % V_AHEAD] = value(t, i + V_AHEAD);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    auto arrived = [&](int t) __attribute__((always_inline)) {   // the wave's copies of tile t; the next one's are on their way
      if (t + 1 < t_end) wait_copies<LOADS>();
      else wait_copies<0>();
      mend_tile(t);
    };
    if (t0 < t_end) {
      load_tile(t0);
      if (t0 + 1 < t_end) load_tile(t0 + 1);
      arrived(t0);
      barrier();
    }
    // Two barriers a tile.  Of each SIMD's two waves one finishes a tile while the other forms sums: the second four waves are half a tile
    // behind, so that softmax and matrix instructions go together (16 x 14 thousand tokens, 128 columns: 104 us, 118 with all in step).
    if (WAVES == 4 || wave < 4) {
      for (int t = t0; t < t_end; ++t) {
        hand_over(t);
        barrier();
        if (t + 2 < t_end) load_tile(t + 2);              // all are done with tile t - 1
        finish(t);
        if (t + 1 < t_end) arrived(t + 1);
        barrier();
      }
    } else {
      for (int t = t0; t < t_end; ++t) {
        if (t > t0) finish(t - 1);
        barrier();
        if (t + 2 < t_end) load_tile(t + 2);
        hand_over(t);
        if (t + 1 < t_end) arrived(t + 1);
        barrier();
      }
      if (t0 < t_end) finish(t_end - 1);
    }

    // ---- the result, or a piece of it (places formed anew: held over the loop they would take registers) ----
    l += __shfl_xor(l, 32);
    const int here = this_lane(), col = cb * 32 + (here & 31), half = here >> 5;
    if (first + col < pairs) {
      if (t0 == 0 && t1 == tiles) {
        const float inv = l == 0.f ? 0.f : 1.f / l;
        const int row = (first + col) / H;
        uint16_t* const dst = a.out.data + (long)(s.row0 + row) * a.out.token_stride + (long)(first + col - row * H) * a.out.head_stride + chs * NCT * 32 + 4 * half;
#pragma unroll
        for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            *reinterpret_cast<u32x2*>(dst + 32 * ct + 8 * e) = u32x2{pack2<T>(o[ct][4 * e] * inv, o[ct][4 * e + 1] * inv),
                                                                    pack2<T>(o[ct][4 * e + 2] * inv, o[ct][4 * e + 3] * inv)};
      } else {
        const long slot = 2l * blockIdx.x + (t0 == 0);
        float* const dst = a.o + (slot * M + col) * R + chs * NCT * 32 + 4 * half;
#pragma unroll
        for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            *reinterpret_cast<f32x4*>(dst + 32 * ct + 8 * e) = f32x4{o[ct][4 * e], o[ct][4 * e + 1], o[ct][4 * e + 2], o[ct][4 * e + 3]};
        if (half == 0 && chs == 0) *reinterpret_cast<f32x2*>(a.ml + 2 * (slot * M + col)) = f32x2{m, l};
      }
    }
    at += t1 - t0;
    if (t1 == tiles && unit == __builtin_amdgcn_readfirstlane(wt.units) - 1) {   // the next sequence that has rows
      begin = at;
      do ++b;
      while (at < end && weight_of(b).units == 0);
    }
  }
}

// Up to 16 columns, which a wave takes with all their channels (queries 72, results 128 registers): every wave of a workgroup copies and works
// tiles of 32 tokens by itself, nothing is shared and no wave waits for another before the end.  A wave's one tile of LDS is loaded again
// when it has been read; three of four waves wait for memory at any time, which is what keeps it busy.  Products of 16 x 16: a lane gets the
// scores of 8 neighbouring tokens of its column, the right operand of the second product.  Bound by memory, at 6.8 TB/s, behind 15 us that do
// not shrink with the cache (finding the work, first tiles, joining waves): 64 sequences of 2000 to 8192 tokens, 16 heads, 378 MB in 77 us.
template <typename T, int R>
__global__ __launch_bounds__(256, 1) void latent_narrow_kernel(LatentArgs a) {
  constexpr int ROT = R == 512 ? 64 : 32, W = R + ROT, M = 16, WAVES = 4, TT = kLatentTile, NK = R / 32, NR = ROT / 32, NCT = R / 16;
  constexpr int EACH = 1024 / (R * 2), COPIES = TT / EACH, ROT_EACH = 512 / ROT, ROT_COPIES = TT / ROT_EACH;   // rows of a copy, copies
  typedef typename Vec8<T>::type tx8;
  struct Tile { char c[TT * R * 2], r[TT * ROT * 2]; };
  union Space {
    Tile tile[WAVES];
    float o[WAVES][M][R + 4];
  };
  __shared__ __align__(1024) Space s_space;
  __shared__ float s_m[WAVES][M], s_l[WAVES][M];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, G = lane >> 4;
  const int H = a.q.heads, P = a.c.page_tokens;
  const auto weight_of = [&](int b) { return latent_weight<M>(a, b); };
  LineStart here;
  if (!line_start(a.line, a.bt.batch, weight_of, here)) return;
  const long end = here.end;
  long at = here.at, begin = here.begin;
  int b = here.b;

  // Pieces of a row are exchanged by bits of the token, so that 16 lanes that read one piece of 16 rows (keys: tokens 8 i + 0..3), and 32 that
  // read two pieces of eight (values), touch all banks.
  auto swap_of = [](int t) { return (t & 3) << 2 | (t >> 3 & 1) << 1 | (t >> 4 & 1); };
  auto rot_swap_of = [](int t) { return ROT == 64 ? (t >> 1 & 1) | (t >> 3 & 3) << 1 : t >> 3 & 3; };
  const int k_token = 8 * (col >> 2) + (col & 3);         // + 4: the second product's
  const int k_at = k_token * R * 2 + ((G ^ swap_of(k_token)) << 4), rot_at = k_token * ROT * 2 + ((G ^ rot_swap_of(k_token)) << 4);   // ^ 64 k (% 4), ^ 64 k
  const int v_token = 8 * G + (col >> 2);                 // + 4: the second half
  const int v_at = v_token * R * 2 + (((col & 3) >> 1 ^ swap_of(v_token)) << 4) + (col & 1) * 8;   // ^ 32 (c % 8), + 256 (c / 8)
  char* const s_c = s_space.tile[wave].c;
  char* const s_r = s_space.tile[wave].r;
  const uint32_t c_to = lds_of(s_c), r_to = lds_of(s_r);

  for (; at < end;) {
    const Sequence s = sequence_of_wave(a.bt, P, b);
    const Weight wt = weight_of(b);
    const int n = min(s.n, a.max_rows), len = s.len, before = s.old;
    const int unit = __builtin_amdgcn_readfirstlane((int)over(at - begin, wt.tiles)), tiles = __builtin_amdgcn_readfirstlane(wt.tiles);
    const int p0 = __builtin_amdgcn_readfirstlane((int)(at - begin - (long)unit * tiles)), p1 = (int)min((long)tiles, p0 + (end - at));
    const int pairs = n * H, first = unit * M;
    const int my_pair = min(first + col, pairs - 1), my_row = my_pair / H;
    const uint16_t* const q_row = a.q.data + (long)(s.row0 + my_row) * a.q.token_stride + (long)(my_pair % H) * a.q.head_stride + 8 * G;
    tx8 q[NK + NR];
#pragma unroll
    for (int k = 0; k < NK + NR; ++k) q[k] = __builtin_bit_cast(tx8, *reinterpret_cast<const u32x4*>(q_row + 32 * k));
    const int rows_lo = first / H;
    uint64_t bits = 0;
    int see_hi = a.causal ? min(before + my_row + 1, len) : len, all_hi = a.causal ? min(before + rows_lo + 1, len) : len;
    if (a.seen) {
      bits = a.seen[s.row0 + my_row];
      if (s.n < 64) bits &= (1ull << s.n) - 1;
      see_hi = all_hi = min(before, len);
    }
    const int t0 = WAVES * p0, t_end = (int)min((long)WAVES * p1, (long)(len + TT - 1) / TT);
    f32x4 o[NCT];
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct) o[ct] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;

    int pages = -1, pages_from = t0 + wave;               // of 64 of this wave's tiles from pages_from on, one a lane
    auto load_pages = [&](int from) __attribute__((always_inline)) {
      pages_from = from;
      const int t = from + lane * WAVES;
      const int page = t < t_end ? a.bt.page_table[(long)b * a.bt.table_stride + t * TT / P] : -1;
      pages = page >= 0 && page < a.c.pages ? page : -1;
    };
    int page = -1;                                        // of the tile on its way
    auto load_tile = [&](int t) __attribute__((always_inline)) {
      if (t - pages_from >= 64 * WAVES) load_pages(t);
      page = __builtin_amdgcn_readlane(pages, (t - pages_from) / WAVES);
      const uint16_t* const from = a.c.rows + ((long)max(page, 0) * P + t * TT % P) * W;
      int here = lane;
      asm volatile("" : "+v"(here));                      // (else the copies' offsets are held over the loop)
      const int row = here / (64 / EACH), slot = here % (64 / EACH), rot_row = here / (ROT / 8), rot_slot = here % (ROT / 8);
#pragma unroll
      for (int i = 0; i < COPIES; ++i) copy_to_lds<true>(from + i * EACH * W, row * W * 2 + ((slot ^ swap_of(i * EACH + row)) << 4), c_to + 1024 * i);
#pragma unroll
      for (int i = 0; i < ROT_COPIES; ++i)
        copy_to_lds<true>(from + i * ROT_EACH * W + R, rot_row * W * 2 + ((rot_slot ^ rot_swap_of(i * ROT_EACH + rot_row)) << 4), r_to + 1024 * i);
    };

    load_pages(t0 + wave);
    __syncthreads();                                      // the last unit's results have been read
    if (t0 + wave < t_end) load_tile(t0 + wave);
    for (int t = t0 + wave; t < t_end; t += WAVES) {
      wait_copies<0>();
      const int left = page < 0 ? 0 : len - t * TT;
      if (left < TT) {                                    // zeros behind the last token, keys of NaN on a page that does not exist
        for (int i = 0; i < COPIES; ++i)
          if (i * EACH + lane / (64 / EACH) >= left) *reinterpret_cast<u32x4*>(s_c + 1024 * i + 16 * lane) = u32x4{0, 0, 0, 0};
        if (page < 0)
          for (int i = 0; i < ROT_COPIES; ++i) *reinterpret_cast<u32x4*>(s_r + 1024 * i + 16 * lane) = kNanPiece;
      }
      f32x4 u[2];
      u[0] = u[1] = f32x4{0.f, 0.f, 0.f, 0.f};
      constexpr int KS = 2 * (NK + NR), AHEAD = 12, V_AHEAD = 8;   // LDS reads on their way ahead of the products that take them
      auto key = [&](int i) __attribute__((always_inline)) {
        const int k = i / 2, h = i % 2;
        if (k < NK) return __builtin_bit_cast(tx8, *(LdsPieces)((LdsBytes)s_c + 4 * h * R * 2 + (k_at ^ 64 * (k % 4)) + 256 * (k / 4)));
        return __builtin_bit_cast(tx8, *(LdsPieces)((LdsBytes)s_r + 4 * h * ROT * 2 + (rot_at ^ 64 * (k - NK))));
      };
      auto value = [&](int c) __attribute__((always_inline)) {
        const LdsBytes from = (LdsBytes)s_c + (v_at ^ 32 * (c % 8)) + 256 * (c / 8);
        return turned_rows<tx8>(from, from + 4 * R * 2);
      };
      tx8 kf[AHEAD], vf[V_AHEAD];
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) kf[i] = key(i);
#pragma unroll
      for (int i = 0; i < KS; ++i) {
        u[i % 2] = mma16(kf[i % AHEAD], q[i / 2], u[i % 2]);
        if (i + AHEAD < KS) kf[i % AHEAD] = key(i + AHEAD);
        if (i >= KS - V_AHEAD) vf[i - (KS - V_AHEAD)] = value(i - (KS - V_AHEAD));
        __builtin_amdgcn_sched_barrier(0);
      }
      if (t * TT + TT > all_hi) {
        const int from = t * TT + 8 * G;
        const uint32_t seen = low_bits(see_hi - from) | (bits_from(bits, from - before) & low_bits(len - from));
#pragma unroll
        for (int e = 0; e < 8; ++e) u[e >> 2][e & 3] = seen >> e & 1 ? u[e >> 2][e & 3] : -INFINITY;
      }
      float top = u[0][0];
#pragma unroll
      for (int e = 1; e < 8; ++e) top = fmaxf(top, u[e >> 2][e & 3]);
      top *= a.scale_log2;
      if (__any(top > m + kLazy)) {
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float m_new = fmaxf(m, top), alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - m_new);
        m = m_new;
        l *= alpha;
#pragma unroll
        for (int ct = 0; ct < NCT; ++ct) o[ct] *= alpha;
      }
      const float base = m == -INFINITY ? 0.f : -m;
      tx8 p;                                              // in the rows' type; the sum, in fp32, is of what they were rounded to
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] = to_element<tx8>(__builtin_amdgcn_exp2f(__builtin_fmaf(u[e >> 2][e & 3], a.scale_log2, base)));
      l = add_eight(l, p);
#pragma unroll
      for (int c = 0; c < NCT; ++c) {
        o[c] = mma16(vf[c % V_AHEAD], p, o[c]);
        if (c + V_AHEAD < NCT) vf[c % V_AHEAD] = value(c + V_AHEAD);
        __builtin_amdgcn_sched_barrier(0);
      }
      if (t + WAVES < t_end) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the tile has been read
        load_tile(t + WAVES);
      }
    }

    // ---- waves joined, then the result or a piece of it ----
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    __syncthreads();                                      // all tiles have been read
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct) *reinterpret_cast<f32x4*>(&s_space.o[wave][col][16 * ct + 4 * G]) = o[ct];
    if (G == 0) { s_m[wave][col] = m; s_l[wave][col] = l; }
    __syncthreads();
    const bool whole = p0 == 0 && p1 == tiles;
    const long slot = 2l * blockIdx.x + (p0 == 0);
    const int cols = min(pairs - first, M);
#pragma unroll
    for (int i = 0; i < M / WAVES; ++i) {
      const int c = i * WAVES + wave;
      if (c >= cols) break;
      float top = s_m[0][c], f[WAVES], ll = 0.f;
#pragma unroll
      for (int w = 1; w < WAVES; ++w) top = fmaxf(top, s_m[w][c]);
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {
        f[w] = __builtin_amdgcn_exp2f(s_m[w][c] - (top == -INFINITY ? 0.f : top));
        ll = __builtin_fmaf(s_l[w][c], f[w], ll);
      }
      const int row = (first + c) / H;
      uint16_t* const dst = a.out.data + (long)(s.row0 + row) * a.out.token_stride + (long)(first + c - row * H) * a.out.head_stride;
      const float inv = ll == 0.f ? 0.f : 1.f / ll;
#pragma unroll
      for (int ch = 4 * lane; ch < R; ch += 256) {
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
          const f32x4 y = *reinterpret_cast<const f32x4*>(&s_space.o[w][c][ch]);
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = __builtin_fmaf(y[e], f[w], x[e]);
        }
        if (whole) *reinterpret_cast<u32x2*>(dst + ch) = u32x2{pack2<T>(x[0] * inv, x[1] * inv), pack2<T>(x[2] * inv, x[3] * inv)};
        else *reinterpret_cast<f32x4*>(a.o + (slot * M + c) * R + ch) = x;
      }
      if (!whole && lane == 0) *reinterpret_cast<f32x2*>(a.ml + 2 * (slot * M + c)) = f32x2{top, ll};
    }
    at += p1 - p0;
    if (p1 == tiles && unit == __builtin_amdgcn_readfirstlane(wt.units) - 1) {   // the next sequence that has rows
      begin = at;
      do ++b;
      while (at < end && weight_of(b).units == 0);
    }
  }
}

template <typename T, int R, int M>
__global__ __launch_bounds__(256) void latent_join_kernel(LatentArgs a) {
  constexpr int GROUPS = M / kJoinColumns<R>;
  const int H = a.q.heads, item = (int)(blockIdx.x / GROUPS), col = (int)(blockIdx.x % GROUPS) * kJoinColumns<R>;
  const int b = item_owner(a.bt.starts, a.bt.rows, a.bt.batch, item, H, M, 1);
  const Sequence s = sequence_of_wave(a.bt, a.c.page_tokens, b);
  const int pairs = min(s.n, a.max_rows) * H, first = (item - item_first(a.bt.starts, a.bt.rows, b, H, M, 1)) * M;
  if (first < 0 || first + col >= pairs) return;
  const auto weight_of = [&](int i) { return latent_weight<M>(a, i); };
  const int tiles = weight_of(b).tiles;
  const LineSums sums = line_sums(a.bt.batch, b, weight_of);
  const Pieces p = pieces_of(sums.before + (long)(first / M) * tiles, tiles, line_quota(a.line, sums.total));
  if (p.first == p.last) return;
  join_columns<T, R>((int)(p.last - p.first) + 1, [&](int i) { return slot_of(p, p.first + i); }, a.o, a.ml, M, col, min(pairs - first, M), [&](int c) {
    const int pair = first + c;
    return a.out.data + (long)(s.row0 + pair / H) * a.out.token_stride + (long)(pair % H) * a.out.head_stride;
  });
}

// Columns of a workgroup: the fewest that hold a sequence's (row, head) pairs, 128 where there are more, since every tile of columns reads the
// tokens again: 16 sequences of 14 thousand tokens with 128 heads 120 us in 128, 156 in 64, 231 in 32; 24 drafted rows of 32 heads behind 8 x 7
// thousand 152, 221, 337; 64 sequences with 16 heads 85 us in the narrow kernel's 16, 91 in 32.  What each takes of its own: 64 sequences of 2000 to
// 8192 tokens with 16, 32 and 64 heads 84, 102 and 131 us.
struct LatentPlan {
  int cols;                // of a workgroup
  long items, workgroups;
};

static bool latent_plan(int batch, long rows, int heads, int max_rows, int max_seq_len, LatentPlan* p) {
  if (batch <= 0 || rows < 0 || heads <= 0 || max_rows < 0 || max_seq_len < 0 || rows * heads >= (1l << 31) - 256) return false;
  const long cols = (long)max_rows * heads;
  p->cols = cols <= 16 ? 16 : cols <= 32 ? 32 : cols <= 64 ? 64 : 128;
  p->items = rows * heads / p->cols + batch;
  if (p->items * (p->cols / kJoinColumns<512>) >= kMaxThreads / 256) return false;
  p->workgroups = 256;   // a compute unit's LDS holds one (two of 256 channels and up to 32 columns, which are launched as one all the same)
  return true;
}
static size_t latent_bytes(const dq_latent_cache* c, const LatentPlan& p) {
  return (size_t)(2 * p.workgroups * p.cols) * (c->latent_dim + 2) * sizeof(float);
}

template <typename T, int R, int CB>
static void launch_latent_blocks(const LatentArgs& a, const LatentPlan& p, hipStream_t st) {
  hipLaunchKernelGGL((latent_attn_kernel<T, R, CB>), dim3((unsigned)p.workgroups), dim3(64 * LatentShape<T, R, CB>::WAVES), 0, st, a);
}
template <typename T, int R, int M>
static void launch_latent_join(const LatentArgs& a, const LatentPlan& p, hipStream_t st) {
  hipLaunchKernelGGL((latent_join_kernel<T, R, M>), dim3((unsigned)(p.items * (M / kJoinColumns<R>))), dim3(256), 0, st, a);
}
template <typename T, int R>
static void launch_latent(const LatentArgs& a, const LatentPlan& p, hipStream_t st) {
  switch (p.cols) {
    case 16:
      hipLaunchKernelGGL((latent_narrow_kernel<T, R>), dim3((unsigned)p.workgroups), dim3(256), 0, st, a);
      launch_latent_join<T, R, 16>(a, p, st);
      break;
    case 32:
      launch_latent_blocks<T, R, 1>(a, p, st);
      launch_latent_join<T, R, 32>(a, p, st);
      break;
    case 64:
      launch_latent_blocks<T, R, 2>(a, p, st);
      launch_latent_join<T, R, 64>(a, p, st);
      break;
    default:
      launch_latent_blocks<T, R, 4>(a, p, st);
      launch_latent_join<T, R, 128>(a, p, st);
  }
}

}  // namespace dq

using namespace dq;

extern "C" size_t dq_latent_workspace_bytes(const dq_latent_cache* cache, int32_t batch, int32_t rows, int32_t q_heads, int32_t max_rows,
                                            int32_t max_seq_len) {
  LatentPlan p;
  if (!latent_cache_ok(cache) || !latent_plan(batch, rows, q_heads, max_rows, max_seq_len, &p)) return 0;
  return latent_bytes(cache, p);                          // (smaller calls with the same heads have no more columns)
}

extern "C" int32_t dq_latent_attention(const dq_latent_cache* cache, const dq_paged_batch* batch, const dq_heads* q, const dq_heads* out,
                                       const uint64_t* seen, int32_t max_rows, int32_t max_seq_len, float softmax_scale, void* workspace,
                                       size_t workspace_bytes, uint32_t flags, void* hip_stream) {
  if (!latent_cache_ok(cache) || !latent_batch_ok(batch, cache, true) || !heads_ok(q, false) || !heads_ok(out, false)) return DQ_EINVAL;
  if (q->heads != out->heads || !workspace || ((uintptr_t)workspace & 15) || (flags & ~DQ_PAGED_CAUSAL) || !(softmax_scale > 0.f) || !scale_ok(softmax_scale)) return DQ_EINVAL;
  if (heads_meet(q, batch->rows, cache->latent_dim + cache->rot_dim, out, batch->rows, cache->latent_dim)) return DQ_EINVAL;
  if (seen && (((uintptr_t)seen & 7) || !(flags & DQ_PAGED_CAUSAL) || max_rows > 64)) return DQ_EINVAL;
  LatentPlan p;
  if (!latent_plan(batch->batch, batch->rows, q->heads, max_rows, max_seq_len, &p)) return DQ_EINVAL;
  if (workspace_bytes < latent_bytes(cache, p)) return DQ_ENOSPACE;
  if (batch->rows == 0 || max_rows == 0) return DQ_OK;
  LatentArgs a = {};
  a.c = *cache; a.bt = *batch; a.q = *q; a.out = *out;
  a.seen = seen;
  a.max_rows = max_rows;
  a.causal = (flags & DQ_PAGED_CAUSAL) ? 1 : 0;
  a.scale_log2 = fmaxf(softmax_scale * 1.44269504088896340736f, 1e-37f);
  a.line = {(int)p.workgroups, p.cols == 16 ? 1 : 2};
  a.o = reinterpret_cast<float*>(workspace);
  a.ml = a.o + 2 * p.workgroups * p.cols * cache->latent_dim;
  hipStream_t st = (hipStream_t)hip_stream;
  if (cache->dtype == DQ_BF16) { if (cache->latent_dim == 512) launch_latent<__bf16, 512>(a, p, st); else launch_latent<__bf16, 256>(a, p, st); }
  else { if (cache->latent_dim == 512) launch_latent<_Float16, 512>(a, p, st); else launch_latent<_Float16, 256>(a, p, st); }
  DQ_HIP_CHECK(hipGetLastError());
  return DQ_OK;
}
