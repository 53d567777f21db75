// Attention of drafted rows over the paged 8-bit cache and, by bit masks, over each other.
#include "dq_latent.h"

namespace dq {

struct TreeArgs {
  dq_paged_cache c;
  dq_paged_batch bt;
  dq_heads q, k, v, out;
  const uint64_t* seen;
  int group;               // query heads per kv head
  int max_rows;            // rows of any sequence at most, 64
  int window;              // 0: none
  float scale_log2;
  Line line;
  float *o, *ml;           // pieces: [slot, column, D], [slot, column, 2]
};

constexpr int kTreeRows = 64;
// Tiles of the line that a unit's drafted rows count for: they are a chain of their own (values to LDS, keys, masks) and would otherwise make
// the workgroups that have them the last ones (8 sequences of 2 to 9 thousand tokens, window 4096, 64 units: 27 us, 30 counted as one tile).
constexpr int kDraftedTiles = 6;

struct TreeSequence {
  int row0, n;             // its drafted rows
  int place0;              // place of a row that sees itself alone
  int len;                 // cached tokens
  int first_tile;          // of the cached tokens that any row sees
  Weight w;                // units: kv head after kv head, a head's column tiles; tiles: of 64 cached tokens, and the drafted rows'
};
template <int M>
__device__ __forceinline__ TreeSequence tree_sequence(const TreeArgs& a, int b) {
  const Sequence s = sequence_of(a.bt, a.c.page_tokens, b);
  TreeSequence t;
  t.row0 = s.row0;
  t.n = min(s.n, a.max_rows);
  t.place0 = s.old + s.n;
  t.len = s.len;
  t.first_tile = a.window ? max(t.place0 - a.window, 0) / kPagedTile : 0;   // (a row that sees none has the place before)
  const int code_tiles = (s.len + kPagedTile - 1) / kPagedTile;
  t.w.units = t.n ? a.c.kv_heads * ((t.n * a.group + M - 1) / M) : 0;
  t.w.tiles = max(code_tiles - t.first_tile, 0) + kDraftedTiles;
  return t;
}

// A workgroup of four waves takes M = 32 CB (row, query head) columns of a kv head; CB blocks of 32 columns, and 4 / CB groups of waves that
// share the tiles of 64 tokens and are joined through LDS.  Codes come to LDS as they lie in memory, and go to f16 on their way into the
// products.  Scores are formed transposed, in products of 32 x 32: row r of a product stands for token (r & 3) + 4 (r >> 3) + 16 (r >> 2 & 1), so a
// lane ends up with the scores of 16 neighbouring tokens of its column, twice, and takes the value codes of those in 16-byte pieces.  16 sequences
// of 32768 tokens, 8 kv heads of 128, 64 columns, 1.08 GB: 203 us (166 are the reading), matrix instructions busy for a third of it and vector
// instructions, two thirds of them from codes to f16 and exponentials, for 55 %.
template <typename T, int D, bool FP8, int CB>
__global__ __launch_bounds__(256, 2) void tree_attn_kernel(TreeArgs a) {
  constexpr int M = 32 * CB, TG = 4 / CB, NC = D / 32, PD = D / 8;
  typedef typename Vec8<T>::type tx8;
  constexpr int NB = CB, PIECES = D / 16, COPIES = D / 8 / CB;   // tiles in LDS of a group of waves; 16-byte pieces of a key row; a wave's copies of a tile
  union Space {
    char codes[TG][NB][2][kPagedTile * D];                // keys, values as the cache holds them
    char v[kTreeRows * D * 2];                            // drafted values, row by row
    float o[TG > 1 ? 4 : 1][32][D + 1];
  };
  __shared__ __align__(1024) Space s_space;
  __shared__ float s_m[4][32], s_l[4][32];
  __shared__ uint64_t s_bad;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r32 = lane & 31, hl = lane >> 5;
  const int cb = wave % CB, tg = wave / CB, H = a.c.kv_heads, P = a.c.page_tokens, runs = P / kPagedTile;
  const auto weight_of = [&](int b) { return tree_sequence<M>(a, b).w; };
  LineStart here;
  if (!line_start(a.line, a.bt.batch, weight_of, here)) return;
  const long end = here.end;
  long at = here.at, begin = here.begin;
  int b = here.b;
  const int k_row = (r32 & 3) | (r32 >> 3) << 2 | (r32 >> 2 & 1) << 4;   // + 32 tt: the token of this lane's row

  while (at < end) {
    TreeSequence s = tree_sequence<M>(a, b);
    auto uniform = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
    s.row0 = uniform(s.row0); s.n = uniform(s.n); s.place0 = uniform(s.place0); s.len = uniform(s.len); s.first_tile = uniform(s.first_tile);
    const int n = s.n, len = s.len, tiles = uniform(s.w.tiles), units = uniform(s.w.units), col_tiles = units / H;
    const int unit = uniform((int)over(at - begin, tiles)), h = unit / col_tiles, first = unit % col_tiles * M;
    const int t0 = uniform((int)(at - begin - (long)unit * tiles)), t1 = (int)min((long)tiles, t0 + (end - at));
    const int pairs = n * a.group;
    const int my_pair = min(first + cb * 32 + r32, pairs - 1), my_row = my_pair / a.group;
    uint64_t bits = a.seen[s.row0 + my_row];
    if (n < 64) bits &= (1ull << n) - 1;
    const int see_lo = window_start(s.place0 + __popcll(bits) - 1, a.window), all_lo = a.window ? window_start(s.place0 + n, a.window) : 0;

    // ---- queries: 8 channels 32 c + 16 hl + 8 half of the column, in f16 ----
    const uint16_t* const q_row = a.q.data + (long)(s.row0 + my_row) * a.q.token_stride + (long)(h * a.group + my_pair % a.group) * a.q.head_stride + 16 * hl;
    f16x8 q[NC][2];
    float sc = a.scale_log2;
    {
      int shift = 0;
      if constexpr (__is_same(T, __bf16)) {
        float amax = 0.f;
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
            float x[8];
            unpack8<T>(*reinterpret_cast<const u32x4*>(q_row + 32 * c + 8 * hf), x);
#pragma unroll
            for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(x[e]));
          }
        amax = fmaxf(amax, __shfl_xor(amax, 32));
        shift = fit_shift(amax);
        sc = __builtin_ldexpf(sc, -shift);
      }
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          const u32x4 w = *reinterpret_cast<const u32x4*>(q_row + 32 * c + 8 * hf);
          if constexpr (__is_same(T, __bf16)) {
            float x[8];
            unpack8<T>(w, x);
#pragma unroll
            for (int e = 0; e < 8; ++e) q[c][hf][e] = (_Float16)__builtin_ldexpf(x[e], shift);
          } else {
            q[c][hf] = __builtin_bit_cast(f16x8, w);
          }
        }
    }
    f32x16 o[NC];
#pragma unroll
    for (int ct = 0; ct < NC; ++ct)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[ct][e] = 0.f;
    float m = -INFINITY, l = 0.f;

    // Softmax of a tile's 32 products of this lane (token 32 (e / 16) + 16 hl + e % 16 of the tile), in place: u -> p = 2^(u f + add - m).
    auto softmax = [&](f32x16 (&u)[2], float f, float add, float inv_sv) __attribute__((always_inline)) {
      float top = u[0][0];
#pragma unroll
      for (int e = 1; e < 32; ++e) top = fmaxf(top, u[e >> 4][e & 15]);
      top = __builtin_fmaf(top, f, add);
      if (__any(top > m + kLazy)) {
        top = fmaxf(top, __shfl_xor(top, 32));
        const float m_new = fmaxf(m, top);
        const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - m_new);
        m = m_new;
        l *= alpha;
#pragma unroll
        for (int ct = 0; ct < NC; ++ct) o[ct] *= alpha;
      }
      const float base = m == -INFINITY ? add : add - m;
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 32; ++e) {
        u[e >> 4][e & 15] = __builtin_amdgcn_exp2f(__builtin_fmaf(u[e >> 4][e & 15], f, base));
        sum += u[e >> 4][e & 15];
      }
      l = __builtin_fmaf(sum, inv_sv, l);
    };
    // Scores of tokens from `from` on that the column does not see (lo .. hi - 1 are seen); NaN factors poison those who see the tokens.
    auto hide = [&](f32x16 (&u)[2], float& f, int from, int lo, int hi) __attribute__((always_inline)) {
      int first_token = from + 16 * hl;
      asm volatile("" : "+v"(first_token)::"memory");     // (a branch, and nothing of it ahead of the loop)
      const float poison = f - f;
      f = f == f ? f : 1.f;
      const int a_lo = lo - first_token, a_hi = hi - first_token;
#pragma unroll
      for (int e = 0; e < 32; ++e) {
        const int t = 32 * (e >> 4) + (e & 15);
        u[e >> 4][e & 15] = t < a_lo || t >= a_hi ? -INFINITY : u[e >> 4][e & 15] + poison;
      }
    };

    // ---- full pages ----
    // A tile's codes lie in one piece; they are copied to LDS past the registers, by the waves that read them (as 16-byte loads of rows they came in
    // quarters of lines, and once for every wave: 273 us for what now takes 203).  Pieces are exchanged by bits of the row so that 16 lanes touch all banks.
    auto key_swap = [](int t) { return PIECES == 8 ? (t >> 1 & 3) | (t >> 4 & 1) << 2 : (t >> 2 & 1) | (t >> 4 & 1) << 1; };
    const int code_tiles = len / P * runs;
    const int code_first = s.first_tile + t0, last_code = min(s.first_tile + t1, code_tiles);
    __syncthreads();                                      // what the last unit left in LDS has been read
    for (int batch0 = code_first; batch0 < last_code; batch0 += 64 * TG) {
      const int t_l = batch0 + lane * TG + tg;            // the next 64 tiles' blocks and scales, one per lane
      int blk = -1;
      float sk = 0.f, lsv = 0.f, isv = 0.f;
      if (t_l < last_code) {
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
      // (every group of waves goes through the barriers of the one with most tiles)
      const int most = min(64, (last_code - batch0 + TG - 1) / TG), count = min(64, max(last_code - batch0 - tg + TG - 1, 0) / TG);
      auto copy_tile = [&](int i) __attribute__((always_inline)) {
        const int block = __builtin_amdgcn_readlane(blk, i);
        int l = lane;
        asm volatile("" : "+v"(l));                       // (else the offsets are held over the loop)
        const int row = l / PIECES, key = row * D + ((l % PIECES ^ key_swap(row)) << 4), value = l / 4 * 64 + ((l % 4 ^ (l >> 4 & 3)) << 4);
        const uint8_t* const ks = block < 0 ? reinterpret_cast<const uint8_t*>(g_no_codes) : a.c.k_codes + (long)block * (kPagedTile * D);
        const uint8_t* const vs = block < 0 ? reinterpret_cast<const uint8_t*>(g_no_codes) : a.c.v_codes + (long)block * (kPagedTile * D);
        const uint32_t to = lds_of(s_space.codes[tg][i % NB][0]);
#pragma unroll
        for (int j = 0; j < COPIES; ++j) {
          const int c = j * CB + cb, part = c % PIECES;   // keys' pieces first
          const int turn = PIECES == 8 ? (part >> 1 & 1) << 2 : (part & 1) << 1;
          copy_to_lds<CB < 4>(reinterpret_cast<const uint16_t*>((c < PIECES ? ks : vs) + 1024 * part), c < PIECES ? key ^ turn << 4 : value, to + 1024 * c);
        }
      };
      auto key_codes = [&](int i, int c, int tt) __attribute__((always_inline)) {
        return *(LdsPieces)((LdsBytes)s_space.codes[tg][i % NB][0] + (32 * tt + k_row) * D + ((2 * c + hl ^ key_swap(k_row)) << 4));
      };
      auto value_codes = [&](int i, int ct, int tt) __attribute__((always_inline)) {
        return *(LdsPieces)((LdsBytes)s_space.codes[tg][i % NB][1] + (32 * ct + r32) * 64 + ((2 * tt + hl ^ (r32 >> 2 & 3)) << 4));
      };
      if (batch0 > code_first && CB > 1) __syncthreads();   // the last 64 tiles have been read
      else asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
      for (int i = 0; i < (NB > 1 ? NB - 1 : 1); ++i)
        if (i < count) copy_tile(i);
      for (int i = 0; i < most; ++i) {
        if constexpr (CB == 1) {
          wait_copies<0>();                               // (a wave's own tile: the other waves compute meanwhile)
          if (i >= count) break;
        } else {
          if (NB > 2 && i + NB - 2 < count) wait_copies<(NB - 2) * COPIES>();
          else wait_copies<0>();
          barrier();                                      // the tile is there, and all are done with the one before it
          if (i + NB - 1 < count) copy_tile(i + NB - 1);
          if (i >= count) continue;
        }
        float f = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, sk), i));
        const float add = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, lsv), i));
        const float inv_sv = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, isv), i));
        f32x16 u[2];
#pragma unroll
        for (int e = 0; e < 32; ++e) u[e >> 4][e & 15] = 0.f;
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int hf = 0; hf < 2; ++hf)
#pragma unroll
            for (int tt = 0; tt < 2; ++tt) {
              const u32x4 w = key_codes(i, c, tt);
              u[tt] = mma32(hf ? codes_f16<FP8>(w.z, w.w) : codes_f16<FP8>(w.x, w.y), q[c][hf], u[tt]);
            }
        f = keep_sign(f * sc);
        const int from = (batch0 + i * TG + tg) * kPagedTile;
        if (from < all_lo) hide(u, f, from, see_lo, INT32_MAX);
        softmax(u, f, add, inv_sv);
        // 11 bits, as the codes' products want them (the sum keeps fp32)
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) {
          f16x8 p[2];
#pragma unroll
          for (int e = 0; e < 16; ++e) p[e >> 3][e & 7] = (_Float16)u[tt][e];
#pragma unroll
          for (int ct = 0; ct < NC; ++ct) {
            const u32x4 w = value_codes(i, ct, tt);
            o[ct] = mma32(codes_f16<FP8>(w.x, w.y), p[0], o[ct]);
            o[ct] = mma32(codes_f16<FP8>(w.z, w.w), p[1], o[ct]);
          }
        }
        if (CB == 1 && i + 1 < count) {
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the tile has been read
          copy_tile(i + 1);
        }
      }
    }

    // Products of 16-bit rows, keys `key(tt, channel)` and values `value(ct, tt, half)`, in their own type.
    auto row_tile = [&](auto key, auto value, float f, int from, int lo, int hi, uint64_t hidden, uint64_t bad) __attribute__((always_inline)) {
      // (a half's pieces are asked for together, and the queries' once more, in their own type)
      f32x16 u[2];
      tx8 rows_q[NC][2];
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) rows_q[c][hf] = __builtin_bit_cast(tx8, *reinterpret_cast<const u32x4*>(q_row + 32 * c + 8 * hf));
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
        u32x4 keys[NC][2];
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) keys[c][hf] = key(tt, 32 * c + 8 * hf);
#pragma unroll
        for (int e = 0; e < 16; ++e) u[tt][e] = 0.f;
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) u[tt] = mma32(__builtin_bit_cast(tx8, keys[c][hf]), rows_q[c][hf], u[tt]);
        __builtin_amdgcn_sched_barrier(0);
      }
      hide(u, f, from, lo, hi);
      int shift = 16 * hl;
      asm volatile("" : "+v"(shift));
      const uint64_t mine = hidden >> shift, poison = bad >> shift;
#pragma unroll
      for (int e = 0; e < 32; ++e) {
        const int t = 32 * (e >> 4) + (e & 15);
        const float w = poison >> t & 1 ? __builtin_nanf("") : u[e >> 4][e & 15];
        u[e >> 4][e & 15] = mine >> t & 1 ? -INFINITY : w;
      }
      softmax(u, f, 0.f, 1.f);
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
        tx8 values[NC][2];
#pragma unroll
        for (int ct = 0; ct < NC; ++ct)
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) values[ct][hf] = value(ct, tt, hf);
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          // in the rows' type, which their products need: 8 bits with bf16 rows, one more such rounding for each of these tokens
          u32x4 p;
#pragma unroll
          for (int e = 0; e < 4; ++e) p[e] = pack2<T>(u[tt][8 * hf + 2 * e], u[tt][8 * hf + 2 * e + 1]);
#pragma unroll
          for (int ct = 0; ct < NC; ++ct) o[ct] = mma32(values[ct][hf], __builtin_bit_cast(tx8, p), o[ct]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    };

    // ---- the page being filled ----
    for (int tile = max(code_tiles, s.first_tile + t0); tile < s.first_tile + min(t1, tiles - kDraftedTiles); ++tile) {
      if ((tile - s.first_tile - t0) % TG != tg) continue;
      const int slot = a.bt.tail_slots ? a.bt.tail_slots[b] : b;
      const bool ok = slot >= 0 && slot < a.c.slots;
      const int left = ok ? len - tile * kPagedTile : 0;
      const long from = (((long)(ok ? slot : 0) * H + h) * runs + (tile - code_tiles)) * kPagedTile * D;
      int here = lane;
      asm volatile("" : "+v"(here));                      // (else its places are formed ahead of all loops and held there)
      const int half = here >> 5;
      const uint16_t* const kt = a.c.k_tail + from + ((here & 3) | (here >> 3 & 3) << 2 | (here >> 2 & 1) << 4) * D + 16 * half;
      const uint16_t* const vt = a.c.v_tail + from + (here & 31) * kPagedTile + 16 * half;
      row_tile([&](int tt, int ch) { return *reinterpret_cast<const u32x4*>(kt + 32 * tt * D + ch); },
               [&](int ct, int tt, int hf) {
                 u32x4 w = *reinterpret_cast<const u32x4*>(vt + ct * 32 * kPagedTile + 32 * tt + 8 * hf);
                 // rows behind the last token may hold anything: 0 * NaN is not 0
#pragma unroll
                 for (int e = 0; e < 4; ++e) w[e] = keep_tokens(w[e], left - 32 * tt - 16 * half - 8 * hf - 2 * e);
                 return __builtin_bit_cast(tx8, w);
               },
               ok ? keep_sign(a.scale_log2) : __builtin_nanf(""), tile * kPagedTile, see_lo, len, 0, 0);
    }

    // ---- the drafted rows: values through LDS, for their transposed reads ----
    if (t1 == tiles) {
      __syncthreads();                                    // the codes have been read
      if (tid == 0) s_bad = 0;
      __syncthreads();
      auto swap_of = [](int t) { return PD == 16 ? (t & 3) << 2 | (t >> 2 & 3) : (t >> 1 & 1) << 2 | (t >> 2 & 3); };
      constexpr uint32_t kExp = __is_same(T, __bf16) ? 0x7F80u : 0x7C00u;
#pragma unroll
      for (int i = tid; i < kTreeRows * PD; i += 256) {   // (whole waves)
        const int row = i / PD, piece = i % PD;
        u32x4 w = {}, kw = {};
        if (row < n) {
          w = *reinterpret_cast<const u32x4*>(a.v.data + (long)(s.row0 + row) * a.v.token_stride + (long)h * a.v.head_stride + 8 * piece);
          kw = *reinterpret_cast<const u32x4*>(a.k.data + (long)(s.row0 + row) * a.k.token_stride + (long)h * a.k.head_stride + 8 * piece);
        }
        // a row that is not finite has values of zero and scores of NaN, for those who see it
        bool any = false;
#pragma unroll
        for (int e = 0; e < 4; ++e) any |= (w[e] & kExp) == kExp || (w[e] >> 16 & kExp) == kExp || (kw[e] & kExp) == kExp || (kw[e] >> 16 & kExp) == kExp;
        const bool bad = (__ballot(any) >> (lane / PD * PD) & ((1ull << PD) - 1)) != 0;
        if (bad) w = u32x4{0, 0, 0, 0};
        if (bad && piece == 0) atomicOr(reinterpret_cast<unsigned long long*>(&s_bad), 1ull << row);
        *reinterpret_cast<u32x4*>(s_space.v + row * D * 2 + ((piece ^ swap_of(row)) << 4)) = w;
      }
      __syncthreads();
      if (tg == 0) {
        int here = lane;
        asm volatile("" : "+v"(here));                    // (else its places are formed ahead of all loops and held there)
        const int half = here >> 5, i16 = here & 15, v_token = 16 * half + (i16 >> 2), v_piece = 2 * (here >> 4 & 1) + ((i16 & 3) >> 1);
        const int key_row = (here & 3) | (here >> 3 & 3) << 2 | (here >> 2 & 1) << 4;
        const uint16_t* const k_head = a.k.data + (long)s.row0 * a.k.token_stride + (long)h * a.k.head_stride + 16 * half;
        const LdsBytes from = (LdsBytes)s_space.v + (i16 & 1) * 8;
        auto v_at = [&](int token, int ct) { return from + token * D * 2 + (((v_piece ^ swap_of(token)) << 4) ^ 64 * ct); };
        row_tile([&](int tt, int ch) {
                   const int row = key_row + 32 * tt;
                   return row < n ? *reinterpret_cast<const u32x4*>(k_head + (long)row * a.k.token_stride + ch) : u32x4{0, 0, 0, 0};
                 },
                 [&](int ct, int tt, int hf) { return turned_rows<tx8>(v_at(v_token + 32 * tt + 8 * hf, ct), v_at(v_token + 32 * tt + 8 * hf + 4, ct)); },
                 keep_sign(a.scale_log2), 0, 0, kTreeRows, ~bits, s_bad);
      }
    }

    // ---- groups of waves joined, then the result or a piece of it ----
    l += __shfl_xor(l, 32);
    const bool whole = t0 == 0 && t1 == tiles;
    const long slot = 2l * blockIdx.x + (t0 == 0);
    auto out_of = [&](int col) {
      const int pair = first + col;
      return a.out.data + (long)(s.row0 + pair / a.group) * a.out.token_stride + (long)(h * a.group + pair % a.group) * a.out.head_stride;
    };
    if constexpr (TG == 1) {
      const int col = cb * 32 + r32;
      if (first + col < pairs) {
        if (whole) {
          const float inv = l == 0.f ? 0.f : 1.f / l;
          uint16_t* const dst = out_of(col);
#pragma unroll
          for (int ct = 0; ct < NC; ++ct)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              *reinterpret_cast<u32x2*>(dst + 32 * ct + 8 * e + 4 * hl) = u32x2{pack2<T>(o[ct][4 * e] * inv, o[ct][4 * e + 1] * inv),
                                                                               pack2<T>(o[ct][4 * e + 2] * inv, o[ct][4 * e + 3] * inv)};
        } else {
          float* const dst = a.o + (slot * M + col) * D;
#pragma unroll
          for (int ct = 0; ct < NC; ++ct)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              *reinterpret_cast<f32x4*>(dst + 32 * ct + 8 * e + 4 * hl) = f32x4{o[ct][4 * e], o[ct][4 * e + 1], o[ct][4 * e + 2], o[ct][4 * e + 3]};
          if (hl == 0) *reinterpret_cast<f32x2*>(a.ml + 2 * (slot * M + col)) = f32x2{m, l};
        }
      }
    } else {
      __syncthreads();                                    // drafted values, or the last unit's results, have been read
#pragma unroll
      for (int ct = 0; ct < NC; ++ct)
#pragma unroll
        for (int e = 0; e < 16; ++e) s_space.o[wave][r32][32 * ct + 8 * (e >> 2) + 4 * hl + (e & 3)] = o[ct][e];
      if (hl == 0) { s_m[wave][r32] = m; s_l[wave][r32] = l; }
      __syncthreads();
      const int cols = min(pairs - first, M);
      for (int idx = 2 * tid; idx < cols * D; idx += 512) {
        const int col = idx / D, ch = idx % D, w0 = col / 32, cc = col % 32;
        float top = -INFINITY;
#pragma unroll
        for (int g = 0; g < TG; ++g) top = fmaxf(top, s_m[w0 + g * CB][cc]);
        const float base = top == -INFINITY ? 0.f : top;
        float x = 0.f, y = 0.f, ll = 0.f;
#pragma unroll
        for (int g = 0; g < TG; ++g) {
          const int w = w0 + g * CB;
          const float f = __builtin_amdgcn_exp2f(s_m[w][cc] - base);
          x = __builtin_fmaf(s_space.o[w][cc][ch], f, x);
          y = __builtin_fmaf(s_space.o[w][cc][ch + 1], f, y);
          ll = __builtin_fmaf(s_l[w][cc], f, ll);
        }
        if (whole) {
          const float inv = ll == 0.f ? 0.f : 1.f / ll;
          *reinterpret_cast<uint32_t*>(out_of(col) + ch) = pack2<T>(x * inv, y * inv);
        } else {
          *reinterpret_cast<f32x2*>(a.o + (slot * M + col) * D + ch) = f32x2{x, y};
          if (ch == 0) *reinterpret_cast<f32x2*>(a.ml + 2 * (slot * M + col)) = f32x2{top, ll};
        }
      }
    }
    at += t1 - t0;
    if (t1 == tiles && unit == units - 1) {               // the next sequence that has rows
      begin = at;
      do ++b;
      while (at < end && uniform(weight_of(b).units) == 0);
    }
  }
}

template <typename T, int D, int CB>
__global__ __launch_bounds__(256) void tree_join_kernel(TreeArgs a) {
  constexpr int M = 32 * CB;
  constexpr unsigned GROUPS = M / kJoinColumns<D>;
  const int H = a.c.kv_heads, col = (int)(blockIdx.x % GROUPS) * kJoinColumns<D>, h = (int)(blockIdx.x / GROUPS % (unsigned)H);
  const int item = (int)(blockIdx.x / GROUPS / (unsigned)H);
  const int b = item_owner(a.bt.starts, a.bt.rows, a.bt.batch, item, a.group, M, 1);
  const TreeSequence s = tree_sequence<M>(a, b);
  const int j = item - item_first(a.bt.starts, a.bt.rows, b, a.group, M, 1), col_tiles = s.w.units / H, first = j * M, pairs = s.n * a.group;
  if (j < 0 || first + col >= pairs) return;
  const auto weight_of = [&](int i) { return tree_sequence<M>(a, i).w; };
  const LineSums sums = line_sums(a.bt.batch, b, weight_of);
  const Pieces p = pieces_of(sums.before + ((long)h * col_tiles + j) * s.w.tiles, s.w.tiles, line_quota(a.line, sums.total));
  if (p.first == p.last) return;
  join_columns<T, D>((int)(p.last - p.first) + 1, [&](int i) { return slot_of(p, p.first + i); }, a.o, a.ml, M, col, min(pairs - first, M), [&](int c) {
    const int pair = first + c;
    return a.out.data + (long)(s.row0 + pair / a.group) * a.out.token_stride + (long)(h * a.group + pair % a.group) * a.out.head_stride;
  });
}

// Columns of a workgroup: the fewest of 32, 64 and 128 that hold a kv head's (row, query head) pairs, since every tile of columns reads the codes
// again: 64 columns over 16 x 32768 tokens 204 us, 337 as twice 32 and 309 in a half empty 128; 30 to 64 over 4 x 8 to 16 thousand 131, 189, 196;
// 104 over 8 x 2 to 4 thousand 27 in 128, 32 as twice 64.
struct TreePlan {
  int cb;
  long items, workgroups;
};
constexpr int kTreeGroups = 512;   // workgroups: two a compute unit

static bool tree_plan(const dq_paged_cache* c, int batch, long rows, int q_heads, int max_rows, int max_seq_len, TreePlan* p) {
  if (batch <= 0 || rows < 0 || q_heads <= 0 || q_heads % c->kv_heads || max_rows < 0 || max_rows > kTreeRows || max_seq_len < 0) return false;
  const long group = q_heads / c->kv_heads, cols = max_rows * group;
  if (rows * group >= (1l << 31) - 256) return false;
  p->cb = cols <= 32 ? 1 : cols <= 64 ? 2 : 4;
  p->items = rows * group / (32 * p->cb) + batch;
  if (p->items * c->kv_heads * 32 * p->cb >= kMaxThreads / 256) return false;
  p->workgroups = kTreeGroups;
  return true;
}
static size_t tree_bytes(long workgroups, int cb, int head_dim) { return (size_t)(2 * workgroups * 32 * cb) * (head_dim + 2) * sizeof(float); }

template <typename T, int D, int CB>
static void launch_tree(const TreeArgs& a, const TreePlan& p, hipStream_t st) {
  const dim3 grid((unsigned)p.workgroups);
  if (a.c.codes == DQ_CODES_E4M3) hipLaunchKernelGGL((tree_attn_kernel<T, D, true, CB>), grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((tree_attn_kernel<T, D, false, CB>), grid, dim3(256), 0, st, a);
  hipLaunchKernelGGL((tree_join_kernel<T, D, CB>), dim3((unsigned)(p.items * a.c.kv_heads * (32 * CB / kJoinColumns<D>))), dim3(256), 0, st, a);
}
template <typename T, int D>
static void launch_tree_cols(const TreeArgs& a, const TreePlan& p, hipStream_t st) {
  if (p.cb == 1) launch_tree<T, D, 1>(a, p, st);
  else if (p.cb == 2) launch_tree<T, D, 2>(a, p, st);
  else launch_tree<T, D, 4>(a, p, st);
}

}  // namespace dq

using namespace dq;

extern "C" size_t dq_paged_tree_workspace_bytes(const dq_paged_cache* cache, int32_t batch, int32_t rows, int32_t q_heads, int32_t max_rows,
                                                int32_t max_seq_len) {
  TreePlan p;
  if (!paged_cache_ok(cache) || !tree_plan(cache, batch, rows, q_heads, max_rows, max_seq_len, &p)) return 0;
  return tree_bytes(kTreeGroups, p.cb, cache->head_dim);  // (smaller calls have fewer columns)
}

extern "C" int32_t dq_paged_tree_attention(const dq_paged_cache* cache, const dq_paged_batch* batch, const dq_heads* q, const dq_heads* k,
                                           const dq_heads* v, const dq_heads* out, const uint64_t* seen, int32_t max_rows, int32_t max_seq_len,
                                           float softmax_scale, int32_t window, void* workspace, size_t workspace_bytes, uint32_t flags,
                                           void* hip_stream) {
  if (!paged_cache_ok(cache) || !paged_batch_ok(batch, cache, true)) return DQ_EINVAL;
  if (!heads_ok(q, false) || !heads_ok(k, false) || !heads_ok(v, false) || !heads_ok(out, false)) return DQ_EINVAL;
  if (q->heads != out->heads || k->heads != cache->kv_heads || v->heads != cache->kv_heads) return DQ_EINVAL;
  if (!seen || ((uintptr_t)seen & 7) || !workspace || ((uintptr_t)workspace & 15) || flags || !scale_ok(softmax_scale)) return DQ_EINVAL;
  if (window != 0 && window < kTreeRows) return DQ_EINVAL;
  TreePlan p;
  if (!tree_plan(cache, batch->batch, batch->rows, q->heads, max_rows, max_seq_len, &p)) return DQ_EINVAL;
  if (workspace_bytes < tree_bytes(p.workgroups, p.cb, cache->head_dim)) return DQ_ENOSPACE;
  if (batch->rows == 0 || max_rows == 0) return DQ_OK;
  // every column tile of a kv head reads its drafted rows, and one that is done writes
  if (heads_meet(k, batch->rows, cache->head_dim, out, batch->rows, cache->head_dim) || heads_meet(v, batch->rows, cache->head_dim, out, batch->rows, cache->head_dim) ||
      !heads_in_place(q, out, batch->rows, cache->head_dim))
    return DQ_EINVAL;
  TreeArgs a = {};
  a.c = *cache; a.bt = *batch; a.q = *q; a.k = *k; a.v = *v; a.out = *out;
  a.seen = seen;
  a.group = q->heads / cache->kv_heads;
  a.max_rows = max_rows;
  a.window = window;
  a.scale_log2 = (softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)cache->head_dim)) * 1.44269504088896340736f;
  a.line = {(int)p.workgroups, 1};
  a.o = reinterpret_cast<float*>(workspace);
  a.ml = a.o + 2 * p.workgroups * 32 * p.cb * cache->head_dim;
  hipStream_t st = (hipStream_t)hip_stream;
  if (cache->dtype == DQ_BF16) { if (cache->head_dim == 128) launch_tree_cols<__bf16, 128>(a, p, st); else launch_tree_cols<__bf16, 64>(a, p, st); }
  else { if (cache->head_dim == 128) launch_tree_cols<_Float16, 128>(a, p, st); else launch_tree_cols<_Float16, 64>(a, p, st); }
  DQ_HIP_CHECK(hipGetLastError());
  return DQ_OK;
}
