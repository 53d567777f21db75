// Attention of many query rows per sequence (prompts, pieces of prompts) over the paged 8-bit cache, and the entry points
// of both attention kernels.
#include "dq_paged_attn.h"

namespace dq {

constexpr int kPromptWaves = 4;
constexpr int kPromptSplits = 32;   // at most, of a tile of rows (their weights fit LDS)

// Rows of a transposed 32-token score product stand for tokens with bits 2 and 3 of their place exchanged: a lane's 16 scores are
// then tokens 8 h .. 8 h + 7 and 16 + 8 h .. of the 32 (h = lane / 32), the right operand that the product with the values wants.
// One workgroup of four waves per (tile of rows, kv head, split): 32 (row, query head) pairs a wave.  The tile's
// codes are turned to f16 once and shared through LDS (two buffers of 64 tokens); keys as [token][channel], values as
// [channel][token], as they are stored.
// Scores are formed transposed, as in the decode kernel: probabilities go from the first product's result registers to
// the second's operand registers without leaving the lane.
//
// Bound by the matrix instructions and what shares their waves: 4 x 32 query heads, prompts of 3500 to 4096 tokens of 128 channels,
// 485 GFLOP within the mask, 515 us, 940 TFLOP/s, against 1100 of a large f16 matrix product (1200 to 1350 of nothing but matrix
// instructions with as many vector instructions as here between them, in registers); matrix units are busy 44 % of the cycles, LDS 40 %.
// Two pieces of 400 to 512 rows behind 15 thousand tokens, 246 GFLOP, 255 us.  64 rows a wave (one workgroup a compute unit) took
// 693 us for 526, three workgroups a compute unit with one buffer spilled (660), codes stored to LDS after the second product 535;
// scores a tile ahead, between the exponentials of the tile before, made prompts no faster (515) and pieces slower (275).
template <typename T, int D, bool FP8>
__global__ __launch_bounds__(64 * kPromptWaves, 2) void paged_prompt_kernel(PagedAttnArgs a) {
  constexpr int NK = D / 16, NCT = D / 32, NB = D / 64, M = 32 * kPromptWaves;
  constexpr int THREADS = 64 * kPromptWaves;
  constexpr int KP = D / 8 + 1, VP = 9;                   // 16-byte pieces of a key row and of a channel's run in LDS
  typedef typename Vec8<T>::type tx8;
  __shared__ __align__(16) u32x4 s_k[2][64 * KP], s_v[2][D * VP];
  __shared__ int s_last;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r32 = lane & 31, hl = lane >> 5;
  const int H = a.c.kv_heads, P = a.c.page_tokens;
  const int h = (int)(blockIdx.x % H), split = (int)(blockIdx.x / H) % a.splits, item = (int)(blockIdx.x / H) / a.splits;
  const int b = a.seq_tiles ? item / a.seq_tiles : item_owner(a.bt.starts, a.bt.rows, a.bt.batch, item, a.group, M, 1);
  const Sequence s = sequence_of_wave(a.bt, P, b);
  const int n = a.seq_tiles ? min(s.n, a.max_rows) : s.n, len = s.len, before = s.old;
  const int row_tiles = (int)(((long)n * a.group + M - 1) / M);
  const int j = a.seq_tiles ? item % a.seq_tiles : item - item_first(a.bt.starts, a.bt.rows, b, a.group, M, 1);
  if (j < 0 || j >= row_tiles) return;
  const int row_tile = row_tiles - 1 - j;                 // the longest first
  const int pairs = n * a.group, first = row_tile * M;
  const int rows_lo = first / a.group, rows_hi = min(first + M - 1, pairs - 1) / a.group;
  // tokens that any / every row of the tile sees
  const int any_hi = a.causal ? min(max(before + rows_hi + 1, 0), len) : len;
  const int any_lo = window_start(before + rows_lo, a.window);
  const int all_hi = a.causal ? before + rows_lo + 1 : len, all_lo = window_start(before + rows_hi, a.window);
  const int runs = P / kPagedTile, code_tiles = len / P * runs;
  int t_first = any_lo / kPagedTile, t_last = (any_hi + kPagedTile - 1) / kPagedTile;
  if (t_last < t_first) t_last = t_first;
  {
    const int share = (t_last - t_first + a.splits - 1) / a.splits;
    t_first = min(t_first + split * share, t_last);
    t_last = min(t_first + share, t_last);
  }

  // ---- queries ----
  const int my_pair = min(first + wave * 32 + r32, pairs - 1), my_row = my_pair / a.group, place = before + my_row;
  const int see_hi = a.causal ? min(place + 1, len) : len, see_lo = window_start(place, a.window);
  const uint16_t* const q_row =
      a.q.data + (long)(s.row0 + my_row) * a.q.token_stride + (long)(h * a.group + my_pair % a.group) * a.q.head_stride + 8 * hl;
  float sc = a.scale_log2;
  f16x8 q[NK];
  {
    float amax = 0.f;
    u32x4 w[NK];
#pragma unroll
    for (int k = 0; k < NK; ++k) {
      w[k] = *reinterpret_cast<const u32x4*>(q_row + 16 * k);
      if constexpr (__is_same(T, __bf16)) {
        float x[8];
        unpack8<T>(w[k], x);
#pragma unroll
        for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(x[e]));
      }
    }
    int shift = 0;
    if constexpr (__is_same(T, __bf16)) {
      amax = fmaxf(amax, __shfl_xor(amax, 32));
      shift = fit_shift(amax);
      sc = __builtin_ldexpf(sc, -shift);
    }
#pragma unroll
    for (int k = 0; k < NK; ++k) {
      if constexpr (__is_same(T, __bf16)) {
        float x[8];
        unpack8<T>(w[k], x);
#pragma unroll
        for (int e = 0; e < 8; ++e) q[k][e] = (_Float16)__builtin_ldexpf(x[e], shift);
      } else {
        q[k] = __builtin_bit_cast(f16x8, w[k]);
      }
    }
  }
  float m = -INFINITY, l = 0.f;
  f32x16 o[NCT];
#pragma unroll
  for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[ct][e] = 0.f;

  // Places of 16-byte pieces in LDS: rows an odd number of pieces apart, so that neighbouring lanes, which read the same piece of
  // neighbouring rows, touch all banks, and what a lane reads lies at fixed offsets from one address.  Keys lie in the order of the
  // score product's rows (above).
  auto k_at = [&](int token, int piece) { return ((token & ~12) | (token & 4) << 1 | (token & 8) >> 1) * KP + piece; };
  auto v_at = [&](int ch, int piece) { return ch * VP + piece; };

  // ---- a tile of 64 tokens ----
  // Codes of the tile after it, on their way from memory to LDS; slice k of NK is turned to f16 between the matrix
  // instructions of the scores, which leave the vector unit idle.
  u32x4 kc[NB], vc[NB];
  auto store_slice = [&](int buf, int k) __attribute__((always_inline)) {
    const int i = k / 4, half = k & 1, piece = i * THREADS + tid;   // 16 codes: two pieces of keys, two of values
    if ((k & 2) == 0) {
      const int token = piece / (D / 16), kp = 2 * (piece % (D / 16)) + half;
      s_k[buf][k_at(token, kp)] = __builtin_bit_cast(u32x4, half ? codes_f16<FP8>(kc[i].z, kc[i].w) : codes_f16<FP8>(kc[i].x, kc[i].y));
    } else {
      s_v[buf][v_at(piece / 4, 2 * (piece % 4) + half)] = __builtin_bit_cast(u32x4, half ? codes_f16<FP8>(vc[i].z, vc[i].w) : codes_f16<FP8>(vc[i].x, vc[i].y));
    }
  };

  // Tile in buffer `buf`, elements of the type of `zero` (f16 of codes, or the rows' own type); `slice(k)` is done after the
  // k-th pair of score products.  p = 2^(s f + add - m); lane: tokens 32 tt + 16 (e / 8) + 8 hl + e % 8.
  auto work_tile = [&](int buf, int tile, auto zero, const auto& qf, float f, float add, float inv_sv, auto mask, auto slice) __attribute__((always_inline)) {
    typedef decltype(zero) ex8;
    const u32x4* const k_from = s_k[buf] + r32 * KP + hl;   // row r32 of the first 32
    const u32x4* const v_from = s_v[buf] + r32 * VP + hl;
    f32x16 u[2];
#pragma unroll
    for (int e = 0; e < 32; ++e) u[e >> 4][e & 15] = 0.f;
    __builtin_amdgcn_s_setprio(1);   // matrix instructions go ahead of the other workgroup's softmax: 507 us, 526 without
#pragma unroll
    for (int k = 0; k < NK; ++k) {
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
        const ex8 kf = __builtin_bit_cast(ex8, k_from[32 * tt * KP + 2 * k]);
        u[tt] = mma32(kf, qf[k], u[tt]);
      }
      slice(k);
    }
    __builtin_amdgcn_s_setprio(0);
    if constexpr (decltype(mask)::value) {
      const float poison = f - f;                         // NaN where the block is: for those who see it, not through a masked -inf
      f = f == f ? f : 1.f;
#pragma unroll
      for (int e = 0; e < 32; ++e) {
        const int t = tile * kPagedTile + 32 * (e >> 4) + 16 * (e >> 3 & 1) + 8 * hl + (e & 7);
        u[e >> 4][e & 15] = t < see_lo || t >= see_hi ? -INFINITY : u[e >> 4][e & 15] + poison;
      }
    }
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
      for (int ct = 0; ct < NCT; ++ct) o[ct] *= alpha;
    }
    const float base = m == -INFINITY ? add : add - m;
    float sum = 0.f;
    // Probabilities of 16 tokens (8 a lane) are made between the products of the 16 before them; in the products' type (f16 over
    // codes, the rows' own over the tail), the sum in fp32.
    ex8 p, p_next;
    auto probabilities = [&](int g, ex8& to) __attribute__((always_inline)) {
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(u[g >> 1][8 * (g & 1) + e], f, base));
        to[e] = to_element<ex8>(x[e]);
      }
      sum += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
    };
    probabilities(0, p);
    __builtin_amdgcn_s_setprio(1);   // matrix instructions go ahead of the other workgroup's softmax: 507 us, 526 without
#pragma unroll
    for (int g = 0; g < 4; ++g) {
#pragma unroll
      for (int ct = 0; ct < NCT; ++ct) {
        const ex8 vf = __builtin_bit_cast(ex8, v_from[32 * ct * VP + 2 * g]);
        o[ct] = mma32(vf, p, o[ct]);
      }
      if (g < 3) {
        probabilities(g + 1, p_next);
        p = p_next;
      }
    }
    l = __builtin_fmaf(sum, inv_sv, l);
    __builtin_amdgcn_s_setprio(0);
  };

  // `total` tiles of full pages, the i-th of them tile_of(i).
  auto run = [&](int total, auto tile_of, auto mask) __attribute__((always_inline)) {
    for (int batch0 = 0; batch0 < total; batch0 += 64) {
      int blk = 0;
      bool held = false;
      uint64_t values = 0;                                // where the tile's codes are (the choice cost prompts 1 % in load_tile)
      float sk = 0.f, lsv = 0.f, isv = 0.f;
      if (batch0 + lane < total) {
        const int t = tile_of(batch0 + lane), page = a.bt.page_table[(long)b * a.bt.table_stride + t / runs];
        const bool ok = page >= 0 && page < a.c.pages;
        const long block = (long)(ok ? page : 0) * H + h;
        blk = (int)(block * runs) + t % runs;
        values = (uint64_t)(ok ? a.c.v_codes + (long)blk * (kPagedTile * D) : reinterpret_cast<const uint8_t*>(g_no_codes));
        sk = ok ? a.c.k_scales[block] : __builtin_nanf("");
        const float sv = ok ? a.c.v_scales[block] : 1.f;
        lsv = __builtin_amdgcn_logf(sv);
        isv = 1.f / sv;
        held = ok;
      }
      place_zero_blocks<D, FP8>(a.c.v_codes, blk, held, lsv, isv);
      const int count = min(64, total - batch0);
      auto load_tile = [&](int i) __attribute__((always_inline)) {   // (behind the last one: that one again, never used)
        const int j = min(i, count - 1);
        const GlobalBytes ks = (GlobalBytes)a.c.k_codes + (long)__builtin_amdgcn_readlane(blk, j) * (kPagedTile * D);
        const GlobalBytes vs = (GlobalBytes)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(values >> 32), j) << 32 |
                                             (uint32_t)__builtin_amdgcn_readlane((int)values, j));
#pragma unroll
        for (int k = 0; k < NB; ++k) {
          kc[k] = *(GlobalPieces)(ks + 16l * (k * THREADS + tid));
          vc[k] = *(GlobalPieces)(vs + 16l * (k * THREADS + tid));
        }
      };
      load_tile(0);
      __syncthreads();                                    // buffer 0 has been read
#pragma unroll
      for (int k = 0; k < NK; ++k) store_slice(0, k);
      load_tile(1);
      __syncthreads();
      for (int i = 0; i < count; ++i) {
        const float f = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, sk), i));
        const float add = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, lsv), i));
        const float inv_sv = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, isv), i));
        work_tile(i & 1, tile_of(batch0 + i), f16x8{}, q, keep_sign(f * sc), add, inv_sv, mask,
                  [&](int k) __attribute__((always_inline)) {
                    store_slice((i + 1) & 1, k);
                    if (k == NK - 1) load_tile(i + 2);
                  });
        __syncthreads();
      }
    }
  };
  // Tiles that every row sees whole, then those that need the mask (two loops: with both kinds in one, registers run out).
  const int code_end = min(t_last, code_tiles);
  const int whole_lo = min(max(t_first, (all_lo + kPagedTile - 1) / kPagedTile), max(code_end, t_first));
  const int whole_hi = max(min(code_end, max(all_hi, 0) / kPagedTile), whole_lo);
  run(whole_hi - whole_lo, [&](int i) { return whole_lo + i; }, Whole{});
  const int ahead = whole_lo - t_first;
  run(ahead + max(code_end - whole_hi, 0), [&](int i) { return i < ahead ? t_first + i : whole_hi + i - ahead; }, Masked{});

  // ---- the page being filled: 16-bit rows ----
  for (int tile = max(t_first, code_tiles); tile < t_last; ++tile) {
    const int slot = a.bt.tail_slots ? a.bt.tail_slots[b] : b;
    const bool ok = slot >= 0 && slot < a.c.slots;
    const int left = ok ? len - tile * kPagedTile : 0;
    const long at = (((long)(ok ? slot : 0) * H + h) * runs + (tile - code_tiles)) * kPagedTile * D;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2 * NB; ++i) {
      const int piece = i * THREADS + tid;                // 8 values
      const u32x4 kw = *reinterpret_cast<const u32x4*>(a.c.k_tail + at + 8l * piece);
      u32x4 vw = *reinterpret_cast<const u32x4*>(a.c.v_tail + at + 8l * piece);
      const int t = 8 * (piece % 8);
#pragma unroll
      for (int e = 0; e < 4; ++e) vw[e] = keep_tokens(vw[e], left - t - 2 * e);
      s_k[0][k_at(piece / (D / 8), piece % (D / 8))] = kw;
      s_v[0][v_at(piece / 8, piece % 8)] = vw;
    }
    __syncthreads();
    tx8 qt[NK];
#pragma unroll
    for (int k = 0; k < NK; ++k) qt[k] = __builtin_bit_cast(tx8, *reinterpret_cast<const u32x4*>(q_row + 16 * k));
    const float f = ok ? keep_sign(a.scale_log2) : __builtin_nanf("");
    work_tile(0, tile, tx8{}, qt, f, 0.f, 1.f, Masked{}, [](int) {});
  }

  // ---- outputs, or partials for the workgroup that joins the splits ----
  auto out_of = [&](int col) {
    const int pair = first + col;
    return a.out.data + (long)(s.row0 + pair / a.group) * a.out.token_stride + (long)(h * a.group + pair % a.group) * a.out.head_stride;
  };
  const int unit = item * H + h;
  l += __shfl_xor(l, 32);
  if (const int col = wave * 32 + r32; first + col >= pairs) {
    // a row of another tile, or none
  } else if (a.splits == 1) {
    const float inv = l == 0.f ? 0.f : 1.f / l;
    uint16_t* const dst = out_of(col);
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        *reinterpret_cast<u32x2*>(dst + 32 * ct + 8 * e + 4 * hl) = u32x2{pack2<T>(o[ct][4 * e] * inv, o[ct][4 * e + 1] * inv),
                                                                         pack2<T>(o[ct][4 * e + 2] * inv, o[ct][4 * e + 3] * inv)};
  } else {
    float* const p = a.partials + ((long)unit * a.splits + split) * (D + 2) * M + col;   // channel by channel: rows lie side by side
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
      for (int e = 0; e < 16; ++e)
        __hip_atomic_store(p + (32 * ct + 8 * (e >> 2) + 4 * hl + (e & 3)) * M, o[ct][e], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (hl == 0) {
      __hip_atomic_store(p + D * M, m, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      __hip_atomic_store(p + (D + 1) * M, l, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
  }
  if (a.splits == 1 || !last_of_splits(a.counters + unit, a.splits, s_last)) return;
  // The splits' results: a thread takes a row and every (THREADS / M)-th run of eight channels of it.
  static_assert(M <= THREADS && THREADS % M == 0 && sizeof(s_k) >= kPromptSplits * M * sizeof(float), "rows a thread, weights in LDS");
  float* const weight = reinterpret_cast<float*>(s_k);    // [split][row]
  const int col = tid % M, ns = a.splits;
  const float* const part = a.partials + (long)unit * ns * (D + 2) * M + col;
  auto load = [](const float* p) __attribute__((always_inline)) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
  float top = -INFINITY, sum = 0.f;
  if (tid < M) {
    for (int i = 0; i < ns; ++i) {
      const float x = load(part + ((long)i * (D + 2) + D) * M);
      weight[i * M + col] = x;
      top = fmaxf(top, x);
    }
    const float at = top == -INFINITY ? 0.f : top;
    for (int i = 0; i < ns; ++i) {
      const float w = __builtin_amdgcn_exp2f(weight[i * M + col] - at);
      weight[i * M + col] = w;
      sum = __builtin_fmaf(load(part + ((long)i * (D + 2) + D + 1) * M), w, sum);
    }
    reinterpret_cast<float*>(s_v)[col] = sum == 0.f ? 0.f : 1.f / sum;
  }
  __syncthreads();
  if (first + col >= pairs) return;
  const float inv = reinterpret_cast<float*>(s_v)[col];
  for (int c = 8 * (tid / M); c < D; c += 8 * (THREADS / M)) {
    float x[8] = {};
    for (int i = 0; i < ns; ++i) {
      const float w = weight[i * M + col];
      float y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = load(part + ((long)i * (D + 2) + c + e) * M);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = __builtin_fmaf(y[e], w, x[e]);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] *= inv;
    *reinterpret_cast<u32x4*>(out_of(col) + c) = pack8<T>(x);
  }
}

constexpr int kPromptRows = 32 * kPromptWaves;

template <typename T, int D>
static void launch_prompt(const PagedAttnArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)((long)a.units * a.splits)), block(64 * kPromptWaves);
  if (a.c.codes == DQ_CODES_E4M3) hipLaunchKernelGGL((paged_prompt_kernel<T, D, true>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((paged_prompt_kernel<T, D, false>), grid, block, 0, st, a);
}

int32_t launch_paged_prompt(const PagedAttnArgs& a, hipStream_t st) {
  if (a.c.dtype == DQ_BF16) { if (a.c.head_dim == 128) launch_prompt<__bf16, 128>(a, st); else launch_prompt<__bf16, 64>(a, st); }
  else { if (a.c.head_dim == 128) launch_prompt<_Float16, 128>(a, st); else launch_prompt<_Float16, 64>(a, st); }
  DQ_HIP_CHECK(hipGetLastError());
  return DQ_OK;
}

// ---- launch shape ----
struct PagedShape {
  bool decode;
  long units;
  int seq_tiles;           // prompt: PagedAttnArgs::seq_tiles
  int splits, cols;        // splits: of every unit (prompt), of a sequence of the longest length if all were (decode)
  long shares, groups;     // decode: PagedAttnArgs::shares; workgroups that may hand over partial results (0: none)
};

constexpr int kPagedCounters = 4096;      // units that may be split, with a ticket each at a fixed place: calls of all sizes may share a workspace
constexpr int kMostSplitGroups = 1024;    // workgroups of a launch whose splits the library chose (below); tiles of rows: half of them may be empty

// Splits of a unit: as many as give `wanted` workgroups, or the next count that leaves few of them idle in the last round, at most
// cap.  The smallest n within 4 % of the fullest rounds (so that a larger cap never means fewer splits).
static int pick_splits(long units, int cap, int wanted) {
  auto fill = [&](int n) { const long w = units * n; return (float)w / (float)(w <= wanted ? wanted : (w + wanted - 1) / wanted * wanted); };
  float best = 0.f;
  for (int n = 1; n <= cap && (n == 1 || units * n <= 2 * wanted); ++n) best = fmaxf(best, fill(n));
  int n = 1;
  while (fill(n) < 0.96f * best) ++n;
  return n;
}

// Decode kernel: a workgroup per compute unit, two where 128 units or more of 64 channels (half the bytes on a wave's way) would
// leave them with long shares.  Measured over 1 to 1024 units of 2 to 2000 tiles, 13 split counts each: the picks are 1.4 % behind the
// best on average; 128 units of 512 tiles of 128 channels 160 us in two splits, 165 in 6; 128 of 47 tiles of 64 channels 11.6 us in 4, 14.5 in 2.
static int decode_splits(long units, int tiles, int head_dim, int cols) {
  return pick_splits(units, decode_cap(tiles, head_dim, cols), head_dim == 64 && units >= 128 ? 512 : 256);
}

// Prompt kernel: two workgroups a compute unit; a split hands over 66 KB, so at most 0.75 sqrt(tiles).  8 units of 500 tiles 71 us in 16
// splits, 521 in one, 85 in 32; 64 of 300 tiles 102 us in 8, 174 in 2, 128 in 12.
static int prompt_cap(int tiles) {
  const int cap = (int)(0.75f * sqrtf((float)tiles));
  return cap < 1 ? 1 : cap < kPromptSplits ? cap : kPromptSplits;
}

// What the entry points agree on: kernel, units and splits from the host's bounds.
static bool paged_shape(const dq_paged_cache* c, int batch, long rows, int q_heads, int max_rows, int max_seq_len, int window, uint32_t flags,
                        PagedShape* s) {
  if (batch <= 0 || rows < 0 || q_heads <= 0 || q_heads % c->kv_heads || max_rows < 0 || max_seq_len < 0) return false;
  const int group = q_heads / c->kv_heads;
  int tiles = max_seq_len / kPagedTile + 1;
  if (window > 0 && ((long)window + max_rows) / kPagedTile + 2 < tiles) tiles = (int)(((long)window + max_rows) / kPagedTile + 2);
  s->decode = (long)max_rows * group <= 16;
  const long most = (long)batch * max_rows;
  if ((most < rows ? most : rows) * group >= (1l << 31)) return false;
  // Tiles of rows: dealt by starts there are `rows` rows of them and one a sequence that may stay empty.  Where the bound on rows gives
  // every sequence tiles of its own with no more in all (one sequence, equal ones, rows behind the last sequence's), it does: a sequence
  // with more rows than the bound then takes nothing from the others.
  const long seq_tiles = ((long)max_rows * group + kPromptRows - 1) / kPromptRows, dealt = rows * group / kPromptRows + batch;
  s->seq_tiles = !s->decode && seq_tiles <= dealt / batch ? (int)seq_tiles : 0;
  const long items = s->decode ? batch : s->seq_tiles ? batch * seq_tiles : dealt;
  if (items >= (1l << 24)) return false;
  s->units = items * c->kv_heads;
  s->cols = s->decode ? 16 : kPromptRows;
  if (s->units >= (1l << 24)) return false;
  s->splits = s->decode ? decode_splits(s->units, tiles, c->head_dim, max_rows * group) : pick_splits(s->units, prompt_cap(tiles), 512);
  if (const int v = (int)(flags >> 8 & 0x7Fu)) s->splits = !s->decode && v > kPromptSplits ? kPromptSplits : v;   // the caller's override
  if (s->units > kPagedCounters) s->splits = 1;
  s->shares = 0;
  s->groups = s->splits == 1 ? 0 : s->units * s->splits;
  if (s->decode) {
    // also where every sequence gets one slot on average, long ones are split if their lengths differ
    const bool some = s->splits > 1 || ((flags >> 8 & 0x7Fu) == 0 && batch > 1 && batch <= 64 && s->units <= kMostSplitGroups && decode_cap(tiles, c->head_dim, max_rows * group) > 1);
    if (some) s->shares = (long)s->splits * batch;
    s->groups = some ? (s->shares + (batch <= 64 ? batch : 0)) * c->kv_heads : 0;
  }
  return true;
}

static size_t paged_bytes(long groups, int cols, int head_dim) {
  return (size_t)kWsHeaderBytes + kPagedCounters * sizeof(int32_t) + (size_t)groups * cols * (head_dim + 2) * sizeof(float);
}

}  // namespace dq

using namespace dq;

extern "C" size_t dq_paged_workspace_bytes(const dq_paged_cache* cache, int32_t batch, int32_t rows, int32_t q_heads, int32_t max_rows,
                                           int32_t max_seq_len) {
  PagedShape s;
  if (!paged_cache_ok(cache) || !paged_shape(cache, batch, rows, q_heads, max_rows, max_seq_len, 0, 0, &s)) return 0;
  // smaller calls have fewer units and may have more splits: their product is what is bounded
  const int tiles = max_seq_len / kPagedTile + 1;
  const long decode_units = (long)batch * cache->kv_heads;
  auto most = [](long units, int splits, long groups) { const long n = units * splits; return splits == 1 ? 0l : n < groups ? n : groups; };
  const int cap = decode_cap(tiles, cache->head_dim, 1) == 1 ? 1 : kMaxSplits + 1;
  size_t bytes = paged_bytes(most(decode_units, cap, 2 * kMostSplitGroups), 16, cache->head_dim);
  if (!s.decode) {
    const size_t p = paged_bytes(most(s.units, prompt_cap(tiles), 2 * kMostSplitGroups), kPromptRows, cache->head_dim);
    if (p > bytes) bytes = p;
  }
  return bytes;
}

extern "C" int32_t dq_paged_attention(const dq_paged_cache* cache, const dq_paged_batch* batch, const dq_heads* q, const dq_heads* out,
                                      int32_t max_rows, int32_t max_seq_len, float softmax_scale, int32_t window, void* workspace,
                                      size_t workspace_bytes, uint32_t flags, void* hip_stream) {
  if (!paged_cache_ok(cache) || !paged_batch_ok(batch, cache, true) || !heads_ok(q, false) || !heads_ok(out, false)) return DQ_EINVAL;
  if (q->heads != out->heads || q->heads % cache->kv_heads || !workspace || ((uintptr_t)workspace & 15)) return DQ_EINVAL;
  if ((flags & ~(DQ_PAGED_CAUSAL | DQ_PAGED_SPLITS(0x7F))) || (flags >> 8 & 0x7Fu) > (uint32_t)kMaxSplits || window < 0 || (window && !(flags & DQ_PAGED_CAUSAL)))
    return DQ_EINVAL;
  if (softmax_scale != softmax_scale) return DQ_EINVAL;
  PagedShape s;
  if (!paged_shape(cache, batch->batch, batch->rows, q->heads, max_rows, max_seq_len, window, flags, &s)) return DQ_EINVAL;
  if (workspace_bytes < paged_bytes(s.groups, s.cols, cache->head_dim)) return DQ_ENOSPACE;
  if (batch->rows == 0 || max_rows == 0) return DQ_OK;
  PagedAttnArgs a = {};
  a.c = *cache; a.bt = *batch; a.q = *q; a.out = *out;
  a.group = q->heads / cache->kv_heads;
  a.max_rows = max_rows;
  a.window = window;
  a.causal = (flags & DQ_PAGED_CAUSAL) ? 1 : 0;
  a.scale_log2 = (softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)cache->head_dim)) * 1.44269504088896340736f;
  a.splits = s.splits;
  a.seq_tiles = s.seq_tiles;
  a.shares = (int)s.shares;
  a.units = (int)s.units;
  char* ws = reinterpret_cast<char*>(workspace);
  a.counters = reinterpret_cast<int32_t*>(ws + kWsHeaderBytes);
  a.partials = reinterpret_cast<float*>(ws + kWsHeaderBytes + kPagedCounters * sizeof(int32_t));
  hipStream_t st = (hipStream_t)hip_stream;
  return s.decode ? launch_paged_decode(a, st) : launch_paged_prompt(a, st);
}
