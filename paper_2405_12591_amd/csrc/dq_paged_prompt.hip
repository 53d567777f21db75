// Attention of many query rows per sequence (prompts, pieces of prompts) over the paged 8-bit cache, and the entry points
// of both attention kernels.
#include "dq_paged_attn.h"

namespace dq {

constexpr int kPromptWaves = 4;

// Token of row r of a transposed 32-token score product: chosen so that a lane's 16 scores are tokens 8 h .. 8 h + 7 and
// 16 + 8 h .. of the 32 (h = lane / 32), the right operand that the product with the values wants.
__device__ __forceinline__ int score_token(int r) { return 16 * (r >> 4) + 8 * ((r >> 2) & 1) + 4 * ((r >> 3) & 1) + (r & 3); }

// One workgroup of four waves per (tile of rows, kv head, split): RB * 32 (row, query head) pairs a wave.  The tile's
// codes are turned to f16 once and shared through LDS (two buffers of 64 tokens, pieces of 16 bytes swizzled so that 16
// neighbouring lanes touch all banks); keys as [token][channel], values as [channel][token], as they are stored.
// Scores are formed transposed, as in the decode kernel: probabilities go from the first product's result registers to
// the second's operand registers without leaving the lane.
template <typename T, int D, bool FP8, int RB>
__global__ __launch_bounds__(64 * kPromptWaves, RB == 1 ? 2 : 1) void paged_prompt_kernel(PagedAttnArgs a) {
  constexpr int NK = D / 16, NCT = D / 32, NB = D / 64, M = 32 * RB * kPromptWaves;
  constexpr int THREADS = 64 * kPromptWaves;
  typedef typename Vec8<T>::type tx8;
  __shared__ __align__(16) u32x4 s_k[2][64 * D / 8], s_v[2][64 * D / 8];
  __shared__ int s_last;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r32 = lane & 31, hl = lane >> 5;
  const int H = a.c.kv_heads, P = a.c.page_tokens;
  const int h = (int)(blockIdx.x % H), split = (int)(blockIdx.x / H) % a.splits, item = (int)(blockIdx.x / H) / a.splits;
  const int b = item_owner(a.bt.starts, a.bt.rows, a.bt.batch, item, a.group, M, 1);
  Sequence s = sequence_of(a.bt, P, b);
  s.len = min(s.len, a.max_seq_len);
  const int n = s.n, len = s.len;
  const int row_tiles = (int)(((long)n * a.group + M - 1) / M);
  const int j = item - item_first(a.bt.starts, a.bt.rows, b, a.group, M, 1);
  if (j < 0 || j >= row_tiles) return;
  const int row_tile = row_tiles - 1 - j;                 // the longest first
  const int pairs = n * a.group, first = row_tile * M;
  const int rows_lo = first / a.group, rows_hi = min(first + M - 1, pairs - 1) / a.group;
  // tokens that any / every row of the tile sees
  const int any_hi = a.causal ? min(max(len - n + rows_hi + 1, 0), len) : len;
  const int any_lo = a.window ? max(len - n + rows_lo + 1 - a.window, 0) : 0;
  const int all_hi = a.causal ? len - n + rows_lo + 1 : len, all_lo = a.window ? len - n + rows_hi + 1 - a.window : 0;
  const int runs = P / kPagedTile, code_tiles = len / P * runs;
  int t_first = any_lo / kPagedTile, t_last = (any_hi + kPagedTile - 1) / kPagedTile;
  if (t_last < t_first) t_last = t_first;
  {
    const int share = (t_last - t_first + a.splits - 1) / a.splits;
    t_first = min(t_first + split * share, t_last);
    t_last = min(t_first + share, t_last);
  }

  // ---- queries ----
  int see_lo[RB], see_hi[RB];
  float sc[RB], m[RB], l[RB];
  f16x8 q[RB][NK];
  f32x16 o[RB][NCT];
  const uint16_t* q_row[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int pair = min(first + (wave * RB + rb) * 32 + r32, pairs - 1);
    const int i = pair / a.group, place = len - n + i;
    see_hi[rb] = a.causal ? min(place + 1, len) : len;
    see_lo[rb] = a.window ? place + 1 - a.window : 0;
    q_row[rb] = a.q.data + (long)(s.row0 + i) * a.q.token_stride + (long)(h * a.group + pair % a.group) * a.q.head_stride + 8 * hl;
    float amax = 0.f;
    u32x4 w[NK];
#pragma unroll
    for (int k = 0; k < NK; ++k) {
      w[k] = *reinterpret_cast<const u32x4*>(q_row[rb] + 16 * k);
      if constexpr (__is_same(T, __bf16)) {
        float x[8];
        unpack8<T>(w[k], x);
#pragma unroll
        for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(x[e]));
      }
    }
    sc[rb] = a.scale_log2;
    int shift = 0;
    if constexpr (__is_same(T, __bf16)) {
      amax = fmaxf(amax, __shfl_xor(amax, 32));
      shift = fit_shift(amax);
      sc[rb] = __builtin_ldexpf(sc[rb], -shift);
    }
#pragma unroll
    for (int k = 0; k < NK; ++k) {
      if constexpr (__is_same(T, __bf16)) {
        float x[8];
        unpack8<T>(w[k], x);
#pragma unroll
        for (int e = 0; e < 8; ++e) q[rb][k][e] = (_Float16)__builtin_ldexpf(x[e], shift);
      } else {
        q[rb][k] = __builtin_bit_cast(f16x8, w[k]);
      }
    }
    m[rb] = -INFINITY;
    l[rb] = 0.f;
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[rb][ct][e] = 0.f;
  }

  auto k_at = [&](int token, int piece) { return token * (D / 8) + (D == 128 ? piece ^ (token & 15) : piece ^ ((token >> 1) & 7)); };
  auto v_at = [&](int ch, int piece) { return ch * 8 + (piece ^ ((ch >> 1) & 7)); };

  // Softmax of 32 tokens' scores from t0 on (lane: 8 hl .. and 16 + 8 hl ..), u -> p.
  auto softmax = [&](f32x16& u, int rb, int t0, float inv_sv, bool masked) __attribute__((always_inline)) {
    if (masked) {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int t = t0 + 16 * (e >> 3) + 8 * hl + (e & 7);
        if (t < see_lo[rb] || t >= see_hi[rb]) u[e] = -INFINITY;
      }
    }
    float top = u[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) top = fmaxf(top, u[e]);
    if (__any(top > m[rb] + kLazy)) {
      top = fmaxf(top, __shfl_xor(top, 32));
      const float m_new = fmaxf(m[rb], top);
      const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[rb] - m_new);
      m[rb] = m_new;
      l[rb] *= alpha;
#pragma unroll
      for (int ct = 0; ct < NCT; ++ct) o[rb][ct] *= alpha;
    }
    const float base = m[rb] == -INFINITY ? 0.f : m[rb];
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      u[e] = __builtin_amdgcn_exp2f(u[e] - base);
      sum += u[e];
    }
    l[rb] = __builtin_fmaf(sum, inv_sv, l[rb]);
  };

  // A tile of 64 tokens in buffer `buf`, elements of type E (f16 of codes, or the rows' own type).
  auto work_tile = [&](int buf, int tile, auto zero, const auto& qf, auto scale_of, float add, float inv_sv) __attribute__((always_inline)) {
    typedef decltype(zero) ex8;
    const bool masked = tile * kPagedTile < all_lo || tile * kPagedTile + kPagedTile > all_hi;
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      f32x16 u[RB];
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int e = 0; e < 16; ++e) u[rb][e] = 0.f;
      const int token = 32 * tt + score_token(r32);
#pragma unroll
      for (int k = 0; k < NK; ++k) {
        const ex8 kf = __builtin_bit_cast(ex8, s_k[buf][k_at(token, 2 * k + hl)]);
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) u[rb] = mma32(kf, qf[rb][k], u[rb]);
      }
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const float f = scale_of(rb);
#pragma unroll
        for (int e = 0; e < 16; ++e) u[rb][e] = __builtin_fmaf(u[rb][e], f, add);
        softmax(u[rb], rb, tile * kPagedTile + 32 * tt, inv_sv, masked);
      }
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        ex8 p[RB];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
          for (int e = 0; e < 8; ++e) p[rb][e] = to_element<ex8>(u[rb][8 * half + e]);
#pragma unroll
        for (int ct = 0; ct < NCT; ++ct) {
          const ex8 vf = __builtin_bit_cast(ex8, s_v[buf][v_at(32 * ct + r32, 4 * tt + 2 * half + hl)]);
#pragma unroll
          for (int rb = 0; rb < RB; ++rb) o[rb][ct] = mma32(vf, p[rb], o[rb][ct]);
        }
      }
    }
  };

  // ---- full pages: a tile's codes in registers while the one before is worked ----
  u32x4 kc[NB], vc[NB];
  auto store_tile = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const int piece = i * THREADS + tid;                // 16 codes
      const int token = piece / (D / 16), kp = 2 * (piece % (D / 16)), ch = piece / 4, vp = 2 * (piece % 4);
      s_k[buf][k_at(token, kp)] = __builtin_bit_cast(u32x4, codes_f16<FP8>(kc[i].x, kc[i].y));
      s_k[buf][k_at(token, kp + 1)] = __builtin_bit_cast(u32x4, codes_f16<FP8>(kc[i].z, kc[i].w));
      s_v[buf][v_at(ch, vp)] = __builtin_bit_cast(u32x4, codes_f16<FP8>(vc[i].x, vc[i].y));
      s_v[buf][v_at(ch, vp + 1)] = __builtin_bit_cast(u32x4, codes_f16<FP8>(vc[i].z, vc[i].w));
    }
  };
  const int code_end = min(t_last, code_tiles);
  for (int batch0 = t_first; batch0 < code_end; batch0 += 64) {
    const int t_l = batch0 + lane;
    int blk = 0;
    float sk = 0.f, lsv = 0.f, isv = 0.f;
    if (t_l < code_end) {
      const int page = a.bt.page_table[(long)b * a.bt.table_stride + t_l / runs];
      const bool ok = page >= 0 && page < a.c.pages;
      const long block = (long)(ok ? page : 0) * H + h;
      blk = (int)(block * runs) + t_l % runs;
      sk = ok ? a.c.k_scales[block] : __builtin_nanf("");
      const float sv = ok ? a.c.v_scales[block] : 1.f;
      lsv = __builtin_amdgcn_logf(sv);
      isv = 1.f / sv;
    }
    const int count = min(64, code_end - batch0);
    auto load_tile = [&](int i) __attribute__((always_inline)) {
      const long at = (long)__builtin_amdgcn_readlane(blk, i) * (kPagedTile * D);
#pragma unroll
      for (int k = 0; k < NB; ++k) {
        kc[k] = *reinterpret_cast<const u32x4*>(a.c.k_codes + at + 16l * (k * THREADS + tid));
        vc[k] = *reinterpret_cast<const u32x4*>(a.c.v_codes + at + 16l * (k * THREADS + tid));
      }
    };
    load_tile(0);
    __syncthreads();                                      // buffer 0 has been read
    store_tile(0);
    __syncthreads();
    for (int i = 0; i < count; ++i) {
      if (i + 1 < count) load_tile(i + 1);
      const float f = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, sk), i));
      const float add = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, lsv), i));
      const float inv_sv = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, isv), i));
      work_tile(i & 1, batch0 + i, f16x8{}, q, [&](int rb) { return f * sc[rb]; }, add, inv_sv);
      if (i + 1 < count) store_tile((i + 1) & 1);
      __syncthreads();
    }
  }

  // ---- the page being filled: 16-bit rows ----
  for (int tile = max(t_first, code_tiles); tile < t_last; ++tile) {
    const int slot = a.bt.tail_slots ? a.bt.tail_slots[b] : b;
    const bool ok = slot >= 0 && slot < a.c.slots;
    const int left = len - tile * kPagedTile;
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
    tx8 qt[RB][NK];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
#pragma unroll
      for (int k = 0; k < NK; ++k) qt[rb][k] = __builtin_bit_cast(tx8, *reinterpret_cast<const u32x4*>(q_row[rb] + 16 * k));
      see_hi[rb] = min(see_hi[rb], len);
    }
    const float f = ok ? a.scale_log2 : __builtin_nanf("");
    work_tile(0, tile, tx8{}, qt, [&](int) { return f; }, 0.f, 1.f);
  }

  // ---- outputs, or partials for the workgroup that joins the splits ----
  auto out_of = [&](int col) {
    const int pair = first + col;
    return a.out.data + (long)(s.row0 + pair / a.group) * a.out.token_stride + (long)(h * a.group + pair % a.group) * a.out.head_stride;
  };
  const int unit = item * H + h;
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    l[rb] += __shfl_xor(l[rb], 32);
    const int col = (wave * RB + rb) * 32 + r32;
    if (first + col >= pairs) continue;
    if (a.splits == 1) {
      const float inv = l[rb] == 0.f ? 0.f : 1.f / l[rb];
      uint16_t* const dst = out_of(col);
#pragma unroll
      for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          *reinterpret_cast<u32x2*>(dst + 32 * ct + 8 * e + 4 * hl) = u32x2{pack2<T>(o[rb][ct][4 * e] * inv, o[rb][ct][4 * e + 1] * inv),
                                                                           pack2<T>(o[rb][ct][4 * e + 2] * inv, o[rb][ct][4 * e + 3] * inv)};
    } else {
      float* const p = a.partials + (((long)unit * a.splits + split) * M + col) * (D + 2);
#pragma unroll
      for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          __hip_atomic_store(p + 32 * ct + 8 * (e >> 2) + 4 * hl + (e & 3), o[rb][ct][e], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      if (hl == 0) {
        __hip_atomic_store(p + D, m[rb], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __hip_atomic_store(p + D + 1, l[rb], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
    }
  }
  if (a.splits > 1) join_splits<T, D>(a, unit, M, min(M, pairs - first), &s_last, out_of);
}

constexpr int kPromptBlocks = 1;   // 32-row blocks of a wave
constexpr int kPromptRows = 32 * kPromptBlocks * kPromptWaves;

template <typename T, int D>
static void launch_prompt(const PagedAttnArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)((long)a.units * a.splits)), block(64 * kPromptWaves);
  if (a.c.codes == DQ_CODES_E4M3) hipLaunchKernelGGL((paged_prompt_kernel<T, D, true, kPromptBlocks>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((paged_prompt_kernel<T, D, false, kPromptBlocks>), grid, block, 0, st, a);
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
  int splits, cols;
};

static int up_div(int a, int b) { return (a + b - 1) / b; }

// What the two queries below agree on: kernel, units and splits from the host's bounds.
static bool paged_shape(const dq_paged_cache* c, int batch, long rows, int q_heads, int max_rows, int max_seq_len, PagedShape* s) {
  if (batch <= 0 || rows < 0 || q_heads <= 0 || q_heads % c->kv_heads || max_rows < 0 || max_seq_len < 0) return false;
  const int group = q_heads / c->kv_heads;
  const int tiles = max_seq_len / kPagedTile + 1;
  s->decode = (long)max_rows * group <= 16;
  if (s->decode) {
    s->units = (long)batch * c->kv_heads;
    s->cols = 16;
  } else {
    if (rows * group >= (1l << 31)) return false;
    s->units = (rows * group / kPromptRows + batch) * c->kv_heads;
    s->cols = kPromptRows;
  }
  if (s->units >= (1l << 24)) return false;
  // workgroups the chip holds at once: two per compute unit
  const long want = s->decode ? 768 : 512;
  int n = (int)((want + s->units - 1) / s->units);
  const int most = s->decode ? up_div(tiles, 4) : up_div(tiles, 8);   // a tile a wave at least, or eight tiles a workgroup
  if (n > most) n = most;
  if (n > kMaxSplits) n = kMaxSplits;
  s->splits = n < 1 ? 1 : n;
  return true;
}

static size_t paged_bytes(const PagedShape& s, int head_dim) {
  if (s.splits == 1) return kWsHeaderBytes;
  return kWsHeaderBytes + align_up((size_t)s.units * sizeof(int32_t), 256) + (size_t)s.units * s.splits * s.cols * (head_dim + 2) * sizeof(float);
}

}  // namespace dq

using namespace dq;

extern "C" size_t dq_paged_workspace_bytes(const dq_paged_cache* cache, int32_t batch, int32_t rows, int32_t q_heads, int32_t max_rows,
                                           int32_t max_seq_len) {
  PagedShape s;
  if (!paged_cache_ok(cache) || !paged_shape(cache, batch, rows, q_heads, max_rows, max_seq_len, &s)) return 0;
  return paged_bytes(s, cache->head_dim);
}

extern "C" int32_t dq_paged_attention(const dq_paged_cache* cache, const dq_paged_batch* batch, const dq_heads* q, const dq_heads* out,
                                      int32_t max_rows, int32_t max_seq_len, float softmax_scale, int32_t window, void* workspace,
                                      size_t workspace_bytes, uint32_t flags, void* hip_stream) {
  if (!paged_cache_ok(cache) || !paged_batch_ok(batch, cache, true) || !heads_ok(q, false) || !heads_ok(out, false)) return DQ_EINVAL;
  if (q->heads != out->heads || q->heads % cache->kv_heads || !workspace || ((uintptr_t)workspace & 15)) return DQ_EINVAL;
  if ((flags & ~DQ_PAGED_CAUSAL) || window < 0 || (window && !(flags & DQ_PAGED_CAUSAL))) return DQ_EINVAL;
  if (softmax_scale != softmax_scale) return DQ_EINVAL;
  PagedShape s;
  if (!paged_shape(cache, batch->batch, batch->rows, q->heads, max_rows, max_seq_len, &s)) return DQ_EINVAL;
  if (workspace_bytes < paged_bytes(s, cache->head_dim)) return DQ_ENOSPACE;
  if (batch->rows == 0 || max_rows == 0) return DQ_OK;
  PagedAttnArgs a = {};
  a.c = *cache; a.bt = *batch; a.q = *q; a.out = *out;
  a.group = q->heads / cache->kv_heads;
  a.max_rows = max_rows;
  a.max_seq_len = max_seq_len;
  a.window = window;
  a.causal = (flags & DQ_PAGED_CAUSAL) ? 1 : 0;
  a.scale_log2 = (softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)cache->head_dim)) * 1.44269504088896340736f;
  a.splits = s.splits;
  a.units = (int)s.units;
  char* ws = reinterpret_cast<char*>(workspace);
  a.counters = reinterpret_cast<int32_t*>(ws + kWsHeaderBytes);
  a.partials = reinterpret_cast<float*>(ws + kWsHeaderBytes + align_up((size_t)s.units * sizeof(int32_t), 256));
  hipStream_t st = (hipStream_t)hip_stream;
  return s.decode ? launch_paged_decode(a, st) : launch_paged_prompt(a, st);
}
