// Attention over keys and values expanded from latents: ragged prompts, heads of D channels and ROT more key channels that all heads share.
#include "dq_latent.h"

namespace dq {

struct ExpandedArgs {
  dq_expanded x;
  int max_rows, causal;
  float scale_log2;
  int splits;              // of every tile of rows
  int seq_tiles;           // tiles of rows that every sequence gets, whatever it has (0: dealt by starts)
  int far;                 // strides too large for 32-bit offsets
  float *o, *ml;           // pieces: [unit * splits + split, row, D], [.., 2]
};

constexpr int kExpandedRows = 128, kExpandedTile = 64;

struct ExpandedSequence {
  int row0, n, token0, len;
};
__device__ __forceinline__ ExpandedSequence expanded_sequence(const dq_expanded& x, int b) {
  auto uniform = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
  ExpandedSequence s;
  s.row0 = uniform(min(max(x.starts[b], 0), x.rows));
  s.n = uniform(min(max(x.starts[b + 1], s.row0), x.rows)) - s.row0;
  s.token0 = uniform(min(max(x.kv_starts[b], 0), x.tokens));
  s.len = uniform(min(max(x.kv_starts[b + 1], s.token0), x.tokens)) - s.token0;
  return s;
}

// One workgroup of four waves per (tile of 128 rows, head, split), 32 rows a wave.  Tiles of 64 tokens are copied to LDS past the registers, a
// tile ahead; scores are formed transposed, as in the kernel over latents, and the values' operand comes from rows as they lie by
// transposing LDS reads.  Four prompts of 3500 to 4096 with 32 heads of 128 + 64, 606 GFLOP: 640 us, 947 TFLOP/s, 70 % of a large product's rate;
// between the products every wave has its exponentials to form.
template <typename T, int D>
__global__ __launch_bounds__(256, 2) void expanded_attn_kernel(ExpandedArgs a) {
  constexpr int ROT = D / 2, W = D + ROT, TT = kExpandedTile, M = kExpandedRows, NK = D / 16, NR = ROT / 16, NCT = D / 32;
  constexpr int PD = D / 8, PR = ROT / 8;                 // pieces of a row
  constexpr int COPIES = TT * PD / 256, ROT_COPIES = TT * PR / 256;   // a wave's, of keys or values
  typedef typename Vec8<T>::type tx8;
  __shared__ __align__(1024) char s_k[2][TT * D * 2], s_r[2][TT * ROT * 2], s_v[2][TT * D * 2];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r32 = lane & 31, hl = lane >> 5;
  const dq_expanded& x = a.x;
  const int H = x.q.heads, h = (int)(blockIdx.x % (unsigned)H), split = (int)(blockIdx.x / (unsigned)H) % a.splits, item = (int)(blockIdx.x / (unsigned)H) / a.splits;
  const int b = a.seq_tiles ? item / a.seq_tiles : item_owner(x.starts, x.rows, x.batch, item, 1, M, 1);
  const ExpandedSequence s = expanded_sequence(x, b);
  const int n = min(s.n, a.max_rows), len = s.len, before = s.len - s.n;
  const int row_tiles = (n + M - 1) / M, j = a.seq_tiles ? item % a.seq_tiles : item - item_first(x.starts, x.rows, b, 1, M, 1);
  if (j < 0 || j >= row_tiles) return;
  const int first = (row_tiles - 1 - j) * M;              // the longest first
  const int rows_hi = min(first + M - 1, n - 1);
  const int any_hi = a.causal ? min(max(before + rows_hi + 1, 0), len) : len, all_hi = a.causal ? min(before + first + 1, len) : len;
  int t_first = 0, t_last = (any_hi + TT - 1) / TT;
  {
    const int share = (t_last + a.splits - 1) / a.splits;
    t_first = min(split * share, t_last);
    t_last = min(t_first + share, t_last);
  }
  const int my_row = min(first + wave * 32 + r32, n - 1), see_hi = a.causal ? min(before + my_row + 1, len) : len;
  const uint16_t* const q_row = x.q.data + (long)(s.row0 + my_row) * x.q.token_stride + (long)h * x.q.head_stride + 8 * hl;
  tx8 q[NK + NR];
#pragma unroll
  for (int k = 0; k < NK + NR; ++k) q[k] = __builtin_bit_cast(tx8, *reinterpret_cast<const u32x4*>(q_row + 16 * k));

  // Pieces of a row in LDS are exchanged by bits of the token, so that the lanes that read one piece of 16 rows, or four pieces of four
  // rows, touch all banks.
  auto k_swap = [](int t) { return PD == 16 ? t & 15 : t >> 1 & 7; };
  auto r_swap = [](int t) { return PR == 8 ? t >> 1 & 7 : t >> 2 & 3; };
  auto v_swap = [](int t) { return PD == 16 ? (t & 3) << 2 | (t >> 2 & 3) : (t >> 1 & 1) << 2 | (t >> 2 & 3); };
  const int k_token = (r32 & ~12) | (r32 & 4) << 1 | (r32 & 8) >> 1;   // + 32: the other half of the tile, with the same exchange
  const int k_at = k_token * D * 2 + ((hl ^ k_swap(k_token)) << 4), r_at = k_token * ROT * 2 + ((hl ^ r_swap(k_token)) << 4);   // ^ 32 k
  const int i16 = lane & 15, v_token = 8 * hl + (i16 >> 2), v_piece = 2 * (lane >> 4 & 1) + ((i16 & 3) >> 1);   // + 4 j + 16 step, + 4 ct
  const int v_at0 = v_token * D * 2 + ((v_piece ^ v_swap(v_token)) << 4) + (i16 & 1) * 8;
  const int v_at1 = (v_token + 4) * D * 2 + ((v_piece ^ v_swap(v_token + 4)) << 4) + (i16 & 1) * 8;   // both ^ 64 ct

  const uint16_t* const k_head = x.k.data + (long)h * x.k.head_stride;
  const uint16_t* const v_head = x.v.data + (long)h * x.v.head_stride;
  auto load_tile = [&](int t) __attribute__((always_inline)) {
    const int buf = t & 1, left = len - t * TT;
    const long token0 = (long)s.token0 + (long)t * TT;
    // copy i of a wave: rows (wave + 4 i) 64 / pieces and on, so that the exchange is the same for all i
    auto rows = [&](const uint16_t* from, long stride, int pieces, int copies, char* to, auto swap) __attribute__((always_inline)) {
      const int each = 64 / pieces, in = lane / pieces, slot = lane % pieces;
      if (left >= TT && !a.far) {
#pragma unroll
        for (int i = 0; i < copies; ++i) {
          copy_to_lds(from + (token0 + each * (wave + 4 * i)) * stride, (uint32_t)in * (uint32_t)stride * 2 + ((slot ^ swap(each * wave + in)) << 4),
                      lds_of(to) + 1024 * (wave + 4 * i));
        }
      } else {
        int l = lane;
        asm volatile("" : "+v"(l));                       // (else its addresses are formed ahead of the loop and held there)
#pragma unroll 1
        for (int i = 0; i < copies; ++i) {
          const int row = each * (wave + 4 * i) + l / pieces;
          copy_to_lds(row < left ? from + (token0 + row) * stride + 8 * (l % pieces ^ swap(row)) : reinterpret_cast<const uint16_t*>(g_blank),
                      lds_of(to) + 1024 * (wave + 4 * i));
        }
      }
    };
    rows(k_head, x.k.token_stride, PD, COPIES, s_k[buf], k_swap);
    rows(x.k_rot, x.k_rot_stride, PR, ROT_COPIES, s_r[buf], r_swap);
    rows(v_head, x.v.token_stride, PD, COPIES, s_v[buf], v_swap);
  };

  f32x16 o[NCT];
#pragma unroll
  for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[ct][e] = 0.f;
  float m = -INFINITY, l = 0.f;
  if (t_first < t_last) load_tile(t_first);
  for (int t = t_first; t < t_last; ++t) {
    wait_copies<0>();
    const bool masked = t * TT + TT > all_hi;
    if (masked) {
      // A value that is not finite must not reach rows that do not see it (0 * inf): in tiles with a mask its token becomes one of zero
      // values and keys of NaN, for those who see it.  Every wave looks at the rows it has copied.
      constexpr uint32_t kExp = __is_same(T, __bf16) ? 0x7F80u : 0x7C00u;
#pragma unroll
      for (int i = 0; i < COPIES; ++i) {
        u32x4* const v = reinterpret_cast<u32x4*>(s_v[t & 1]) + 64 * (wave + 4 * i) + lane;
        const u32x4 w = *v;
        bool bad = false;
#pragma unroll
        for (int e = 0; e < 4; ++e) bad |= (w[e] & kExp) == kExp || (w[e] >> 16 & kExp) == kExp;
        const uint64_t lanes = __ballot(bad);
        if (lanes == 0 || !(lanes >> (lane / PD * PD) & ((1ull << PD) - 1))) continue;
        *v = u32x4{0, 0, 0, 0};
        reinterpret_cast<u32x4*>(s_k[t & 1])[64 * (wave + 4 * i) + lane] = kNanPiece;
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
    barrier();
    if (t + 1 < t_last) load_tile(t + 1);
    const LdsBytes k_from = (LdsBytes)s_k[t & 1], r_from = (LdsBytes)s_r[t & 1], v_from = (LdsBytes)s_v[t & 1];
    f32x16 u[2];
#pragma unroll
    for (int e = 0; e < 32; ++e) u[e >> 4][e & 15] = 0.f;
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int k = 0; k < NK; ++k) {
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) u[tt] = mma32(__builtin_bit_cast(tx8, *(LdsPieces)(k_from + 32 * tt * D * 2 + (k_at ^ 32 * k))), q[k], u[tt]);
      if (k % 2) __builtin_amdgcn_sched_barrier(0);         // (all reads ahead of the first product would take 96 registers)
    }
#pragma unroll
    for (int k = 0; k < NR; ++k)
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) u[tt] = mma32(__builtin_bit_cast(tx8, *(LdsPieces)(r_from + 32 * tt * ROT * 2 + (r_at ^ 32 * k))), q[NK + k], u[tt]);
    __builtin_amdgcn_s_setprio(0);
    if (masked) {
      int from = 8 * hl;
      asm volatile("" : "+v"(from)::"memory");            // (a branch, and nothing of it ahead of the loop: 64 registers)
      const int sees = see_hi - t * TT - from;
#pragma unroll
      for (int e = 0; e < 32; ++e) {
        const int in = 32 * (e >> 4) + 16 * (e >> 3 & 1) + (e & 7);
        u[e >> 4][e & 15] = in < sees ? u[e >> 4][e & 15] : -INFINITY;
      }
    }
    float top = u[0][0];
#pragma unroll
    for (int e = 1; e < 32; ++e) top = fmaxf(top, u[e >> 4][e & 15]);
    top *= a.scale_log2;
    if (__any(top > m + kLazy)) {
      top = fmaxf(top, __shfl_xor(top, 32));
      const float m_new = fmaxf(m, top);
      const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - m_new);
      m = m_new;
      l *= alpha;
#pragma unroll
      for (int ct = 0; ct < NCT; ++ct) o[ct] *= alpha;
    }
    const float base = m == -INFINITY ? 0.f : -m;
#pragma unroll
    for (int g = 0; g < 4; ++g) {                         // 16 tokens, 8 a lane; probabilities in the rows' type, the sum, in fp32, of those
      tx8 p;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        p[e] = to_element<tx8>(__builtin_amdgcn_exp2f(__builtin_fmaf(u[g >> 1][8 * (g & 1) + e], a.scale_log2, base)));
      }
      l = add_eight(l, p);
      const LdsBytes from = v_from + 16 * g * D * 2;
#pragma unroll
      for (int ct = 0; ct < NCT; ++ct) o[ct] = mma32(turned_rows<tx8>(from + (v_at0 ^ 64 * ct), from + (v_at1 ^ 64 * ct)), p, o[ct]);
    }
  }

  l += __shfl_xor(l, 32);
  const int col = wave * 32 + r32;
  if (first + col >= n) return;
  if (a.splits == 1) {
    const float inv = l == 0.f ? 0.f : 1.f / l;
    uint16_t* const dst = x.out.data + (long)(s.row0 + my_row) * x.out.token_stride + (long)h * x.out.head_stride;
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        *reinterpret_cast<u32x2*>(dst + 32 * ct + 8 * e + 4 * hl) = u32x2{pack2<T>(o[ct][4 * e] * inv, o[ct][4 * e + 1] * inv),
                                                                         pack2<T>(o[ct][4 * e + 2] * inv, o[ct][4 * e + 3] * inv)};
    return;
  }
  const long at = (((long)item * H + h) * a.splits + split) * M + col;
#pragma unroll
  for (int ct = 0; ct < NCT; ++ct)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      *reinterpret_cast<f32x4*>(a.o + at * D + 32 * ct + 8 * e + 4 * hl) = f32x4{o[ct][4 * e], o[ct][4 * e + 1], o[ct][4 * e + 2], o[ct][4 * e + 3]};
  if (hl == 0) *reinterpret_cast<f32x2*>(a.ml + 2 * at) = f32x2{m, l};
}

template <typename T, int D>
__global__ __launch_bounds__(256) void expanded_join_kernel(ExpandedArgs a) {
  constexpr int M = kExpandedRows;
  const dq_expanded& x = a.x;
  constexpr unsigned GROUPS = M / kJoinColumns<D>;
  const int H = x.q.heads, col = (int)(blockIdx.x % GROUPS) * kJoinColumns<D>;
  const long unit = blockIdx.x / GROUPS;
  const int h = (int)(unit % H), item = (int)(unit / H);
  const int b = a.seq_tiles ? item / a.seq_tiles : item_owner(x.starts, x.rows, x.batch, item, 1, M, 1);
  const ExpandedSequence s = expanded_sequence(x, b);
  const int n = min(s.n, a.max_rows), row_tiles = (n + M - 1) / M;
  const int j = a.seq_tiles ? item % a.seq_tiles : item - item_first(x.starts, x.rows, b, 1, M, 1);
  const int first = (row_tiles - 1 - j) * M;
  if (j < 0 || j >= row_tiles || first + col >= n) return;
  join_columns<T, D>(a.splits, [&](int i) { return unit * a.splits + i; }, a.o, a.ml, M, col, min(n - first, M), [&](int c) {
    return x.out.data + (long)(s.row0 + first + c) * x.out.token_stride + (long)h * x.out.head_stride;
  });
}

struct ExpandedPlan {
  long units;
  int seq_tiles, splits;
};
constexpr int kExpandedGroups = 2048;   // workgroups of a launch that splits

// Tiles of rows are dealt by starts, with one a sequence that may stay empty, or, where the bound on rows gives every sequence tiles of
// its own with no more in all, by that.  Splits of a tile where tiles leave compute units idle: the fewest within 4 % of the
// fullest rounds of the workgroups that are resident (two pieces of 400 to 512 rows of 40 heads of 64 channels behind 15 thousand tokens: 269 us in
// 2 splits, 307 in 3, 274 in 7).
static bool expanded_plan(int batch, long rows, int heads, int head_dim, int max_rows, int max_seq_len, ExpandedPlan* p) {
  if (batch <= 0 || rows < 0 || heads <= 0 || max_rows < 0 || max_seq_len < 0) return false;
  const long seq_tiles = ((long)max_rows + kExpandedRows - 1) / kExpandedRows, dealt = rows / kExpandedRows + batch;
  p->seq_tiles = seq_tiles <= dealt / batch ? (int)seq_tiles : 0;
  p->units = (p->seq_tiles ? batch * seq_tiles : dealt) * heads;
  if (p->units >= (1l << 24)) return false;
  const int cap = (int)(0.75f * sqrtf((float)(max_seq_len / kExpandedTile + 1)));
  const long resident = head_dim == 64 ? 768 : 512;        // workgroups: three or two a compute unit
  auto fill = [&](int n) { const long w = p->units * n; return (float)w / (float)((w + resident - 1) / resident * resident); };
  float best = 0.f;
  p->splits = 1;
  if (p->units == 0 || p->units >= kExpandedGroups / 2) return true;
  for (int n = 1; n <= cap && p->units * n <= kExpandedGroups; ++n) best = fmaxf(best, fill(n));
  while (fill(p->splits) < 0.96f * best) ++p->splits;
  return true;
}
static size_t expanded_bytes(const ExpandedPlan& p, int splits, int head_dim) {
  return kWsHeaderBytes + (splits > 1 ? (size_t)p.units * p.splits * kExpandedRows * (head_dim + 2) * sizeof(float) : 0);
}
static bool expanded_dims_ok(int head_dim, int rot_dim) { return (head_dim == 128 && rot_dim == 64) || (head_dim == 64 && rot_dim == 32); }

template <typename T, int D>
static void launch_expanded(const ExpandedArgs& a, const ExpandedPlan& p, hipStream_t st) {
  hipLaunchKernelGGL((expanded_attn_kernel<T, D>), dim3((unsigned)(p.units * a.splits)), dim3(256), 0, st, a);
  if (a.splits > 1) hipLaunchKernelGGL((expanded_join_kernel<T, D>), dim3((unsigned)(p.units * (kExpandedRows / kJoinColumns<D>))), dim3(256), 0, st, a);
}

}  // namespace dq

using namespace dq;

extern "C" size_t dq_expanded_workspace_bytes(int32_t batch, int32_t rows, int32_t heads, int32_t head_dim, int32_t max_rows, int32_t max_seq_len) {
  ExpandedPlan p;
  if ((head_dim != 128 && head_dim != 64) || !expanded_plan(batch, rows, heads, head_dim, max_rows, max_seq_len, &p)) return 0;
  // smaller calls have fewer units and may have more splits: both together are bounded
  const int cap = (int)(0.75f * sqrtf((float)(max_seq_len / kExpandedTile + 1)));
  if (cap < 2) return kWsHeaderBytes;
  const ExpandedPlan most = {p.units * cap < kExpandedGroups ? p.units * cap : kExpandedGroups, 0, 1};
  return expanded_bytes(most, 2, head_dim);
}

extern "C" int32_t dq_expanded_attention(const dq_expanded* call, int32_t max_rows, int32_t max_seq_len, float softmax_scale, void* workspace,
                                         size_t workspace_bytes, uint32_t flags, void* hip_stream) {
  if (!call) return DQ_EINVAL;
  dq_expanded one = *call;
  const dq_expanded* const x = &one;
  if (one.tokens == 0) one.k.data = one.v.data = const_cast<uint16_t*>(one.k_rot = one.out.data);   // tensors of no tokens have no address, and are not read
  if (!x->starts || !x->kv_starts || x->batch <= 0 || x->rows < 0 || x->tokens < 0 || !expanded_dims_ok(x->head_dim, x->rot_dim)) return DQ_EINVAL;
  if (x->dtype != DQ_F16 && x->dtype != DQ_BF16) return DQ_EINVAL;
  if (!heads_ok(&x->q, false) || !heads_ok(&x->k, false) || !heads_ok(&x->v, false) || !heads_ok(&x->out, false)) return DQ_EINVAL;
  if (x->q.heads != x->k.heads || x->q.heads != x->v.heads || x->q.heads != x->out.heads) return DQ_EINVAL;
  const dq_heads rot = {const_cast<uint16_t*>(x->k_rot), 0, x->k_rot_stride, 0, 1};
  if (heads_meet(&x->q, x->rows, x->head_dim + x->rot_dim, &x->out, x->rows, x->head_dim) || heads_meet(&x->k, x->tokens, x->head_dim, &x->out, x->rows, x->head_dim) ||
      heads_meet(&x->v, x->tokens, x->head_dim, &x->out, x->rows, x->head_dim) || heads_meet(&rot, x->tokens, x->rot_dim, &x->out, x->rows, x->head_dim))
    return DQ_EINVAL;
  if (!x->k_rot || ((uintptr_t)x->k_rot & 15) || x->k_rot_stride < 0 || (x->k_rot_stride & 7)) return DQ_EINVAL;
  if (!workspace || ((uintptr_t)workspace & 15) || (flags & ~DQ_PAGED_CAUSAL) || !scale_ok(softmax_scale)) return DQ_EINVAL;
  if (x->tokens >= kMostTokens || x->rows >= kMostTokens) return DQ_EINVAL;
  ExpandedPlan p;
  if (!expanded_plan(x->batch, x->rows, x->q.heads, x->head_dim, max_rows, max_seq_len, &p)) return DQ_EINVAL;
  if (p.units * p.splits >= kMaxThreads / 256 || (p.splits > 1 && p.units * kExpandedRows >= kMaxThreads / 256)) return DQ_EINVAL;
  if (workspace_bytes < expanded_bytes(p, p.splits, x->head_dim)) return DQ_ENOSPACE;
  if (x->rows == 0 || max_rows == 0) return DQ_OK;
  ExpandedArgs a = {};
  a.x = *x;
  a.max_rows = max_rows;
  a.causal = (flags & DQ_PAGED_CAUSAL) ? 1 : 0;
  a.scale_log2 = fmaxf((softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)(x->head_dim + x->rot_dim))) * 1.44269504088896340736f, 1e-37f);
  a.splits = p.splits;
  a.seq_tiles = p.seq_tiles;
  const int64_t limit = 1 << 27;                          // 15 rows in 32-bit byte offsets
  a.far = x->k.token_stride >= limit || x->v.token_stride >= limit || x->k_rot_stride >= limit;
  a.o = reinterpret_cast<float*>(reinterpret_cast<char*>(workspace) + kWsHeaderBytes);
  a.ml = a.o + p.units * p.splits * kExpandedRows * x->head_dim;
  hipStream_t st = (hipStream_t)hip_stream;
  if (x->dtype == DQ_BF16) { if (x->head_dim == 128) launch_expanded<__bf16, 128>(a, p, st); else launch_expanded<__bf16, 64>(a, p, st); }
  else { if (x->head_dim == 128) launch_expanded<_Float16, 128>(a, p, st); else launch_expanded<_Float16, 64>(a, p, st); }
  DQ_HIP_CHECK(hipGetLastError());
  return DQ_OK;
}
