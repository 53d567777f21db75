// The paged cache of latents: rows in (norm, rotation) and out.
#include "dq_latent.h"

namespace dq {

struct LatentAppendArgs {
  dq_latent_cache c;
  dq_paged_batch bt;
  const uint16_t *latent, *k_rot, *weight;
  long latent_stride, k_rot_stride;
  float eps;
  dq_heads q, q_out;               // heads == 0: none
  dq_rotary rot;                   // rot_dim == 0: none
  int head_groups;                 // of the queries; 0: none
};

// Which sequence each of a workgroup's packed rows belongs to: every thread looks at its sequences, all at once, and names the rows
// they have here.  (A search by row would be a chain of loads.)
struct RowPlace {
  int b, i;                        // b < 0: of no sequence
};
template <int ROWS>
__device__ __forceinline__ void place_rows(const int32_t* starts, int rows, int batch, int first, RowPlace (&s_place)[ROWS]) {
  for (int r = threadIdx.x; r < ROWS; r += blockDim.x) s_place[r].b = -1;
  __syncthreads();
  for (int b = threadIdx.x; b < batch; b += blockDim.x) {
    const int lo = min(max(starts ? starts[b] : b, 0), rows), hi = min(max(starts ? starts[b + 1] : b + 1, lo), rows);
    for (int r = max(lo, first); r < min(hi, first + ROWS); ++r) s_place[r - first] = {b, r - lo};
  }
  __syncthreads();
}

// Whether any of a piece's eight values is infinite or NaN.
template <typename T> __device__ __forceinline__ bool not_finite(const u32x4& v) {
  constexpr uint32_t kExp = __is_same(T, __bf16) ? 0x7F80u : 0x7C00u;
  bool bad = false;
#pragma unroll
  for (int e = 0; e < 4; ++e) bad |= (v[e] & kExp) == kExp || (v[e] >> 16 & kExp) == kExp;
  return bad;
}

// Of 256 / (ROT / 16) rows a workgroup takes a quarter's latents and shared key channels, or the queries' heads of a group.  A wave norms four
// rows of 512 channels (eight of 256), all asked for together (all the rows' latents in one workgroup, four times as many after one another: 11.7 us
// for 128 rows of 128 heads where this takes 6.1, 10.5 and 5.9 for 16 rows).  A thread keeps 16 of the rotated channels of one row, whose angles it
// forms once for all heads of its group.
constexpr int kLatentParts = 4;
constexpr int kTurnedHeads = 8;   // of a group (28 thousand rows of 16 heads in prompts: 47 us, 51 with four, 52 with sixteen; 16 rows: 5.9, 5.5 with four)
template <typename T, int R, bool INTERLEAVED>
__global__ __launch_bounds__(256) void latent_append_kernel(LatentAppendArgs a) {
  constexpr int ROT = R == 512 ? 64 : 32, W = R + ROT, LANES = ROT / 16, ROWS = 256 / LANES;
  constexpr int AT_ONCE = 512 / R, PASSES = ROWS / kLatentParts / (4 * AT_ONCE);   // rows of a wave and pass, passes
  __shared__ RowPlace s_place[ROWS];
  __shared__ int s_token[ROWS];
  __shared__ long s_row[ROWS];     // of the cache, or -1
  __shared__ bool s_bad[ROWS];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, P = a.c.page_tokens;
  const int groups = a.head_groups + kLatentParts, group = (int)(blockIdx.x % (unsigned)groups), first = (int)(blockIdx.x / (unsigned)groups) * ROWS;
  const bool latents = group < kLatentParts;
  const int row0 = group * (ROWS / kLatentParts);         // (latents) the first of its rows here
  if (latents && first + row0 >= a.bt.rows) return;
  place_rows(a.bt.starts, a.bt.rows, a.bt.batch, first, s_place);
  if (tid < ROWS) {
    const RowPlace at = s_place[tid];
    long row = -1;
    int token = 0;
    if (at.b >= 0) {
      const Sequence s = sequence_of(a.bt, P, at.b);
      token = s.old + at.i;
      if (latents && token >= 0 && token < s.len) {
        const int page = a.bt.page_table[(long)at.b * a.bt.table_stride + token / P];
        if (page >= 0 && page < a.c.pages) row = (long)page * P + token % P;
      }
    }
    s_token[tid] = token;
    s_row[tid] = row;
    s_bad[tid] = false;
  }
  __syncthreads();

  if (latents) {
    const int piece = lane % (R / 8);                     // 8 channels
    u32x4 w = {};
    if (a.weight) w = *reinterpret_cast<const u32x4*>(a.weight + 8 * piece);
    u32x4 v[PASSES];
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
      const int r = row0 + (i * 4 + wave) * AT_ONCE + lane / (R / 8);
      v[i] = s_row[r] >= 0 ? *reinterpret_cast<const u32x4*>(a.latent + (long)(first + r) * a.latent_stride + 8 * piece) : u32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
      const int r = row0 + (i * 4 + wave) * AT_ONCE + lane / (R / 8);
      if (a.weight) {
        float x[8], y[8], sum = 0.f;
        unpack8<T>(v[i], x);
        unpack8<T>(w, y);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum = __builtin_fmaf(x[e], x[e], sum);
        sum = row_reduce<16>(sum, [](float p, float q) { return p + q; });
        sum += __shfl_xor(sum, 16);
        if constexpr (R == 512) sum += __shfl_xor(sum, 32);
        const float f = 1.0f / sqrtf(sum * (1.0f / R) + a.eps);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = x[e] * f * y[e];
        v[i] = pack8<T>(x);
      }
      const uint64_t any = __ballot(not_finite<T>(v[i])) >> (R == 512 ? 0 : lane & 32) & (R == 512 ? ~0ull : 0xFFFFFFFFull);
      if (any) v[i] = u32x4{0, 0, 0, 0};
      const long row = s_row[r];
      if (row < 0) continue;
      *reinterpret_cast<u32x4*>(a.c.rows + row * W + 8 * piece) = v[i];
      if (any && piece == 0) s_bad[r] = true;
    }
    __syncthreads();
  }

  const int unit = tid % LANES, r = tid / LANES;
  const bool live = latents ? r >= row0 && r < row0 + ROWS / kLatentParts && s_row[r] >= 0 : s_place[r].b >= 0;
  if (!__any(live)) return;
  RowLayout l = row_layout(unit, a.rot.rot_dim, INTERLEAVED);
  if (!live) l.pair0 = -1;
  UnitTurns ut;
  load_turns(a.rot, l, first + r, s_token[r], ut);
  u32x4 v[2] = {};
  const int h0 = (group - kLatentParts) * kTurnedHeads, h1 = min(h0 + kTurnedHeads, a.q.heads);
  const uint16_t* const q = a.q.data + (long)(first + r) * a.q.token_stride;
  const uint16_t* const k = a.k_rot + (long)(first + r) * a.k_rot_stride;
  if (live) load_unit(v, latents ? k : q + h0 * a.q.head_stride, l);
  float cs[8], sn[8];
  make_turns(l, ut, cs, sn);
  if (!latents) {
    rotate_row<T, LANES, INTERLEAVED>(v, q, a.q_out.data + (long)(first + r) * a.q_out.token_stride, a.q.head_stride, a.q_out.head_stride, h0, h1, live,
                                      l, nullptr, 0.f, 0.f, cs, sn);
  } else if (live) {
    u32x4 none[2] = {};
    ready_unit<T, LANES, INTERLEAVED>(v, none, false, l.pair0 >= 0, 0.f, 0.f, cs, sn);
    // Key channels that came or were turned out of the type's range count as the latent's do: an infinite score would hide the token from
    // half of the queries.  (A row's lanes are here together.  Its latent is finite, and stays: zeros over it, whose stores no row
    // comes to, took 1.1 us of 62 for 28 thousand rows.)
    const uint64_t lanes = __ballot(not_finite<T>(v[0]) || not_finite<T>(v[1]));
    if (s_bad[r] || (lanes >> (lane / LANES * LANES) & ((1u << LANES) - 1))) v[0] = v[1] = kNanPiece;
    uint16_t* const to = a.c.rows + s_row[r] * W + R;
    *reinterpret_cast<u32x4*>(to + l.at0) = v[0];
    *reinterpret_cast<u32x4*>(to + l.at1) = v[1];
  }
}

struct LatentReadArgs {
  dq_latent_cache c;
  dq_paged_batch bt;
  const int32_t *first, *out_starts;
  uint16_t* out;
  long out_stride;
};

// A workgroup copies 32 rows, 16 bytes a lane, all asked for before the first is stored.
template <int W>
__global__ __launch_bounds__(256) void latent_read_kernel(LatentReadArgs a) {
  constexpr int ROWS = 32, PIECES = W / 8, EACH = (ROWS * PIECES + 255) / 256, ROT = W == 576 ? 64 : 32;
  __shared__ RowPlace s_place[ROWS];
  __shared__ long s_row[ROWS];     // of the cache; -1: a page that does not exist; -2: not to be written
  const int tid = threadIdx.x, first = (int)blockIdx.x * ROWS, P = a.c.page_tokens;
  place_rows(a.out_starts, a.bt.rows, a.bt.batch, first, s_place);
  if (tid < ROWS) {
    const RowPlace at = s_place[tid];
    long row = -2;
    if (at.b >= 0) {
      const int len = min(max(a.bt.seq_lens[at.b], 0), a.bt.table_width * P);
      // (starts before row 0 count: i is the row's distance from the first that is there)
      const long token = (long)(a.first ? max(a.first[at.b], 0) : 0) + at.i + (min(max(a.out_starts[at.b], 0), a.bt.rows) - (long)a.out_starts[at.b]);
      if (token < len) {
        const int page = a.bt.page_table[(long)at.b * a.bt.table_stride + token / P];
        row = page >= 0 && page < a.c.pages ? (long)page * P + token % P : -1;
      }
    }
    s_row[tid] = row;
  }
  __syncthreads();
  u32x4 v[EACH];
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const int p = min(i * 256 + tid, ROWS * PIECES - 1), c = p % PIECES;
    const long row = s_row[p / PIECES];
    const uint32_t none = 8 * c >= W - ROT ? 0x7FFF7FFFu : 0u;
    v[i] = row >= 0 ? *reinterpret_cast<const u32x4*>(a.c.rows + row * W + 8 * c) : u32x4{none, none, none, none};
  }
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const int p = i * 256 + tid;
    if (p < ROWS * PIECES && s_row[p / PIECES] != -2)
      __builtin_nontemporal_store(v[i], reinterpret_cast<u32x4*>(a.out + (first + p / PIECES) * a.out_stride + 8 * (p % PIECES)));
  }
}

template <typename T, int R>
static void launch_latent_append(const LatentAppendArgs& a, dim3 grid, hipStream_t st) {
  if (a.rot.interleaved) hipLaunchKernelGGL((latent_append_kernel<T, R, true>), grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((latent_append_kernel<T, R, false>), grid, dim3(256), 0, st, a);
}

}  // namespace dq

using namespace dq;

static bool rows_ok(const void* p, int64_t stride) { return p && !((uintptr_t)p & 15) && stride >= 0 && !(stride & 7); }

extern "C" int32_t dq_latent_append(const dq_latent_cache* cache, const dq_paged_batch* batch, const uint16_t* latent, int64_t latent_stride,
                                    const uint16_t* k_rot, int64_t k_rot_stride, const uint16_t* weight, float eps, const dq_heads* q,
                                    const dq_heads* q_out, const dq_rotary* rot, void* hip_stream) {
  if (!latent_cache_ok(cache) || !latent_batch_ok(batch, cache, true) || (!q) != (!q_out)) return DQ_EINVAL;
  if (!rows_ok(latent, latent_stride) || !rows_ok(k_rot, k_rot_stride) || ((uintptr_t)weight & 15) || (weight && !(eps >= 0.f))) return DQ_EINVAL;
  if (q && (!heads_ok(q, false) || !heads_ok(q_out, false) || q->heads != q_out->heads)) return DQ_EINVAL;
  if (!rotary_ok(rot, cache->rot_dim, batch->rows, false) || (rot && rot->rot_dim != cache->rot_dim)) return DQ_EINVAL;
  if (batch->rows == 0) return DQ_OK;
  // queries are turned by other workgroups than take the rows in
  const dq_heads c = {const_cast<uint16_t*>(latent), 0, latent_stride, 0, 1}, r = {const_cast<uint16_t*>(k_rot), 0, k_rot_stride, 0, 1};
  if (q && (heads_meet(&c, batch->rows, cache->latent_dim, q_out, batch->rows, cache->rot_dim) ||
            heads_meet(&r, batch->rows, cache->rot_dim, q_out, batch->rows, cache->rot_dim) || !heads_in_place(q, q_out, batch->rows, cache->rot_dim)))
    return DQ_EINVAL;
  LatentAppendArgs a = {};
  a.c = *cache; a.bt = *batch;
  a.latent = latent; a.latent_stride = latent_stride;
  a.k_rot = k_rot; a.k_rot_stride = k_rot_stride;
  a.weight = weight; a.eps = eps;
  if (q) { a.q = *q; a.q_out = *q_out; }
  if (rot) a.rot = *rot;
  const int rows_per_block = 256 / (cache->rot_dim / 16);
  const long blocks = (batch->rows + (long)rows_per_block - 1) / rows_per_block;
  const long groups = q ? (q->heads + (kTurnedHeads - 1l)) / kTurnedHeads : 0, workgroups = blocks * (groups + kLatentParts);
  if (workgroups >= kMaxThreads / 256) return DQ_EINVAL;
  a.head_groups = (int)groups;
  const dim3 grid((unsigned)workgroups);
  hipStream_t st = (hipStream_t)hip_stream;
  if (cache->dtype == DQ_BF16) { if (cache->latent_dim == 512) launch_latent_append<__bf16, 512>(a, grid, st); else launch_latent_append<__bf16, 256>(a, grid, st); }
  else { if (cache->latent_dim == 512) launch_latent_append<_Float16, 512>(a, grid, st); else launch_latent_append<_Float16, 256>(a, grid, st); }
  DQ_HIP_CHECK(hipGetLastError());
  return DQ_OK;
}

extern "C" int32_t dq_latent_read(const dq_latent_cache* cache, const dq_paged_batch* batch, const int32_t* first, const int32_t* out_starts,
                                  uint16_t* out, int64_t out_stride, void* hip_stream) {
  if (!latent_cache_ok(cache) || !latent_batch_ok(batch, cache, false) || !out_starts || !rows_ok(out, out_stride) ||
      (batch->rows != 1 && out_stride < cache->latent_dim + cache->rot_dim))   // (a stride over one row says nothing)
    return DQ_EINVAL;
  if (batch->rows == 0) return DQ_OK;
  const LatentReadArgs a = {*cache, *batch, first, out_starts, out, out_stride};
  const dim3 grid((unsigned)((batch->rows + 31l) / 32));
  if (cache->latent_dim == 512) hipLaunchKernelGGL((latent_read_kernel<576>), grid, dim3(256), 0, (hipStream_t)hip_stream, a);
  else hipLaunchKernelGGL((latent_read_kernel<288>), grid, dim3(256), 0, (hipStream_t)hip_stream, a);
  DQ_HIP_CHECK(hipGetLastError());
  return DQ_OK;
}
