// Rows into the paged 8-bit cache (norm and rotation of the keys, and of the queries beside them, on the way), and
// out of it.
#include "dq_paged.h"

namespace dq {

struct AppendArgs {
  dq_paged_cache c;
  dq_paged_batch bt;
  dq_heads k, v, q, q_out;   // q.heads == 0: none
  dq_head_norm norm;
  dq_rotary rot;             // rot_dim == 0: none
  int heads_per_group;       // kv heads a workgroup takes of its page, one after the other
  int head_groups;
  int page_blocks;           // workgroups that work pages; the others take query rows
  int q_heads_per_group, q_head_groups;
};

// One page of one sequence, PASSES rows of every thread: places and sources of the rows.
// Keys of a page: thread (row r = pass * RP + tid / LPR, unit tid % LPR), the unit's channels laid for the rotation.
// Values: rows PASSES * (tid / LPR) + pass, neighbours in the value layout, 16 neighbouring channels.
template <typename T, int D, int P, bool FP8>
struct PageWork {
  static constexpr int LPR = D / 16, RP = kPagedThreads / LPR, PASSES = P / RP;
  static_assert(PASSES == 1 || PASSES == 2 || PASSES == 4, "rows a thread");
};

__device__ __forceinline__ bool finite_pair(uint32_t w, uint32_t exponent) {   // both 16-bit values
  return ((w & exponent) != exponent) & ((w & (exponent << 16)) != (exponent << 16));
}

// Pages are worked by one workgroup per (page, group of kv heads): the angles of a page's rows are formed once per group.
// Reads 4 bytes and writes 2 per cached element pair (k, v); about 40 flops an element.  Bound by memory where
// prompts are long, by latency for a generated token (its page is read only when it fills).
template <typename T, int D, int P, bool FP8>
__global__ __launch_bounds__(kPagedThreads) void paged_append_kernel(AppendArgs a) {
  typedef PageWork<T, D, P, FP8> W;
  constexpr int LPR = W::LPR, RP = W::RP, PASSES = W::PASSES;
  constexpr uint32_t kExponent = __is_same(T, __bf16) ? 0x7F80u : 0x7C00u;
  constexpr uint32_t kNanPair = __is_same(T, __bf16) ? 0x7FC07FC0u : 0x7E007E00u;
  constexpr int VS = 68;                                  // bytes of a channel's run in LDS: 64 and a word against bank conflicts
  __shared__ __align__(16) uint8_t s_v[(P / 64) * D * VS];
  __shared__ float s_amax[2][4];
  __shared__ int s_bad[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, unit = tid % LPR;
  const RowLayout l = row_layout(unit, a.rot.rot_dim, a.rot.interleaved);
  const float inv_dim = 1.0f / D;

  if ((int)blockIdx.x >= a.page_blocks) {                 // query rows
    const int item = (int)blockIdx.x - a.page_blocks;
    const int group = item % a.q_head_groups;
    const long row = (long)(item / a.q_head_groups) * RP + tid / LPR;
    bool live = row < a.bt.rows;
    int place = 0;
    if (live) {
      const int b = item_owner(a.bt.starts, a.bt.rows, a.bt.batch, (int)row, 1, 1, 0);
      const Sequence s = sequence_of(a.bt, P, b);
      live = row < s.row0 + s.n;                          // rows behind the last sequence's stay as they are
      place = s.len - s.n + (int)(row - s.row0);
    }
    float cs[8], sn[8];
    RowLayout turned = l;
    if (!live) turned.pair0 = -1;
    unit_turns(a.rot, turned, row, place, cs, sn);
    const int h0 = group * a.q_heads_per_group;
    rotate_row<T, LPR>(a.q.data + row * a.q.token_stride, a.q_out.data + row * a.q_out.token_stride, a.q.head_stride, a.q_out.head_stride, h0,
                       min(h0 + a.q_heads_per_group, a.q.heads), live, l, a.norm.q_weight, a.norm.eps, inv_dim, cs, sn, a.rot.interleaved);
    return;
  }

  const int item = (int)blockIdx.x / a.head_groups, h_first = ((int)blockIdx.x % a.head_groups) * a.heads_per_group;
  const int h_last = min(h_first + a.heads_per_group, a.c.kv_heads);
  const int b = item_owner(a.bt.starts, a.bt.rows, a.bt.batch, item, 1, P, 2);
  const Sequence s = sequence_of(a.bt, P, b);
  if (s.n == 0 || s.len == 0) return;
  const int old = s.len - s.n;                            // may be negative: those rows are left out
  const int first_page = max(old, 0) / P, last_page = (s.len - 1) / P;
  int page = first_page + item - item_first(a.bt.starts, a.bt.rows, b, 1, P, 2);
  if (page < first_page || page > last_page) return;
  const int slot = a.bt.tail_slots ? a.bt.tail_slots[b] : b;
  const bool slot_ok = slot >= 0 && slot < a.c.slots;
  // Where a page fills whose first rows lie in the tail and rows remain behind it, those go into the same tail: the
  // workgroup that reads the old rows also writes the new ones, afterwards.
  const bool tail_read_first = old > first_page * P && (first_page + 1) * P <= s.len;
  const bool partial_last = s.len % P != 0;
  if (page == last_page && page != first_page && partial_last && tail_read_first) return;
  const bool then_last = page == first_page && tail_read_first && partial_last;

  float wk[16];
  if (a.norm.k_weight) {
    unpack8<T>(*reinterpret_cast<const u32x4*>(a.norm.k_weight + l.at0), wk);
    unpack8<T>(*reinterpret_cast<const u32x4*>(a.norm.k_weight + l.at1), wk + 8);
  }
  for (int part = 0; part < (then_last ? 2 : 1); ++part) {
    if (part) {
      page = last_page;
      __syncthreads();                                    // the old tail rows of all heads have been read
    }
    const int base = page * P;                            // first token of the page
    const bool full = base + P <= s.len;
    const int page_id = full ? a.bt.page_table[(long)b * a.bt.table_stride + page] : 0;
    if (full ? (page_id < 0 || page_id >= a.c.pages) : !slot_ok) continue;   // no such page: its rows are dropped
    const int lo = max(old, base) - base, hi = min(s.len - base, P);         // new rows of the page: [lo, hi)
    float cs[PASSES][8], sn[PASSES][8];
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
      const int r = i * RP + tid / LPR;
      RowLayout turned = l;
      if (r < lo || r >= hi) turned.pair0 = -1;
      unit_turns(a.rot, turned, s.row0 + (base + r - old), base + r, cs[i], sn[i]);
    }
    for (int h = h_first; h < h_last; ++h) {
      const long tail_block = ((long)slot * a.c.kv_heads + h) * P * D;
      uint16_t* const k_tail = a.c.k_tail + tail_block;
      uint16_t* const v_tail = a.c.v_tail + tail_block;
      // ---- rows ----
      u32x4 kr[PASSES][2], vr[PASSES][2];
#pragma unroll
      for (int i = 0; i < PASSES; ++i) {
        const int r = i * RP + tid / LPR, rv = PASSES * (tid / LPR) + i;
        kr[i][0] = kr[i][1] = vr[i][0] = vr[i][1] = u32x4{0, 0, 0, 0};
        if (r >= lo && r < hi) {
          const uint16_t* src = a.k.data + (s.row0 + (base + r - old)) * a.k.token_stride + h * a.k.head_stride;
          kr[i][0] = *reinterpret_cast<const u32x4*>(src + l.at0);
          kr[i][1] = *reinterpret_cast<const u32x4*>(src + l.at1);
        } else if (r < lo && full && slot_ok) {
          kr[i][0] = *reinterpret_cast<const u32x4*>(k_tail + (long)r * D + l.at0);
          kr[i][1] = *reinterpret_cast<const u32x4*>(k_tail + (long)r * D + l.at1);
        }
        if (rv >= lo && rv < hi) {
          const uint16_t* src = a.v.data + (s.row0 + (base + rv - old)) * a.v.token_stride + h * a.v.head_stride + 16 * unit;
          vr[i][0] = *reinterpret_cast<const u32x4*>(src);
          vr[i][1] = *reinterpret_cast<const u32x4*>(src + 8);
        }
      }
      if (full && slot_ok) {                              // old value rows: from the channel runs of the tail
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
          const int rv = PASSES * (tid / LPR) + i;
          if (rv < lo) {
            const uint16_t* src = v_tail + (long)(rv / 64) * 64 * D + 16 * unit * 64 + rv % 64;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              vr[i][0][j / 2] |= (uint32_t)src[j * 64] << (16 * (j & 1));
              vr[i][1][j / 2] |= (uint32_t)src[(8 + j) * 64] << (16 * (j & 1));
            }
          }
        }
      }
      // ---- keys: norm, rotation, the rounding the tail keeps ----
#pragma unroll
      for (int i = 0; i < PASSES; ++i) {
        const int r = i * RP + tid / LPR;
        float x[16];
        unpack8<T>(kr[i][0], x);
        unpack8<T>(kr[i][1], x + 8);
        if (a.norm.k_weight) norm_unit<LPR>(x, wk, a.norm.eps, inv_dim);
        if (l.pair0 >= 0) turn_unit(x, cs[i], sn[i], a.rot.interleaved);
        const bool fresh = r >= lo && r < hi;             // the tail's rows are ready
        const u32x4 y0 = pack8<T>(x), y1 = pack8<T>(x + 8);
        if (fresh) { kr[i][0] = y0; kr[i][1] = y1; }
      }
      // ---- rows that are not finite: NaN keys, zero values.  Key and value pieces of a row lie in different threads ----
      int bad = 0;
#pragma unroll
      for (int i = 0; i < PASSES; ++i) {
        bool k_ok = true, v_ok = true;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          k_ok &= finite_pair(kr[i][0][j], kExponent) & finite_pair(kr[i][1][j], kExponent);
          v_ok &= finite_pair(vr[i][0][j], kExponent) & finite_pair(vr[i][1][j], kExponent);
        }
        bad |= (!k_ok | !v_ok);
      }
      if (__syncthreads_or(bad)) {                        // (no row of ordinary data comes here)
        uint8_t* const flag = s_v;                        // one byte a row
        for (int r = tid; r < P; r += kPagedThreads) flag[r] = 0;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
          bool k_ok = true, v_ok = true;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            k_ok &= finite_pair(kr[i][0][j], kExponent) & finite_pair(kr[i][1][j], kExponent);
            v_ok &= finite_pair(vr[i][0][j], kExponent) & finite_pair(vr[i][1][j], kExponent);
          }
          if (!k_ok) flag[i * RP + tid / LPR] = 1;
          if (!v_ok) flag[PASSES * (tid / LPR) + i] = 1;
        }
        __syncthreads();
        bad = 0;
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
          if (flag[i * RP + tid / LPR]) {
            bad = 1;
            const uint32_t fill = full ? 0u : kNanPair;   // in a full page the scale says it
            kr[i][0] = kr[i][1] = u32x4{fill, fill, fill, fill};
          }
          if (flag[PASSES * (tid / LPR) + i]) vr[i][0] = vr[i][1] = u32x4{0, 0, 0, 0};
        }
        __syncthreads();
      }
      if (!full) {
        // ---- the page goes on: its new rows into the tail ----
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
          const int r = i * RP + tid / LPR, rv = PASSES * (tid / LPR) + i;
          if (r >= lo && r < hi) {
            *reinterpret_cast<u32x4*>(k_tail + (long)r * D + l.at0) = kr[i][0];
            *reinterpret_cast<u32x4*>(k_tail + (long)r * D + l.at1) = kr[i][1];
          }
          if (rv >= lo && rv < hi) {
            uint16_t* dst = v_tail + (long)(rv / 64) * 64 * D + 16 * unit * 64 + rv % 64;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              dst[j * 64] = (uint16_t)(vr[i][0][j / 2] >> (16 * (j & 1)));
              dst[(8 + j) * 64] = (uint16_t)(vr[i][1][j / 2] >> (16 * (j & 1)));
            }
          }
        }
        continue;
      }
      // ---- the page is full: one step for the block's keys, one for its values ----
      float k_amax = 0.f, v_amax = 0.f;
#pragma unroll
      for (int i = 0; i < PASSES; ++i) {
        float x[16];
        unpack8<T>(kr[i][0], x);
        unpack8<T>(kr[i][1], x + 8);
#pragma unroll
        for (int j = 0; j < 16; ++j) k_amax = fmaxf(k_amax, fabsf(x[j]));
        unpack8<T>(vr[i][0], x);
        unpack8<T>(vr[i][1], x + 8);
#pragma unroll
        for (int j = 0; j < 16; ++j) v_amax = fmaxf(v_amax, fabsf(x[j]));
      }
      for (int o = 32; o; o >>= 1) {
        k_amax = fmaxf(k_amax, __shfl_xor(k_amax, o));
        v_amax = fmaxf(v_amax, __shfl_xor(v_amax, o));
      }
      const int any_bad = __any(bad);
      if (lane == 0) { s_amax[0][wave] = k_amax; s_amax[1][wave] = v_amax; s_bad[wave] = any_bad; }
      __syncthreads();
      k_amax = fmaxf(fmaxf(s_amax[0][0], s_amax[0][1]), fmaxf(s_amax[0][2], s_amax[0][3]));
      v_amax = fmaxf(fmaxf(s_amax[1][0], s_amax[1][1]), fmaxf(s_amax[1][2], s_amax[1][3]));
      const bool nan_block = s_bad[0] | s_bad[1] | s_bad[2] | s_bad[3] | (lo > 0 && !slot_ok);   // (rows of no slot)
      const float rk = inverse_step<FP8>(k_amax), rv_step = inverse_step<FP8>(v_amax);
      const long block = (long)page_id * a.c.kv_heads + h;
      if (tid == 0) {
        a.c.k_scales[block] = nan_block ? __builtin_nanf("") : rk > 0.f ? 1.f / rk : 1.f;
        a.c.v_scales[block] = rv_step > 0.f ? 1.f / rv_step : 1.f;
      }
      uint8_t* const k_codes = a.c.k_codes + block * P * D;
      uint8_t* const v_codes = a.c.v_codes + block * P * D;
      uint32_t vc[PASSES][4];
#pragma unroll
      for (int i = 0; i < PASSES; ++i) {
        const int r = i * RP + tid / LPR;
        float x[16];
        unpack8<T>(kr[i][0], x);
        unpack8<T>(kr[i][1], x + 8);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const u32x2 w = {codes4<FP8>(x[8 * j] * rk, x[8 * j + 1] * rk, x[8 * j + 2] * rk, x[8 * j + 3] * rk),
                           codes4<FP8>(x[8 * j + 4] * rk, x[8 * j + 5] * rk, x[8 * j + 6] * rk, x[8 * j + 7] * rk)};
          *reinterpret_cast<u32x2*>(k_codes + (long)r * D + (j ? l.at1 : l.at0)) = w;
        }
        unpack8<T>(vr[i][0], x);
        unpack8<T>(vr[i][1], x + 8);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          vc[i][j] = codes4<FP8>(x[4 * j] * rv_step, x[4 * j + 1] * rv_step, x[4 * j + 2] * rv_step, x[4 * j + 3] * rv_step);
      }
      // values channel by channel: the thread's rows are neighbours of a channel's run
      const int rv0 = PASSES * (tid / LPR);
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        uint8_t* dst = s_v + (rv0 / 64) * D * VS + (16 * unit + j) * VS + rv0 % 64;
        uint32_t w = 0;
#pragma unroll
        for (int i = 0; i < PASSES; ++i) w |= (vc[i][j / 4] >> (8 * (j & 3)) & 255u) << (8 * i);
        if constexpr (PASSES == 4) *reinterpret_cast<uint32_t*>(dst) = w;
        else if constexpr (PASSES == 2) *reinterpret_cast<uint16_t*>(dst) = (uint16_t)w;
        else *dst = (uint8_t)w;
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < P * D / 16 / kPagedThreads; ++i) {
        const int piece = i * kPagedThreads + tid;        // 16 codes of a channel's run
        const uint32_t* src = reinterpret_cast<const uint32_t*>(s_v + (piece / 4) * VS + 16 * (piece % 4));
        *reinterpret_cast<u32x4*>(v_codes + 16l * piece) = u32x4{src[0], src[1], src[2], src[3]};
      }
      // (the next head's first barrier, or the next page's, keeps s_v and s_amax until all have read them)
    }
  }
}

struct ReadArgs {
  dq_paged_cache c;
  dq_paged_batch bt;
  const int32_t* first;
  const int32_t* out_starts;
  dq_heads k, v;
};

// One workgroup per (page, kv head).  Reads one byte and writes two per element.
template <typename T, int D, int P, bool FP8>
__global__ __launch_bounds__(kPagedThreads) void paged_read_kernel(ReadArgs a) {
  constexpr int LPR = D / 16, RP = kPagedThreads / LPR, PASSES = P / RP;
  constexpr int RS = D / 2 + 1;                           // words of a token's row in LDS, an odd number
  __shared__ uint32_t s_v[64 * RS];
  const int tid = threadIdx.x, h = blockIdx.y;
  const int b = item_owner(a.out_starts, a.bt.rows, a.bt.batch, (int)blockIdx.x, 1, P, 2);
  const int len = min(max(a.bt.seq_lens[b], 0), a.bt.table_width * P);
  const int first = a.first ? max(a.first[b], 0) : 0;
  const int page = first / P + (int)blockIdx.x - item_first(a.out_starts, a.bt.rows, b, 1, P, 2);
  const int base = page * P;
  if (first >= len || page < first / P || base >= len) return;
  const long out0 = (long)a.out_starts[b] - first;        // row of token 0
  const long row_end = min((long)a.bt.rows, (long)a.out_starts[b + 1]);
  const bool full = base + P <= len;
  const int id = full ? a.bt.page_table[(long)b * a.bt.table_stride + page] : a.bt.tail_slots ? a.bt.tail_slots[b] : b;
  const bool ok = id >= 0 && id < (full ? a.c.pages : a.c.slots);
  const long block = (long)(ok ? id : 0) * a.c.kv_heads + h;
  const float nan = __builtin_nanf("");
  const float ks = full ? (ok ? a.c.k_scales[block] : nan) : (ok ? 1.f : nan);
  const float vs = full ? (ok ? a.c.v_scales[block] : nan) : (ok ? 1.f : nan);
  const int lo = max(first - base, 0), hi = min(len - base, P);
  const int unit = tid % LPR;
  auto live = [&](int r) { const long at = out0 + base + r; return r >= lo && r < hi && at >= 0 && at < row_end; };
#pragma unroll
  for (int i = 0; i < PASSES; ++i) {
    const int r = i * RP + tid / LPR;
    if (!live(r)) continue;
    float x[16];
    if (full) {
      const u32x4 w = *reinterpret_cast<const u32x4*>(a.c.k_codes + block * P * D + (long)r * D + 16 * unit);
#pragma unroll
      for (int j = 0; j < 4; ++j) values4<FP8>(w[j], x + 4 * j);
    } else {
      const uint16_t* src = a.c.k_tail + block * P * D + (long)r * D + 16 * unit;
      unpack8<T>(*reinterpret_cast<const u32x4*>(src), x);
      unpack8<T>(*reinterpret_cast<const u32x4*>(src + 8), x + 8);
    }
#pragma unroll
    for (int j = 0; j < 16; ++j) x[j] *= ks;
    uint16_t* dst = a.k.data + (out0 + base + r) * a.k.token_stride + h * a.k.head_stride + 16 * unit;
    *reinterpret_cast<u32x4*>(dst) = pack8<T>(x);
    *reinterpret_cast<u32x4*>(dst + 8) = pack8<T>(x + 8);
  }
  // values: a thread takes two channels of four tokens and leaves a word (both channels) per token
  for (int run = 0; run < P / 64; ++run) {
    if (run) __syncthreads();
#pragma unroll
    for (int i = 0; i < D / 2 * 16 / kPagedThreads; ++i) {
      const int piece = i * kPagedThreads + tid, pair = piece / 16, t4 = 4 * (piece % 16);
      float x[4], y[4];
      const long at = block * P * D + (long)run * 64 * D + 2 * pair * 64 + t4;
      if (full) {
        values4<FP8>(*reinterpret_cast<const uint32_t*>(a.c.v_codes + at), x);
        values4<FP8>(*reinterpret_cast<const uint32_t*>(a.c.v_codes + at + 64), y);
      } else {
        const u32x2 u = *reinterpret_cast<const u32x2*>(a.c.v_tail + at), w = *reinterpret_cast<const u32x2*>(a.c.v_tail + at + 64);
        unpack2<T>(u.x, x[0], x[1]);
        unpack2<T>(u.y, x[2], x[3]);
        unpack2<T>(w.x, y[0], y[1]);
        unpack2<T>(w.y, y[2], y[3]);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) s_v[(t4 + j) * RS + pair] = pack2<T>(x[j] * vs, y[j] * vs);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 64 * D / 8 / kPagedThreads; ++i) {
      const int piece = i * kPagedThreads + tid, r = piece / (D / 8), c8 = piece % (D / 8);
      if (!live(run * 64 + r)) continue;
      const uint32_t* src = s_v + r * RS + 4 * c8;
      *reinterpret_cast<u32x4*>(a.v.data + (out0 + base + run * 64 + r) * a.v.token_stride + h * a.v.head_stride + 8 * c8) =
          u32x4{src[0], src[1], src[2], src[3]};
    }
  }
}

template <template <typename, int, int, bool> class Launch, typename... Args>
static void for_format(const dq_paged_cache* c, Args... args) {
  const bool bf = c->dtype == DQ_BF16, fp8 = c->codes == DQ_CODES_E4M3, wide = c->head_dim == 128, big = c->page_tokens == 128;
#define DQ_ONE(T, D, P, F) Launch<T, D, P, F>::go(args...)
#define DQ_CODE(T, D, P) do { if (fp8) DQ_ONE(T, D, P, true); else DQ_ONE(T, D, P, false); } while (0)
#define DQ_PAGE(T, D) do { if (big) DQ_CODE(T, D, 128); else DQ_CODE(T, D, 64); } while (0)
#define DQ_DIM(T) do { if (wide) DQ_PAGE(T, 128); else DQ_PAGE(T, 64); } while (0)
  if (bf) DQ_DIM(__bf16); else DQ_DIM(_Float16);
#undef DQ_ONE
#undef DQ_CODE
#undef DQ_PAGE
#undef DQ_DIM
}

template <typename T, int D, int P, bool F> struct LaunchAppend {
  static void go(AppendArgs a, dim3 grid, hipStream_t st) {
    hipLaunchKernelGGL((paged_append_kernel<T, D, P, F>), grid, dim3(kPagedThreads), 0, st, a);
  }
};
template <typename T, int D, int P, bool F> struct LaunchRead {
  static void go(ReadArgs a, dim3 grid, hipStream_t st) {
    hipLaunchKernelGGL((paged_read_kernel<T, D, P, F>), grid, dim3(kPagedThreads), 0, st, a);
  }
};

}  // namespace dq

using namespace dq;

extern "C" int32_t dq_paged_append(const dq_paged_cache* cache, const dq_paged_batch* batch, const dq_heads* k, const dq_heads* v,
                                   const dq_heads* q, const dq_heads* q_out, const dq_head_norm* norm, const dq_rotary* rot,
                                   void* hip_stream) {
  if (!paged_cache_ok(cache) || !paged_batch_ok(batch, cache, true) || (!q) != (!q_out)) return DQ_EINVAL;
  if (!heads_ok(k, false) || !heads_ok(v, false) || k->heads != cache->kv_heads || v->heads != cache->kv_heads) return DQ_EINVAL;
  if (q && (!heads_ok(q, false) || !heads_ok(q_out, false) || q->heads != q_out->heads)) return DQ_EINVAL;
  if (!norm_ok(norm) || !rotary_ok(rot, cache->head_dim, batch->rows, false)) return DQ_EINVAL;
  if (batch->rows == 0) return DQ_OK;
  AppendArgs a = {};
  a.c = *cache; a.bt = *batch; a.k = *k; a.v = *v;
  if (q) { a.q = *q; a.q_out = *q_out; }
  if (norm) a.norm = *norm;
  if (rot) a.rot = *rot;
  const int rows_per_block = kPagedThreads / (cache->head_dim / 16);
  const long items = batch->rows / cache->page_tokens + 2l * batch->batch;
  const long q_items = q ? (batch->rows + rows_per_block - 1) / rows_per_block : 0;
  // Heads that share a page's angles: four where the pages alone fill the chip.
  int per = 4, q_per = 8;
  while (per > 1 && items * ((cache->kv_heads + per - 1) / per) < 1024) per /= 2;
  while (q && q_per > 1 && q_items * ((q->heads + q_per - 1) / q_per) < 1024) q_per /= 2;
  a.heads_per_group = per;
  a.head_groups = (cache->kv_heads + per - 1) / per;
  a.q_heads_per_group = q_per;
  a.q_head_groups = q ? (q->heads + q_per - 1) / q_per : 1;
  const long page_blocks = items * a.head_groups, blocks = page_blocks + q_items * a.q_head_groups;
  if (blocks >= (1l << 31)) return DQ_EINVAL;
  a.page_blocks = (int)page_blocks;
  for_format<LaunchAppend>(cache, a, dim3((unsigned)blocks), (hipStream_t)hip_stream);
  DQ_HIP_CHECK(hipGetLastError());
  return DQ_OK;
}

extern "C" int32_t dq_paged_read(const dq_paged_cache* cache, const dq_paged_batch* batch, const int32_t* first, const int32_t* out_starts,
                                 const dq_heads* k_out, const dq_heads* v_out, void* hip_stream) {
  if (!paged_cache_ok(cache) || !paged_batch_ok(batch, cache, false) || !out_starts) return DQ_EINVAL;
  if (!heads_ok(k_out, false) || !heads_ok(v_out, false) || k_out->heads != cache->kv_heads || v_out->heads != cache->kv_heads) return DQ_EINVAL;
  if (cache->kv_heads > kMaxGridY) return DQ_EINVAL;
  if (batch->rows == 0) return DQ_OK;
  ReadArgs a = {*cache, *batch, first, out_starts, *k_out, *v_out};
  const long items = batch->rows / cache->page_tokens + 2l * batch->batch;
  if (items >= (1l << 31)) return DQ_EINVAL;
  for_format<LaunchRead>(cache, a, dim3((unsigned)items, (unsigned)cache->kv_heads), (hipStream_t)hip_stream);
  DQ_HIP_CHECK(hipGetLastError());
  return DQ_OK;
}
