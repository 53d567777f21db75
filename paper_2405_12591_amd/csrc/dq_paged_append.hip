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

// Largest magnitudes as 16-bit patterns, which order as integers; those from `exponent` on are not finite.  Both values of
// a word at a time.
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t larger_pair(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}
__device__ __forceinline__ uint32_t largest(const u32x4& v, uint32_t m) {
#pragma unroll
  for (int j = 0; j < 4; ++j) m = larger_pair(m, v[j] & 0x7FFF7FFFu);
  return m;
}
__device__ __forceinline__ uint32_t higher_half(uint32_t m) { return max(m >> 16, m & 0xFFFFu); }
template <int CTRL>
__device__ __forceinline__ uint32_t larger_of_lanes(uint32_t x) {
  return larger_pair(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, true));
}

// Pages are worked by one workgroup per (page, group of kv heads); a thread has 16 channels of one key row, laid for the
// rotation, and 8 channels of two neighbouring value rows, as the value layout wants them.  The angles of a key row's
// unit are formed once and kept for all heads of the group.
// Reads 4 bytes and writes 2 per cached element pair (k, v); about 40 flops an element.  Bound by memory where
// prompts are long: 28.6 thousand tokens of 32 heads of 128 channels, pages of 128, 190 us, 3.7 TB/s (its workgroups of 16 waves
// wait at two barriers a head, one a compute unit), and 272 us with 32 query heads, 4.3 TB/s.  By latency for a generated token
// (its page is read only when it fills): 7 us for 16 sequences.  By both in between: of the 24 us for 7 thousand rows
// of 8 heads 10 are vector instructions, most of them angles, which few rows share with few heads.
template <typename T, int D, int P, bool FP8, bool INTERLEAVED>
__global__ __launch_bounds__(P * D / 16, 4) void paged_append_kernel(AppendArgs a) {
  constexpr int THREADS = P * D / 16, LPR = D / 16, RP = P, WAVES = THREADS / 64;
  constexpr uint32_t kExponent = __is_same(T, __bf16) ? 0x7F80u : 0x7C00u;
  constexpr uint32_t kNanPair = __is_same(T, __bf16) ? 0x7FC07FC0u : 0x7E007E00u;
  constexpr int VS = 68;                                  // bytes of a channel's run in LDS: 64 and a word against bank conflicts
  __shared__ __align__(16) uint8_t s_v[(P / 64) * D * VS];
  __shared__ f32x4 s_turn[4][THREADS];                    // the thread's eight cosines and sines, for all heads of its group (16 registers less)
  __shared__ uint32_t s_amax[2][WAVES];
  const int thread = threadIdx.x;
  constexpr float inv_dim = 1.0f / D;

  if ((int)blockIdx.x >= a.page_blocks) {                 // query rows
    const int tid = thread;
    const RowLayout l = row_layout(tid % LPR, a.rot.rot_dim, INTERLEAVED);
    const int item = (int)blockIdx.x - a.page_blocks;
    const int group = item % a.q_head_groups;
    const long row = (long)(item / a.q_head_groups) * RP + tid / LPR;
    bool live = row < a.bt.rows;
    int place = 0, b = (int)row;
    if (a.bt.starts) {                                    // the row's sequence: bisection in LDS, a row a thread
      int32_t* const known = reinterpret_cast<int32_t*>(s_v);
      constexpr int kKnown = sizeof(s_v) / 4;
      const int stride = (a.bt.batch + kKnown - 1) / kKnown;   // more sequences than LDS holds: every stride-th, then in memory
      for (int i = tid; i * stride < a.bt.batch; i += THREADS) known[i] = a.bt.starts[i * stride];
      __syncthreads();
      int lo = 0, hi = (a.bt.batch - 1) / stride;
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (min(max(known[mid], 0), a.bt.rows) <= row) lo = mid; else hi = mid - 1;
      }
      lo *= stride;
      hi = min(lo + stride, a.bt.batch) - 1;
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (min(max(a.bt.starts[mid], 0), a.bt.rows) <= row) lo = mid; else hi = mid - 1;
      }
      b = lo;
    }
    if (live) {
      const Sequence s = sequence_of(a.bt, P, b);
      live = row >= s.row0 && row < s.row0 + s.n;         // rows before the first sequence's and behind the last's stay as they are
      place = s.old + (int)(row - s.row0);
    }
    RowLayout turned = l;
    if (!live) turned.pair0 = -1;
    UnitTurns ut;
    load_turns(a.rot, turned, row, place, ut);
    const int h0 = group * a.q_heads_per_group;
    const uint16_t* const q = a.q.data + row * a.q.token_stride;
    u32x4 v[2] = {};
    if (live) load_unit(v, q + h0 * a.q.head_stride, l);
    float cs[8], sn[8];
    make_turns(turned, ut, cs, sn);
    rotate_row<T, LPR, INTERLEAVED>(v, q, a.q_out.data + row * a.q_out.token_stride, a.q.head_stride, a.q_out.head_stride, h0,
                                    min(h0 + a.q_heads_per_group, a.q.heads), live, l, a.norm.q_weight, a.norm.eps, inv_dim, cs, sn);
    return;
  }

  const int item = (int)blockIdx.x / a.head_groups, h_first = ((int)blockIdx.x % a.head_groups) * a.heads_per_group;
  const int h_last = min(h_first + a.heads_per_group, a.c.kv_heads);
  const int b = item_owner(a.bt.starts, a.bt.rows, a.bt.batch, item, 1, P, 2);
  const Sequence s = sequence_of_wave(a.bt, P, b);
  if (s.n == 0 || s.len == 0) return;
  const int old = s.old;                                  // rows of tokens before 0 or past the table are left out
  const int first_page = max(old, 0) / P, last_page = (s.len - 1) / P;
  int page = first_page + item - item_first(a.bt.starts, a.bt.rows, b, 1, P, 2);
  if (page < first_page || page > last_page) return;
  const int slot = a.bt.tail_slots ? __builtin_amdgcn_readfirstlane(a.bt.tail_slots[b]) : b;
  const bool slot_ok = slot >= 0 && slot < a.c.slots;
  // Where a page fills whose first rows lie in the tail and rows remain behind it, those go into the same tail: the
  // workgroup that reads the old rows also writes the new ones, afterwards.
  const bool tail_read_first = old > first_page * P && (first_page + 1) * P <= s.len;
  const bool partial_last = s.len % P != 0;
  if (page == last_page && page != first_page && partial_last && tail_read_first) return;
  const bool then_last = page == first_page && tail_read_first && partial_last;

  const int tid = thread, lane = tid & 63, wave = tid >> 6;
  const RowLayout l = row_layout(tid % LPR, a.rot.rot_dim, INTERLEAVED);
  const int r = tid / LPR, v8 = tid % (D / 8), rv = 2 * (tid / (D / 8));   // key row; value channels and first row
  u32x4 wk[2] = {};
  if (a.norm.k_weight) load_unit(wk, a.norm.k_weight, l);

  // The thread's new rows of a page: where they come from, and the angles of the key row (to LDS).
  struct NewRows {
    const uint16_t *k, *v;                                // of kv head 0
    bool k_new, v_new[2];
  };
  auto new_rows = [&](int base, int lo, int hi) __attribute__((always_inline)) {
    NewRows n;
    n.k_new = r >= lo && r < hi;
    n.v_new[0] = rv >= lo && rv < hi;
    n.v_new[1] = rv + 1 >= lo && rv + 1 < hi;
    n.k = a.k.data + (s.row0 + (base + r - old)) * a.k.token_stride;
    n.v = a.v.data + (s.row0 + (base + rv - old)) * a.v.token_stride + 8 * v8;
    return n;
  };
  auto angles = [&](int base, const NewRows& n) __attribute__((always_inline)) {
    RowLayout turned = l;
    if (!n.k_new) turned.pair0 = -1;
    UnitTurns ut;
    float cs[8], sn[8];
    load_turns(a.rot, turned, s.row0 + (base + r - old), base + r, ut);
    make_turns(turned, ut, cs, sn);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      s_turn[i][tid] = f32x4{cs[4 * i], cs[4 * i + 1], cs[4 * i + 2], cs[4 * i + 3]};
      s_turn[2 + i][tid] = f32x4{sn[4 * i], sn[4 * i + 1], sn[4 * i + 2], sn[4 * i + 3]};
    }
  };
  auto load_rows = [&](const NewRows& n, int h, u32x4 (&kn)[2], u32x4 (&vn)[2]) __attribute__((always_inline)) {
    if (n.k_new) load_unit(kn, n.k + h * a.k.head_stride, l);
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (n.v_new[i]) vn[i] = *reinterpret_cast<const u32x4*>(n.v + i * a.v.token_stride + h * a.v.head_stride);
  };
  auto ready_key = [&](u32x4 (&kr)[2]) __attribute__((always_inline)) {   // norm, rotation, the rounding the tail keeps
    float cs[8], sn[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      cs[i] = s_turn[i / 4][tid][i % 4];
      sn[i] = s_turn[2 + i / 4][tid][i % 4];
    }
    ready_unit<T, LPR, INTERLEAVED>(kr, wk, a.norm.k_weight != nullptr, l.pair0 >= 0, a.norm.eps, inv_dim, cs, sn);
  };
  // Largest magnitudes of the workgroup's key and value pieces, as patterns in the high and low half.
  auto amax_of = [&](const u32x4 (&kr)[2], const u32x4 (&vr)[2], int buf) __attribute__((always_inline)) {
    uint32_t m = higher_half(largest(kr[1], largest(kr[0], 0))) << 16 | higher_half(largest(vr[1], largest(vr[0], 0)));
    m = larger_of_lanes<0xB1>(m);
    m = larger_of_lanes<0x4E>(m);
    m = larger_of_lanes<0x141>(m);
    m = larger_of_lanes<0x140>(m);
    m = larger_pair(m, (uint32_t)__shfl_xor((int)m, 16));
    m = larger_pair(m, (uint32_t)__shfl_xor((int)m, 32));
    if (lane == 0) s_amax[buf][wave] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) m = larger_pair(m, s_amax[buf][w]);
    return m;
  };
  // Rows that are not finite become NaN keys (`fill`) and zero values (no row of ordinary data comes here).  A row's key and
  // value pieces lie in different threads.
  auto drop_rows = [&](u32x4 (&kr)[2], u32x4 (&vr)[2], uint32_t fill) __attribute__((always_inline)) {
    uint8_t* const flag = s_v;                            // one byte a row
    if (tid < P) flag[tid] = 0;
    __syncthreads();
    if (higher_half(largest(kr[1], largest(kr[0], 0))) >= kExponent) flag[r] = 1;
    if (higher_half(largest(vr[0], 0)) >= kExponent) flag[rv] = 1;
    if (higher_half(largest(vr[1], 0)) >= kExponent) flag[rv + 1] = 1;
    __syncthreads();
    if (flag[r]) kr[0] = kr[1] = u32x4{fill, fill, fill, fill};
    if (flag[rv]) vr[0] = u32x4{0, 0, 0, 0};
    if (flag[rv + 1]) vr[1] = u32x4{0, 0, 0, 0};
    __syncthreads();
  };
  const int v_at = (rv / 64) * 64 * D + 8 * v8 * 64 + rv % 64;   // the first row's place in a block of the value layout; + 64 j: channel 8 v8 + j

  if ((page + 1) * P <= s.len) {
    // ---- a full page ----
    const int base = page * P, lo = max(old - base, 0);   // rows from lo on are new, the others in the tail
    const int page_id = a.bt.page_table[(long)b * a.bt.table_stride + page];
    if (page_id >= 0 && page_id < a.c.pages) {            // no such page: its rows are dropped
      const NewRows rows = new_rows(base, lo, P);
      angles(base, rows);
      u32x4 kn[2] = {}, vn[2] = {};                       // the head to come
      load_rows(rows, h_first, kn, vn);
      for (int h = h_first; h < h_last; ++h) {
        u32x4 kr[2] = {kn[0], kn[1]}, vr[2] = {vn[0], vn[1]};
        if (h + 1 < h_last) load_rows(rows, h + 1, kn, vn);   // on their way while this head is worked
        if (lo > 0 && slot_ok) {                          // old rows; the values' from the channel runs, both rows in a load
          const long tail_block = ((long)slot * a.c.kv_heads + h) * P * D;
          if (r < lo) load_unit(kr, a.c.k_tail + tail_block + (long)r * D, l);
          if (rv < lo) {
            const uint32_t keep0 = 0xFFFFu, keep1 = rv + 1 < lo ? 0xFFFF0000u : 0u;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const uint32_t w = *reinterpret_cast<const uint32_t*>(a.c.v_tail + tail_block + v_at + j * 64), x = w & keep0, y = w & keep1;
              vr[0][j / 2] |= (j & 1) ? x << 16 : x;
              vr[1][j / 2] |= (j & 1) ? y : y >> 16;
            }
          }
        }
        if (rows.k_new) ready_key(kr);
        // one step for the block's keys, one for its values
        uint32_t top = amax_of(kr, vr, 0);
        bool nan_block = lo > 0 && !slot_ok;              // (rows of no slot)
        if (higher_half(top) >= kExponent) {
          drop_rows(kr, vr, 0u);                          // (the scale says it)
          top = amax_of(kr, vr, 1);
          nan_block = true;
        }
        float k_amax, v_amax;
        unpack2<T>(top, v_amax, k_amax);
        const float k_step = inverse_step<FP8>(k_amax), v_step = inverse_step<FP8>(v_amax);
        const long block = (long)page_id * a.c.kv_heads + h;
        if (tid == 0) {
          a.c.k_scales[block] = nan_block ? __builtin_nanf("") : k_step > 0.f ? 1.f / k_step : 1.f;
          a.c.v_scales[block] = v_step > 0.f ? 1.f / v_step : 1.f;
        }
        uint8_t* const k_codes = a.c.k_codes + block * P * D + (long)r * D;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float x[8];
          unpack8<T>(kr[i], x);
          *reinterpret_cast<u32x2*>(k_codes + (i ? l.at1 : l.at0)) =
              u32x2{codes4<FP8>(x[0] * k_step, x[1] * k_step, x[2] * k_step, x[3] * k_step),
                    codes4<FP8>(x[4] * k_step, x[5] * k_step, x[6] * k_step, x[7] * k_step)};
        }
        // values channel by channel: the thread's two rows are neighbours of a channel's run
#pragma unroll
        for (int i = 0; i < 2; ++i) {                     // four channels at a time
          float x[4], y[4];
          unpack2<T>(vr[0][2 * i], x[0], x[1]);
          unpack2<T>(vr[0][2 * i + 1], x[2], x[3]);
          unpack2<T>(vr[1][2 * i], y[0], y[1]);
          unpack2<T>(vr[1][2 * i + 1], y[2], y[3]);
#pragma unroll
          for (int j = 0; j < 4; j += 2) {                // codes of (row, row + 1) of two channels
            const uint32_t w = codes4<FP8>(x[j] * v_step, y[j] * v_step, x[j + 1] * v_step, y[j + 1] * v_step);
            uint8_t* dst = s_v + ((rv / 64) * D + 8 * v8 + 4 * i + j) * VS + rv % 64;
            *reinterpret_cast<uint16_t*>(dst) = (uint16_t)w;
            *reinterpret_cast<uint16_t*>(dst + VS) = (uint16_t)(w >> 16);
          }
        }
        __syncthreads();
        const uint32_t* src = reinterpret_cast<const uint32_t*>(s_v + (tid / 4) * VS + 16 * (tid % 4));   // 16 codes of a channel's run
        *reinterpret_cast<u32x4*>(a.c.v_codes + block * P * D + 16l * tid) = u32x4{src[0], src[1], src[2], src[3]};
        // (the next head's first barrier keeps s_v and s_amax until all have read them)
      }
    }
    if (!then_last) return;
    page = last_page;
    __syncthreads();                                      // the old tail rows of all heads have been read
  }
  // ---- a page that goes on: its new rows into the tail ----
  if (!slot_ok) return;
  const int base = page * P;
  const NewRows rows = new_rows(base, max(old - base, 0), s.len - base);
  angles(base, rows);
  for (int h = h_first; h < h_last; ++h) {
    u32x4 kr[2] = {}, vr[2] = {};
    load_rows(rows, h, kr, vr);
    if (rows.k_new) ready_key(kr);
    if (__syncthreads_or(higher_half(largest(kr[1], largest(kr[0], largest(vr[1], largest(vr[0], 0))))) >= kExponent)) drop_rows(kr, vr, kNanPair);
    const long tail_block = ((long)slot * a.c.kv_heads + h) * P * D;
    if (rows.k_new) store_unit(a.c.k_tail + tail_block + (long)r * D, l, kr);
    uint16_t* const v_tail = a.c.v_tail + tail_block + v_at;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t x = vr[0][j / 2] >> (16 * (j & 1)) & 0xFFFFu, y = vr[1][j / 2] >> (16 * (j & 1)) & 0xFFFFu;
      if (rows.v_new[0] && rows.v_new[1]) *reinterpret_cast<uint32_t*>(v_tail + j * 64) = x | y << 16;
      else if (rows.v_new[0]) v_tail[j * 64] = (uint16_t)x;
      else if (rows.v_new[1]) v_tail[j * 64 + 1] = (uint16_t)y;
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

// One workgroup per (page, kv head), a page's heads neighbours in the grid: its rows are written by workgroups that run together.
// Reads one byte and writes two per element, 16 neighbouring bytes a lane, past the caches' own order.  Bound by memory: 28.6
// thousand tokens of 32 heads of 128 channels, 710 MB, 139 us, 5.1 TB/s (145 with the values asked for behind the keys, 150 with the heads
// far apart as well, 190 with 32 bytes a lane in two stores).
template <typename T, int D, int P, bool FP8>
__global__ __launch_bounds__(kPagedThreads) void paged_read_kernel(ReadArgs a) {
  constexpr int LPR = D / 8, RP = kPagedThreads / LPR, PASSES = P / RP, VP = D / 2 * 16 / kPagedThreads;
  constexpr int RS = D / 2 + 1;                           // words of a token's row in LDS, an odd number
  __shared__ uint32_t s_v[64 * RS];
  const int tid = threadIdx.x;
  const int h = (int)(blockIdx.x % (unsigned)a.c.kv_heads), item = (int)(blockIdx.x / (unsigned)a.c.kv_heads);
  const int b = item_owner(a.out_starts, a.bt.rows, a.bt.batch, item, 1, P, 2);
  const int len = min(max(a.bt.seq_lens[b], 0), a.bt.table_width * P);
  const int first = a.first ? max(a.first[b], 0) : 0;
  const int page = first / P + item - item_first(a.out_starts, a.bt.rows, b, 1, P, 2);
  const int base = page * P;
  if (first >= len || page < first / P || page > (len - 1) / P) return;
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
  // keys and the first run of values are asked for together
  u32x4 kw[PASSES] = {};
  u32x2 vw[VP][2];
  auto load_v = [&](int run) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < VP; ++i) {
      const int piece = i * kPagedThreads + tid;
      const long at = block * P * D + (long)run * 64 * D + 2 * (piece / 16) * 64 + 4 * (piece % 16);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        if (full) vw[i][j].x = *reinterpret_cast<const uint32_t*>(a.c.v_codes + at + 64 * j);
        else vw[i][j] = *reinterpret_cast<const u32x2*>(a.c.v_tail + at + 64 * j);
      }
    }
  };
#pragma unroll
  for (int i = 0; i < PASSES; ++i) {
    const int r = i * RP + tid / LPR;
    const long at = block * P * D + (long)r * D + 8 * unit;
    if (!live(r)) continue;
    if (full) {
      const u32x2 w = *reinterpret_cast<const u32x2*>(a.c.k_codes + at);
      kw[i].x = w.x;
      kw[i].y = w.y;
    } else {
      kw[i] = *reinterpret_cast<const u32x4*>(a.c.k_tail + at);
    }
  }
  load_v(0);
#pragma unroll
  for (int i = 0; i < PASSES; ++i) {
    const int r = i * RP + tid / LPR;
    if (!live(r)) continue;
    float x[8];
    if (full) {
      values4<FP8>(kw[i].x, x);
      values4<FP8>(kw[i].y, x + 4);
    } else {
      unpack8<T>(kw[i], x);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] *= ks;
    __builtin_nontemporal_store(pack8<T>(x), reinterpret_cast<u32x4*>(a.k.data + (out0 + base + r) * a.k.token_stride + h * a.k.head_stride + 8 * unit));
  }
  // values: a thread takes two channels of four tokens and leaves a word (both channels) per token
  for (int run = 0; run < P / 64; ++run) {
    if (run) {
      __syncthreads();
      load_v(run);
    }
#pragma unroll
    for (int i = 0; i < VP; ++i) {
      const int piece = i * kPagedThreads + tid, pair = piece / 16, t4 = 4 * (piece % 16);
      float x[4], y[4];
      if (full) {
        values4<FP8>(vw[i][0].x, x);
        values4<FP8>(vw[i][1].x, y);
      } else {
        unpack2<T>(vw[i][0].x, x[0], x[1]);
        unpack2<T>(vw[i][0].y, x[2], x[3]);
        unpack2<T>(vw[i][1].x, y[0], y[1]);
        unpack2<T>(vw[i][1].y, y[2], y[3]);
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
      uint16_t* const dst = a.v.data + (out0 + base + run * 64 + r) * a.v.token_stride + h * a.v.head_stride + 8 * c8;
      __builtin_nontemporal_store(u32x4{src[0], src[1], src[2], src[3]}, reinterpret_cast<u32x4*>(dst));
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
    if (a.rot.interleaved) hipLaunchKernelGGL((paged_append_kernel<T, D, P, F, true>), grid, dim3(P * D / 16), 0, st, a);
    else hipLaunchKernelGGL((paged_append_kernel<T, D, P, F, false>), grid, dim3(P * D / 16), 0, st, a);
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
  const long rows_per_block = cache->page_tokens;
  const long items = batch->rows / cache->page_tokens + 2l * batch->batch;
  const long q_items = q ? (batch->rows + rows_per_block - 1) / rows_per_block : 0;
  // Heads that share a page's angles: four where pages alone take the place of every resident workgroup (16 waves a compute
  // unit), fewer where they do not.  Pages of 128, 128 channels: 4096 tokens of 32 heads 26 us (34 with two heads a workgroup), 28
  // thousand of 8 heads 53 (63 with one).  Eight: 3 % faster with query rows beside large pages, up to 10 % slower on pages of 64.
  const int resident = (1 << 18) / (cache->page_tokens * cache->head_dim / 16);
  int per = 4, q_per = 8;
  auto groups = [](long heads, int each) { return (int)((heads + each - 1) / each); };
  while (per > 1 && items * groups(cache->kv_heads, per) < resident) per /= 2;
  while (q && q_per > 1 && q_items * groups(q->heads, q_per) < 1024) q_per /= 2;
  a.heads_per_group = per;
  a.head_groups = groups(cache->kv_heads, per);
  a.q_heads_per_group = q_per;
  a.q_head_groups = q ? groups(q->heads, q_per) : 1;
  const long page_blocks = items * a.head_groups, blocks = page_blocks + q_items * a.q_head_groups;
  if (blocks * (cache->page_tokens * cache->head_dim / 16) >= kMaxThreads) return DQ_EINVAL;
  a.page_blocks = (int)page_blocks;
  for_format<LaunchAppend>(cache, a, dim3((unsigned)blocks), (hipStream_t)hip_stream);
  DQ_HIP_CHECK(hipGetLastError());
  return DQ_OK;
}

extern "C" int32_t dq_paged_read(const dq_paged_cache* cache, const dq_paged_batch* batch, const int32_t* first, const int32_t* out_starts,
                                 const dq_heads* k_out, const dq_heads* v_out, void* hip_stream) {
  if (!paged_cache_ok(cache) || !paged_batch_ok(batch, cache, false) || !out_starts) return DQ_EINVAL;
  if (!heads_ok(k_out, false) || !heads_ok(v_out, false) || k_out->heads != cache->kv_heads || v_out->heads != cache->kv_heads) return DQ_EINVAL;
  if (batch->rows == 0) return DQ_OK;
  ReadArgs a = {*cache, *batch, first, out_starts, *k_out, *v_out};
  const long items = batch->rows / cache->page_tokens + 2l * batch->batch;
  if (items * cache->kv_heads >= kMaxThreads / kPagedThreads) return DQ_EINVAL;
  for_format<LaunchRead>(cache, a, dim3((unsigned)(items * cache->kv_heads)), (hipStream_t)hip_stream);
  DQ_HIP_CHECK(hipGetLastError());
  return DQ_OK;
}
