// What the two attention kernels over the paged cache share.
#pragma once
#include "dq_paged.h"

namespace dq {

struct PagedAttnArgs {
  dq_paged_cache c;
  dq_paged_batch bt;
  dq_heads q, out;
  int group;               // query heads per kv head
  int max_rows;            // rows of any sequence at most
  int window;              // 0: none
  int causal;
  float scale_log2;        // softmax scale * log2(e)
  int splits;              // prompt kernel: of every tile of rows
  int seq_tiles;           // prompt kernel: tiles of rows that every sequence gets, whatever it has (0: dealt by starts)
  int shares;              // decode kernel: slots that are meant to have equal shares of all tiles (0: a slot per sequence)
  float* partials;         // decode: [slot, kv head, column, D + 2]; prompt: [unit, split, D + 2, row]
  int32_t* counters;       // [unit], zero between calls
  int units;               // what the splits of are joined: (sequence, kv head), or (tile of query rows, kv head)
};

// Most splits of a sequence in the decode kernel: 1.2 sqrt(tiles), where a split's ticket and merge (2 us with up to four
// columns) outweigh shorter shares, 0.9 with more columns; none below 12 tiles, 24 with 64 channels or more columns.
__host__ __device__ inline int decode_cap(int tiles, int head_dim, int cols) {
  if (tiles < (head_dim == 64 || cols > 4 ? 24 : 12)) return 1;
  const int cap = (int)((cols > 4 ? 0.9f : 1.2f) * sqrtf((float)tiles));
  return cap < kMaxSplits ? cap : kMaxSplits;
}

// First token that a row in this place sees (a place before 0, which sees none, must not wrap round with a large window).
__device__ __forceinline__ int window_start(int place, int window) { return window ? max(max(place + 1, 0) - window, 0) : 0; }

constexpr float kLazy = 8.f;   // a running maximum may fall behind by so many powers of two before sums are rescaled

// Eight codes as f16, exactly.  8-bit floats have an instruction for it; integers ride in the low bits of 1024 + 128 + c.
template <bool FP8>
__device__ __forceinline__ f16x8 codes_f16(uint32_t lo, uint32_t hi) {
  f16x8 r;
  if constexpr (FP8) {
    const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)lo, 1.0f, true);
    const f16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)hi, 1.0f, true);
    r = f16x8{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
  } else {
    const uint32_t base = 0x64646464u;
    const f16x2 off = {(_Float16)1152.f, (_Float16)1152.f};
    lo ^= 0x80808080u;
    hi ^= 0x80808080u;
    const f16x2 a = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(base, lo, 0x04010400u)) - off;
    const f16x2 b = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(base, lo, 0x04030402u)) - off;
    const f16x2 c = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(base, hi, 0x04010400u)) - off;
    const f16x2 d = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(base, hi, 0x04030402u)) - off;
    r = f16x8{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
  }
  return r;
}

// A row's power of two that brings its largest value to [2^7, 2^8): bf16 queries then fit f16 exactly (what lies 2^22
// below the row's largest loses bits below 2^-32 of it).
__device__ __forceinline__ int fit_shift(float amax) {
  const int e = (int)(__builtin_bit_cast(uint32_t, amax) >> 23 & 255);
  return amax > 0.f ? min(max(134 - e, -120), 120) : 0;
}

__device__ __forceinline__ f32x4 mma16(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 mma32(f16x8 a, f16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 mma32(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }

template <typename T> struct Vec8;
template <> struct Vec8<_Float16> { typedef f16x8 type; };
template <> struct Vec8<__bf16> { typedef bf16x8 type; };

template <typename V> struct Element;
template <> struct Element<f16x8> { typedef _Float16 type; };
template <> struct Element<bf16x8> { typedef __bf16 type; };
template <typename V> __device__ __forceinline__ typename Element<V>::type to_element(float x) { return (typename Element<V>::type)x; }

// Compile-time switch of a lambda: with the test inside one body the compiler makes the mask's 64 comparisons and
// selects part of every tile (a third of the vector instructions of a prompt).
struct Masked { static constexpr bool value = true; };
struct Whole { static constexpr bool value = false; };

// Scores are scaled inside the exponential's argument; a factor of 0 (an underflow) would make NaN of a masked -inf.
__device__ __forceinline__ float keep_sign(float f) { return f < 1e-37f ? 1e-37f : f; }   // (NaN stays)

// Codes that a page which does not exist has: its tokens are NaN by the factor of their scores, for those who see them, and must
// not reach the others as 0 * NaN of whatever another page holds.
__device__ const u32x4 g_no_codes[kPagedTile * 128 / 16] = {};
// A tile's codes (its number, or -1).  The address space is named: a choice between two plain pointers became flat loads, which LDS waits count too.
typedef const uint8_t __attribute__((address_space(1))) * GlobalBytes;
typedef const u32x4 __attribute__((address_space(1))) * GlobalPieces;
__device__ __forceinline__ GlobalBytes codes_of(const uint8_t* codes, int tile, int bytes) {
  return tile < 0 ? (GlobalBytes)g_no_codes : (GlobalBytes)codes + (long)tile * bytes;
}

// A block of zero values has the scale 1, which says nothing of its size: as it is, it would hold the running maximum far above blocks
// of small values, whose probabilities would lose bits in f16 or vanish.  Any scale 2^k serves it as well (codes of 0; k cancels in the
// sum): 2^-40 of the least of the wave's other blocks, so that it stays out of their way also where its tokens weigh most, and no less
// than 2^-95, which keeps the sum in fp32.  lsv, isv: log2 and inverse of the scale of the lane's block `tile` (where `ok`).  A wave
// with no scale of exactly 1 passes by.
template <int D, bool FP8>
__device__ __forceinline__ void place_zero_blocks(const uint8_t* v_codes, int tile, bool ok, float& lsv, float& isv) {
  const bool one = ok && isv == 1.f;
  uint64_t asks = __ballot(one);
  if (asks == 0) return;
  float least = ok && !one ? lsv : INFINITY;
  for (int o = 1; o < 64; o *= 2) least = fminf(least, __shfl_xor(least, o));
  const float k = least == INFINITY ? -60.f : fmaxf(floorf(least) - 40.f, -95.f);
  const int lane = threadIdx.x & 63;
  for (; asks; asks &= asks - 1) {
    const int i = __builtin_ctzll(asks);
    const u32x4* const from = reinterpret_cast<const u32x4*>(v_codes + (long)__builtin_amdgcn_readlane(tile, i) * (kPagedTile * D));
    uint32_t any = 0;
#pragma unroll
    for (int p = 0; p < D / 16; ++p) {
      const u32x4 w = from[64 * p + lane];
      any |= w.x | w.y | w.z | w.w;
    }
    if (__any((any & (FP8 ? 0x7F7F7F7Fu : ~0u)) != 0) || lane != i) continue;
    lsv = k;
    isv = __builtin_amdgcn_exp2f(-k);
  }
}

// Two 16-bit tokens of a value word, zero where the token lies behind the last one (`left` tokens count from the word's first).
__device__ __forceinline__ uint32_t keep_tokens(uint32_t w, int left) { return left >= 2 ? w : left == 1 ? (w & 0xFFFFu) : 0u; }

// Whether this workgroup is the last of its unit's splits to hand in its partial results.  They are device-scope stores; every
// wave waits for its own, then one thread takes a ticket at the memory side, so the holder of the last ticket finds all of
// them performed; it reads them with device-scope loads.
__device__ __forceinline__ bool last_of_splits(int32_t* counter, int splits, int& s_last) {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
  __syncthreads();
  if (threadIdx.x == 0) {
    const int ticket = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    s_last = ticket == splits - 1;
    if (s_last) __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);   // clean for the next call
  }
  __syncthreads();
  return s_last;
}

// Two neighbouring floats of partial results, at device scope.
__device__ __forceinline__ void store_pair(float* p, float a, float b) {
  __hip_atomic_store(reinterpret_cast<uint64_t*>(p), __builtin_bit_cast(uint64_t, f32x2{a, b}), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ f32x2 load_pair(const float* p) {
  return __builtin_bit_cast(f32x2, __hip_atomic_load(reinterpret_cast<const uint64_t*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}

struct JoinSpace {   // LDS
  float m[16][kMaxSplits], l[16][kMaxSplits], inv[16];
  int last;
};

// Joins the partial results of `ns` splits, `step` floats apart from `base` on, and writes the outputs.
// cols: valid columns; out_of(col): pointer to the column's output row.
template <typename T, int D, typename Out>
__device__ __forceinline__ void join_splits(int32_t* counter, int ns, const float* base, long step, int cols, JoinSpace& js, Out out_of) {
  if (!last_of_splits(counter, ns, js.last)) return;
  // Sixteen columns at a time: every (column, split)'s maximum and sum and a thread's first two elements of eight splits in one
  // round trip, weights to LDS, then what is left of the elements.
  const int tid = threadIdx.x, threads = blockDim.x;
  for (int c0 = 0; c0 < cols; c0 += 16) {
    const int nc = min(16, cols - c0);
    const float* const from = base + (long)c0 * (D + 2);
    auto elements = [&](int idx, int s, f32x2 (&u)[8]) __attribute__((always_inline)) {   // (the last split's again behind it)
#pragma unroll
      for (int k = 0; k < 8; ++k) u[k] = load_pair(from + min(s + k, ns - 1) * step + idx / D * (D + 2) + idx % D);
    };
    f32x2 u[8];
    if (2 * tid < nc * D) elements(2 * tid, 0, u);
    for (int i = tid; i < nc * ns; i += threads) {
      const f32x2 ml = load_pair(from + (i % ns) * step + (i / ns) * (D + 2) + D);
      js.m[i / ns][i % ns] = ml.x;
      js.l[i / ns][i % ns] = ml.y;
    }
    __syncthreads();
    for (int col = tid; col < nc; col += threads) {
      float M = -INFINITY, l = 0.f;
      for (int s = 0; s < ns; ++s) M = fmaxf(M, js.m[col][s]);
      const float at = M == -INFINITY ? 0.f : M;
      for (int s = 0; s < ns; ++s) {
        const float w = __builtin_amdgcn_exp2f(js.m[col][s] - at);
        js.m[col][s] = w;
        l = __builtin_fmaf(js.l[col][s], w, l);
      }
      js.inv[col] = l == 0.f ? 0.f : 1.f / l;
    }
    __syncthreads();
    for (int idx = 2 * tid; idx < nc * D; idx += 2 * threads) {
      const int col = idx / D;
      float x = 0.f, y = 0.f;
      for (int s = 0; s < ns; s += 8) {
        if (s > 0 || idx >= 2 * threads) elements(idx, s, u);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          if (s + k >= ns) break;
          x = __builtin_fmaf(u[k].x, js.m[col][s + k], x);
          y = __builtin_fmaf(u[k].y, js.m[col][s + k], y);
        }
      }
      *reinterpret_cast<uint32_t*>(out_of(c0 + col) + idx % D) = pack2<T>(x * js.inv[col], y * js.inv[col]);
    }
    __syncthreads();
  }
}

int32_t launch_paged_decode(const PagedAttnArgs& a, hipStream_t st);
int32_t launch_paged_prompt(const PagedAttnArgs& a, hipStream_t st);

}  // namespace dq
