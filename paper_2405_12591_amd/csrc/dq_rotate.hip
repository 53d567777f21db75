// Norm of query and key heads and their position rotation in one pass over the rows.
#include "dq_paged.h"

namespace dq {

struct RotateArgs {
  dq_heads q, q_out, k, k_out;   // heads == 0: none
  int batch, tokens, head_dim;
  dq_head_norm norm;
  dq_rotary rot;                 // rot_dim == 0: none
  int heads_per_group;           // heads one workgroup takes of its rows, queries and keys counted through
  int head_groups;
};

// A thread keeps one unit (16 channels) of one token for all heads of its group, so the eight angles of the unit are
// formed once and turn every head.  Bound by memory: 2 bytes in and 2 out per element against about 7 flops.  A token's
// groups of heads are neighbours in the grid, so that its row is read and written by workgroups that run together, and the
// results are stored past the caches' own order (`store_unit`): 16384 tokens of 40 heads of 128 channels with norm and three axes,
// 336 MB, 66 us (5.1 TB/s, as a copy of that size); 71 with the groups far apart, 69 with plain stores, 75 with both.
template <typename T, int LANES, bool INTERLEAVED>
__global__ __launch_bounds__(kPagedThreads) void rotate_heads_kernel(RotateArgs a) {
  const int unit = threadIdx.x % LANES;
  const int group = (int)(blockIdx.x % (unsigned)a.head_groups);
  const long column = (long)(blockIdx.x / (unsigned)a.head_groups) * (kPagedThreads / LANES) + threadIdx.x / LANES;
  const bool live = column < (long)a.batch * a.tokens && 16 * unit < a.head_dim;
  const int b = live && a.batch > 1 ? (int)(column / a.tokens) : 0;
  const long t = live ? column - (long)b * a.tokens : 0;
  const RowLayout l = row_layout(unit, a.rot.rot_dim, INTERLEAVED);
  const int h0 = group * a.heads_per_group, h1 = min(h0 + a.heads_per_group, a.q.heads + a.k.heads);
  const uint16_t* const q = a.q.data + b * a.q.batch_stride + t * a.q.token_stride;
  const uint16_t* const k = a.k.data + b * a.k.batch_stride + t * a.k.token_stride;
  const int k0 = max(h0 - a.q.heads, 0);
  RowLayout turned = l;
  if (!live) turned.pair0 = -1;
  UnitTurns ut;
  load_turns(a.rot, turned, column, 0, ut);
  u32x4 v[2] = {};
  if (live) load_unit(v, h0 < a.q.heads ? q + h0 * a.q.head_stride : k + k0 * a.k.head_stride, l);
  float cs[8], sn[8];
  make_turns(turned, ut, cs, sn);
  const float inv_dim = 1.0f / (float)a.head_dim;
  if (h0 < a.q.heads) {
    rotate_row<T, LANES, INTERLEAVED>(v, q, a.q_out.data + b * a.q_out.batch_stride + t * a.q_out.token_stride, a.q.head_stride, a.q_out.head_stride, h0,
                                      min(h1, a.q.heads), live, l, a.norm.q_weight, a.norm.eps, inv_dim, cs, sn);
    if (live && h1 > a.q.heads) load_unit(v, k, l);
  }
  if (h1 > a.q.heads)
    rotate_row<T, LANES, INTERLEAVED>(v, k, a.k_out.data + b * a.k_out.batch_stride + t * a.k_out.token_stride, a.k.head_stride, a.k_out.head_stride, k0,
                                      h1 - a.q.heads, live, l, a.norm.k_weight, a.norm.eps, inv_dim, cs, sn);
}

template <typename T, int LANES>
static void launch_rotate2(const RotateArgs& a, dim3 grid, hipStream_t st) {
  if (a.rot.interleaved) hipLaunchKernelGGL((rotate_heads_kernel<T, LANES, true>), grid, dim3(kPagedThreads), 0, st, a);
  else hipLaunchKernelGGL((rotate_heads_kernel<T, LANES, false>), grid, dim3(kPagedThreads), 0, st, a);
}

template <typename T>
static void launch_rotate(const RotateArgs& a, int lanes, dim3 grid, hipStream_t st) {
  switch (lanes) {
    case 2: launch_rotate2<T, 2>(a, grid, st); break;
    case 4: launch_rotate2<T, 4>(a, grid, st); break;
    case 8: launch_rotate2<T, 8>(a, grid, st); break;
    default: launch_rotate2<T, 16>(a, grid, st); break;
  }
}

}  // namespace dq

using namespace dq;

extern "C" int32_t dq_rotate_heads(const dq_heads* q, const dq_heads* q_out, const dq_heads* k, const dq_heads* k_out, int32_t batch,
                                   int32_t tokens, int32_t head_dim, int32_t dtype, const dq_head_norm* norm, const dq_rotary* rot,
                                   void* hip_stream) {
  if ((!q) != (!q_out) || (!k) != (!k_out) || (!q && !k) || (!norm && !rot)) return DQ_EINVAL;
  if (batch <= 0 || tokens < 0 || head_dim < 32 || head_dim > 256 || head_dim % 16) return DQ_EINVAL;
  if (dtype != DQ_F16 && dtype != DQ_BF16) return DQ_EINVAL;
  if (q && (!heads_ok(q, true) || !heads_ok(q_out, true) || q->heads != q_out->heads)) return DQ_EINVAL;
  if (k && (!heads_ok(k, true) || !heads_ok(k_out, true) || k->heads != k_out->heads)) return DQ_EINVAL;
  const long rows = (long)batch * tokens;
  if (!norm_ok(norm) || !rotary_ok(rot, head_dim, rows, true) || rows >= (1l << 31)) return DQ_EINVAL;
  if (rows == 0) return DQ_OK;
  RotateArgs a = {};
  if (q) { a.q = *q; a.q_out = *q_out; }
  if (k) { a.k = *k; a.k_out = *k_out; }
  a.batch = batch; a.tokens = tokens; a.head_dim = head_dim;
  if (norm) a.norm = *norm;
  if (rot) a.rot = *rot;
  int lanes = 2;
  while (16 * lanes < head_dim) lanes *= 2;
  const long groups = (rows + kPagedThreads / lanes - 1) / (kPagedThreads / lanes);
  const long heads = (long)a.q.heads + a.k.heads;
  // Heads a workgroup takes: eight share the angles where the rows alone fill the chip, fewer where they do not.
  int per = 8;
  while (per > 1 && groups * ((heads + per - 1) / per) < 1024) per /= 2;
  a.heads_per_group = per;
  const long head_groups = (heads + per - 1) / per;
  if (heads > INT32_MAX || groups * head_groups >= kMaxThreads / kPagedThreads) return DQ_EINVAL;
  a.head_groups = (int)head_groups;
  const dim3 grid((unsigned)(groups * a.head_groups));
  if (dtype == DQ_BF16) launch_rotate<__bf16>(a, lanes, grid, (hipStream_t)hip_stream);
  else launch_rotate<_Float16>(a, lanes, grid, (hipStream_t)hip_stream);
  DQ_HIP_CHECK(hipGetLastError());
  return DQ_OK;
}
