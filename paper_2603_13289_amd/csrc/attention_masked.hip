// Grouped-query attention of a ragged batch: scores capped by a tanh or biased by distance, a key range for every row.
#include <climits>

#include "common.h"

namespace rc {

// One wavefront per (row, head): 64 keys at a time, a lane a key for the scores, two elements of the head a lane for the values.
template <typename T>
__global__ void __launch_bounds__(256)
masked_attn_row_kernel(MaskedAttnArgs a) {
  const int lane = threadIdx.x & 63;
  const long item = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int row = (int)(item / a.n_q_heads), head = (int)(item - (long)row * a.n_q_heads);
  if (row >= a.n_rows) return;
  int s = 0, e = a.n_seq;   // the last sequence that begins at or before the row
  while (e - s > 1) {
    const int m = (s + e) >> 1;
    if (a.row_start[m] <= row) s = m; else e = m;
  }
  const int first = a.row_start[s];
  if (row < first || row >= a.row_start[s + 1] || row - first >= a.max_rows_per_seq) return;
  const int seq = a.seq ? min(max(a.seq[s], 0), a.n_table_rows - 1) : s;
  const int dh = a.g.head_dim, kvh = head / (a.n_q_heads / a.g.n_kv_heads);
  const int pos = a.row_pos[row];
  const int lo = max(a.row_lo ? a.row_lo[row] : 0, 0), hi = min(a.row_hi ? a.row_hi[row] : pos, a.max_len - 1);
  const T* const q = reinterpret_cast<const T*>(a.q) + ((size_t)row * a.n_q_heads + head) * dh;
  const float slope = a.slopes ? a.slopes[head] : 0.f;
  float m = -INFINITY, l = 0.f, o0 = 0.f, o1 = 0.f;
  for (int k0 = lo; k0 <= hi; k0 += 64) {
    const int key = min(k0 + lane, hi);
    const size_t off = kv_row_offset(a.g, seq, key, kvh);
    const T* const k = reinterpret_cast<const T*>(a.k_pool) + off;
    float x = 0.f;
    for (int d = 0; d < dh; ++d) x += to_f32(q[d]) * to_f32(k[d]);
    x *= a.scale;
    if (a.cap > 0.f) x = a.cap * tanhf(x / a.cap);
    x -= slope * fabsf((float)(pos - key));
    if (k0 + lane > hi) x = -INFINITY;
    float mx = x;
    for (int w = 32; w > 0; w >>= 1) mx = fmaxf(mx, __shfl_xor(mx, w, 64));
    const float m_new = fmaxf(m, mx), m_use = m_new == -INFINITY ? 0.f : m_new;
    const float corr = __expf(m - m_use), p = k0 + lane > hi ? 0.f : __expf(x - m_use);
    m = m_new;
    l = l * corr + p;
    o0 *= corr;
    o1 *= corr;
    for (int j = 0; j < min(64, hi - k0 + 1); ++j) {
      const float w = __shfl(p, j, 64);
      const T* const v = reinterpret_cast<const T*>(a.v_pool) + kv_row_offset(a.g, seq, k0 + j, kvh);
      o0 += w * to_f32(v[lane]);
      if (dh == 128) o1 += w * to_f32(v[lane + 64]);
    }
  }
  for (int w = 32; w > 0; w >>= 1) l += __shfl_xor(l, w, 64);
  T* const out = reinterpret_cast<T*>(a.out) + ((size_t)row * a.n_q_heads + head) * dh;
  const float inv = lo > hi ? 0.f : 1.f / l;
  out[lane] = from_f32<T>(o0 * inv);
  if (dh == 128) out[lane + 64] = from_f32<T>(o1 * inv);
}

size_t masked_attention_partial_floats(const MaskedAttnArgs&, bool) { return 0; }

hipError_t launch_masked_attention(const MaskedAttnArgs& a, bool is_bf16, float*, hipStream_t st) {
  const unsigned grid = (unsigned)(((long)a.n_rows * a.n_q_heads + 3) / 4);
  if (is_bf16) masked_attn_row_kernel<bf16><<<grid, 256, 0, st>>>(a);
  else masked_attn_row_kernel<float><<<grid, 256, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace rc
