// Rows of a ragged batch: block tables, slots and key ranges from request lengths; per-head norms with rotary positions, written into
// paged caches; moves of cached rows under the same rotary positions.
#include <algorithm>
#include <climits>

#include "common.h"

namespace rc {

static constexpr int kThreads = 256;

// ------------------------------------------------------------------ block tables, slots and key ranges
// Two prefix sums over the sequences (rows, new blocks), then independent rows.  The sums are short, so every workgroup makes them for itself
// and one launch does: a thread adds up a run of consecutive sequences, the 256 runs are scanned in LDS.  Bound by latency: 32 single tokens
// 4.5 us, 256 sequences of 256k rows in documents 8.4 us (5.4 MB).
struct MapScan {
  long long rows[kThreads];     // of the sequences before a thread's run
  long long blocks[kThreads];
  long long wave_rows[kThreads / 64], wave_blocks[kThreads / 64];
};

// One sequence of the batch as its lengths say.
struct MapSeq { long long cached, total; int have, need; bool in_table; };
__device__ inline MapSeq map_seq(const rc_batch_map_args& a, int s) {
  MapSeq q;
  q.cached = max(a.n_cached[s], 0);
  q.total = q.cached + max(a.n_new[s], 0);
  q.in_table = q.total <= (long long)a.max_blocks_per_seq * a.block_size;
  q.have = (int)((q.cached + a.block_size - 1) / a.block_size);
  q.need = q.in_table ? (int)((q.total + a.block_size - 1) / a.block_size) - q.have : 0;
  return q;
}

__global__ void __launch_bounds__(kThreads)
batch_map_kernel(rc_batch_map_args a, int run) {
  __shared__ MapScan scan;
  __shared__ int refused_of[kThreads / 64], taken_of[kThreads / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int first_free = a.free_first ? min(max(*a.free_first, 0), a.n_free) : 0;
  const int avail = a.n_free - first_free;

  const int s_begin = min((long long)tid * run, (long long)a.n_seq), s_end = min(s_begin + run, a.n_seq);
  long long rows = 0, blocks = 0;
  for (int s = s_begin; s < s_end; ++s) {
    const MapSeq q = map_seq(a, s);
    rows += q.total - q.cached;
    blocks += q.need;
  }
  long long r_in = rows, b_in = blocks;   // inclusive within the wavefront
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const long long r = __shfl_up(r_in, o, 64), b = __shfl_up(b_in, o, 64);
    if (lane >= o) { r_in += r; b_in += b; }
  }
  if (lane == 63) { scan.wave_rows[wave] = r_in; scan.wave_blocks[wave] = b_in; }
  __syncthreads();
  long long r0 = r_in - rows, b0 = b_in - blocks, all_rows = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) {
    if (w < wave) { r0 += scan.wave_rows[w]; b0 += scan.wave_blocks[w]; }
    all_rows += scan.wave_rows[w];
  }
  scan.rows[tid] = r0;
  scan.blocks[tid] = b0;
  __syncthreads();

  if (blockIdx.x == 0) {   // what belongs to sequences, not rows
    long long r = r0, b = b0;
    int refused = 0, taken = 0;
    for (int s = s_begin; s < s_end; ++s) {
      const MapSeq q = map_seq(a, s);
      const long long n = q.total - q.cached;
      const bool served = q.in_table && (q.need == 0 || b + q.need <= avail) && (n == 0 || r + n <= a.max_rows);
      a.row_start[s] = (int)min(r, (long long)a.max_rows);
      if (a.kv_len) a.kv_len[s] = (int)(served ? q.total : q.cached);
      if (served && q.need > 0) taken = max(taken, (int)(b + q.need));
      refused += !served;
      r += n;
      b += q.need;
    }
    if (tid == 0) a.row_start[a.n_seq] = (int)min(all_rows, (long long)a.max_rows);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      refused += __shfl_xor(refused, o, 64);
      taken = max(taken, __shfl_xor(taken, o, 64));
    }
    if (lane == 0) { refused_of[wave] = refused; taken_of[wave] = taken; }
    __syncthreads();
    if (tid == 0 && a.counts) {
      for (int w = 1; w < kThreads / 64; ++w) { refused += refused_of[w]; taken = max(taken, taken_of[w]); }
      a.counts[0] = (int)min(all_rows, (long long)a.max_rows);
      a.counts[1] = first_free + taken;
      a.counts[2] = refused;
    }
  }

  const int live = (int)min(all_rows, (long long)a.max_rows);
  for (long long row = (long long)blockIdx.x * kThreads + tid; row < live; row += (long long)gridDim.x * kThreads) {
    const int r = (int)row;
    // the last run that begins at or before the row, then the last such sequence of it: empty ones begin where the next does
    int t = 0;
#pragma unroll
    for (int step = kThreads / 2; step > 0; step >>= 1)
      if (scan.rows[t + step] <= r) t += step;
    int s = t * run;
    if (s >= a.n_seq) s = a.n_seq - 1;
    long long start = scan.rows[t], b = scan.blocks[t];
    MapSeq q = map_seq(a, s);
    while (s + 1 < a.n_seq && start + (q.total - q.cached) <= r) {
      start += q.total - q.cached;
      b += q.need;
      q = map_seq(a, ++s);
    }
    const bool served = q.in_table && (q.need == 0 || b + q.need <= avail) && start + (q.total - q.cached) <= a.max_rows;
    const long long pos = q.cached + (r - start);
    int slot = -1, lo = 0, hi = -1;
    if (served) {
      const int at = (int)pos / a.block_size, in = (int)pos - at * a.block_size;
      int32_t* const entry = a.block_table + (size_t)s * a.max_blocks_per_seq + at;
      int blk;
      if (at < q.have) {
        blk = *entry;
      } else {
        blk = a.free_blocks[first_free + (int)b + (at - q.have)];
        if (in == 0) *entry = blk;   // a new block begins with one of the new rows
      }
      if (blk >= 0 && blk < a.n_blocks) slot = blk * a.block_size + in;
      int end = (int)q.total;
      if (a.doc_start) {
        int u = min(max(a.doc_start[s], 0), a.n_docs), v = min(max(a.doc_start[s + 1], u), a.n_docs);   // first document behind pos
        const int first = u, last = v;
        while (u < v) {
          const int m = (u + v) >> 1;
          if (a.doc_first[m] <= (int)pos) u = m + 1; else v = m;
        }
        if (u > first) lo = max(a.doc_first[u - 1], 0);
        if (u < last) end = min(end, a.doc_first[u]);
      }
      hi = (int)pos;
      if (a.prefix_len) hi = max(hi, a.prefix_len[s] - 1);
      hi = min(hi, end - 1);
    }
    if (a.row_seq) a.row_seq[r] = s;
    if (a.row_pos) a.row_pos[r] = (int)min(pos, (long long)INT_MAX);
    if (a.row_slot) a.row_slot[r] = slot;
    if (a.row_lo) a.row_lo[r] = lo;
    if (a.row_hi) a.row_hi[r] = hi;
  }
}

hipError_t launch_batch_map(const rc_batch_map_args& a, hipStream_t st) {
  const int run = (a.n_seq + kThreads - 1) / kThreads;
  const unsigned grid = (unsigned)std::min(std::max(1ll, ((long long)a.max_rows + kThreads - 1) / kThreads), 2048ll);
  batch_map_kernel<<<grid, kThreads, 0, st>>>(a, run);
  return hipGetLastError();
}

// ------------------------------------------------------------------ rotary positions
// Angle in 64 bits as a number of turns; whole quarter turns are dropped there, the rest (at most 1/8 turn) is exact enough as a float.
__device__ inline float2 rotary_entry(double pos, double turns, float amplitude) {
  const double t = 4.0 * pos * turns;
  const double whole = rint(t);
  float s, c;
  sincospif(0.5f * (float)(t - whole), &s, &c);
  const int quarter = (int)((long long)whole & 3);
  const float x = quarter & 1 ? -s : c, y = quarter & 1 ? c : s;
  return quarter & 2 ? make_float2(-amplitude * x, -amplitude * y) : make_float2(amplitude * x, amplitude * y);
}

// 2 CH elements of a head belong to a lane t of head_dim / (2 CH): two runs of CH, the elements of CH rotary pairs (CH t .. CH t + CH - 1) where
// 2 CH t < rotary_dim, else as many that pass through.  A run is 16 bytes of T: CH is 4 for float and 8 for bf16, 4 there where the
// rotated part is no multiple of 16.
template <int CH> struct HeadLane { int off0, off1; bool rotated; };
template <int CH>
__device__ inline HeadLane<CH> head_lane(int t, int layout, int rotary_dim) {
  HeadLane<CH> h;
  h.rotated = 2 * CH * t < rotary_dim;
  const bool apart = h.rotated && layout == RC_ROTARY_HALF;
  h.off0 = apart ? CH * t : 2 * CH * t;
  h.off1 = apart ? rotary_dim / 2 + CH * t : 2 * CH * t + CH;
  return h;
}
// cs: (cos, sin) of the lane's pairs
template <int CH>
__device__ inline void rotate_pairs(float (&x0)[CH], float (&x1)[CH], const float2* cs, int layout) {
  if (layout == RC_ROTARY_HALF) {
#pragma unroll
    for (int e = 0; e < CH; ++e) {
      const float2 t = cs[e];
      const float a = x0[e], b = x1[e];
      x0[e] = a * t.x - b * t.y;
      x1[e] = b * t.x + a * t.y;
    }
  } else {
#pragma unroll
    for (int e = 0; e < CH; e += 2) {
      const float2 t = cs[e / 2], u = cs[CH / 2 + e / 2];
      const float a = x0[e], b = x0[e + 1], c = x1[e], d = x1[e + 1];
      x0[e] = a * t.x - b * t.y;
      x0[e + 1] = b * t.x + a * t.y;
      x1[e] = c * u.x - d * u.y;
      x1[e + 1] = d * u.x + c * u.y;
    }
  }
}

// CH consecutive elements
template <int CH>
__device__ inline void load_run(const float* p, float (&v)[CH]) {
#pragma unroll
  for (int i = 0; i < CH; i += 4) {
    const float4 t = *reinterpret_cast<const float4*>(p + i);
    v[i] = t.x; v[i + 1] = t.y; v[i + 2] = t.z; v[i + 3] = t.w;
  }
}
__device__ inline void load_run(const bf16* p, float (&v)[8]) { Vec16<bf16>::load(p, v); }
__device__ inline void load_run(const bf16* p, float (&v)[4]) {
  const uint2 t = *reinterpret_cast<const uint2*>(p);
  v[0] = __uint_as_float(t.x << 16); v[1] = __uint_as_float(t.x & 0xffff0000u);
  v[2] = __uint_as_float(t.y << 16); v[3] = __uint_as_float(t.y & 0xffff0000u);
}
// the same, of what nobody reads again: not kept in the caches on the way (5120 rows of float projections 39.6 -> 37.5 us; for cache rows and for
// stores it is no gain: 32768 moved rows 57 -> 59 us with such loads, 87 with such stores)
template <typename T, int CH>
__device__ inline void load_run_once(const T* p, float (&v)[CH]) {
  typedef unsigned u32xn __attribute__((ext_vector_type(CH * sizeof(T) >= 16 ? 4 : 2)));
  constexpr int PER = sizeof(u32xn) / sizeof(T);
#pragma unroll
  for (int i = 0; i < CH; i += PER) {
    const u32xn t = __builtin_nontemporal_load(reinterpret_cast<const u32xn*>(p + i));
#pragma unroll
    for (int e = 0; e < PER; ++e)
      v[i + e] = sizeof(T) == 4 ? __uint_as_float(t[e * sizeof(T) / 4]) : __uint_as_float(e & 1 ? t[e / 2] & 0xffff0000u : t[e / 2] << 16);
  }
}
template <int CH>
__device__ inline void store_run(float* p, const float (&v)[CH]) {
#pragma unroll
  for (int i = 0; i < CH; i += 4) *reinterpret_cast<float4*>(p + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
}
__device__ inline void store_run(bf16* p, const float (&v)[8]) { Vec16<bf16>::store(p, v); }
__device__ inline void store_run(bf16* p, const float (&v)[4]) {
  *reinterpret_cast<uint2*>(p) = make_uint2((uint32_t)f32_to_bf16(v[0]).v | ((uint32_t)f32_to_bf16(v[1]).v << 16),
                                            (uint32_t)f32_to_bf16(v[2]).v | ((uint32_t)f32_to_bf16(v[3]).v << 16));
}

// ------------------------------------------------------------------ per-head norm, rotation, scatter
// A workgroup per row: its (cos, sin) once for all heads, then head_dim / (2 CH) lanes a head; the loads of kHeadsAhead heads a lane stand in front of
// the work on the first one.  Bound by HBM: 5120 rows of 32 + 2 x 8 heads of 128, float in and bf16 out (199 MB), 37 us or 5.4 TB/s; 16 such
// rows 5.4 us, which is the launch and three loads one behind the other.
static constexpr int kHeadsAhead = 2;
template <typename TI, typename T, int CH>
__global__ void __launch_bounds__(kThreads)
norm_rotary_kernel(NormRotaryArgs a, RotaryArg rot) {
  __shared__ float2 cs_of[RC_ROTARY_MAX_PAIRS];
  const int r = blockIdx.x;
  if (a.n_live && r >= *a.n_live) return;
  const int dh = a.g.head_dim, lph = dh / (2 * CH), per_pass = kThreads / lph;
  const int t = threadIdx.x % lph, h0 = threadIdx.x / lph;
  const HeadLane<CH> at = head_lane<CH>(t, rot.layout, rot.rotary_dim);
  const int nq = a.n_q_heads, nkv = a.g.n_kv_heads, heads = nq + 2 * nkv;
  const TI* const row = reinterpret_cast<const TI*>(a.qkv) + (size_t)r * a.stride;
  float x0[kHeadsAhead][CH], x1[kHeadsAhead][CH];
  auto load = [&](int h) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < kHeadsAhead; ++u) {
      const TI* const p = row + (size_t)min(h + u * per_pass, heads - 1) * dh;
      load_run_once(p + at.off0, x0[u]);
      load_run_once(p + at.off1, x1[u]);
    }
  };
  load(h0);
  const int slot = a.slot[r];
  const bool to_cache = slot >= 0 && slot < a.g.rows;
  if ((int)threadIdx.x < rot.rotary_dim / 2)
    cs_of[threadIdx.x] = rotary_entry((double)a.pos[r], rot.turns[threadIdx.x], rot.amplitude);
  __syncthreads();
  for (int h1 = h0; h1 < heads; h1 += kHeadsAhead * per_pass) {
    if (h1 != h0) load(h1);
#pragma unroll
    for (int u = 0; u < kHeadsAhead; ++u) {
      const int h = h1 + u * per_pass;
      if (h >= heads) break;
      auto put = [&](T* p) __attribute__((always_inline)) {
        store_run(p + at.off0, x0[u]);
        store_run(p + at.off1, x1[u]);
      };
      if (h >= nq + nkv) {
        if (to_cache) put(reinterpret_cast<T*>(a.v_pool) + slot_offset(a.g, slot, h - nq - nkv));
        continue;
      }
      const T* const gain = reinterpret_cast<const T*>(h < nq ? a.g_q : a.g_k);
      if (gain) {
        float ss = 0.f, g0[CH], g1[CH];
#pragma unroll
        for (int e = 0; e < CH; e += 4) ss = add_squares(ss, make_float4(x0[u][e], x0[u][e + 1], x0[u][e + 2], x0[u][e + 3]));
#pragma unroll
        for (int e = 0; e < CH; e += 4) ss = add_squares(ss, make_float4(x1[u][e], x1[u][e + 1], x1[u][e + 2], x1[u][e + 3]));
        for (int o = lph >> 1; o > 0; o >>= 1) ss += __shfl_xor(ss, o, 64);
        const float inv = 1.0f / sqrtf(ss / (float)dh + a.eps);
        load_run(gain + at.off0, g0);
        load_run(gain + at.off1, g1);
#pragma unroll
        for (int e = 0; e < CH; ++e) { x0[u][e] = x0[u][e] * inv * g0[e]; x1[u][e] = x1[u][e] * inv * g1[e]; }
      }
      if (h >= nq && to_cache && a.k_pre) put(reinterpret_cast<T*>(a.k_pre) + slot_offset(a.g, slot, h - nq));
      if (at.rotated) rotate_pairs(x0[u], x1[u], cs_of + CH * t, rot.layout);
      if (h < nq) put(reinterpret_cast<T*>(a.q_out) + ((size_t)r * nq + h) * dh);
      else if (to_cache) put(reinterpret_cast<T*>(a.k_pool) + slot_offset(a.g, slot, h - nq));
    }
  }
}

hipError_t launch_norm_rotary(const NormRotaryArgs& a, const RotaryArg& rot, bool qkv_bf16, bool pool_bf16, hipStream_t st) {
  if (a.n <= 0) return hipSuccess;
  const bool wide = rot.rotary_dim % 16 == 0;
  if (pool_bf16 && wide) {
    if (qkv_bf16) norm_rotary_kernel<bf16, bf16, 8><<<a.n, kThreads, 0, st>>>(a, rot);
    else norm_rotary_kernel<float, bf16, 8><<<a.n, kThreads, 0, st>>>(a, rot);
  } else if (pool_bf16) {
    if (qkv_bf16) norm_rotary_kernel<bf16, bf16, 4><<<a.n, kThreads, 0, st>>>(a, rot);
    else norm_rotary_kernel<float, bf16, 4><<<a.n, kThreads, 0, st>>>(a, rot);
  } else {
    if (qkv_bf16) norm_rotary_kernel<bf16, float, 4><<<a.n, kThreads, 0, st>>>(a, rot);
    else norm_rotary_kernel<float, float, 4><<<a.n, kThreads, 0, st>>>(a, rot);
  }
  return hipGetLastError();
}

// ------------------------------------------------------------------ rows to other slots and positions
// head_dim / (2 CH) lanes a (row, head): a lane reads and writes its pairs of the key and its elements of the value, so that a row may stay in its
// slot.  The (cos, sin) of a workgroup's rows are worked out once, under the loads.  Bound by HBM: 32768 rows of 8 heads of 128, bf16 (269 MB), 46 us or
// 5.8 TB/s.
template <typename T, int CH>
__global__ void __launch_bounds__(kThreads)
rotary_move_kernel(RotaryMoveArgs a, RotaryArg rot) {
  extern __shared__ float2 cs_rows[];   // [row of the workgroup][pair]
  const int dh = a.gs.head_dim, lph = dh / (2 * CH), groups = kThreads / lph, nkv = a.gs.n_kv_heads, pairs = rot.rotary_dim / 2;
  const long g0 = (long)blockIdx.x * groups;
  const int r0 = (int)(g0 / nkv);
  const int n = a.n_live ? min(a.n, *a.n_live) : a.n;
  if (r0 >= n) return;
  const int t = threadIdx.x % lph;
  const long rh = g0 + threadIdx.x / lph;
  const int r = (int)(rh / nkv), head = (int)(rh - (long)r * nkv);
  const int rr = min(r, n - 1);
  const int from = a.src_slot[rr], to = a.dst_slot[rr];
  const bool moves = r < n && from >= 0 && from < a.gs.rows && to >= 0 && to < a.gd.rows;
  const HeadLane<CH> at = head_lane<CH>(t, rot.layout, rot.rotary_dim);
  const size_t so = slot_offset(a.gs, moves ? from : 0, head);
  const T* const k = reinterpret_cast<const T*>(a.k_src) + so;
  const T* const v = reinterpret_cast<const T*>(a.v_src) + so;
  float x0[CH], x1[CH], v0[CH], v1[CH];
  load_run(k + at.off0, x0);
  load_run(k + at.off1, x1);
  load_run(v + at.off0, v0);
  load_run(v + at.off1, v1);
  const int rows = (int)((g0 + groups - 1) / nkv) - r0 + 1;
  for (int i = threadIdx.x; i < rows * pairs; i += kThreads) {
    const int row = i / pairs, p = i - row * pairs, at_row = min(r0 + row, n - 1);
    const double by = (double)a.new_pos[at_row] - (a.old_pos ? (double)a.old_pos[at_row] : 0.0);
    cs_rows[i] = rotary_entry(by, rot.turns[p], a.old_pos ? 1.f : rot.amplitude);
  }
  __syncthreads();
  if (!moves) return;
  if (at.rotated) rotate_pairs(x0, x1, cs_rows + (size_t)(r - r0) * pairs + CH * t, rot.layout);
  const size_t dof = slot_offset(a.gd, to, head);
  T* const ko = reinterpret_cast<T*>(a.k_dst) + dof;
  T* const vo = reinterpret_cast<T*>(a.v_dst) + dof;
  store_run(ko + at.off0, x0);
  store_run(ko + at.off1, x1);
  store_run(vo + at.off0, v0);
  store_run(vo + at.off1, v1);
}

template <typename T, int CH>
static hipError_t launch_move(const RotaryMoveArgs& a, const RotaryArg& rot, hipStream_t st) {
  const int groups = kThreads / (a.gs.head_dim / (2 * CH)), nkv = a.gs.n_kv_heads;
  const unsigned grid = (unsigned)(((long)a.n * nkv + groups - 1) / groups);
  const int rows = (groups - 1) / nkv + 2;   // that the groups of a workgroup can touch
  rotary_move_kernel<T, CH><<<grid, kThreads, (size_t)rows * (rot.rotary_dim / 2) * sizeof(float2), st>>>(a, rot);
  return hipGetLastError();
}

hipError_t launch_rotary_move(const RotaryMoveArgs& a, const RotaryArg& rot, bool pool_bf16, hipStream_t st) {
  if (a.n <= 0) return hipSuccess;
  if (!pool_bf16) return launch_move<float, 4>(a, rot, st);
  return rot.rotary_dim % 16 == 0 ? launch_move<bf16, 8>(a, rot, st) : launch_move<bf16, 4>(a, rot, st);
}

}  // namespace rc
