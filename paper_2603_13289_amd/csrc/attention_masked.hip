// Grouped-query attention of a ragged batch: scores capped by a tanh or biased by distance, a key range for every row.
//
// A row and head of a key head's group is a column of the products.  Per 32 or 64 keys, on 32x32x16 matrix instructions,
//   S^T[key][column] = K[key][:] . Q[column][:]     A: K rows from LDS, B: Q in registers
//   O^T[d][column]  += V^T[d][key] P[key][column]   A: V rows from LDS, transposed by the read; B: P, S^T's registers as they stand
// so that a column's scores lie in two lanes (c, c + 32) and its softmax takes one exchange between them.  P's element order is a
// permutation of the keys inside a group of 16 (a lane of half h has keys 4h .. 4h + 3 and 8 + 4h .. 8 + 4h + 3); the transposing read
// takes four keys at a time, so it follows that order for nothing.
//
// Rows in LDS are padded: K's lie 272 bytes apart, so that the lanes that fetch one 16-byte piece of consecutive keys meet every bank once, V's 320, which
// does so for the four keys of a transposing read; every address is a lane's base plus a constant (SQ_LDS_BANK_CONFLICT: 0).
#include <algorithm>
#include <climits>
#include <type_traits>

#include "common.h"

namespace rc {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;
typedef __attribute__((__vector_size__(8 * sizeof(float)))) float f32x8;
typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16;
typedef __attribute__((__vector_size__(4 * sizeof(short)))) short s16x4;
typedef __attribute__((__vector_size__(4 * sizeof(unsigned)))) unsigned u32x4;   // (an array of uint4 went to scratch memory)

static constexpr int DH = 128;
static constexpr int BKV = 64;            // keys per tile of the tile kernel
static constexpr int TILE_COLS = 128, WIDE_COLS = 256;   // columns of a tile: four or eight wavefronts, 32 each
static constexpr int ROW_COLS = 32;       // columns of the few-row kernel
static constexpr int F32_COLS = 16;       // columns of the float kernel
static constexpr int ROW_KEYS = 32;       // keys a wavefront of it takes at a time
static constexpr int KROW = DH * 2 + 16, VROW = DH * 2 + 64;   // bytes between rows in LDS
static constexpr int PROW = DH + 4;       // floats between the columns of a partial result
static constexpr int K_TILE = BKV * KROW, V_TILE = BKV * VROW, kTileBytes = 2 * (K_TILE + V_TILE);
static constexpr int kAhead = 4;          // LDS operand fragments in flight ahead of the product that uses them
static constexpr float kRescaleSlack = 8.f;   // log2 units the running maximum may lead the reference exponent
static constexpr float kLog2e = 1.4426950408889634f;

__device__ inline float pair_max(float x) {   // over lanes l, l ^ 32
  const unsigned u = __float_as_uint(x);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// Rows r0 .. r1 - 1 of a sequence, whatever the device says inside [0, n_rows].
struct SeqRows { int s, r0, r1, table_row; };
__device__ inline int row_in_batch(const MaskedAttnArgs& a, int start) { return min(max(start, 0), a.n_rows); }
__device__ inline SeqRows rows_of_seq(const MaskedAttnArgs& a, int s, int start, int end) {
  SeqRows q;
  q.s = s;
  q.r0 = row_in_batch(a, start);
  q.r1 = min(max(end, q.r0), min(a.n_rows, q.r0 + a.max_rows_per_seq));
  q.table_row = a.seq ? min(max(a.seq[s], 0), a.n_table_rows - 1) : s;
  return q;
}
__device__ inline SeqRows rows_of_seq(const MaskedAttnArgs& a, int s) { return rows_of_seq(a, s, a.row_start[s], a.row_start[s + 1]); }
// Keys that a row sees; (kNoKey, -1) where it sees none.
static constexpr int kNoKey = 1 << 30;   // no key is that far (host)
struct Range { int lo, hi; };
__device__ inline Range range_of_row(const MaskedAttnArgs& a, int row) {
  const int lo = max(a.row_lo ? a.row_lo[row] : 0, 0), hi = min(a.row_hi ? a.row_hi[row] : a.row_pos[row], a.max_len - 1);
  return lo <= hi ? Range{lo, hi} : Range{kNoKey, -1};
}
// The last sequence s whose place(first row, s) is at most x; places ascend.  64 candidates a step, and the starts of the last 64 stay in the lanes.
template <typename F>
__device__ inline SeqRows find_seq(const MaskedAttnArgs& a, int x, F place) {
  const int lane = threadIdx.x & 63;
  int base = 0, n = a.n_seq;
  while (true) {
    const int step = (n - base + 63) / 64, i = base + lane * step;
    const int start = a.row_start[min(i, a.n_seq)];
    const unsigned long long at = __ballot(i < n && place(row_in_batch(a, start), i) <= x);
    const int k = __builtin_amdgcn_readfirstlane(at ? 63 - __clzll((long long)at) : 0);
    base += k * step;
    if (step <= 1) return rows_of_seq(a, base, __builtin_amdgcn_readlane(start, k), k < 63 ? __builtin_amdgcn_readlane(start, k + 1) : a.row_start[base + 1]);
    n = min(n, base + step);
  }
}

// Scores in units of log2 (what a weight is 2 to the power of), up to a line: score = raw * MUL + add, MUL and add the same for all keys, so
// that the line and the reference exponent's subtraction are one operation.  The cap: cap tanh(x / cap) = cap - 2 cap / (exp(2 x / cap) + 1), whose
// quotient is the raw score (it falls as the score rises); its error of 2^-23 changes a weight by as much times the cap (kMostCap: 2^-11), where weights
// are rounded to 2^-9 in any case.
// Bounded scores: a cap without a bias bounds them by itself, so that its softmax needs no running maximum: with the reference exponent fixed at a quarter of
// the cap, weights lie between 2^-100 and 2^60 up to kMostBounded, and no score has to wait for another; values between 2^-26 and 2^48
// keep their digits in the products' sums, wherever the scores lie (up to a million keys).
enum ScoreKind : int { kPlain = 0, kBias = 1, kCap = 2, kCapBias = 3, kBounded = 4 };
static constexpr float kMostBounded = 80.f;   // log2 units: a cap of 55
template <int KIND>
struct Score {
  static constexpr bool CAP = KIND >= kCap, BIAS = KIND == kBias || KIND == kCapBias, kFixed = KIND == kBounded;
  static constexpr bool kFalls = CAP && !BIAS;
  float in, out, mul, add, slope, from;   // from: key offset of the lane's element 0 minus the row's position
  __device__ Score(const MaskedAttnArgs& a)
      : in(CAP ? fminf(2.f * kLog2e * a.scale / a.cap, 3e38f) : a.scale * kLog2e), out(-2.f * kLog2e * a.cap),
        mul(BIAS ? 1.f : CAP ? out : in), add(CAP ? kLog2e * a.cap : 0.f), slope(0.f), from(0.f) {}
  __device__ __forceinline__ float raw(float dot, float offset) const {
    float x = dot;
    if constexpr (CAP) x = __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(x * in) + 1.f);
    if constexpr (BIAS) x = fmaf(-slope, fabsf(from + offset), x * (CAP ? out : in));
    return x;
  }
  static __device__ __forceinline__ float none() { return kFalls ? INFINITY : -INFINITY; }   // the raw score of a key that is not seen
  static __device__ __forceinline__ float larger(float x, float y) { return kFalls ? fminf(x, y) : fmaxf(x, y); }
  __device__ __forceinline__ float first_reference() const { return kFixed ? 0.25f * add : -INFINITY; }
};

// Two values: halves that are not finite become zeros (they would turn a weight of 0 into NaN); bad: there was one.
__device__ inline uint32_t only_finite(uint32_t w, bool& bad) {
  const bool lo = (w & 0x7f80u) == 0x7f80u, hi = (w & 0x7f800000u) == 0x7f800000u;
  bad |= lo | hi;
  return w & (lo ? 0xffff0000u : ~0u) & (hi ? 0xffffu : ~0u);
}
__device__ inline u32x4 only_finite(u32x4 v, bool& bad) {
  return u32x4{only_finite(v[0], bad), only_finite(v[1], bad), only_finite(v[2], bad), only_finite(v[3], bad)};
}
// What such values of keys key0 .. key1 - 1 add to the columns that see them: an infinity or NaN, whatever the weight.  Behind the main loop, over
// the whole range, in the rare case that the staging met one.
__device__ __forceinline__ void add_not_finite(const bf16* v_pool, const KvGeom& g, int seq, int kvh, int key0, int key1, Range r, f32x16 (&acc_o)[4]) {
  const int half = (threadIdx.x >> 5) & 1;
#pragma unroll 1
  for (int key = key0; key < key1; ++key) {
    const bool sees = r.lo <= key && key <= r.hi;
    if (!__any(sees)) continue;
    const bf16* const v = v_pool + kv_row_offset(g, seq, key, kvh) + 4 * half;
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float x = to_f32(v[32 * db + 8 * (e >> 2) + (e & 3)]);
        if (sees && !(fabsf(x) < INFINITY)) acc_o[db][e] += x;
      }
  }
}

// The running softmax of a column over 32 B keys (in two lanes).  The reference exponent follows the maximum lazily: the sums are rescaled only
// when a column's maximum has grown by more than kRescaleSlack since the last time, so weights stay below 2^kRescaleSlack instead of 1; any
// reference gives the same quotient.
template <int KIND, int B>
__device__ __forceinline__ float move_reference(const Score<KIND>& score, const f32x16 (&s)[B], float& m_run, float& l_run, f32x16 (&acc_o)[4]) {
  if constexpr (Score<KIND>::kFixed) return score.add - m_run;
  float mx = s[0][0];
#pragma unroll
  for (int b = 0; b < B; ++b)
#pragma unroll
    for (int e = 0; e < 16; ++e) mx = Score<KIND>::larger(mx, s[b][e]);
  mx = pair_max(fmaf(mx, score.mul, score.add));
  const float m_new = fmaxf(m_run, mx);
  if (__any(m_new > m_run + kRescaleSlack)) {
    const float corr = __builtin_amdgcn_exp2f(m_run - (m_new == -INFINITY ? 0.f : m_new));
    l_run *= corr;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc_o[i][e] *= corr;
    m_run = m_new;
  }
  return score.add - (m_run == -INFINITY ? 0.f : m_run);
}
// The sum takes the weights as they are multiplied, rounded: where few keys count, their roundings then cancel in the quotient (tokens behind
// a handful of keys: error against 64 bits 0.0017 -> 0.00085, of which 0.0008 are the output's own rounding); and it takes two at a time.
__device__ __forceinline__ void add_weights(bf16x8 p, float& sum) {
  typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;
  const bf16x2 ones = {(__bf16)1.f, (__bf16)1.f};
#pragma unroll
  for (int j = 0; j < 8; j += 2) sum = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{p[j], p[j + 1]}, ones, sum, false);
}
// the weights of eight scores
template <int KIND>
__device__ __forceinline__ bf16x8 weights(const Score<KIND>& score, const f32x16& s, int u, float add, float& sum) {
  f32x8 w;
#pragma unroll
  for (int j = 0; j < 8; ++j) w[j] = __builtin_amdgcn_exp2f(fmaf(s[8 * u + j], score.mul, add));
  const bf16x8 p = __builtin_convertvector(w, bf16x8);
  add_weights(p, sum);
  return p;
}

// K operand: key block b (32 keys), d step i (16 of them); k: the lane's place, kv_lane_k
__device__ __forceinline__ int k_lane(int lane) { return (lane & 31) * KROW + (lane >> 5) * 16; }
__device__ __forceinline__ bf16x8 k_fragment(const unsigned char* k, int b, int i) {
  return __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(k + b * 32 * KROW + 32 * i));
}
// V^T operand of keys 16 t .. 16 t + 15 and d = 32 db .. 32 db + 31; v: the lane's place
__device__ __forceinline__ int v_lane(int lane) { return (4 * (lane >> 5) + ((lane >> 2) & 3)) * VROW + 32 * ((lane >> 4) & 1) + 8 * (lane & 3); }
__device__ __forceinline__ bf16x8 v_fragment(const unsigned char* v, int t, int db) {
  typedef __attribute__((__vector_size__(8 * sizeof(short)))) short s16x8;
  auto at = [&](int key) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(v + key * VROW + 64 * db));
  };
  return __builtin_bit_cast(bf16x8, (s16x8)__builtin_shufflevector(at(16 * t), at(16 * t + 8), 0, 1, 2, 3, 4, 5, 6, 7));
}

// The reference exponent that a part of a range is merged with: NaN where its sum is, so that a part whose scores are all NaN, and which has no maximum, shows.
__device__ inline float2 part_sum(float m, float l) { return make_float2(l != l ? l : m, l); }

__device__ inline void store4(float* p, float a, float b, float c, float d) { *reinterpret_cast<float4*>(p) = make_float4(a, b, c, d); }

// how a batch's key ranges are cut
struct MaskedSplit { int n_chunks, chunk; };   // chunk: keys

__device__ inline uint2 pack4(float a, float b, float c, float d) {
  return make_uint2((uint32_t)f32_to_bf16(a).v | ((uint32_t)f32_to_bf16(b).v << 16), (uint32_t)f32_to_bf16(c).v | ((uint32_t)f32_to_bf16(d).v << 16));
}

__device__ inline void store4(bf16* p, float a, float b, float c, float d) { *reinterpret_cast<uint2*>(p) = pack4(a, b, c, d); }

// ------------------------------------------------------------------ tiles of 128 or 256 columns
// A wavefront has 32 columns (queries and outputs stay in its registers) and walks over the keys in steps of 64, which the workgroup stages through
// LDS for all of its wavefronts, double buffered.  Bound by the power that products and exponentials draw together (the clock falls to 1.7-1.85 GHz):
// 4096 rows over 8192 keys, 32 query and 8 key heads, on 16-slot pages, 497 us without a cap (1106 TFLOP/s), 585 with one (940), 560 with a bias; packed documents of
// up to 2300 keys, 6702 rows of 40 heads, 138 us (635 TFLOP/s of what is multiplied: ten steps a workgroup on average, before which its look-ups, queries
// and first tile take as long as two).
// Slots: the tiles of sequence s begin at slot row_start[s] / rows_per_tile + s, which leaves room for all of them without a sum
// over the sequences (ceil(n / R) <= floor((a + n) / R) - floor(a / R) + 1).
struct MaskedTile { int first, n_valid, table_row, unused; };

// The tiles of all slots, those with the longest ranges first, empty ones last: workgroups start in order, and a long one that starts late runs on alone (packed
// documents of up to 2300 keys 147 -> 138 us).  A tile's length is taken from its first row's first key to its last row's last, in steps of a quarter of
// an octave, inside which the later rows go first and neighbours stay neighbours, which share K and V in the caches.  One workgroup, a counting sort, 4.9 us.
static constexpr int kMostOrdered = 4096, kOrderThreads = 1024, kOrderBins = 128;
__global__ void __launch_bounds__(kOrderThreads)
masked_attn_order_kernel(MaskedAttnArgs a, int n_slots, int rows_per_tile, MaskedTile* __restrict__ order) {
  __shared__ int starts[kMostOrdered + 1], count[kOrderBins], before[kOrderBins / 64];
  constexpr int PER = kMostOrdered / kOrderThreads;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  for (int i = tid; i <= a.n_seq; i += kOrderThreads) starts[i] = row_in_batch(a, a.row_start[i]);   // n_seq <= n_slots <= kMostOrdered (host)
  if (tid < kOrderBins) count[tid] = 0;
  __syncthreads();
  MaskedTile tile[PER];
  int bin[PER], rank[PER];
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int slot = n_slots - 1 - (tid + k * kOrderThreads);
    bin[k] = -1;
    if (slot < 0) continue;
    int s = 0;
    for (int n = a.n_seq; n - s > 1;) {
      const int m = (s + n) >> 1;
      if (starts[m] / rows_per_tile + m <= slot) s = m; else n = m;
    }
    const SeqRows sq = rows_of_seq(a, s, starts[s], starts[s + 1]);
    const int first = sq.r0 + (slot - (sq.r0 / rows_per_tile + s)) * rows_per_tile;
    const int n_valid = first < sq.r0 ? 0 : max(min(rows_per_tile, sq.r1 - first), 0);
    tile[k] = {first, n_valid, sq.table_row, 0};
    bin[k] = kOrderBins - 1;
    if (n_valid > 0) {
      const int keys = max(range_of_row(a, first + n_valid - 1).hi - range_of_row(a, first).lo, 0);
      bin[k] -= 1 + (int)((__float_as_uint((float)(keys + BKV)) >> 21) - (__float_as_uint((float)BKV) >> 21));   // up to 2^30 keys: 24 octaves
    }
  }
#pragma unroll
  for (int k = 0; k < PER; ++k)
    for (int at = k * kOrderThreads; at < min(n_slots, (k + 1) * kOrderThreads); at += 64) {   // a wavefront at a time
      if (wave == (at >> 6) % (kOrderThreads / 64) && bin[k] >= 0) rank[k] = atomicAdd(&count[bin[k]], 1);
      __syncthreads();
    }
  int upto = tid < kOrderBins ? count[tid] : 0;   // inclusive within the wavefront
  const int own = upto;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int x = __shfl_up(upto, o, 64);
    if (lane >= o) upto += x;
  }
  if (tid < kOrderBins && lane == 63) before[wave] = upto;
  __syncthreads();
  if (tid < kOrderBins) {
    for (int w = 0; w < wave; ++w) upto += before[w];
    count[tid] = upto - own;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < PER; ++k)
    if (bin[k] >= 0) order[count[bin[k]] + rank[k]] = tile[k];
}

template <int KIND, bool GROUPED, int NW>
__global__ void __launch_bounds__(64 * NW, 8 / NW)
masked_attn_tile_kernel(MaskedAttnArgs a, MaskedSplit sp, int n_slots, int rows_per_tile, const MaskedTile* __restrict__ order, float* __restrict__ part_o,
                        float2* __restrict__ part_ml) {
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];   // two K tiles, two V tiles
  __shared__ int bad_v;
  constexpr int COLS = 32 * NW, STEP = 4 * NW, PER = BKV / STEP;   // columns; rows that the threads load at a time, and how often
  const int kvh = (int)blockIdx.x % a.g.n_kv_heads;
  const int item = (int)blockIdx.x / a.g.n_kv_heads;
  const int slot = n_slots - 1 - item / sp.n_chunks, chunk = item % sp.n_chunks;   // late rows see the most keys: they go first
  const int G = a.n_q_heads / a.g.n_kv_heads;
  int first, n_valid, table_row;
  if (order) {
    const MaskedTile tile = order[item];
    first = tile.first;
    n_valid = tile.n_valid;
    table_row = tile.table_row;
  } else {
    const SeqRows sq = find_seq(a, slot, [&](int r0, int i) { return r0 / rows_per_tile + i; });
    first = sq.r0 + (slot - (sq.r0 / rows_per_tile + sq.s)) * rows_per_tile;
    n_valid = first < sq.r0 ? 0 : min(rows_per_tile, sq.r1 - first);
    table_row = sq.table_row;
  }
  if (n_valid <= 0) return;

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), ql = lane & 31, half = lane >> 5;
  int lo_min = INT_MAX, lo_max = 0, hi_min = INT_MAX, hi_max = -1;
  for (int i = lane; i < n_valid; i += 64) {
    const Range r = range_of_row(a, first + i);
    lo_min = min(lo_min, r.lo); lo_max = max(lo_max, r.lo); hi_min = min(hi_min, r.hi); hi_max = max(hi_max, r.hi);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    lo_min = min(lo_min, __shfl_xor(lo_min, o, 64)); lo_max = max(lo_max, __shfl_xor(lo_max, o, 64));
    hi_min = min(hi_min, __shfl_xor(hi_min, o, 64)); hi_max = max(hi_max, __shfl_xor(hi_max, o, 64));
  }
  lo_min = __builtin_amdgcn_readfirstlane(lo_min); lo_max = __builtin_amdgcn_readfirstlane(lo_max);
  hi_min = __builtin_amdgcn_readfirstlane(hi_min); hi_max = __builtin_amdgcn_readfirstlane(hi_max);
  const bool is_split = sp.n_chunks > 1;
  const int key_end = is_split ? min(hi_max + 1, (chunk + 1) * sp.chunk) : hi_max + 1;   // chunk sizes are whole tiles, chunks * size < 2^31 (host)
  const int t_begin = hi_max < 0 ? 0 : max(lo_min, chunk * sp.chunk) / BKV, t_end = (key_end + BKV - 1) / BKV;
  if (t_begin >= t_end && is_split) return;

  const int col = wave * 32 + ql, my = col / G;
  const bool live = col < rows_per_tile * G && my < n_valid;
  const int row = first + min(my, n_valid - 1), head = kvh * G + col % G;
  const Range mine = range_of_row(a, row);
  const unsigned seen = mine.hi < 0 ? 0u : (unsigned)(mine.hi - mine.lo) + 1u;

  // Queries come in whole rows and are handed around through the memory of the tiles to come (a wavefront's own part of it): with a lane asking for pieces of
  // its own row, a load touched 64 cache lines.
  const unsigned row_head = (unsigned)row * (unsigned)a.n_q_heads + (unsigned)head;   // below 2^31 (host)
  unsigned char* const own_rows = lds + wave * 32 * KROW;
  static_assert(COLS * KROW <= kTileBytes, "room for the queries");
  auto row_at = [&](int i) __attribute__((always_inline)) { return (size_t)(unsigned)__shfl((int)row_head, 4 * i + (lane >> 4), 64) * 256 + (lane & 15) * 16; };
  u32x4 q_in[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) q_in[i] = *reinterpret_cast<const u32x4*>(reinterpret_cast<const char*>(a.q) + row_at(i));
  Score<KIND> score(a);
  constexpr bool CAP = Score<KIND>::CAP, BIAS = Score<KIND>::BIAS;
  if constexpr (BIAS) score.slope = a.slopes[head] * kLog2e;
  const int pos = a.row_pos[row];

  // A lane looks up the block of one key of a tile, three tiles ahead; a thread loads 16 bytes of four rows.  GROUPED: the 16 keys of a group lie one
  // behind the other, so that loads go to a group's scalar address and a constant lane offset; else every key's row is handed around.  Behind
  // the last key that one is repeated (its group).
  const int32_t* const table = a.g.block_table + (size_t)table_row * a.g.max_blocks;
  const int last_key = min(t_end * BKV, a.max_len) - 1, ask_key = GROUPED ? last_key & ~15 : last_key;
  const int last_block = a.g.max_blocks - 1, block_size = a.g.block_size, head_rows = a.g.n_kv_heads, pool_blocks = a.g.n_blocks - 1;
  const KvGeom geom = a.g;
  const char* const k_pool = reinterpret_cast<const char*>(a.k_pool);
  const char* const v_pool = reinterpret_cast<const char*>(a.v_pool);
  struct Asked { int block, slot; };
  auto ask = [&](int t) __attribute__((always_inline)) -> Asked {
    const int key = min(t * BKV + lane, ask_key), at = block_of(geom, key);
    return {table[min(at, last_block)], key - at * block_size};
  };
  auto row_of = [&](Asked q) __attribute__((always_inline)) { return (unsigned)(min(max(q.block, 0), pool_blocks) * head_rows + kvh) * (unsigned)block_size + q.slot; };
  u32x4 rk[PER], rv[PER];
  const unsigned lane_off = (GROUPED ? ((tid >> 4) & 15) * 256 : 0) + (tid & 15) * 16;
  auto row_bytes = [&](unsigned row, int i) __attribute__((always_inline)) -> size_t {
    if constexpr (GROUPED) return (size_t)(unsigned)__builtin_amdgcn_readlane((int)row, STEP * i + 4 * (wave & ~3)) * 256;
    return (size_t)(unsigned)__shfl((int)row, (tid >> 4) + STEP * i, 64) * 256;
  };
  auto load = [&](const char* pool, size_t at) __attribute__((always_inline)) { return *reinterpret_cast<const u32x4*>(pool + at + lane_off); };
  auto fetch = [&](Asked q) __attribute__((always_inline)) {
    const unsigned row = row_of(q);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const size_t at = row_bytes(row, i);
      rk[i] = load(k_pool, at);
      rv[i] = load(v_pool, at);
    }
  };
  // tiles t_whole .. t_ragged - 1: every row of the tile sees all of their keys
  const int t_whole = (lo_max + BKV - 1) / BKV, t_ragged = (hi_min + 1) / BKV;
  unsigned char* const k_wr = lds + (tid >> 4) * KROW + (tid & 15) * 16;
  unsigned char* const v_wr = lds + 2 * K_TILE + (tid >> 4) * VROW + (tid & 15) * 16;
  auto stage_k = [&](auto buf) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < PER; ++i) *reinterpret_cast<u32x4*>(k_wr + decltype(buf)::value * K_TILE + i * STEP * KROW) = rk[i];
  };
  auto stage_v = [&](auto buf, int i) __attribute__((always_inline)) {
    *reinterpret_cast<u32x4*>(v_wr + decltype(buf)::value * V_TILE + i * STEP * VROW) = rv[i];
  };
  auto clean_v = [&](int t) __attribute__((always_inline)) {
    if ((t >= t_whole && t < t_ragged) || t >= t_end) return;
    bool bad = false;
#pragma unroll
    for (int i = 0; i < PER; ++i) rv[i] = only_finite(rv[i], bad);
    if (bad) bad_v = 1;
  };

  f32x16 acc_o[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc_o[i][e] = 0.f;
  float m_run = score.first_reference(), l_run = 0.f;

  const std::integral_constant<int, 0> buf0;
  const std::integral_constant<int, 1> buf1;
  Asked asked = {};   // of the tile two on
  bf16x8 qf[8];
  auto hand_queries = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 8; ++i) *reinterpret_cast<u32x4*>(own_rows + (4 * i + (lane >> 4)) * KROW + (lane & 15) * 16) = q_in[i];
    asm volatile("" ::: "memory");   // a wavefront's LDS accesses stay in order
#pragma unroll
    for (int i = 0; i < 8; ++i) qf[i] = k_fragment(own_rows + k_lane(lane), 0, i);
  };
  if (tid == 0) bad_v = 0;
  if (t_begin < t_end) {
    const Asked q0 = ask(t_begin), q1 = ask(t_begin + 1);
    asked = ask(t_begin + 2);
    fetch(q0);
    hand_queries();
    __syncthreads();   // the queries are in registers: K and V may come where they were
    clean_v(t_begin);
    stage_k(buf0);
#pragma unroll
    for (int i = 0; i < PER; ++i) stage_v(buf0, i);
    fetch(q1);
  }
  __syncthreads();
  const unsigned char* const k_rd = lds + k_lane(lane);
  const unsigned char* const v_rd = lds + 2 * K_TILE + v_lane(lane);
  // Step t multiplies the tile in buffer t % 2 (counted from t_begin), stages tile t + 1, whose rows are in registers, into the other and asks for tile
  // t + 2; past the end of the range its last rows once more, which nobody multiplies.
  //
  // The matrix unit and the vector ALUs run side by side where independent work stands side by side in the instruction stream (a SIMD's two
  // wavefronts drift into the same phase): the first key block's scores are worked on under the second one's products, the second
  // one's weights under the products with the first one's.
  auto tile_step = [&](int t, auto buf, auto whole) __attribute__((always_inline)) {
    constexpr int KOFF = decltype(buf)::value * K_TILE, VOFF = decltype(buf)::value * V_TILE;
    constexpr bool WHOLE = decltype(whole)::value, EARLY = Score<KIND>::kFixed && WHOLE;   // EARLY: block 0's weights under block 1's products as well
    const std::integral_constant<int, 1 - decltype(buf)::value> other;
    const unsigned row2 = row_of(asked);
    asked = ask(t + 3);
    if constexpr (BIAS) score.from = (float)(t * BKV + 4 * half - pos);
    f32x16 acc_s[2];
    auto raw = [&](int b, int e) __attribute__((always_inline)) { acc_s[b][e] = score.raw(acc_s[b][e], (float)(32 * b + 8 * (e >> 2) + (e & 3))); };
    f32x16 zero;
#pragma unroll
    for (int e = 0; e < 16; ++e) zero[e] = 0.f;
    bf16x8 kf[kAhead], p[4];
    float sum = 0.f, add = score.add - m_run;   // move_reference's where that moves
    f32x8 w;
    auto weight = [&](int b, int j) __attribute__((always_inline)) {
      w[j & 7] = __builtin_amdgcn_exp2f(fmaf(acc_s[b][j], score.mul, add));
      if ((j & 7) != 7) return;
      p[2 * b + (j >> 3)] = __builtin_convertvector(w, bf16x8);
      add_weights(p[2 * b + (j >> 3)], sum);
    };
#pragma unroll
    for (int i = 0; i < kAhead; ++i) kf[i] = k_fragment(k_rd + KOFF, 0, i);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int b = i >> 3;
      acc_s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[i % kAhead], qf[i & 7], (i & 7) == 0 ? zero : acc_s[b], 0, 0, 0);
      if (i + kAhead < 16) kf[i % kAhead] = k_fragment(k_rd + KOFF, (i + kAhead) >> 3, (i + kAhead) & 7);
      if (i >= 8 && (CAP || BIAS)) {
        raw(0, 2 * (i - 8));
        raw(0, 2 * (i - 8) + 1);
        if constexpr (EARLY) {
          weight(0, 2 * (i - 8));
          weight(0, 2 * (i - 8) + 1);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    bf16x8 vf[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) vf[i] = v_fragment(v_rd + VOFF, i >> 2, i & 3);
    __builtin_amdgcn_sched_barrier(0);
    clean_v(t + 1);
    stage_k(other);
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (!EARLY) {
#pragma unroll
      for (int e = 0; e < 16; ++e) raw(1, e);
      if constexpr (!WHOLE) {
        const int key0 = t * BKV + 4 * half - mine.lo;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if ((unsigned)(key0 + 32 * b + 8 * (e >> 2) + (e & 3)) >= seen) acc_s[b][e] = score.none();
      }
      add = move_reference(score, acc_s, m_run, l_run, acc_o);
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      if constexpr (!EARLY) {
#pragma unroll
        for (int j = 0; j < 8; ++j) weight(0, 8 * u + j);
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = u * PER / 2; i < (u + 1) * PER / 2; ++i) stage_v(other, i);
      __builtin_amdgcn_sched_barrier(0);
    }
    size_t at = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      acc_o[i & 3] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[i % kAhead], p[i >> 2], acc_o[i & 3], 0, 0, 0);
      if (i + kAhead < 16) vf[i % kAhead] = v_fragment(v_rd + VOFF, (i + kAhead) >> 2, (i + kAhead) & 3);
      if (i < 8) {
#pragma unroll
        for (int j = 2 * i; j < 2 * i + 2; ++j) {
          if constexpr (EARLY) raw(1, j);
          weight(1, j);
        }
      }
      if (i % 4 == 0 && i / 4 < PER) {
        at = row_bytes(row2, i / 4);
        rk[i / 4] = load(k_pool, at);
      }
      if (i % 4 == 2 && i / 4 < PER) rv[i / 4] = load(v_pool, at);
      __builtin_amdgcn_sched_barrier(0);
    }
    l_run += sum;
    __syncthreads();   // tile t consumed, tile t + 1 staged
  };
  const std::true_type whole;
  const std::false_type part;
  const int t_lim = min(t_ragged, t_end);
  int t = t_begin;
  auto part_tiles = [&](int end) __attribute__((always_inline)) {   // an even number of steps, but at the end of the range
    for (; t < end; t += 2) {
      tile_step(t, buf0, part);
      if (t + 1 < t_end) tile_step(t + 1, buf1, part);
    }
  };
  part_tiles(min(t_whole, t_end));
  for (; t + 1 < t_lim; t += 2) {
    tile_step(t, buf0, whole);
    tile_step(t + 1, buf1, whole);
  }
  part_tiles(t_end);
  if (bad_v) {
    // whole tiles were not looked at and have multiplied theirs: once more does no harm
    add_not_finite(reinterpret_cast<const bf16*>(a.v_pool), a.g, table_row, kvh, t_begin * BKV, min(t_end * BKV, a.max_len), mine, acc_o);
  }

  const float l_tot = l_run + __shfl_xor(l_run, 32, 64);
  if (is_split) {
    if (!live) return;
    const size_t at = ((size_t)(slot * (long)sp.n_chunks + chunk) * a.g.n_kv_heads + kvh) * COLS + col;
    if (half == 0) part_ml[at] = part_sum(m_run, l_tot);
    float* const o = part_o + at * PROW + 4 * half;
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
      for (int e = 0; e < 16; e += 4)
        *reinterpret_cast<float4*>(o + 32 * db + 2 * e) = make_float4(acc_o[db][e], acc_o[db][e + 1], acc_o[db][e + 2], acc_o[db][e + 3]);
    return;
  }
  // outputs leave as whole rows, the way the queries came
  const float inv = seen ? 1.0f / l_tot : 0.f;
#pragma unroll
  for (int db = 0; db < 4; ++db)
#pragma unroll
    for (int e = 0; e < 16; e += 4)
      *reinterpret_cast<uint2*>(own_rows + ql * KROW + 64 * db + 4 * e + 8 * half) = pack4(acc_o[db][e] * inv, acc_o[db][e + 1] * inv, acc_o[db][e + 2] * inv, acc_o[db][e + 3] * inv);
  asm volatile("" ::: "memory");
  const unsigned long long live_cols = __ballot(live);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const size_t to = row_at(i);
    const u32x4 o = *reinterpret_cast<const u32x4*>(own_rows + (4 * i + (lane >> 4)) * KROW + (lane & 15) * 16);
    if (live_cols >> (4 * i + (lane >> 4)) & 1) *reinterpret_cast<u32x4*>(reinterpret_cast<char*>(a.out) + to) = o;
  }
}

// ------------------------------------------------------------------ few rows a sequence: at most 32 columns
// A workgroup takes a sequence's columns and a range of keys; its wavefronts take every fourth block of 32 keys of the range with a softmax of
// their own and share nothing before the end.  Bound by HBM: K and V pass once, the products are a fifth of the time.  16 sequences of 1.4k to 9.5k keys
// (394 MB) in 68 us, 5.8 TB/s, where a large copy reaches 6.0; one of 5k keys (21 MB) in 8.1 us, most of which is the chain of look-ups and loads.
static constexpr int kRowWaveBytes = ROW_KEYS * (KROW + VROW);   // a wavefront's K and V, at the end its sums
static_assert(kRowWaveBytes >= ROW_COLS * PROW * 4, "room for the sums");
template <int KIND>
__global__ void __launch_bounds__(256, 2)
masked_attn_rows_kernel(MaskedAttnArgs a, MaskedSplit sp, float* __restrict__ part_o, float2* __restrict__ part_ml) {
  extern __shared__ __attribute__((aligned(16))) unsigned char lds_rows[];
  __shared__ float2 ml[4][ROW_COLS];
  const int kvh = (int)blockIdx.x % a.g.n_kv_heads;
  const int item = (int)blockIdx.x / a.g.n_kv_heads;
  const int s = item / sp.n_chunks, chunk = item - s * sp.n_chunks;
  const int G = a.n_q_heads / a.g.n_kv_heads;
  const SeqRows sq = rows_of_seq(a, s);
  const int n_cols = (sq.r1 - sq.r0) * G;   // at most 32 (host)
  if (n_cols <= 0) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 31, half = lane >> 5;
  // the blocks of the first keys, beside the rows' ranges, for ranges that begin with the chunk
  const bool is_split = sp.n_chunks > 1;
  const int32_t* const table = a.g.block_table + (size_t)sq.table_row * a.g.max_blocks;
  const int max_key = a.max_len - 1, last_block = a.g.max_blocks - 1, block_size = a.g.block_size;
  const KvGeom geom = a.g;
  struct Asked { int block, slot; };
  auto ask = [&](int b) __attribute__((always_inline)) -> Asked {
    const int key = min(b * ROW_KEYS + col, max_key), at = block_of(geom, key);
    return {table[min(at, last_block)], key - at * block_size};
  };
  const int b_chunk = chunk * (sp.chunk / ROW_KEYS);
  Asked q0 = ask(b_chunk + wave), next = ask(b_chunk + wave + 4);
  const int row = sq.r0 + min(col, n_cols - 1) / G, head = kvh * G + min(col, n_cols - 1) % G;
  const Range mine = range_of_row(a, row);
  const unsigned seen = mine.hi < 0 ? 0u : (unsigned)(mine.hi - mine.lo) + 1u;
  int lo_min = mine.lo, lo_max = mine.lo, hi_min = mine.hi, hi_max = mine.hi;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    lo_min = min(lo_min, __shfl_xor(lo_min, o, 64)); lo_max = max(lo_max, __shfl_xor(lo_max, o, 64));
    hi_min = min(hi_min, __shfl_xor(hi_min, o, 64)); hi_max = max(hi_max, __shfl_xor(hi_max, o, 64));
  }
  lo_min = __builtin_amdgcn_readfirstlane(lo_min); lo_max = __builtin_amdgcn_readfirstlane(lo_max);
  hi_min = __builtin_amdgcn_readfirstlane(hi_min); hi_max = __builtin_amdgcn_readfirstlane(hi_max);
  const int key_end = is_split ? min(hi_max + 1, (chunk + 1) * sp.chunk) : hi_max + 1;
  const int b_begin = hi_max < 0 ? 0 : max(lo_min, chunk * sp.chunk) / ROW_KEYS, b_end = (key_end + ROW_KEYS - 1) / ROW_KEYS;
  if (b_begin >= b_end && is_split) return;

  bf16x8 qf[8];
  {
    const bf16* const q = reinterpret_cast<const bf16*>(a.q) + ((size_t)row * a.n_q_heads + head) * DH + 8 * half;
#pragma unroll
    for (int i = 0; i < 8; ++i) qf[i] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(q + 16 * i));
  }
  Score<KIND> score(a);
  constexpr bool BIAS = Score<KIND>::BIAS;
  if constexpr (BIAS) score.slope = a.slopes[head] * kLog2e;
  const int pos = a.row_pos[row];

  u32x4 rk[8], rv[8];
  auto fetch = [&](Asked q) __attribute__((always_inline)) {
    const unsigned pool_row = (unsigned)(min(max(q.block, 0), geom.n_blocks - 1) * geom.n_kv_heads + kvh) * (unsigned)block_size + q.slot;
    size_t off[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) off[i] = (size_t)(unsigned)__shfl((int)pool_row, 4 * i + (lane >> 4), 64) * 256 + (lane & 15) * 16;
    // read once, by nobody else: not kept in the caches on the way (16 ragged sequences 91 -> 75 us, one of 40k keys 44.5 -> 35)
#pragma unroll
    for (int i = 0; i < 8; ++i) rk[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(reinterpret_cast<const char*>(a.k_pool) + off[i]));
#pragma unroll
    for (int i = 0; i < 8; ++i) rv[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(reinterpret_cast<const char*>(a.v_pool) + off[i]));
  };

  f32x16 acc_o[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc_o[i][e] = 0.f;
  float m_run = score.first_reference(), l_run = 0.f;
  unsigned char* const k = lds_rows + wave * kRowWaveBytes;
  unsigned char* const v = k + ROW_KEYS * KROW;
  int b = b_begin + wave;
  bool bad = false;
  if (b < b_end) {
    if (b_begin != b_chunk) {   // uniform
      q0 = ask(b);
      next = ask(b + 4);
    }
    fetch(q0);
    for (; b < b_end; b += 4) {
      const bool whole = b * ROW_KEYS >= lo_max && b * ROW_KEYS + ROW_KEYS - 1 <= hi_min;
      if (!whole) {
#pragma unroll
        for (int i = 0; i < 8; ++i) rv[i] = only_finite(rv[i], bad);
      }
      // this wavefront's own memory, and its LDS accesses stay in order: no barrier
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int key = 4 * i + (lane >> 4), piece = lane & 15;
        *reinterpret_cast<u32x4*>(k + key * KROW + 16 * piece) = rk[i];
        *reinterpret_cast<u32x4*>(v + key * VROW + 16 * piece) = rv[i];
      }
      asm volatile("" ::: "memory");
      if (b + 4 < b_end) {
        fetch(next);
        next = ask(b + 8);
      }
      f32x16 acc_s[1];
#pragma unroll
      for (int e = 0; e < 16; ++e) acc_s[0][e] = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        acc_s[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k_fragment(k + k_lane(lane), 0, i), qf[i], acc_s[0], 0, 0, 0);
      if constexpr (BIAS) score.from = (float)(b * ROW_KEYS + 4 * half - pos);
#pragma unroll
      for (int e = 0; e < 16; ++e) acc_s[0][e] = score.raw(acc_s[0][e], (float)(8 * (e >> 2) + (e & 3)));
      if (!whole) {
        const int key0 = b * ROW_KEYS + 4 * half - mine.lo;
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if ((unsigned)(key0 + 8 * (e >> 2) + (e & 3)) >= seen) acc_s[0][e] = score.none();
      }
      bf16x8 p[2];
      const float add = move_reference(score, acc_s, m_run, l_run, acc_o);
#pragma unroll
      for (int u = 0; u < 2; ++u) p[u] = weights(score, acc_s[0], u, add, l_run);
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int db = 0; db < 4; ++db)
          acc_o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v_fragment(v + v_lane(lane), u, db), p[u], acc_o[db], 0, 0, 0);
      asm volatile("" ::: "memory");
    }
    if (__any(bad)) {
      for (b = b_begin + wave; b < b_end; b += 4)
        add_not_finite(reinterpret_cast<const bf16*>(a.v_pool), a.g, sq.table_row, kvh, b * ROW_KEYS, min(b * ROW_KEYS + ROW_KEYS, a.max_len), mine, acc_o);
    }
  }

  // the four wavefronts' sums, in their order
  const float l_tot = l_run + __shfl_xor(l_run, 32, 64);
  if (half == 0) ml[wave][col] = part_sum(m_run, l_tot);
  __syncthreads();
  float m_all = ml[0][col].x;
#pragma unroll
  for (int w = 1; w < 4; ++w) m_all = fmaxf(m_all, ml[w][col].x);
  const float mine_by = m_run == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run - m_all);
  float* const sums = reinterpret_cast<float*>(k);
  if (col < n_cols) {
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
      for (int e = 0; e < 16; e += 4)
        *reinterpret_cast<float4*>(sums + col * PROW + 32 * db + 2 * e + 4 * half) =
            m_run == -INFINITY ? make_float4(0.f, 0.f, 0.f, 0.f)
                               : make_float4(acc_o[db][e] * mine_by, acc_o[db][e + 1] * mine_by, acc_o[db][e + 2] * mine_by, acc_o[db][e + 3] * mine_by);
  }
  __syncthreads();
  for (int i = tid; i < n_cols * (DH / 4); i += 256) {
    const int c = i / (DH / 4), d = (i - c * (DH / 4)) * 4;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    float m = ml[0][c].x, l = 0.f;
#pragma unroll
    for (int w = 1; w < 4; ++w) m = fmaxf(m, ml[w][c].x);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float4 x = *reinterpret_cast<const float4*>(lds_rows + w * kRowWaveBytes + (c * PROW + d) * 4);
      o.x += x.x; o.y += x.y; o.z += x.z; o.w += x.w;
      l += ml[w][c].x == -INFINITY ? 0.f : ml[w][c].y * __builtin_amdgcn_exp2f(ml[w][c].x - m);
    }
    if (is_split) {
      const size_t at = ((size_t)item * a.g.n_kv_heads + kvh) * ROW_COLS + c;
      if (d == 0) part_ml[at] = part_sum(m, l);
      *reinterpret_cast<float4*>(part_o + at * PROW + d) = o;
    } else {
      const int r = sq.r0 + c / G, h = kvh * G + c % G;
      const Range range = range_of_row(a, r);
      const float inv = range.hi < 0 ? 0.f : 1.0f / l;
      *reinterpret_cast<uint2*>(reinterpret_cast<bf16*>(a.out) + ((size_t)r * a.n_q_heads + h) * DH + d) = pack4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
    }
  }
}

// ------------------------------------------------------------------ merge of the chunks
// A wavefront per (row, head); lane c has chunk c's exponent and sum, D / 4 lanes with four elements each read the outputs of every second (fourth)
// chunk.  A chunk left a result for a column exactly if the tile's range reaches into it, which it does where the row's own range does.
// Bound by a chain of dependent reads (4.7 us).  ROWS (results of the few-row kernel): what is read does not hang on the rows' places, so
// that the results of the first chunks are asked for beside the row's range.
static constexpr int kMaxChunks = 64;   // a lane each
template <typename T, int D, int COLS, bool ROWS>
__global__ void __launch_bounds__(256)
masked_attn_merge_kernel(MaskedAttnArgs a, MaskedSplit sp, int rows_per_tile, const float* __restrict__ part_o, const float2* __restrict__ part_ml) {
  const long item = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int row_or = (int)(item / a.n_q_heads), head = (int)(item - (long)row_or * a.n_q_heads);   // ROWS: row in_seq of sequence s, in turn
  constexpr int LANES = D / 4, TURNS = 64 / LANES;   // of a chunk; chunks side by side
  const int lane = threadIdx.x & 63, d = (lane % LANES) * 4, turn = lane / LANES;
  const int G = a.n_q_heads / a.g.n_kv_heads, kvh = head / G;
  int in_seq, row;
  SeqRows sq;
  if constexpr (ROWS) {
    const int s = row_or / a.max_rows_per_seq;
    in_seq = row_or - s * a.max_rows_per_seq;
    if (s >= a.n_seq) return;
    sq = rows_of_seq(a, s);
  } else {
    row = row_or;
    if (row >= a.n_rows) return;
    sq = find_seq(a, row, [](int r0, int) { return r0; });
    if (row < sq.r0 || row >= sq.r1) return;
    in_seq = row - sq.r0;
  }
  const int h = head - kvh * G;
  long slot;
  int col;
  if constexpr (ROWS) { slot = sq.s; col = in_seq * G + h; }
  else if constexpr (COLS == F32_COLS) { const long c = (long)in_seq * G + h; slot = (long)sq.r0 * G / COLS + sq.s + c / COLS; col = (int)(c % COLS); }
  else { slot = sq.r0 / rows_per_tile + sq.s + in_seq / rows_per_tile; col = in_seq % rows_per_tile * G + h; }
  const size_t first = ((size_t)slot * sp.n_chunks * a.g.n_kv_heads + kvh) * COLS + col, step = (size_t)a.g.n_kv_heads * COLS;
  const float2 ml = part_ml[first + min(lane, sp.n_chunks - 1) * step];
  float4 o[4];
  auto fetch = [&](int c) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = *reinterpret_cast<const float4*>(part_o + (first + min(c + TURNS * i + turn, sp.n_chunks - 1) * step) * (D + 4) + d);
  };
  if constexpr (ROWS) {
    fetch(0);
    row = sq.r0 + in_seq;
    if (row >= sq.r1) return;
  }
  const Range r = range_of_row(a, row);
  T* const out = reinterpret_cast<T*>(a.out) + ((size_t)row * a.n_q_heads + head) * D + d;
  if (r.hi < 0) {
    if (turn == 0) store4(out, 0.f, 0.f, 0.f, 0.f);
    return;
  }
  const int c0 = r.lo / sp.chunk, c1 = r.hi / sp.chunk;
  const bool mine = lane >= c0 && lane <= c1 && ml.x != -INFINITY;
  float m = mine ? ml.x : -INFINITY;
#pragma unroll
  for (int k = 32; k > 0; k >>= 1) m = fmaxf(m, __shfl_xor(m, k, 64));
  const unsigned long long parts = __ballot(mine);
  const float w = mine ? __builtin_amdgcn_exp2f(ml.x - m) : 0.f;
  float l = mine ? ml.y * w : 0.f;
#pragma unroll
  for (int k = 32; k > 0; k >>= 1) l += __shfl_xor(l, k, 64);
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  const int from = ROWS ? 0 : c0;
  for (int c = from; c <= c1; c += 4 * TURNS) {
    if (!ROWS || c > 0) fetch(c);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int at = c + TURNS * i + turn;
      const float by = __shfl(w, at & 63, 64);
      // what other parts' places hold may be no number, whatever the factor
      if (at < 64 && (parts >> at & 1)) { acc.x += o[i].x * by; acc.y += o[i].y * by; acc.z += o[i].z * by; acc.w += o[i].w * by; }
    }
  }
#pragma unroll
  for (int k = 32; k >= LANES; k >>= 1) { acc.x += __shfl_xor(acc.x, k, 64); acc.y += __shfl_xor(acc.y, k, 64); acc.z += __shfl_xor(acc.z, k, 64); acc.w += __shfl_xor(acc.w, k, 64); }
  const float inv = 1.0f / l;
  if (turn == 0) store4(out, acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
}

// ------------------------------------------------------------------ float
// 16 columns a workgroup on 16x16x4 matrix instructions; its wavefronts take every eighth (heads of 128: fourth) block of 16 keys of the range with a
// softmax of their own and are merged through LDS.  Bound by latency (float models have a few hundred keys), so K and V go from memory straight to
// registers, the next block's keys under the softmax and its values under the scores.  384 rows over as many keys, four query and two key heads of 64: 12 us.
//   S^T[key][column]: lane holds column lane % 16, keys 4 (lane / 16) + 0..3; O^T[d][column] += V^T[d][key] P: P's operand is S^T's result as it stands
// The tanh is the library's: what the quotient of the bf16 kernels loses (2^-23 of the cap) shows in a float output.
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4;
template <int D>
__global__ void __launch_bounds__(D == 64 ? 512 : 256, 2)
masked_attn_f32_kernel(MaskedAttnArgs a, MaskedSplit sp, int n_slots, float* __restrict__ part_o, float2* __restrict__ part_ml) {
  constexpr int NB = D / 16, NW = D == 64 ? 8 : 4, OROW = D + 4;
  __shared__ __attribute__((aligned(16))) float lds_o[NW][F32_COLS][OROW];
  __shared__ float2 lds_ml[NW][F32_COLS];
  const int kvh = (int)blockIdx.x % a.g.n_kv_heads;
  const int item = (int)blockIdx.x / a.g.n_kv_heads;
  const int slot = n_slots - 1 - item / sp.n_chunks, chunk = item % sp.n_chunks;
  const int G = a.n_q_heads / a.g.n_kv_heads;
  const SeqRows sq = find_seq(a, slot, [&](int r0, int i) { return (int)((long)r0 * G / F32_COLS) + i; });
  const long first = (long)(slot - ((int)((long)sq.r0 * G / F32_COLS) + sq.s)) * F32_COLS;
  const int n_valid = (int)min((long)F32_COLS, (long)(sq.r1 - sq.r0) * G - first);
  if (n_valid <= 0 || first < 0) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), qi = lane & 15, kq = lane >> 4;
  const long col = first + min(qi, n_valid - 1);
  const int row = sq.r0 + (int)(col / G), head = kvh * G + (int)(col % G);
  const Range mine = range_of_row(a, row);
  const unsigned seen = mine.hi < 0 ? 0u : (unsigned)(mine.hi - mine.lo) + 1u;
  int lo_min = mine.lo, lo_max = mine.lo, hi_min = mine.hi, hi_max = mine.hi;
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) {
    lo_min = min(lo_min, __shfl_xor(lo_min, o, 64)); lo_max = max(lo_max, __shfl_xor(lo_max, o, 64));
    hi_min = min(hi_min, __shfl_xor(hi_min, o, 64)); hi_max = max(hi_max, __shfl_xor(hi_max, o, 64));
  }
  lo_min = __builtin_amdgcn_readfirstlane(lo_min); lo_max = __builtin_amdgcn_readfirstlane(lo_max);
  hi_min = __builtin_amdgcn_readfirstlane(hi_min); hi_max = __builtin_amdgcn_readfirstlane(hi_max);
  const bool is_split = sp.n_chunks > 1;
  const int key_end = is_split ? min(hi_max + 1, (chunk + 1) * sp.chunk) : hi_max + 1;
  const int b_begin = hi_max < 0 ? 0 : max(lo_min, chunk * sp.chunk) / 16, b_end = (key_end + 15) / 16;
  if (b_begin >= b_end && is_split) return;

  const float* const q = reinterpret_cast<const float*>(a.q) + ((size_t)row * a.n_q_heads + head) * D + 4 * kq;
  f32x4 fq[NB], fk[NB], acc[NB], fv[NB];   // fv[t][c]: V[key 4 kq + c][16 t + qi]
#pragma unroll
  for (int t = 0; t < NB; ++t) {
    fq[t] = *reinterpret_cast<const f32x4*>(q + 16 * t);
    acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const float slope = a.slopes ? a.slopes[head] : 0.f;
  const int pos = a.row_pos[row];
  const float* const k_pool = reinterpret_cast<const float*>(a.k_pool);
  const float* const v_pool = reinterpret_cast<const float*>(a.v_pool);
  const int32_t* const table = a.g.block_table + (size_t)sq.table_row * a.g.max_blocks;
  const KvGeom geom = a.g;
  const int max_key = a.max_len - 1;
  auto ask = [&](int b) __attribute__((always_inline)) -> int {   // the pool row of key qi of a block
    const int key = min(min(b, b_end - 1) * 16 + qi, max_key), at = block_of(geom, key);
    return (min(max(table[min(at, geom.max_blocks - 1)], 0), geom.n_blocks - 1) * geom.n_kv_heads + kvh) * geom.block_size + (key - at * geom.block_size);
  };
  auto load_k = [&](int pool_row) __attribute__((always_inline)) {
    const float* const p = k_pool + (size_t)(unsigned)pool_row * D + 4 * kq;
#pragma unroll
    for (int t = 0; t < NB; ++t) fk[t] = *reinterpret_cast<const f32x4*>(p + 16 * t);
  };
  auto load_v = [&](int pool_row) __attribute__((always_inline)) {
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const float* const p = v_pool + (size_t)(unsigned)__shfl(pool_row, 4 * kq + c, 64) * D + qi;
#pragma unroll
      for (int t = 0; t < NB; ++t) fv[t][c] = p[16 * t];
    }
  };
  float m_run = -INFINITY, l_run = 0.f;
  bool bad = false;
  int b = b_begin + wave;
  if (b < b_end) {
    int at = ask(b), next = ask(b + NW);
    load_k(at);
    load_v(at);
    for (; b < b_end; b += NW) {
      const bool whole = b * 16 >= lo_max && b * 16 + 15 <= hi_min;
      f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = s0;
#pragma unroll
      for (int t = 0; t < NB; t += 2)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          s0 = __builtin_amdgcn_mfma_f32_16x16x4f32(fk[t][c], fq[t][c], s0, 0, 0, 0);
          s1 = __builtin_amdgcn_mfma_f32_16x16x4f32(fk[t + 1][c], fq[t + 1][c], s1, 0, 0, 0);
        }
      load_k(next);   // behind the range its last block once more
      float x[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        x[r] = (s0[r] + s1[r]) * a.scale;
        if (a.cap > 0.f) x[r] = a.cap * tanhf(x[r] / a.cap);
        x[r] = fmaf(-slope, fabsf((float)(b * 16 + 4 * kq + r - pos)), x[r]);
      }
      if (!whole) {
        const int key0 = b * 16 + 4 * kq - mine.lo;
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if ((unsigned)(key0 + r) >= seen) x[r] = -INFINITY;
#pragma unroll
        for (int t = 0; t < NB; ++t)
#pragma unroll
          for (int c = 0; c < 4; ++c)
            if (!(fabsf(fv[t][c]) < INFINITY)) { fv[t][c] = 0.f; bad = true; }
      }
      float mx = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
      mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64)) * kLog2e;
      const float m_new = fmaxf(m_run, mx), m_use = m_new == -INFINITY ? 0.f : m_new;
      if (__any(m_new > m_run)) {
        const float corr = __builtin_amdgcn_exp2f(m_run - m_use);
        l_run *= corr;
#pragma unroll
        for (int t = 0; t < NB; ++t) acc[t] *= corr;
        m_run = m_new;
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        x[r] = __builtin_amdgcn_exp2f(fmaf(x[r], kLog2e, -m_use));
        l_run += x[r];
      }
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int t = 0; t < NB; ++t) acc[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(fv[t][c], x[c], acc[t], 0, 0, 0);
      load_v(next);
      next = ask(b + 2 * NW);
    }
    if (__any(bad)) {
      for (b = b_begin + wave; b < b_end; b += NW)
        for (int key = b * 16; key < min(b * 16 + 16, a.max_len); ++key) {
          const bool sees = mine.lo <= key && key <= mine.hi;
          const float* const v = v_pool + kv_row_offset(geom, sq.table_row, key, kvh) + 4 * kq;
#pragma unroll
          for (int t = 0; t < NB; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const float y = v[16 * t + r];
              if (sees && !(fabsf(y) < INFINITY)) acc[t][r] += y;
            }
        }
    }
  }

  // the wavefronts' sums, in their order
  float l_tot = l_run + __shfl_xor(l_run, 16, 64);
  l_tot += __shfl_xor(l_tot, 32, 64);
  if (kq == 0) lds_ml[wave][qi] = part_sum(m_run, l_tot);
  __syncthreads();
  float m_all = -INFINITY;
#pragma unroll
  for (int w = 0; w < NW; ++w) m_all = fmaxf(m_all, lds_ml[w][qi].x);
  const float by = m_run == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run - m_all);
#pragma unroll
  for (int t = 0; t < NB; ++t) {
    const f32x4 o = by == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : acc[t] * by;
    *reinterpret_cast<f32x4*>(&lds_o[wave][qi][16 * t + 4 * kq]) = o;
  }
  __syncthreads();
  for (int i = tid; i < n_valid * (D / 4); i += NW * 64) {
    const int c = i / (D / 4), d = (i - c * (D / 4)) * 4;
    float m = -INFINITY, l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < NW; ++w) m = fmaxf(m, lds_ml[w][c].x);
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      o += *reinterpret_cast<const f32x4*>(&lds_o[w][c][d]);
      l += lds_ml[w][c].x == -INFINITY ? 0.f : lds_ml[w][c].y * __builtin_amdgcn_exp2f(lds_ml[w][c].x - m);
    }
    if (is_split) {
      const size_t to = ((size_t)((long)slot * sp.n_chunks + chunk) * a.g.n_kv_heads + kvh) * F32_COLS + c;
      if (d == 0) part_ml[to] = part_sum(m, l);
      store4(part_o + to * OROW + d, o[0], o[1], o[2], o[3]);
    } else {
      const long cc = first + c;
      const int r = sq.r0 + (int)(cc / G), h = kvh * G + (int)(cc % G);
      const float inv = range_of_row(a, r).hi < 0 ? 0.f : 1.0f / l;
      store4(reinterpret_cast<float*>(a.out) + ((size_t)r * a.n_q_heads + h) * D + d, o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
    }
  }
}

// ------------------------------------------------------------------ host
// The few-row kernel serves sequences whose columns fit 32; the grid is then (sequence, chunk), else (tile, chunk).
// Key ranges are cut until there are as many workgroups as compute units (tiles: twice that, as many as run at a time), but into chunks of 256 keys at
// least (tiles: 512; float: eight steps of a workgroup, which the merge's launch costs): more and shorter ones cost more in the merge and in beginnings than they spread.  A token for each of 8 sequences of 16k keys: 110 us
// with 256 workgroups wanted, 111 with 1024, 125 with 4096; of one sequence of 40k keys 44 and 48; of one of 5k keys 16.0 in chunks of 256,
// 18.5 in chunks of 128.
struct MaskedPlan { bool rows, ordered; long slots; int rows_per_tile, cols; MaskedSplit split; };
static MaskedPlan plan_masked(const MaskedAttnArgs& a, bool is_bf16) {
  MaskedPlan p;
  const int G = a.n_q_heads / a.g.n_kv_heads;
  p.rows = is_bf16 && (long)a.max_rows_per_seq * G <= ROW_COLS;
  // Tiles of 256 columns load and stage K and V once for eight wavefronts, and run alone on a compute unit: worth it where ranges are long and there are
  // enough of them.  4096 rows over 8192 keys 622 -> 573 us (uncapped 533 -> 486), selected rows over 18k keys 708 -> 646; but packed documents
  // of up to 2300 keys, in no order, 143 -> 153, windows of 300 keys 183 -> 194, of 1200 417 -> 420.
  const bool wide = (a.n_rows / (WIDE_COLS / G) + 1l) * a.g.n_kv_heads >= 256 && a.max_len >= 4096;
  p.cols = !is_bf16 ? F32_COLS : p.rows ? ROW_COLS : wide ? WIDE_COLS : TILE_COLS;
  p.rows_per_tile = p.cols / G;
  p.slots = !is_bf16 ? (long)a.n_rows * G / F32_COLS + a.n_seq : p.rows ? a.n_seq : a.n_rows / p.rows_per_tile + a.n_seq;
  const bool tiles = is_bf16 && !p.rows;
  const long wgs = p.slots * a.g.n_kv_heads;
  const long unit = tiles ? BKV : 128, least = !is_bf16 ? (a.g.head_dim == 64 ? 1024 : 512) : tiles ? 512 : 256, wanted = tiles ? 512 : 256;
  const long chunks = std::min({wanted / std::max(wgs, 1l), (a.max_len + least - 1) / least, (long)kMaxChunks});
  const long chunk = chunks <= 1 ? 0 : ((a.max_len + chunks - 1) / chunks + unit - 1) / unit * unit;
  p.split.n_chunks = chunk ? (int)((a.max_len + chunk - 1) / chunk) : 1;
  p.split.chunk = (int)chunk;
  // Worth its launch where not all tiles run at a time and ranges do not grow with the rows anyhow.  Many tiles end together by themselves, and apart
  // in time those of a sequence read its K and V again: 200 sequences of 200 to 800 rows 960 -> 1025 us, 64 of them 299 -> 290; where a sequence has
  // few tiles that does not count (1000 of 20 to 60 rows 287 -> 259).
  p.ordered = tiles && p.split.n_chunks == 1 && wgs > (wide ? 256 : 512) && (a.n_seq > 1 || a.row_lo) &&
              p.slots <= (a.max_rows_per_seq <= 4 * p.rows_per_tile ? kMostOrdered : 2048);
  return p;
}

size_t masked_attention_part_bytes(const MaskedAttnArgs& a, bool is_bf16) {
  if (a.n_rows <= 0) return 0;
  const MaskedPlan p = plan_masked(a, is_bf16);
  if (p.ordered) return (size_t)p.slots * sizeof(MaskedTile);
  if (p.split.n_chunks <= 1) return 0;
  return (size_t)p.slots * p.split.n_chunks * a.g.n_kv_heads * p.cols * (a.g.head_dim + 4 + 2) * sizeof(float);
}

template <int KIND, bool GROUPED, int NW>
static hipError_t launch_tiles(const MaskedAttnArgs& a, const MaskedPlan& p, unsigned grid, float* part_o, float2* part_ml, hipStream_t st) {
  static std::atomic<unsigned long long> told{0};
  const hipError_t e = allow_dynamic_lds((const void*)masked_attn_tile_kernel<KIND, GROUPED, NW>, kTileBytes, told);
  if (e != hipSuccess) return e;
  MaskedTile* const order = p.ordered ? reinterpret_cast<MaskedTile*>(part_o) : nullptr;
  if (order) masked_attn_order_kernel<<<1, kOrderThreads, 0, st>>>(a, (int)p.slots, p.rows_per_tile, order);
  masked_attn_tile_kernel<KIND, GROUPED, NW><<<grid, 64 * NW, kTileBytes, st>>>(a, p.split, (int)p.slots, p.rows_per_tile, order, part_o, part_ml);
  return hipGetLastError();
}

template <int KIND>
static hipError_t launch_bf16(const MaskedAttnArgs& a, const MaskedPlan& p, float* part_o, float2* part_ml, hipStream_t st) {
  const long grid = p.slots * p.split.n_chunks * a.g.n_kv_heads;
  if (p.rows) {
    static std::atomic<unsigned long long> told{0};
    const hipError_t e = allow_dynamic_lds((const void*)masked_attn_rows_kernel<KIND>, 4 * kRowWaveBytes, told);
    if (e != hipSuccess) return e;
    masked_attn_rows_kernel<KIND><<<(unsigned)grid, 256, 4 * kRowWaveBytes, st>>>(a, p.split, part_o, part_ml);
  } else {
    // pages of 16, 32, 64, ... slots, or one block a sequence whose slots are a multiple of 16
    const bool grouped = a.g.max_blocks == 1 ? a.g.block_size % 16 == 0 : a.g.bs_shift >= 4;
    if (p.cols == WIDE_COLS)
      return grouped ? launch_tiles<KIND, true, 8>(a, p, (unsigned)grid, part_o, part_ml, st)
                     : launch_tiles<KIND, false, 8>(a, p, (unsigned)grid, part_o, part_ml, st);
    return grouped ? launch_tiles<KIND, true, 4>(a, p, (unsigned)grid, part_o, part_ml, st)
                   : launch_tiles<KIND, false, 4>(a, p, (unsigned)grid, part_o, part_ml, st);
  }
  return hipGetLastError();
}

hipError_t launch_masked_attention(const MaskedAttnArgs& a, bool is_bf16, float* part, hipStream_t st) {
  MaskedPlan p = plan_masked(a, is_bf16);
  if (!part) p.split = {1, 0}, p.ordered = false;
  const long grid = p.slots * p.split.n_chunks * a.g.n_kv_heads, per_row = ((long)a.n_rows * a.n_q_heads + 3) / 4;
  if (grid > INT_MAX || per_row > INT_MAX) return hipErrorInvalidValue;
  float2* const part_ml = reinterpret_cast<float2*>(part + (size_t)grid * p.cols * (a.g.head_dim + 4));
  const bool cap = a.cap > 0.f, bias = a.slopes != nullptr;
  hipError_t e;
  if (!is_bf16) {
    if (a.g.head_dim == 64) masked_attn_f32_kernel<64><<<(unsigned)grid, 512, 0, st>>>(a, p.split, (int)p.slots, part, part_ml);
    else masked_attn_f32_kernel<128><<<(unsigned)grid, 256, 0, st>>>(a, p.split, (int)p.slots, part, part_ml);
    e = hipGetLastError();
  } else if (cap && bias) e = launch_bf16<kCapBias>(a, p, part, part_ml, st);
  else if (bias) e = launch_bf16<kBias>(a, p, part, part_ml, st);
  else if (!cap) e = launch_bf16<kPlain>(a, p, part, part_ml, st);
  else if (a.cap * kLog2e <= kMostBounded) e = launch_bf16<kBounded>(a, p, part, part_ml, st);
  else e = launch_bf16<kCap>(a, p, part, part_ml, st);
  if (e != hipSuccess || p.split.n_chunks <= 1) return e;
  const unsigned rows = (unsigned)per_row, by_seq = (unsigned)(((long)a.n_seq * a.max_rows_per_seq * a.n_q_heads + 3) / 4);
  if (p.rows) masked_attn_merge_kernel<bf16, DH, ROW_COLS, true><<<by_seq, 256, 0, st>>>(a, p.split, p.rows_per_tile, part, part_ml);
  else if (p.cols == WIDE_COLS) masked_attn_merge_kernel<bf16, DH, WIDE_COLS, false><<<rows, 256, 0, st>>>(a, p.split, p.rows_per_tile, part, part_ml);
  else if (is_bf16) masked_attn_merge_kernel<bf16, DH, TILE_COLS, false><<<rows, 256, 0, st>>>(a, p.split, p.rows_per_tile, part, part_ml);
  else if (a.g.head_dim == 64) masked_attn_merge_kernel<float, 64, F32_COLS, false><<<rows, 256, 0, st>>>(a, p.split, 0, part, part_ml);
  else masked_attn_merge_kernel<float, 128, F32_COLS, false><<<rows, 256, 0, st>>>(a, p.split, 0, part, part_ml);
  return hipGetLastError();
}

}  // namespace rc
