// Attention of a ragged batch against its pages, the prefix that the sequences share read once for all of them.
//
// o = sum_j e^(s_j) v_j / sum_j e^(s_j) with s_j = scale * q . k_j splits over any division of the keys: a part gives
// (m, l, o) = (m, sum e^(s - m), sum e^(s - m) v) for any reference m, and parts merge as M = max m, l = sum l e^(m - M), o = sum o e^(m - M).  So the
// shared prefix is one attention of ALL rows of the batch against the same keys, and each sequence's own keys another; what a row gets of both is merged.
//
// Two ways of taking a source of keys, whose query rows - rows x the G query heads of a kv head, packed [row][head] - share them:
//   paged_tiles   64, 128 or 256 packed rows a workgroup, keys and values through LDS: the shared prefix, prompts, verifications (bf16)
//   paged_stream  up to 32 packed rows, keys and values straight into registers: a sequence's own keys while it decodes; fp32
// and one launch has workgroups of both, so that the products of the one run beside the loads of the other.
//
// Scores and outputs are computed transposed (S^T = K Q^T, O^T = V^T P^T): a lane holds scores and outputs of one query row, the weights go from the
// first product's accumulators into the second one without leaving the registers, and both operands come from the pages as 16 bytes per lane.
// Weights are powers of two of scores less a reference, the largest score of the first keys, which moves only to one that exceeds it by
// PA_LAZY: most steps need neither a maximum across lanes nor a scaling of what is summed.  A weight is then at most 2^8, and as exact: the reference is that score rounded up, since a
// weight takes its score unrounded, and from scores of 2^31 on half a step of a float would be more than a power of two can hold.
// The bf16 kernels round the weights to bf16 for the second product (2^-9 of each on average, at random): the error is 0.0022 of the result's norm, where the output's own rounding alone
// leaves 0.0017.  With a second product of what the rounding drops it is 0.0017 too, but that is 8 % of the time in the mean over 27 calls, 37 % of 256 x 5 rows behind 16384 positions and 44 %
// of prompts (62.6 -> 90.0 us).  Their sum is held in fp32: tiles take it of the rounded weights, by dot instructions, streams of the unrounded ones.
//
// What bounds a call (0.5B heads, 14 x 64 over 2, bf16, one MI355X; kernel times):
//   few rows      the dependent steps - lengths, table, keys, scores, values, LDS - of which one token over 1024 positions takes 8.3 us; 16 x 7 rows over 256 to 4096 positions 11.5
//                 us and 3.9 for the merge, where the bytes would take 3.1
//   a prefix      of 16384 positions for 256 x 5 rows: 96 to 103 us, 740 to 790 TFLOP/s; the matrix units are busy for 34 % of that, the vector units (weights: a power of two, a product, half a
//                 conversion and half a sum each) for 44 %, and two waves of a SIMD hardly overlap the one with the other
//   prompts       seven of 100 to 2001 rows behind 1024 positions: 68 to 70 us, 650 TFLOP/s, 28 and 39 %: the same, and compute units with more workgroups than others
//   what is not finite   a row that is done over takes one wave for its keys, a row at a time: seven such prompts with a NaN in every block 28 ms, 16 x 7 rows 1.2 ms
#pragma once
#include <type_traits>

#include "common.h"
#include "pages.h"

namespace ssd {

constexpr int PA_WAVES = 4, PA_THREADS = PA_WAVES * WAVE;        // of a workgroup of tiles; streams that are by themselves have twice as many
constexpr int PA_CHUNK = 64;           // keys in which parts are counted
constexpr float PA_LAZY = 8.0f, PA_LARGE = 256.0f;
constexpr float PA_NONE = -3.402823466e38f;                      // the reference of a row that has seen nothing: no score that is a number is below it
constexpr float PA_FAINT = 0x1p-60f;   // a sum of weights below this is one of weights that have run out, or of none: the largest is 1 less a few steps of its score
typedef __attribute__((ext_vector_type(16))) float f32x16;

struct PagedAttnArgs {
  Pages p;
  const void* q;
  void* out;
  size_t q_stride, out_stride;
  const int32_t *len, *row_start, *table, *shared_table, *shared;
  int32_t* status;
  float* o_part;         // [n_rows * nq][P][hd]
  float* ml_part;        // [n_rows * nq][P][2]
  float scale2;          // scale * log2(e)
  int nq, n_seqs, n_rows, cap, shared_blocks;
  int in_line;           // 1: a sequence's keys are the shared ones and its own behind each other, and there is no source of shared ones
  int P, P_sh;           // parts of a row at most, and those of the shared prefix
  int sh_chunks;         // chunks of a part of the shared prefix
  int own_chunks;        // chunks of a part of a sequence's keys, at least
  int sh_slots, own_slots;             // tiles of query rows of the shared prefix, of the sequences: workgroups are sh_slots x P_sh x nkv and then own_slots x (P - P_sh) x nkv
};
static_assert(sizeof(PagedAttnArgs) % 4 == 0, "");

struct SeqRows {
  int r0, n;             // first row of the launch, number of rows
  int len, start;        // cached positions; first position of its keys here
  int chunks, per;       // chunks of its keys, of one part of them
  int head;              // blocks that are looked up in the shared table
  bool ok;
};
__device__ __forceinline__ SeqRows seq_rows(const PagedAttnArgs& a, int s) {
  SeqRows r;
  const int r0 = a.row_start[s], r1 = a.row_start[s + 1];
  r.len = a.len[s];
  const int own_head = a.shared ? a.shared[s] : a.shared_blocks;
  r.r0 = min(max(r0, 0), a.n_rows);
  r.n = min(max(r1, 0), a.n_rows) - r.r0;
  r.ok = r.n > 0 && r.len >= 0 && r.len <= a.cap << a.p.bt_shift;
  const int sh = a.shared_blocks << a.p.bt_shift;
  const bool joins = sh > 0 && r.len >= sh && own_head >= a.shared_blocks;
  r.start = joins && !a.in_line ? sh : 0;
  r.head = joins && a.in_line ? a.shared_blocks : 0;
  r.chunks = ceil_div(r.len + r.n - r.start, PA_CHUNK);
  r.per = max(a.own_chunks, ceil_div(r.chunks, a.P - a.P_sh));
  return r;
}

// (what the compiler cannot see to be the same in all lanes it keeps in vector registers, and makes a mask of every condition on it)
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// The last sequence s whose base(first row, s) is at most x, as wave_search() finds it, and its rows.  Of the last 64 candidates every lane looks one up whole: what the
// chosen one has is there with what it is chosen by, one step of memory earlier.  (Here and in the merge 1 % in the mean over 27 calls; 64 rows behind 4096 positions 14.3 -> 13.6 us.)
template <typename F>
__device__ __forceinline__ SeqRows find_rows(const PagedAttnArgs& a, int x, int& s, F base) {
  const int lane = threadIdx.x & 63;
  int lo = 0, step = 1;
  while (step * 64 < a.n_seqs) step *= 64;
  for (; step > 1; step /= 64) {
    const int t = lo + lane * step;
    const unsigned long long m = __ballot(t < a.n_seqs && base(min(max(a.row_start[min(t, a.n_seqs - 1)], 0), a.n_rows), t) <= x);
    lo += (63 - __builtin_clzll(m | 1ull)) * step;
  }
  const SeqRows r = seq_rows(a, min(lo + lane, a.n_seqs - 1));
  const int l = 63 - __builtin_clzll(__ballot(lo + lane < a.n_seqs && base(r.r0, lo + lane) <= x) | 1ull);
  auto from = [&](int v) { return __builtin_amdgcn_readlane(v, l); };
  s = lo + l;
  return SeqRows{from(r.r0), from(r.n), from(r.len), from(r.start), from(r.chunks), from(r.per), from(r.head), from(r.ok) != 0};
}

// What a workgroup does: packed rows row0 .. of n_packed, whose first row is seq_r0, against keys k_begin .. k_end - 1.
struct Work {
  const int32_t* table;
  int table_n, head;                   // entries; those that are looked up in the shared table instead
  int row0, n_packed, seq_r0, len;
  int k_begin, k_end;
  int slot;                            // of the partial result; -1: there is no other part, and the row is finished here
  bool shared;                         // every row sees all of the keys
};
// `id`: of this workgroup among those of its source, without the kv head; T: packed rows of a workgroup.  false: nothing to do.
__device__ __forceinline__ bool shared_work(const PagedAttnArgs& a, int id, int T, int G, Work& w) {
  const int part = id % a.P_sh;
  w.row0 = id / a.P_sh * T;
  w.n_packed = min(max(a.row_start[a.n_seqs], 0), a.n_rows) * G;
  w.table = a.shared_table;
  w.table_n = a.shared_blocks;
  w.head = w.seq_r0 = w.len = 0;
  w.k_begin = part * a.sh_chunks * PA_CHUNK;
  w.k_end = min(a.shared_blocks << a.p.bt_shift, w.k_begin + a.sh_chunks * PA_CHUNK);
  w.slot = part;
  w.shared = true;
  return w.row0 < w.n_packed;
}
__device__ __forceinline__ bool own_work(const PagedAttnArgs& a, int id, int T, int G, Work& w) {
  const int parts = a.P - a.P_sh, slot = id / parts, part = id - slot * parts;
  // (sequence s has tiles from r0 G / T + s on: room for a last one that is not full, without a list of tiles)
  int s;
  const SeqRows r = find_rows(a, slot, s, [&](int r0, int x) { return r0 * G / T + x; });
  // The last tile of a sequence, which sees the most keys, comes first: what is given out last, to compute units that are done, has the least to do.  (Seven prompts of up to
  // 2001 rows 69.6 us; ascending 74.9; all sequences' tiles in order of length, which takes a search over lengths, 73.4.)
  const int n_packed = r.n * G, tile = ceil_div(n_packed, T) - 1 - (slot - (r.r0 * G / T + s));
  w.row0 = uniform(tile * T);
  if (w.row0 < 0 || w.row0 >= n_packed) return false;      // (a slot without a tile; behind a first sequence that does not begin at row 0)
  if (!r.ok) {
    if (threadIdx.x == 0 && a.status) atomicOr(a.status, ST_BAD);
    return false;
  }
  if (part >= ceil_div(r.chunks, r.per)) return false;
  w.n_packed = uniform(n_packed);
  w.table = a.table + (size_t)uniform(s) * a.cap;
  w.table_n = a.cap;
  w.head = uniform(r.head);
  w.seq_r0 = uniform(r.r0);
  w.len = uniform(r.len);
  w.k_begin = uniform(r.start + part * r.per * PA_CHUNK);
  w.k_end = uniform(min(r.len + min(r.n - 1, (w.row0 + T - 1) / G) + 1, w.k_begin + r.per * PA_CHUNK));      // (up to the last position that a row of the tile sees)
  w.slot = uniform(r.chunks <= r.per && r.start == 0 ? -1 : a.P_sh + part);
  w.shared = false;
  return true;
}
// The block of key `key`, as the table has it; -1 behind the last key and the table's end.
__device__ __forceinline__ int block_of(const PagedAttnArgs& a, const Work& w, int key) {
  const int b = key >> a.p.bt_shift;
  return key < w.k_end && b < w.table_n ? (b < w.head ? a.shared_table[b] : w.table[b]) : -1;
}
// -1 for what is no block of the pool, and whether a key is without one.
__device__ __forceinline__ int checked_block(const PagedAttnArgs& a, const Work& w, int blk, int key, int& bad) {
  const bool there = blk >= 0 && blk < a.p.n_blocks;
  bad |= !there && key < w.k_end;
  return there ? blk : -1;
}

// No less than the product that `s` is rounded from.
__device__ __forceinline__ float above(float s) { return fmaf(fabsf(s), 0x1p-23f, s); }

// A negative factor leaves its sign with the queries, so that the largest product is the largest score; of 0 the queries become zeros (and a hidden
// key's score stays -inf), but for rows whose query is not finite, which are done over: 0 times that is NaN.
__device__ __forceinline__ float factor(const PagedAttnArgs& a) { return a.scale2 == 0.f ? 1.f : fabsf(a.scale2); }
__device__ __forceinline__ u32x4 factor_into(const PagedAttnArgs& a, u32x4 q, uint32_t signs) { return a.scale2 == 0.f ? u32x4{0, 0, 0, 0} : q ^ signs; }

// Rows that share a tile do not all see its last keys.  The weight of a hidden key is 0, and 0 times a value that is not finite is NaN, so a row with such a key and a result
// that is not finite is done over, by one wave, from the keys that it sees: the products then need no look at the values, and this is as rare as infinities in a cache are.
//   So is a row whose weights sum up to nothing although there are keys before it: its blocks are missing; its scores are so large that steps of a float decide (here they are rounded
// before they are subtracted); or all of them are -inf, and a softmax of these is NaN. Of a part, the reference -inf says so, and becomes NaN if no other part has anything.
__device__ __forceinline__ bool has_hidden(const Work& w, int G, int pr) { return !w.shared && w.len + pr / G + 1 < w.k_end; }
__device__ __forceinline__ bool has_keys(const Work& w, int G, int pr) { return w.shared || w.k_begin < w.len + pr / G + 1; }
__device__ __forceinline__ bool all_finite(f32x4 v) { return v[0] * 0.f + v[1] * 0.f + v[2] * 0.f + v[3] * 0.f == 0.f; }
// The arguments, read from where the launch put them: what only a row that is done over asks for is then in no register before that.  (With them in registers the loops over keys
// have some of their own conditions and constants in vector registers: 1 % of a call's time.)
__device__ __forceinline__ PagedAttnArgs args_again() {
  typedef const __attribute__((address_space(4))) uint32_t* Words;
  struct Copy { uint32_t w[sizeof(PagedAttnArgs) / 4]; } c;
  Words p = (Words)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
#pragma unroll
  for (int i = 0; i < (int)(sizeof(PagedAttnArgs) / 4); ++i) c.w[i] = p[i];
  return __builtin_bit_cast(PagedAttnArgs, c);
}
// A block is missing (a wave calls this; T: packed rows of a workgroup of the shared prefix, 0 of another one).  The prefix is read for all rows, also where none has it in front: then nothing is.
__device__ __forceinline__ void report_pages(const Work& w, int T, int G) {
  const PagedAttnArgs a = args_again();
  const int lane = threadIdx.x & 63;
  if (!a.status) return;
  if (T) {
    bool any = false;
    for (int s = lane; s < a.n_seqs; s += 64) {
      const SeqRows r = seq_rows(a, s);
      any |= r.n > 0 && r.start > 0 && r.r0 * G < w.row0 + T && (r.r0 + r.n) * G > w.row0;
    }
    if (!__any(any)) return;
  }
  if (lane == 0) atomicOr(a.status, ST_PAGE);
}
// Is any block of the workgroup's keys in the pool?  (Without one, as of a prefix that is not there yet, all rows are zeros as they stand: asked once, not of each row.  A wave calls it.)
__device__ __forceinline__ bool any_block(const PagedAttnArgs& a, const Work& w) {
  bool any = false;
  for (int k = w.k_begin & ~(a.p.bt - 1); k < w.k_end && !any; k += 64 << a.p.bt_shift) {
    const int blk = block_of(a, w, k + ((threadIdx.x & 63) << a.p.bt_shift));
    any = __any(blk >= 0 && blk < a.p.n_blocks);
  }
  return any;
}
template <typename DT, int HD>
__device__ __forceinline__ bool odd_query(const PagedAttnArgs& a, const Work& w, int kvh, int G, int pr) {
  const typename DT::T* q = (const typename DT::T*)a.q + (size_t)(w.seq_r0 + pr / G) * a.q_stride + (kvh * G + pr % G) * HD;
  float x = 0.f;
#pragma unroll 8
  for (int d = 0; d < HD; ++d) x = fmaf(DT::ld(q + d), 0.f, x);
  return x != 0.f;
}
template <typename DT, int HD>
__device__ __forceinline__ void redo_row(const PagedAttnArgs& a, const Work& w, int kvh, int G, int pr) {
  typedef typename DT::T T;
  constexpr int D = HD < 64 ? 1 : HD / 64;
  const int lane = threadIdx.x & 63, dim = lane & (HD - 1), row = w.seq_r0 + pr / G, head = kvh * G + pr % G, end = w.shared ? w.k_end : min(w.len + pr / G + 1, w.k_end), tmask = a.p.bt - 1;
  const T* q = (const T*)a.q + (size_t)row * a.q_stride + head * HD;
  float acc[D] = {}, mx = PA_NONE, sum = 0.f;
  const float first = a.scale2 == 0.f ? 0.f : 1.f, then = a.scale2 == 0.f ? 1.f : a.scale2;            // (of a factor of 0, as factor_into() has it)
  bool seen = false;
  for (int k0 = w.k_begin; k0 < end; k0 += 64) {
    const int key = k0 + lane;
    int bad = 0;
    const int blk = key < end ? checked_block(a, w, block_of(a, w, key), key, bad) : -1;
    if (!__any(blk >= 0)) continue;
    seen = true;
    float s = -INFINITY;
    if (blk >= 0) {
      const T* kp = (const T*)a.p.keys + (((size_t)blk * a.p.nkv + kvh) * a.p.bt + (key & tmask)) * HD;
      float dot = 0.f;
#pragma unroll 8
      for (int d = 0; d < HD; ++d) dot = fmaf(DT::ld(q + d) * first, DT::ld(kp + d), dot);
      s = dot * then;
    }
    const float m = wave_max(s);
    if (m > mx) {
      const float keep = __builtin_amdgcn_exp2f(mx - m);
      mx = m;
      sum *= keep;
#pragma unroll
      for (int j = 0; j < D; ++j) acc[j] *= keep;
    }
    const float weight = __builtin_amdgcn_exp2f(s - mx);
    sum += wave_sum(weight);
    const int n = min(64, end - k0);
#pragma unroll 1
    for (int i = 0; i < n; i += 8) {                       // (eight keys' values asked for at once)
      float v[8][D];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int key_i = min(i + e, n - 1), b = max(__builtin_amdgcn_readlane(blk, key_i), 0);
        const T* vp = (const T*)a.p.values + (((size_t)b * a.p.nkv + kvh) * HD + dim) * a.p.bt + ((k0 + key_i) & tmask);
#pragma unroll
        for (int j = 0; j < D; ++j) v[e][j] = DT::ld(vp + 64 * j * a.p.bt);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int key_i = min(i + e, n - 1);
        if (i + e >= n || __builtin_amdgcn_readlane(blk, key_i) < 0) continue;
        const float f = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(weight), key_i));
#pragma unroll
        for (int j = 0; j < D; ++j) acc[j] = fmaf(f, v[e][j], acc[j]);
      }
    }
  }
  const size_t at = ((size_t)row * a.nq + head) * a.P + w.slot;
  if (seen && sum == 0.f) mx = -INFINITY;
#pragma unroll
  for (int j = 0; j < D; ++j) {
    if (lane >= HD) continue;
    if (w.slot < 0) DT::st((T*)a.out + (size_t)row * a.out_stride + head * HD + dim + 64 * j, sum == 0.f ? (seen ? NAN : 0.f) : acc[j] / sum);
    else a.o_part[at * HD + dim + 64 * j] = acc[j];
  }
  if (w.slot >= 0 && lane == 0) { a.ml_part[at * 2] = mx; a.ml_part[at * 2 + 1] = sum; }
}

// ---------------------------------------------------------------------------------------------- few rows: from the pages into registers
//   bf16  16x16x32 products.  Of a pair of 16-key tiles, row m of tile t is key 8 (m / 4) + 4 t + m % 4: lane group g = lane / 16 then ends with the scores of
//         keys 8 g .. 8 g + 7, whose values it holds as the second product's operand.
//   fp32  16x16x4 products: lane group g ends with keys 4 g .. 4 g + 3 of a tile.
// A workgroup has up to RT tiles of 16 rows; its waves take steps of 16 NT keys in turn, each with references, sums and outputs of its own, and meet in
// LDS.  The next step's keys are requested when this one's have been multiplied, its values likewise.  Bound by the loads' latency, of which a wave has one step's in flight: where streams
// are by themselves they have eight waves, and keys that eight waves take in two or three steps need no parts (one token over 1024 positions: 10.2 us, in parts with a merge 14.6).
// Through LDS keys would be written and read once each: no other wave wants them.
template <typename DT, int HD>
struct StreamShape {
  static constexpr bool B16 = sizeof(typename DT::T) == 2;
  static constexpr int FIT = 512 / (HD * (int)sizeof(typename DT::T)), NT = FIT < 4 ? FIT : 4, STEP = 16 * NT;      // keys and values of a step take 64 registers, or 32
  static constexpr int KU = B16 ? HD / 32 : HD / 16;       // 16-byte units of a key, or of a query row, that a lane has
  static constexpr int VU = HD / 16, VT = B16 ? NT / 2 : NT;           // dim tiles; pairs of key tiles, or tiles, that a value operand spans
  static constexpr int LDS = 4 * 16 * (HD + 4) + 2 * 4 * 16;                       // floats: what four waves have of 16 rows
};

template <typename DT, int HD, int RT, int W, bool SHARED>
__device__ __forceinline__ void paged_stream(const PagedAttnArgs& a, int id, float* lds) {
  typedef typename DT::T T;
  typedef StreamShape<DT, HD> S;
  constexpr bool B16 = S::B16;
  constexpr int NT = S::NT, STEP = S::STEP, KU = S::KU, VU = S::VU, VT = S::VT;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), li = lane & 15, g = lane >> 4;
  const int nkv = a.p.nkv, G = a.nq / nkv, kvh = id % nkv, tmask = a.p.bt - 1;
  id /= nkv;
  Work w;
  if (!(SHARED ? shared_work(a, id, 16 * RT, G, w) : own_work(a, id, 16 * RT, G, w))) return;
  const int rows = min(16 * RT, w.n_packed - w.row0);      // (uniform: tiles behind the last row are left out)
  const int pos_lo = w.shared ? 0x7FFFFFFF : w.len + w.row0 / G;
  // block ids of the wave's next 64 / NT steps: lane NT i + t has that of tile t of step i
  int bad = 0;
  auto key_of = [&](int step) { return w.k_begin + ((step + lane / NT) * W + wave) * STEP + lane % NT * 16; };
  int ids = block_of(a, w, key_of(0));
  int pos[RT];
  u32x4 q[RT][KU];
#pragma unroll
  for (int x = 0; x < RT; ++x) {
    const int pr = w.row0 + min(16 * x + li, rows - 1), row = w.seq_r0 + pr / G, head = kvh * G + pr % G;
    pos[x] = w.shared ? 0x7FFFFFFF : w.len + pr / G;
    const u32x4* qp = (const u32x4*)((const T*)a.q + row * a.q_stride + head * HD) + g;
#pragma unroll
    for (int u = 0; u < KU; ++u) q[x][u] = qp[u * 4];
  }
  ids = checked_block(a, w, ids, key_of(0), bad);
  const float scale2 = factor(a);
  if (a.scale2 <= 0.f) {
#pragma unroll
    for (int x = 0; x < RT; ++x)
#pragma unroll
      for (int u = 0; u < KU; ++u) q[x][u] = factor_into(a, q[x][u], B16 ? 0x80008000u : 0x80000000u);
  }
  f32x4 o[RT][VU];
  float m[RT], l[RT];
#pragma unroll
  for (int x = 0; x < RT; ++x) {
    m[x] = PA_NONE;
    l[x] = 0.f;
#pragma unroll
    for (int d = 0; d < VU; ++d) o[x][d] = f32x4{0, 0, 0, 0};
  }
  const size_t head_elems = (size_t)a.p.bt * HD, block_elems = head_elems * nkv;
  const T* keys = (const T*)a.p.keys + kvh * head_elems;
  const T* values = (const T*)a.p.values + kvh * head_elems;
  u32x4 kf[NT][KU], vf[VT][VU];
  // (`base`: of the step's tiles among the ids; `k0`: its first key)
  auto load_keys = [&](int base, int k0) {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int key = k0 + (B16 ? 32 * (t >> 1) + 8 * (li >> 2) + 4 * (t & 1) + (li & 3) : 16 * t + li);
      const int b0 = __builtin_amdgcn_readlane(ids, base + (B16 ? t & ~1 : t)), b1 = B16 ? __builtin_amdgcn_readlane(ids, base + (t | 1)) : b0;
      const int blk = max(B16 && li >= 8 ? b1 : b0, 0);
      const u32x4* kp = (const u32x4*)(keys + (size_t)blk * block_elems + (key & tmask) * HD) + g;
#pragma unroll
      for (int u = 0; u < KU; ++u) kf[t][u] = kp[u * 4];
    }
  };
  auto load_values = [&](int base, int k0) {
#pragma unroll
    for (int t = 0; t < VT; ++t) {
      const int key = k0 + (B16 ? 32 * t + 8 * g : 16 * t + 4 * g);
      const int b0 = __builtin_amdgcn_readlane(ids, base + (B16 ? 2 * t : t)), b1 = B16 ? __builtin_amdgcn_readlane(ids, base + 2 * t + 1) : b0;
      const int blk = max(B16 && g >= 2 ? b1 : b0, 0);
      const T* vp = values + (size_t)blk * block_elems + (key & tmask);
#pragma unroll
      for (int d = 0; d < VU; ++d) vf[t][d] = *(const u32x4*)(vp + (d * 16 + li) * a.p.bt);
    }
  };
  const int n_steps = max(0, ceil_div(w.k_end - w.k_begin, STEP)), mine = (n_steps - wave + W - 1) / W;
  const int first_key = w.k_begin + wave * STEP;
  if (mine > 0) { load_keys(0, first_key); load_values(0, first_key); }
  constexpr int PER = 64 / NT;                             // steps of a wave whose ids are at hand
  unsigned long long have = __ballot(ids >= 0);
  for (int i = 0; i < mine; ++i) {
    const int k0 = first_key + i * W * STEP;
    const int there = (int)(have >> (i % PER * NT)) & ((1 << NT) - 1);
    const bool more = i + 1 < mine, refill = more && (i + 1) % PER == 0;
    if (refill) {                                          // (this step's blocks are in `there`, its loads on their way)
      ids = checked_block(a, w, block_of(a, w, key_of(i + 1)), key_of(i + 1), bad);
      have = __ballot(ids >= 0);
    }
    const int base_next = (i + 1) % PER * NT, k_next = k0 + W * STEP;
    const bool edge = there != (1 << NT) - 1 || k0 + STEP > w.k_end || k0 + STEP - 1 > pos_lo;
    if (edge) {
#pragma unroll
      for (int t = 0; t < VT; ++t) {                       // values that are not there may be anything: they become zeros
        const bool page = there >> (B16 ? 2 * t + (g >> 1) : t) & 1;
        const int n = page ? w.k_end - k0 - (B16 ? 32 * t + 8 * g : 16 * t + 4 * g) : 0;
        u32x4 keep;
#pragma unroll
        for (int e = 0; e < 4; ++e) keep[e] = B16 ? (2 * e < n ? 0xFFFFu : 0u) | (2 * e + 1 < n ? 0xFFFF0000u : 0u) : e < n ? 0xFFFFFFFFu : 0u;
#pragma unroll
        for (int d = 0; d < VU; ++d) vf[t][d] &= keep;
      }
    }
#pragma unroll
    for (int x = 0; x < RT; ++x) {
      if (16 * x >= rows) break;
      f32x4 s[NT];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        s[t] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int u = 0; u < KU; ++u) {
          if constexpr (B16) {
            s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf[t][u]), __builtin_bit_cast(bf16x8, q[x][u]), s[t], 0, 0, 0);
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) s[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kf[t][u][e]), __uint_as_float(q[x][u][e]), s[t], 0, 0, 0);
          }
        }
      }
      if (more && (x == RT - 1 || 16 * (x + 1) >= rows)) load_keys(base_next, k_next);
      if (edge) {
        const int last = min(pos[x], w.k_end - 1) - k0 - (B16 ? 8 : 4) * g;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const int first = B16 ? 32 * (t >> 1) + 4 * (t & 1) : 16 * t;              // of the lane's four keys, less 8 g or 4 g
          const bool page = there >> (B16 ? (t & ~1) + (g >> 1) : t) & 1;
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (!page || first + e > last) s[t][e] = -INFINITY;
        }
      }
      float mx = s[0][0];
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) mx = fmaxf(mx, s[t][e]);
      mx = above(mx * scale2);
      if (__any(mx > m[x] + PA_LAZY)) {
        mx = max_over_groups(mx);
        if (mx > m[x] + PA_LAZY) {
          const float keep = __builtin_amdgcn_exp2f(m[x] - mx);
          m[x] = mx;
          l[x] *= keep;
#pragma unroll
          for (int d = 0; d < VU; ++d) o[x][d] *= keep;
        }
      }
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s[t][e] = __builtin_amdgcn_exp2f(fmaf(s[t][e], scale2, -m[x]));
          l[x] += s[t][e];
        }
#pragma unroll
      for (int t = 0; t < VT; ++t) {
        if constexpr (B16) {
          const f32x4 lo = s[2 * t], hi = s[2 * t + 1];
          const u32x4 pw = {f2_to_bf16x2(lo[0], lo[1]), f2_to_bf16x2(lo[2], lo[3]), f2_to_bf16x2(hi[0], hi[1]), f2_to_bf16x2(hi[2], hi[3])};
#pragma unroll
          for (int d = 0; d < VU; ++d)
            o[x][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vf[t][d]), __builtin_bit_cast(bf16x8, pw), o[x][d], 0, 0, 0);
        } else {
#pragma unroll
          for (int d = 0; d < VU; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[x][d] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vf[t][d][e]), s[t][e], o[x][d], 0, 0, 0);
        }
      }
    }
    if (more) load_values(base_next, k_next);
  }
  if (__builtin_expect(__any(bad), 0)) report_pages(w, SHARED ? 16 * RT : 0, G);
  uint32_t again = 0;                                      // rows of which this lane has written something that is to be done over
  float (*po)[16][HD + 4] = (float (*)[16][HD + 4])lds;
  float (*pm)[16] = (float (*)[16])(lds + 4 * 16 * (HD + 4)), (*pl)[16] = pm + 4;
#pragma unroll
  for (int x = 0; x < RT; ++x) {
    if (16 * x >= rows) break;
    if (x) __syncthreads();
    float ls = sum_over_groups(l[x]);
    auto leave = [&](int at) {
#pragma unroll
      for (int d = 0; d < VU; ++d) *(f32x4*)&po[at][li][d * 16 + g * 4] = o[x][d];
      if (g == 0) { pm[at][li] = m[x]; pl[at][li] = ls; }
    };
    if constexpr (W == 8) {                                // the upper four waves' go to the lower four
      if (wave >= 4) leave(wave - 4);
      __syncthreads();
      if (wave < 4) {
        const float m1 = pm[wave][li], mx = fmaxf(m[x], m1), f0 = __builtin_amdgcn_exp2f(m[x] - mx), f1 = __builtin_amdgcn_exp2f(m1 - mx);
        m[x] = mx;
        ls = ls * f0 + pl[wave][li] * f1;
#pragma unroll
        for (int d = 0; d < VU; ++d) o[x][d] = o[x][d] * f0 + *(const f32x4*)&po[wave][li][d * 16 + g * 4] * f1;
        leave(wave);                                       // (where it has read)
      }
    } else {
      leave(wave);
    }
    __syncthreads();
    for (int i = tid; i < 16 * (HD / 4); i += W * WAVE) {
      const int r = i / (HD / 4), d = (i - r * (HD / 4)) * 4;
      if (16 * x + r >= rows) break;
      float mx = pm[0][r];
#pragma unroll
      for (int y = 1; y < 4; ++y) mx = fmaxf(mx, pm[y][r]);
      float sum = 0.f;
      f32x4 acc = {0, 0, 0, 0};
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        const float f = __builtin_amdgcn_exp2f(pm[y][r] - mx);
        sum = fmaf(pl[y][r], f, sum);
        acc += *(const f32x4*)&po[y][r][d] * f;
      }
      const int pr = w.row0 + 16 * x + r, row = w.seq_r0 + pr / G, head = kvh * G + pr % G;
      if (!SHARED && !all_finite(acc) ? has_hidden(w, G, pr) : sum < PA_FAINT && has_keys(w, G, pr)) again |= 1u << (16 * x + r);
      if (w.slot < 0) {
        T* dst = (T*)a.out + (size_t)row * a.out_stride + head * HD + d;
        acc *= sum == 0.f ? 0.f : 1.f / sum;
        if constexpr (B16) *(uint2*)dst = make_uint2(f2_to_bf16x2(acc[0], acc[1]), f2_to_bf16x2(acc[2], acc[3]));
        else *(f32x4*)dst = acc;
      } else {
        const size_t at = ((size_t)row * a.nq + head) * a.P + w.slot;
        *(f32x4*)(a.o_part + at * HD + d) = acc;
        if (d == 0) { a.ml_part[at * 2] = mx; a.ml_part[at * 2 + 1] = sum; }
      }
    }
  }
  if (__builtin_expect(__any(again) || a.scale2 == 0.f, 0)) {          // (or its code stands before the end that every call comes to)
    // (one wave has written the whole of a row; it writes it again behind that)
    __builtin_amdgcn_s_waitcnt(0x0070);
    const PagedAttnArgs b = args_again();
    if (!any_block(b, w)) return;
    if (b.scale2 == 0.f && lane < rows && (lane & 15) * (HD / 4) / WAVE % W == wave && odd_query<DT, HD>(b, w, kvh, G, w.row0 + lane)) again |= 1u << lane;
    for (int r = 0; r < rows; ++r)
      if (__any(again >> r & 1)) redo_row<DT, HD>(b, w, kvh, G, w.row0 + r);
  }
}

// ---------------------------------------------------------------------------------------------- many rows: through LDS (bf16)
// A workgroup takes 128 QS packed query rows, 32 QS a wave, and a part of the keys, whose 64-key chunks all of its waves read from LDS, where direct
// loads put them a chunk ahead (wave w the 16 keys w of a chunk, which lie in one block).  With KW 2 it takes half the rows: two waves have the same ones, one the
// first 32 keys of every chunk and one the others, and meet in LDS at the end.  (Verifications have few more than 32 rows: two of four waves would be idle.  16 x 7 rows: 15.0 us, with
// 128 15.5, by streams 16.4.)  32x32x16 products: a lane holds the scores of one row
// (lane % 32) for keys 16 (i / 8) + 8 h + i % 8 of a 32-key tile (i: register, h = lane / 32) if row m of the tile's operand is the key whose bits 2 and 3
// are those of m swapped; these are the operand of the second product as they stand.
//   A direct load brings 1 KB of consecutive memory where the layout has it, so keys are parked [group of 16][key][16-byte unit] and values [group of
// 16][dim][8-key half], with unit u of key t at u ^ (t >> (4 - log2 units)) and half x of dim d at x ^ (d >> 3 & 1): the sixteen lanes of a read then
// have sixteen distinct quads of banks.
template <int HD>
struct TileShape {
  static constexpr int J = HD / 32;
  typedef u32x4 Lds[2][2][4][J][64];   // [buffer][keys, values][group][..]
};

template <int HD, int QS, int KW, bool SHARED>
__device__ __forceinline__ void paged_tiles(const PagedAttnArgs& a, int id, typename TileShape<HD>::Lds& kv_lds) {
  constexpr int J = HD / 32, T = 128 * QS / KW, NT = 2 / KW;         // NT: 32-key tiles of a chunk that a wave multiplies, from t0 on
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 31, h = lane >> 5;
  const int nkv = a.p.nkv, G = a.nq / nkv, kvh = id % nkv, tmask = a.p.bt - 1;
  id /= nkv;
  Work w;
  if (!(SHARED ? shared_work(a, id, T, G, w) : own_work(a, id, T, G, w))) return;
  const int n_chunks = max(0, ceil_div(w.k_end - w.k_begin, PA_CHUNK));
  // this wave's rows and what they see
  const int w0 = w.row0 + wave % (4 / KW) * 32 * QS, t0 = KW == 2 ? wave >> 1 : 0;
  const bool has_rows = w0 < w.n_packed;
  const int reach = !has_rows ? -1 : w.shared ? 0x7FFFFFFF : w.len + (min(w0 + 32 * QS, w.n_packed) - 1) / G;
  const int full_to = min(w.k_end, w.shared ? 0x7FFFFFFF : w.len + w0 / G + 1);        // keys before this one are there for all of the wave's rows
  // block ids of 16 chunks at a time: lane i has that of keys 16 i .. of them; and the next 16 chunks', looked at when their turn comes
  int bad = 0;
  auto key_of = [&](int chunk) { return w.k_begin + chunk * PA_CHUNK + lane * 16; };
  int ids = block_of(a, w, key_of(0)), ids_next = block_of(a, w, key_of(16));
  int row[QS], head[QS];
  bf16x8 q[QS][2 * J];
#pragma unroll
  for (int x = 0; x < QS; ++x) {
    const int pr = min(w0 + 32 * x + c, w.n_packed - 1);
    row[x] = w.seq_r0 + pr / G;
    head[x] = kvh * G + pr % G;
    const u32x4* qp = (const u32x4*)((const bf16_t*)a.q + row[x] * a.q_stride + head[x] * HD) + h;
#pragma unroll
    for (int s = 0; s < 2 * J; ++s) q[x][s] = __builtin_bit_cast(bf16x8, qp[2 * s]);
  }
  ids = checked_block(a, w, ids, key_of(0), bad);
  unsigned long long have = __ballot(ids >= 0);            // a bit for each group of 16 keys whose block is there
  const float scale2 = factor(a);
  if (a.scale2 <= 0.f) {
#pragma unroll
    for (int x = 0; x < QS; ++x)
#pragma unroll
      for (int s = 0; s < 2 * J; ++s) q[x][s] = __builtin_bit_cast(bf16x8, factor_into(a, __builtin_bit_cast(u32x4, q[x][s]), 0x80008000u));
  }
  // units of a key; a load's lanes have keys t, t + 64 / UNITS, ..
  constexpr int UNITS = HD / 8, SW = UNITS == 4 ? 2 : UNITS == 8 ? 1 : 0;
  int k_off[J];
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int t = j * (64 / UNITS) + lane / UNITS;
    k_off[j] = (t * HD + ((lane % UNITS) ^ (t >> SW & (UNITS - 1))) * 8) * 2;
  }
  const int v_half = (lane & 1) ^ (lane >> 4 & 1), v_off = ((lane >> 1) * a.p.bt + v_half * 8) * 2, v_dims = 32 * a.p.bt * 2;
  const uint32_t head_bytes = (uint32_t)a.p.bt * HD * 2, block_bytes = head_bytes * nkv;            // (< 2^28)
  const char* keys = (const char*)a.p.keys + (size_t)kvh * head_bytes;
  const char* values = (const char*)a.p.values + (size_t)kvh * head_bytes;
  int tok = (w.k_begin + wave * 16) & tmask;               // of this wave's group of the chunk that is requested next
  auto request = [&](int it) {
    const uint32_t blk = (uint32_t)max(__builtin_amdgcn_readlane(ids, (it & 15) * 4 + wave), 0);
    const size_t at = (size_t)blk * block_bytes;
    const rsrc_t rk = load_rsrc(keys + at + tok * (HD * 2)), rv = load_rsrc(values + at + tok * 2);
#pragma unroll
    for (int j = 0; j < J; ++j) load_to_lds(rk, &kv_lds[it & 1][0][wave][j][0], k_off[j], 0);
#pragma unroll
    for (int j = 0; j < J; ++j) load_to_lds(rv, &kv_lds[it & 1][1][wave][j][0], v_off, j * v_dims);
    tok = (tok + PA_CHUNK) & tmask;
  };
  const int kk = (c & 19) | (c & 4) << 1 | (c & 8) >> 1;   // the key that row c of a tile's operand is
  f32x16 o[QS][J];
  float m[QS], l[QS];
#pragma unroll
  for (int x = 0; x < QS; ++x) {
    m[x] = PA_NONE;
    l[x] = 0.f;
#pragma unroll
    for (int d = 0; d < J; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[x][d][i] = 0.f;
  }
  if (n_chunks > 0) request(0);
  bool first = true;                                       // (the same in all lanes)
  for (int it = 0; it < n_chunks; ++it) {
    const int kbase = w.k_begin + it * PA_CHUNK;
    const int now = (int)(have >> ((it & 15) * 4)) & 15;
    // (the builtin: with a wait in assembly the compiler places waits of its own for the queries, and with them for the chunk that was just requested)
    __builtin_amdgcn_s_waitcnt(0x0070);                    // vmcnt(0) lgkmcnt(0): the chunk has arrived, and nothing is still to be read of the one whose buffer is next
    asm volatile("" ::: "memory");
    if (now != 15 || kbase + PA_CHUNK > w.k_end) {
      // values of this wave's group that are not there may be anything: they become zeros
      const int n_tok = (now >> wave & 1) ? w.k_end - (kbase + wave * 16) : 0;
      if (n_tok < 16) {
#pragma unroll
        for (int j = 0; j < J; ++j) {
          u32x4 v = kv_lds[it & 1][1][wave][j][lane];
          const int n = n_tok - 8 * v_half;
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] &= (2 * e < n ? 0xFFFFu : 0u) | (2 * e + 1 < n ? 0xFFFF0000u : 0u);
          kv_lds[it & 1][1][wave][j][lane] = v;
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      }
    }
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (it + 1 < n_chunks) {
      if ((it & 15) == 15) {
        ids = checked_block(a, w, ids_next, key_of(it + 1), bad);
        have = __ballot(ids >= 0);
        ids_next = block_of(a, w, key_of(it + 17));
      }
      request(it + 1);
    }
    if (kbase + 32 * t0 > reach) continue;
    const bool edge = now != 15 || kbase + PA_CHUNK > full_to;
    // Weights by the references that the rows have; if some row's come out too large - the first chunk's always do - they are taken again, after a look at the
    // largest scores, from the keys, which are still at hand.
    bf16x8 p[QS][2 * NT];
    float sum[QS];
    auto weigh = [&](auto look) {
      f32x16 s[QS][NT];
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int x = 0; x < QS; ++x)
#pragma unroll
          for (int i = 0; i < 16; ++i) s[x][t][i] = 0.f;
      bf16x8 kf[2 * J][NT];
#pragma unroll
      for (int k = 0; k < 2 * J; ++k)
#pragma unroll
        for (int t = 0; t < NT; ++t)
          kf[k][t] = __builtin_bit_cast(bf16x8, (&kv_lds[it & 1][0][2 * (t0 + t) + (kk >> 4)][0][0])[(kk & 15) * UNITS + ((2 * k + h) ^ ((kk & 15) >> SW & (UNITS - 1)))]);
#pragma unroll
      for (int k = 0; k < 2 * J; ++k)                      // (chains side by side, or each product waits for the one before)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int x = 0; x < QS; ++x) s[x][t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[k][t], q[x][k], s[x][t], 0, 0, 0);
      if (edge) {
#pragma unroll
        for (int x = 0; x < QS; ++x) {
          const int pos = w.shared ? 0x7FFFFFFF : w.len + row[x] - w.seq_r0;
          const int last = min(pos, w.k_end - 1) - kbase - 32 * t0 - 8 * h;  // of this lane's keys, less 8 h
#pragma unroll
          for (int y = 0; y < 2 * NT; ++y) {
            int last_y = now >> (2 * t0 + y) & 1 ? last : -1;
            asm volatile("" : "+v"(last_y));                                 // (or the comparisons are made for every chunk)
#pragma unroll
            for (int i = 0; i < 8; ++i)
              if (16 * y + i > last_y) s[x][y >> 1][(y & 1) * 8 + i] = -INFINITY;
          }
        }
      }
      if constexpr (decltype(look)::value) {
#pragma unroll
        for (int x = 0; x < QS; ++x) {
          float mx = s[x][0][0];
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[x][t][i]);
          const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
          mx = above(fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1])) * scale2);
          if (mx > m[x]) {
            const float keep = __builtin_amdgcn_exp2f(m[x] - mx);
            m[x] = mx;
            l[x] *= keep;
#pragma unroll
            for (int d = 0; d < J; ++d) o[x][d] *= keep;
          }
        }
      }
      bool large = false;
#pragma unroll
      for (int x = 0; x < QS; ++x) {
        sum[x] = 0.f;
#pragma unroll
        for (int k = 0; k < 2 * NT; ++k) {
          u32x4 w4;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int i = (k & 1) * 8 + 2 * e;
            const uint32_t two = f2_to_bf16x2(__builtin_amdgcn_exp2f(fmaf(s[x][k >> 1][i], scale2, -m[x])), __builtin_amdgcn_exp2f(fmaf(s[x][k >> 1][i + 1], scale2, -m[x])));
            w4[e] = two;                                   // (a bit cast of a vector's element is one of its first)
            sum[x] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, two), __builtin_bit_cast(bf16x2_t, 0x3F803F80u), sum[x], false);
          }
          p[x][k] = __builtin_bit_cast(bf16x8, w4);
        }
        large |= !(sum[x] <= PA_LARGE);
      }
      return __any(large) != 0;
    };
    // The values' operands are asked for ahead of the weights, which take longer than LDS does, where there are registers for them (with QS 2 it gains
    // nothing): seven prompts 66.8 -> 63.8 us in a graph, 9 sequences of up to 919 rows with heads of 128 38.5 -> 35.5, 2 % in the mean over 29 calls.
    auto values_of = [&](int k, int d) { return __builtin_bit_cast(bf16x8, kv_lds[it & 1][1][2 * t0 + k][d][2 * c + (h ^ (c >> 3 & 1))]); };
    bf16x8 vf[QS == 1 ? 2 * NT : 1][J];
    if constexpr (QS == 1) {
#pragma unroll
      for (int k = 0; k < 2 * NT; ++k)
#pragma unroll
        for (int d = 0; d < J; ++d) vf[k][d] = values_of(k, d);
      __builtin_amdgcn_sched_barrier(0);                   // (or they are made where they are used)
    }
    if (first || weigh(std::false_type())) weigh(std::true_type());
    first = false;
#pragma unroll
    for (int x = 0; x < QS; ++x) l[x] += sum[x];
#pragma unroll
    for (int k = 0; k < 2 * NT; ++k)
#pragma unroll
      for (int d = 0; d < J; ++d) {
        const bf16x8 v = QS == 1 ? vf[QS == 1 ? k : 0][d] : values_of(k, d);
#pragma unroll
        for (int x = 0; x < QS; ++x) o[x][d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, p[x][k], o[x][d], 0, 0, 0);
      }
  }
  if (__builtin_expect(__any(bad), 0)) report_pages(w, SHARED ? T : 0, G);
  if constexpr (KW == 2) {
    // the second wave's references, sums and outputs: [wave][QS][4 J + 1][lane] of four
    static_assert(2 * QS * (4 * J + 1) * 64 <= 16 * J * 64, "");
    f32x4* x4 = (f32x4*)&kv_lds[0][0][0][0][0] + (size_t)(wave & 1) * (QS * (4 * J + 1) * 64) + lane;
    __syncthreads();                                       // (the last chunk has been read)
    if (t0) {
#pragma unroll
      for (int x = 0; x < QS; ++x) {
#pragma unroll
        for (int d = 0; d < J; ++d)
#pragma unroll
          for (int e = 0; e < 4; ++e) x4[(x * (4 * J + 1) + d * 4 + e) * 64] = f32x4{o[x][d][4 * e], o[x][d][4 * e + 1], o[x][d][4 * e + 2], o[x][d][4 * e + 3]};
        x4[(x * (4 * J + 1) + 4 * J) * 64] = f32x4{m[x], l[x], 0.f, 0.f};
      }
    }
    __syncthreads();
    if (t0) return;
#pragma unroll
    for (int x = 0; x < QS; ++x) {
      const f32x4 ml = x4[(x * (4 * J + 1) + 4 * J) * 64];
      const float mx = fmaxf(m[x], ml[0]), f0 = __builtin_amdgcn_exp2f(m[x] - mx), f1 = __builtin_amdgcn_exp2f(ml[0] - mx);
      m[x] = mx;
      l[x] = l[x] * f0 + ml[1] * f1;
#pragma unroll
      for (int d = 0; d < J; ++d)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const f32x4 v = x4[(x * (4 * J + 1) + d * 4 + e) * 64];
#pragma unroll
          for (int i = 0; i < 4; ++i) o[x][d][4 * e + i] = o[x][d][4 * e + i] * f0 + v[i] * f1;
        }
    }
  }
#pragma unroll
  for (int x = 0; x < QS; ++x) {
    const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(l[x]), __float_as_uint(l[x]), false, false);
    const float ls = __uint_as_float(both[0]) + __uint_as_float(both[1]);
    f32x4 any = {0, 0, 0, 0};
#pragma unroll
    for (int d = 0; d < J; ++d)
#pragma unroll
      for (int e = 0; e < 4; ++e) any += f32x4{o[x][d][4 * e], o[x][d][4 * e + 1], o[x][d][4 * e + 2], o[x][d][4 * e + 3]} * 0.f;
    const int pr = w0 + 32 * x + c;
    const bool odd = !SHARED && !all_finite(any);
    if (pr < w.n_packed) {
      // dims 32 d + 8 e + 4 h .. + 3 in registers 4 e ..
      if (w.slot < 0) {
        const float inv = ls == 0.f ? 0.f : 1.f / ls;
        bf16_t* dst = (bf16_t*)a.out + row[x] * a.out_stride + head[x] * HD + 4 * h;
#pragma unroll
        for (int d = 0; d < J; ++d)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            *(uint2*)(dst + 32 * d + 8 * e) = make_uint2(f2_to_bf16x2(o[x][d][4 * e] * inv, o[x][d][4 * e + 1] * inv), f2_to_bf16x2(o[x][d][4 * e + 2] * inv, o[x][d][4 * e + 3] * inv));
      } else {
        const size_t at = ((size_t)row[x] * a.nq + head[x]) * a.P + w.slot;
        float* dst = a.o_part + at * HD + 4 * h;
#pragma unroll
        for (int d = 0; d < J; ++d)
#pragma unroll
          for (int e = 0; e < 4; ++e) *(f32x4*)(dst + 32 * d + 8 * e) = f32x4{o[x][d][4 * e], o[x][d][4 * e + 1], o[x][d][4 * e + 2], o[x][d][4 * e + 3]};
        if (h == 0) { a.ml_part[at * 2] = m[x]; a.ml_part[at * 2 + 1] = ls; }
      }
    }
    if (__builtin_expect(has_rows && (__any(odd || ls < PA_FAINT) || a.scale2 == 0.f), 0)) {
      __builtin_amdgcn_s_waitcnt(0x0070);
      const PagedAttnArgs b = args_again();
      if (!any_block(b, w)) continue;
      const unsigned long long again = __ballot(pr < w.n_packed && ((odd ? has_hidden(w, G, pr) : ls < PA_FAINT && has_keys(w, G, pr)) ||
                                                                    (b.scale2 == 0.f && odd_query<BF16, HD>(b, w, kvh, G, pr))));
      for (uint32_t rows = (uint32_t)(again | again >> 32); rows; rows &= rows - 1) redo_row<BF16, HD>(b, w, kvh, G, w0 + 32 * x + __builtin_ctz(rows));
    }
  }
}

// The shared prefix first: its workgroups have the most to do.  SH: by tiles of 128 or 256 rows (1, 2), by streams (3), none (0); OWN: by tiles of 128 rows (0), by tiles of 64 (3), by streams of up to 16 (1);
// fp32 by streams of up to 16 or 32 rows (1, 2), of four waves where there is no other source (4, 5).
template <int SH, int OWN>
struct PagedShape {
  static constexpr bool STREAMS = OWN != 0 && OWN != 3, TILES = SH == 1 || SH == 2 || !STREAMS;
  static constexpr int RT = OWN > 3 ? OWN - 3 : OWN, W = TILES || OWN > 3 ? PA_WAVES : 8, THREADS = W * WAVE;
};
template <typename DT, int HD, int SH, int OWN>
__global__ void __launch_bounds__((PagedShape<SH, OWN>::THREADS), 2) k_paged_attention(PagedAttnArgs a) {
  typedef PagedShape<SH, OWN> S;
  constexpr int TILE_BYTES = S::TILES ? (int)sizeof(typename TileShape<HD>::Lds) : 0, STREAM_BYTES = S::STREAMS ? StreamShape<DT, HD>::LDS * (int)sizeof(float) : 0;
  __shared__ __align__(16) unsigned char lds[TILE_BYTES > STREAM_BYTES ? TILE_BYTES : STREAM_BYTES];
  int id = blockIdx.x;
  if constexpr (SH > 0) {
    const int n = a.sh_slots * a.P_sh * a.p.nkv;
    if (id < n) {
      if constexpr (SH == 3) paged_stream<DT, HD, S::RT, S::W, true>(a, id, (float*)lds);
      else paged_tiles<HD, SH, 1, true>(a, id, *(typename TileShape<HD>::Lds*)lds);
      return;
    }
    id -= n;
  }
  if constexpr (OWN == 0) paged_tiles<HD, 1, 1, false>(a, id, *(typename TileShape<HD>::Lds*)lds);
  else if constexpr (OWN == 3) paged_tiles<HD, 1, 2, false>(a, id, *(typename TileShape<HD>::Lds*)lds);
  else paged_stream<DT, HD, S::RT, S::W, false>(a, id, (float*)lds);
}

// Rows that have several parts, one wave per row and head: a lane has four dims of every STEP-th part, and all loads go out at once; the parts' factors go from lane
// to lane.  Ascending parts in each lane, then lane by lane in a fixed order.  4 us for being a launch; 256 x 5 rows in 8 parts, 38 MB, 11.6 us.  (The last part to arrive could
// merge, but its release and acquire cost more, and the counters would have to be zeroed.)
template <typename DT, int HD>
__global__ void __launch_bounds__(BLOCK) k_paged_attention_merge(PagedAttnArgs a) {
  typedef typename DT::T T;
  constexpr int LANES = HD / 4, STEP = 64 / LANES;
  const int lane = threadIdx.x & 63, sub = lane / LANES, d = lane % LANES * 4;
  const int at = blockIdx.x * (BLOCK / WAVE) + (threadIdx.x >> 6);
  const int row = at / a.nq, head = at - row * a.nq;
  const float* ml = a.ml_part + (size_t)at * a.P * 2;
  const float* op = a.o_part + (size_t)at * a.P * HD + d;
  if (row >= a.n_rows) return;
  // Everything is asked for at once: where the rows end, the row's sequence (those without rows have the same start: the last of those that begin at or before it), and the first
  // parts before it is known which of them there are.
  const int rows = a.row_start[a.n_seqs];
  float pm = PA_NONE, pl = 0.f;                            // (P <= 64: a lane for every part)
  if (lane < a.P) { pm = ml[lane * 2]; pl = ml[lane * 2 + 1]; }
  f32x4 v[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = *(const f32x4*)(op + (size_t)min(e * STEP + sub, a.P - 1) * HD);
  int s;
  const SeqRows r = find_rows(a, row, s, [&](int r0, int) { return r0; });
  asm volatile("" : "+v"(v[0]), "+v"(v[1]), "+v"(v[2]), "+v"(v[3]), "+v"(pm), "+v"(pl));         // (or the loads are made behind the returns)
  if (row >= rows || !r.ok || row < r.r0 || row >= r.r0 + r.n) return;
  const int first = r.start ? 0 : a.P_sh, n = a.P_sh + ceil_div(r.chunks, r.per);
  if (n - first == 1 && r.start == 0) return;
  if (lane < first || lane >= n) { pm = PA_NONE; pl = 0.f; }
  const float mx = wave_max(pm), f = __builtin_amdgcn_exp2f(pm - mx);
  const float l = wave_sum(pl * f);
  f32x4 o = {0, 0, 0, 0};
  for (int c = 0; c < n; c += 4 * STEP) {
    if (c)
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = *(const f32x4*)(op + (size_t)min(c + e * STEP + sub, n - 1) * HD);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int x = c + e * STEP + sub;
      const float fx = __shfl(f, min(x, n - 1), WAVE);
      if (x >= first && x < n) o += v[e] * fx;
    }
  }
#pragma unroll
  for (int x = LANES; x < 64; x *= 2)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], x, WAVE);
  o *= l == 0.f ? (__any(pm == -INFINITY) ? NAN : 0.f) : 1.f / l;
  if (sub) return;
  T* dst = (T*)a.out + (size_t)row * a.out_stride + head * HD + d;
  if constexpr (sizeof(T) == 2) *(uint2*)dst = make_uint2(f2_to_bf16x2(o[0], o[1]), f2_to_bf16x2(o[2], o[3]));
  else *(f32x4*)dst = o;
}

}  // namespace ssd
