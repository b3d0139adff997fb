// Attention of a ragged batch against its pages, the prefix that the sequences share read once for all of them.
//
// o = sum_j e^(s_j) v_j / sum_j e^(s_j) with s_j = scale * q . k_j splits over any division of the keys: a part gives
// (m, l, o) = (max s, sum e^(s - m), sum e^(s - m) v), and parts merge as M = max m, l = sum l e^(m - M), o = sum o e^(m - M).  So the shared prefix
// is one attention of ALL rows of the batch against the same keys, and each sequence's own keys another; what a row gets of both is merged.
//
// The query rows of a source of keys - rows x the G query heads of a kv head, packed [row][head] - form tiles of 16.  Scores and outputs are
// computed transposed (S^T = K Q^T, O^T = V^T P^T), so a lane holds scores and outputs of one query row, the weights go from the first
// product's accumulators into the second one without leaving the registers, and both operands come from the pages as 16 bytes per lane:
//   bf16  16x16x32 products.  Of a pair of 16-key tiles, row m of tile t is key 8 (m / 4) + 4 t + m % 4: lane group g then ends with the scores of keys
//         8 g .. 8 g + 7, whose values it holds as the second product's operand.
//   fp32  16x16x4 products: lane group g ends with keys 4 g .. 4 g + 3 of a tile.
// The weights are rounded to bf16 for the second product (2^-9 of each, at random: the sum is off by about as much as the output's own
// rounding); their sum is taken of the unrounded ones, in fp32.
#pragma once
#include "common.h"
#include "pages.h"

namespace ssd {

constexpr int PA_WAVES = 4, PA_THREADS = PA_WAVES * WAVE;
constexpr int PA_CHUNK = 64;           // keys that a wave takes at a time

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
  int P, P_sh;           // parts of a row at most, and those of the shared prefix
  int sh_chunks;         // chunks of a part of the shared prefix
  int own_chunks;        // chunks of a part of a sequence's own keys, at least
  int sh_slots, own_slots;             // tiles of query rows of the shared prefix, of the sequences
};

// Largest s in [0, n) with base(s) <= x, for base ascending from base(0) <= x; all lanes of the wave call it.
template <typename F>
__device__ __forceinline__ int wave_search(int n, int x, F base) {
  const int lane = threadIdx.x & 63;
  int lo = 0, step = 1;
  while (step * 64 < n) step *= 64;
  for (;; step /= 64) {
    const int s = lo + lane * step;
    const unsigned long long m = __ballot(s < n && base(s) <= x);
    lo += (63 - __builtin_clzll(m | 1ull)) * step;
    if (step == 1) return lo;
  }
}

struct SeqRows {
  int r0, n;             // first row of the launch, number of rows
  int len, start;        // cached positions; first position that is not read from the shared prefix
  int chunks, per;       // chunks of its own keys, of one part of them
  bool ok;
};
__device__ __forceinline__ SeqRows seq_rows(const PagedAttnArgs& a, int s) {
  SeqRows r;
  r.r0 = min(max(a.row_start[s], 0), a.n_rows);
  r.n = min(max(a.row_start[s + 1], 0), a.n_rows) - r.r0;
  r.len = a.len[s];
  const int limit = a.cap << a.p.bt_shift;
  r.ok = r.n > 0 && r.len >= 0 && r.len <= limit;
  const int sh = a.shared_blocks << a.p.bt_shift;
  const bool joins = sh > 0 && r.len >= sh && (!a.shared || a.shared[s] >= a.shared_blocks);
  r.start = joins ? sh : 0;
  r.chunks = ceil_div(r.len + r.n - r.start, PA_CHUNK);
  r.per = max(a.own_chunks, ceil_div(r.chunks, a.P - a.P_sh));
  return r;
}

template <typename DT, int HD>
struct AttnFrags;

template <int HD>
struct AttnFrags<BF16, HD> {
  static constexpr int KS = HD / 32, DTILES = HD / 16;
  u32x4 q[KS];
  __device__ __forceinline__ void load_q(const void* row, int g) {
    const u32x4* p = (const u32x4*)row + g;
#pragma unroll
    for (int s = 0; s < KS; ++s) q[s] = p[s * 4];
  }
};
template <int HD>
struct AttnFrags<F32, HD> {
  static constexpr int KS = HD / 16, DTILES = HD / 16;
  f32x4 q[KS];
  __device__ __forceinline__ void load_q(const void* row, int g) {
    const f32x4* p = (const f32x4*)row + g;
#pragma unroll
    for (int s = 0; s < KS; ++s) q[s] = p[s * 4];
  }
};

// One workgroup: a tile of 16 query rows against a part of the keys of one source.  Its waves take the part's chunks in turn and meet in LDS.
template <typename DT, int HD>
__global__ void __launch_bounds__(PA_THREADS) k_paged_attention(PagedAttnArgs a) {
  typedef typename DT::T T;
  constexpr bool B16 = sizeof(T) == 2;
  constexpr int DTILES = HD / 16;
  __shared__ float po[PA_WAVES][16][HD + 4];
  __shared__ float pm[PA_WAVES][16], pl[PA_WAVES][16];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), li = lane & 15, g = lane >> 4;
  const int nkv = a.p.nkv, G = a.nq / nkv;
  int id = blockIdx.x;
  const int kvh = id % nkv;
  id /= nkv;
  const bool is_shared = id < a.sh_slots * a.P_sh;
  int part, row0, n_packed, seq_r0, len = 0, k_begin, k_end, part_slot, n_parts = 0;
  const int32_t* table;
  if (is_shared) {
    part = id % a.P_sh;
    row0 = id / a.P_sh * 16;
    seq_r0 = 0;
    n_packed = min(max(a.row_start[a.n_seqs], 0), a.n_rows) * G;
    if (row0 >= n_packed) return;
    table = a.shared_table;
    const int keys = a.shared_blocks << a.p.bt_shift;
    k_begin = part * a.sh_chunks * PA_CHUNK;
    k_end = min(keys, k_begin + a.sh_chunks * PA_CHUNK);
    part_slot = part;
  } else {
    id -= a.sh_slots * a.P_sh;
    const int po_ = a.P - a.P_sh, slot = id / po_;
    part = id - slot * po_;
    const int s = wave_search(a.n_seqs, slot, [&](int x) { return min(max(a.row_start[x], 0), a.n_rows) * G / 16 + x; });
    const SeqRows r = seq_rows(a, s);
    row0 = (slot - (r.r0 * G / 16 + s)) * 16;
    n_packed = r.n * G;
    if (row0 >= n_packed) return;
    if (!r.ok) {
      if (tid == 0 && a.status) atomicOr(a.status, ST_BAD);
      return;
    }
    n_parts = ceil_div(r.chunks, r.per);
    if (part >= n_parts) return;
    seq_r0 = r.r0;
    len = r.len;
    table = a.table + (size_t)s * a.cap;
    k_begin = r.start + part * r.per * PA_CHUNK;
    const int last = r.len + min(r.n - 1, (row0 + 15) / G);        // the last position that a row of the tile sees
    k_end = min(last + 1, k_begin + r.per * PA_CHUNK);
    part_slot = a.P_sh + part;
    n_parts += r.start ? a.P_sh : 0;
  }
  // this lane's query row
  const int pr = min(row0 + li, n_packed - 1);
  const int row = seq_r0 + pr / G, head = kvh * G + pr % G;
  const int pos = is_shared ? 0x7FFFFFFF : len + pr / G;
  AttnFrags<DT, HD> f;
  f.load_q((const T*)a.q + row * a.q_stride + head * HD, g);
  f32x4 o[DTILES];
#pragma unroll
  for (int d = 0; d < DTILES; ++d) o[d] = f32x4{0, 0, 0, 0};
  float m = -INFINITY, l = 0.f;
  int bad = 0;
  auto block_of = [&](int key) {                           // -1: nothing there
    if (key >= k_end) return -1;
    const int b = key >> a.p.bt_shift;
    const int blk = b < (is_shared ? a.shared_blocks : a.cap) ? table[b] : -1;
    if (blk < 0 || blk >= a.p.n_blocks) { bad = 1; return -1; }
    return blk;
  };
  const int tmask = a.p.bt - 1;
  for (int c0 = k_begin + wave * PA_CHUNK; c0 < k_end; c0 += PA_WAVES * PA_CHUNK) {
    float w[4][4];                                         // bf16: [pair * 2 + tile][i] of key 32 pair + 8 g + 4 tile + i; fp32: [tile][i] of key 16 tile + 4 g + i
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int key = c0 + (B16 ? 32 * (t >> 1) + 8 * (li >> 2) + 4 * (t & 1) + (li & 3) : 16 * t + li);
      const int blk = block_of(key);
      const T* kp = (const T*)a.p.keys + (((size_t)max(blk, 0) * nkv + kvh) * a.p.bt + (key & tmask)) * HD;
      f32x4 acc = {0, 0, 0, 0};
      if constexpr (B16) {
#pragma unroll
        for (int s = 0; s < HD / 32; ++s)
          acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, ((const u32x4*)kp)[s * 4 + g]), __builtin_bit_cast(bf16x8, f.q[s]), acc, 0, 0, 0);
      } else {
#pragma unroll
        for (int s = 0; s < HD / 16; ++s) {
          const f32x4 kk = ((const f32x4*)kp)[s * 4 + g];
#pragma unroll
          for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(kk[e], f.q[s][e], acc, 0, 0, 0);
        }
      }
      // which of this lane's four keys are there: one block has them all
      const int k4 = c0 + (B16 ? 32 * (t >> 1) + 8 * g + 4 * (t & 1) : 16 * t + 4 * g);
      const bool page = block_of(k4) >= 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) w[t][i] = page && k4 + i <= pos && k4 + i < k_end ? acc[i] * a.scale2 : -INFINITY;
    }
    float mx = m;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) mx = fmaxf(mx, w[t][i]);
    mx = max_over_groups(mx);
    const float base = mx == -INFINITY ? 0.f : mx;
    const float keep = __builtin_amdgcn_exp2f(m - base);
    m = mx;
    l *= keep;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        w[t][i] = __builtin_amdgcn_exp2f(w[t][i] - base);
        l += w[t][i];
      }
#pragma unroll
    for (int d = 0; d < DTILES; ++d) o[d] *= keep;
    if constexpr (B16) {
#pragma unroll
      for (int pr2 = 0; pr2 < 2; ++pr2) {
        const int k8 = c0 + 32 * pr2 + 8 * g;
        const int blk = block_of(k8);
        u32x4 pw = {f2_to_bf16x2(w[2 * pr2][0], w[2 * pr2][1]), f2_to_bf16x2(w[2 * pr2][2], w[2 * pr2][3]),
                    f2_to_bf16x2(w[2 * pr2 + 1][0], w[2 * pr2 + 1][1]), f2_to_bf16x2(w[2 * pr2 + 1][2], w[2 * pr2 + 1][3])};
        const T* vp = (const T*)a.p.values + ((size_t)max(blk, 0) * nkv + kvh) * HD * a.p.bt + (k8 & tmask);
#pragma unroll
        for (int d = 0; d < DTILES; ++d) {
          u32x4 v = *(const u32x4*)(vp + (size_t)(d * 16 + li) * a.p.bt);
          const int n = blk < 0 ? 0 : k_end - k8;          // tokens of the eight that are there: what lies behind may hold anything
          if (n < 8)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] &= (2 * e < n ? 0xFFFFu : 0u) | (2 * e + 1 < n ? 0xFFFF0000u : 0u);
          o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, pw), o[d], 0, 0, 0);
        }
      }
    } else {
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int k4 = c0 + 16 * t + 4 * g;
        const int blk = block_of(k4);
        const T* vp = (const T*)a.p.values + ((size_t)max(blk, 0) * nkv + kvh) * HD * a.p.bt + (k4 & tmask);
#pragma unroll
        for (int d = 0; d < DTILES; ++d) {
          const f32x4 v = *(const f32x4*)(vp + (size_t)(d * 16 + li) * a.p.bt);
#pragma unroll
          for (int e = 0; e < 4; ++e)
            o[d] = __builtin_amdgcn_mfma_f32_16x16x4f32(blk >= 0 && k4 + e < k_end ? v[e] : 0.f, w[t][e], o[d], 0, 0, 0);
        }
      }
    }
  }
  l = sum_over_groups(l);
  if (__any(bad) && lane == 0 && a.status) atomicOr(a.status, ST_PAGE);
#pragma unroll
  for (int d = 0; d < DTILES; ++d) *(f32x4*)&po[wave][li][d * 16 + g * 4] = o[d];
  if (g == 0) { pm[wave][li] = m; pl[wave][li] = l; }
  __syncthreads();
  for (int i = tid; i < 16 * (HD / 4); i += PA_THREADS) {
    const int r = i / (HD / 4), d = (i - r * (HD / 4)) * 4;
    if (row0 + r >= n_packed) break;
    float mx = pm[0][r];
#pragma unroll
    for (int x = 1; x < PA_WAVES; ++x) mx = fmaxf(mx, pm[x][r]);
    const float base = mx == -INFINITY ? 0.f : mx;
    float ls = 0.f;
    f32x4 acc = {0, 0, 0, 0};
#pragma unroll
    for (int x = 0; x < PA_WAVES; ++x) {
      const float f2 = __builtin_amdgcn_exp2f(pm[x][r] - base);
      ls = fmaf(pl[x][r], f2, ls);
      acc += *(const f32x4*)&po[x][r][d] * f2;
    }
    const size_t at = (size_t)(seq_r0 + (row0 + r) / G) * a.nq + kvh * G + (row0 + r) % G;
    if (n_parts == 1) {
      T* dst = (T*)a.out + (size_t)(seq_r0 + (row0 + r) / G) * a.out_stride + (kvh * G + (row0 + r) % G) * HD + d;
      const float inv = ls == 0.f ? 0.f : 1.f / ls;
#pragma unroll
      for (int e = 0; e < 4; ++e) DT::st(dst + e, acc[e] * inv);
    } else {
      *(f32x4*)(a.o_part + (at * a.P + part_slot) * HD + d) = acc;
      if (d == 0) { a.ml_part[(at * a.P + part_slot) * 2] = mx; a.ml_part[(at * a.P + part_slot) * 2 + 1] = ls; }
    }
  }
}

// ---------------------------------------------------------------------------------------------- many rows against the same keys (bf16)
// The same for sources whose keys many rows share - the shared prefix, prompts.  A workgroup takes 128 QS packed query rows, 32 QS a wave, and a part of the
// keys, whose 64-key chunks all of its waves read from LDS, where direct loads put them a chunk ahead (wave w the 16 keys w of a chunk, which lie
// in one block).  32x32x16 products: a lane holds the scores of one row (lane % 32) for keys 16 (i / 8) + 8 h + i % 8 of a 32-key tile (i: register,
// h = lane / 32) if row m of the tile's operand is the key whose bits 2 and 3 are those of m swapped; these are the operand of the second product as they stand.
//   Weights are powers of two of scores less a reference, which is the largest score of the first chunk and moves only to one that exceeds it by PT_LAZY, so that most chunks need
// neither a maximum across lanes nor a scaling of what is summed; a weight is then up to 2^8, and as exact.
//   LDS of a chunk, 1 KB for each direct load: keys [group of 16][32 dims][8-dim piece][key], values [group of 16][32 dims][8-key half][dim].
constexpr float PT_LAZY = 8.0f, PT_NONE = -3.0e38f;      // the second: the reference of a row that has seen nothing
typedef __attribute__((ext_vector_type(16))) float f32x16;

template <int HD, int QS>
__global__ void __launch_bounds__(PA_THREADS, 2) k_paged_tiles(PagedAttnArgs a) {
  constexpr int J = HD / 32, T = 128 * QS;
  __shared__ u32x4 kv_lds[2][2][4][J][64];                 // [buffer][keys, values][group][32 dims][..]
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 31, h = lane >> 5;
  const int nkv = a.p.nkv, G = a.nq / nkv, tmask = a.p.bt - 1;
  int id = blockIdx.x;
  const int kvh = id % nkv;
  id /= nkv;
  const bool is_shared = id < a.sh_slots * a.P_sh;
  int part, row0, n_packed, seq_r0, len = 0, k_begin, k_end, part_slot, n_parts = 0, table_n;
  const int32_t* table;
  if (is_shared) {
    part = id % a.P_sh;
    row0 = id / a.P_sh * T;
    seq_r0 = 0;
    n_packed = min(max(a.row_start[a.n_seqs], 0), a.n_rows) * G;
    if (row0 >= n_packed) return;
    table = a.shared_table;
    table_n = a.shared_blocks;
    k_begin = part * a.sh_chunks * PA_CHUNK;
    k_end = min(a.shared_blocks << a.p.bt_shift, k_begin + a.sh_chunks * PA_CHUNK);
    part_slot = part;
  } else {
    id -= a.sh_slots * a.P_sh;
    const int po_ = a.P - a.P_sh, slot = id / po_;
    part = id - slot * po_;
    const int s = wave_search(a.n_seqs, slot, [&](int x) { return min(max(a.row_start[x], 0), a.n_rows) * G / T + x; });
    const SeqRows r = seq_rows(a, s);
    row0 = (slot - (r.r0 * G / T + s)) * T;
    n_packed = r.n * G;
    if (row0 >= n_packed) return;
    if (!r.ok) {
      if (tid == 0 && a.status) atomicOr(a.status, ST_BAD);
      return;
    }
    n_parts = ceil_div(r.chunks, r.per);
    if (part >= n_parts) return;
    seq_r0 = r.r0;
    len = r.len;
    table = a.table + (size_t)s * a.cap;
    table_n = a.cap;
    k_begin = r.start + part * r.per * PA_CHUNK;
    k_end = min(r.len + min(r.n - 1, (row0 + T - 1) / G) + 1, k_begin + r.per * PA_CHUNK);
    part_slot = a.P_sh + part;
    n_parts += r.start ? a.P_sh : 0;
  }
  const int n_chunks = max(0, ceil_div(k_end - k_begin, PA_CHUNK));
  // this wave's rows and what they see
  const int w0 = row0 + wave * 32 * QS;
  const bool has_rows = w0 < n_packed;
  const int pos_lo = is_shared ? 0x7FFFFFFF : len + w0 / G, reach = is_shared ? 0x7FFFFFFF : len + (min(w0 + 32 * QS, n_packed) - 1) / G;
  int pos[QS];
  size_t at[QS];                                           // row * nq + head
  bf16x8 q[QS][2 * J];
#pragma unroll
  for (int x = 0; x < QS; ++x) {
    const int pr = min(w0 + 32 * x + c, n_packed - 1), row = seq_r0 + pr / G, head = kvh * G + pr % G;
    pos[x] = is_shared ? 0x7FFFFFFF : len + pr / G;
    at[x] = (size_t)row * a.nq + head;
    const u32x4* qp = (const u32x4*)((const bf16_t*)a.q + row * a.q_stride + head * HD) + h;
#pragma unroll
    for (int s = 0; s < 2 * J; ++s) q[x][s] = __builtin_bit_cast(bf16x8, qp[2 * s]);
  }
  // (a negative factor: its sign goes to the queries, so that the largest product is the largest score)
  const float scale2 = fabsf(a.scale2);
  if (a.scale2 < 0.f) {
#pragma unroll
    for (int x = 0; x < QS; ++x)
#pragma unroll
      for (int s = 0; s < 2 * J; ++s) q[x][s] = __builtin_bit_cast(bf16x8, __builtin_bit_cast(u32x4, q[x][s]) ^ 0x80008000u);
  }
  // block ids of 16 chunks at a time: lane i has that of keys 16 i .. of them; and the next 16 chunks', looked at when their turn comes
  int bad = 0;
  auto look_up = [&](int first) {
    const int key = k_begin + first * PA_CHUNK + lane * 16, b = key >> a.p.bt_shift;
    return key < k_end && b < table_n ? table[b] : -1;
  };
  auto checked = [&](int blk, int first) {
    const bool there = blk >= 0 && blk < a.p.n_blocks;
    bad |= !there && k_begin + first * PA_CHUNK + lane * 16 < k_end;
    return there ? blk : -1;
  };
  int ids = checked(look_up(0), 0), ids_next = look_up(16);
  const int k_lane = ((lane & 15) * HD + (lane >> 4) * 8) * 2, v_lane = (c * a.p.bt + h * 8) * 2;
  const size_t head_bytes = (size_t)a.p.bt * HD * 2;
  auto request = [&](int it) {                             // returns which of the chunk's groups are there
    if (it && it % 16 == 0) { ids = checked(ids_next, it); ids_next = look_up(it + 16); }
    const int blk = __builtin_amdgcn_readlane(ids, (it & 15) * 4 + wave);
    const int tok = (k_begin + it * PA_CHUNK + wave * 16) & tmask;
    const size_t at_ = ((size_t)max(blk, 0) * nkv + kvh) * head_bytes;
    const rsrc_t rk = load_rsrc((const char*)a.p.keys + at_ + tok * HD * 2), rv = load_rsrc((const char*)a.p.values + at_ + tok * 2);
#pragma unroll
    for (int j = 0; j < J; ++j) load_to_lds(rk, &kv_lds[it & 1][0][wave][j][0], k_lane, j * 64);
#pragma unroll
    for (int j = 0; j < J; ++j) load_to_lds(rv, &kv_lds[it & 1][1][wave][j][0], v_lane + j * 32 * a.p.bt * 2, 0);
    return (int)(__ballot(ids >= 0) >> ((it & 15) * 4)) & 15;
  };
  f32x16 o[QS][J];
  float m[QS], l[QS];
#pragma unroll
  for (int x = 0; x < QS; ++x) {
    m[x] = PT_NONE;
    l[x] = 0.f;
#pragma unroll
    for (int d = 0; d < J; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[x][d][i] = 0.f;
  }
  const int kk = (c & ~12) | (c & 4) << 1 | (c & 8) >> 1;  // the key that row c of a tile's operand is
  int there = n_chunks ? request(0) : 0;
  for (int it = 0; it < n_chunks; ++it) {
    const int kbase = k_begin + it * PA_CHUNK;
    // (the builtin: with a wait in assembly the compiler places waits of its own for the queries, and with them for the chunk that was just requested)
    __builtin_amdgcn_s_waitcnt(0x0070);                    // vmcnt(0) lgkmcnt(0)
    asm volatile("" ::: "memory");                         // (the chunk has arrived; and nothing is still to be read of the one whose buffer is next)
    // values of this wave's group that are not there may be anything: they become zeros
    const int n_tok = (there >> wave & 1) ? k_end - (kbase + wave * 16) : 0;
    if (n_tok < 16) {
#pragma unroll
      for (int j = 0; j < J; ++j) {
        u32x4 v = kv_lds[it & 1][1][wave][j][lane];
        const int n = n_tok - 8 * h;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] &= (2 * e < n ? 0xFFFFu : 0u) | (2 * e + 1 < n ? 0xFFFF0000u : 0u);
        kv_lds[it & 1][1][wave][j][lane] = v;
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    const int now = there;
    if (it + 1 < n_chunks) there = request(it + 1);
    if (!has_rows || kbase > reach) continue;
    const bool edge = now != 15 || kbase + PA_CHUNK > k_end || kbase + PA_CHUNK - 1 > pos_lo;
    f32x16 s[QS][2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
      for (int x = 0; x < QS; ++x)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[x][t][i] = 0.f;
#pragma unroll
      for (int k = 0; k < 2 * J; ++k) {
        const bf16x8 kf = __builtin_bit_cast(bf16x8, kv_lds[it & 1][0][2 * t + (kk >> 4)][k >> 1][((k & 1) * 2 + h) * 16 + (kk & 15)]);
#pragma unroll
        for (int x = 0; x < QS; ++x) s[x][t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, q[x][k], s[x][t], 0, 0, 0);
      }
    }
    if (edge) {
#pragma unroll
      for (int x = 0; x < QS; ++x) {
        const int last = min(pos[x], k_end - 1) - kbase - 8 * h;           // of this lane's keys, less 8 h
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int key = 32 * t + 16 * (i >> 3) + (i & 7);
            if (key > last || !(now >> (2 * t + (i >> 3)) & 1)) s[x][t][i] = -INFINITY;
          }
      }
    }
    bf16x8 p[QS][4];
#pragma unroll
    for (int x = 0; x < QS; ++x) {
      float mx = s[x][0][0];
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[x][t][i]);
      mx *= scale2;
      if (__any(mx > m[x] + PT_LAZY)) {
        const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
        mx = fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1]));
        if (mx > m[x] + PT_LAZY) {
          const float keep = __builtin_amdgcn_exp2f(m[x] - mx);
          m[x] = mx;
          l[x] *= keep;
#pragma unroll
          for (int d = 0; d < J; ++d) o[x][d] *= keep;
        }
      }
      float sum = 0.f;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          s[x][t][i] = __builtin_amdgcn_exp2f(fmaf(s[x][t][i], scale2, -m[x]));
          sum += s[x][t][i];
        }
      l[x] += sum;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        u32x4 w;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = f2_to_bf16x2(s[x][k >> 1][(k & 1) * 8 + 2 * e], s[x][k >> 1][(k & 1) * 8 + 2 * e + 1]);
        p[x][k] = __builtin_bit_cast(bf16x8, w);
      }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int d = 0; d < J; ++d) {
        const bf16x8 vf = __builtin_bit_cast(bf16x8, kv_lds[it & 1][1][k][d][lane]);
#pragma unroll
        for (int x = 0; x < QS; ++x) o[x][d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, p[x][k], o[x][d], 0, 0, 0);
      }
  }
  if (__any(bad) && lane == 0 && a.status) atomicOr(a.status, ST_PAGE);
#pragma unroll
  for (int x = 0; x < QS; ++x) {
    const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(l[x]), __float_as_uint(l[x]), false, false);
    const float ls = __uint_as_float(both[0]) + __uint_as_float(both[1]);
    if (w0 + 32 * x + c >= n_packed) continue;
    // dims 32 d + 8 e + 4 h .. + 3 in registers 4 e ..
    if (n_parts == 1) {
      const float inv = ls == 0.f ? 0.f : 1.f / ls;
      const size_t row = at[x] / a.nq, head = at[x] - row * a.nq;
      bf16_t* dst = (bf16_t*)a.out + row * a.out_stride + head * HD + 4 * h;
#pragma unroll
      for (int d = 0; d < J; ++d)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          *(uint2*)(dst + 32 * d + 8 * e) = make_uint2(f2_to_bf16x2(o[x][d][4 * e] * inv, o[x][d][4 * e + 1] * inv), f2_to_bf16x2(o[x][d][4 * e + 2] * inv, o[x][d][4 * e + 3] * inv));
    } else {
      float* dst = a.o_part + (at[x] * a.P + part_slot) * HD + 4 * h;
#pragma unroll
      for (int d = 0; d < J; ++d)
#pragma unroll
        for (int e = 0; e < 4; ++e) *(f32x4*)(dst + 32 * d + 8 * e) = f32x4{o[x][d][4 * e], o[x][d][4 * e + 1], o[x][d][4 * e + 2], o[x][d][4 * e + 3]};
      if (h == 0) { a.ml_part[(at[x] * a.P + part_slot) * 2] = m[x]; a.ml_part[(at[x] * a.P + part_slot) * 2 + 1] = ls; }
    }
  }
}

// One wave per row and head of those that have several parts: merged in ascending order.
template <typename DT, int HD>
__global__ void __launch_bounds__(BLOCK) k_paged_attention_merge(PagedAttnArgs a) {
  typedef typename DT::T T;
  const int lane = threadIdx.x & 63;
  const size_t at = (size_t)blockIdx.x * (BLOCK / WAVE) + (threadIdx.x >> 6);
  const int row = (int)(at / a.nq), head = (int)(at - (size_t)row * a.nq);
  if (row >= min(max(a.row_start[a.n_seqs], 0), a.n_rows)) return;
  // (sequences without rows have the same start: the last of those that begin at or before the row is the row's)
  const int s = wave_search(a.n_seqs, row, [&](int x) { return a.row_start[x]; });
  const SeqRows r = seq_rows(a, s);
  if (!r.ok || row < r.r0 || row >= r.r0 + r.n) return;
  const int first = r.start ? 0 : a.P_sh, n = a.P_sh + ceil_div(r.chunks, r.per);
  if (n - first == 1) return;
  const float* ml = a.ml_part + at * a.P * 2;
  const float* op = a.o_part + at * a.P * HD;
  float mx = -INFINITY;
  for (int c = first; c < n; ++c) mx = fmaxf(mx, ml[c * 2]);
  const float base = mx == -INFINITY ? 0.f : mx;
  float l = 0.f, o[(HD + 63) / 64];
#pragma unroll
  for (int i = 0; i < (HD + 63) / 64; ++i) o[i] = 0.f;
  for (int c = first; c < n; ++c) {
    const float w = __builtin_amdgcn_exp2f(ml[c * 2] - base);
    l = fmaf(ml[c * 2 + 1], w, l);
#pragma unroll
    for (int i = 0; i < (HD + 63) / 64; ++i)
      if (lane + 64 * i < HD) o[i] = fmaf(op[(size_t)c * HD + lane + 64 * i], w, o[i]);
  }
  T* out = (T*)a.out + (size_t)row * a.out_stride + head * HD;
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int i = 0; i < (HD + 63) / 64; ++i)
    if (lane + 64 * i < HD) DT::st(out + lane + 64 * i, o[i] * inv);
}

}  // namespace ssd
