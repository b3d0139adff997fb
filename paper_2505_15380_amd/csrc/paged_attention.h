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
