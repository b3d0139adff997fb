// What a step does to a layer's pages before attention: the blocks that its rows need (once a step), and the rotated keys and the
// values put into them.
#pragma once
#include "common.h"

namespace ssd {

// A layer's pages, as ssd_pages names them.
struct Pages {
  void* keys;            // [n_blocks][nkv][bt][hd]
  void* values;          // [n_blocks][nkv][hd][bt]
  int n_blocks, nkv, bt, hd;
  int bt_shift;          // bt = 1 << bt_shift
};

// Bits of a status word (the public header's SSD_STATUS_*).
constexpr int ST_POOL = 1, ST_TABLE = 2, ST_ROWS = 4, ST_BAD = 8, ST_PAGE = 16;

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

// ---------------------------------------------------------------------------------------------- block tables
constexpr int BT_MAX_SEQS = 4096;      // sequences of a call: three prefix sums of them stand in LDS
constexpr int BT_THREADS = 1024;
constexpr int BT_ROWS_HERE = 4096;     // rows that k_block_tables looks up itself; more go to a launch of their own

struct BlockTableArgs {
  const int32_t *len, *rows, *owned, *shared, *n_free;
  int32_t *table, *stack, *owned_out, *n_free_out, *row_start, *row_seq, *row_pos, *row_slot, *status;
  int B, bt_shift, n_blocks, cap, max_rows;
};

struct SeqNeed {
  int have, need, rows, head;          // blocks of its own held and needed, new rows, blocks in front that are not its own
  int bad;                             // ST_* bits
};
__device__ __forceinline__ SeqNeed seq_need(const BlockTableArgs& a, int s) {
  SeqNeed n;
  const int len = a.len[s];
  n.rows = a.rows[s];
  n.have = a.owned[s];
  n.head = a.shared ? a.shared[s] : 0;
  const int bt = 1 << a.bt_shift;
  const long long end = (long long)len + n.rows;
  const long long blocks = (end + bt - 1) >> a.bt_shift;
  n.bad = 0;
  if (len < 0 || n.rows < 0 || n.have < 0 || n.head < 0 || (long long)n.head + n.have > a.cap) n.bad = ST_BAD;
  else if (n.rows > 0 && ((long long)n.head << a.bt_shift) > len) n.bad = ST_BAD;
  else if (blocks > a.cap) n.bad = ST_TABLE;
  n.need = n.bad ? 0 : max(0, (int)blocks - n.head);
  return n;
}

// Inclusive prefix sums of three numbers per thread of BT_THREADS, added to what `sum` holds of earlier rounds; sum grows by the totals.  w: 3 x 16
// entries of LDS.
__device__ __forceinline__ void block_incl_scan3(unsigned long long (&v)[3], unsigned long long (&sum)[3], unsigned long long* w) {
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    v[k] = wave_inclusive_scan(v[k]);
    if (lane == 63) w[k * 16 + wave] = v[k];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 3; ++k) {                            // (the waves' totals: a prefix sum over 16 lanes)
    const unsigned long long t = wave_inclusive_scan(lane < 16 ? w[k * 16 + lane] : 0ull);
    v[k] += sum[k] + (wave ? lane_u64(t, wave - 1) : 0ull);
    sum[k] += lane_u64(t, 15);
  }
  __syncthreads();
}

// i-th entry of a list whose sequences' entries end at ends[0..B): the sequence it belongs to.
__device__ __forceinline__ int owner_of(const int* ends, int B, int i) {
  int lo = 0, hi = B - 1;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (ends[mid] > i) hi = mid; else lo = mid + 1;
  }
  return lo;
}

// (an id that is no block's, shifted, can be a slot of another block: it gets one that no pool has)
__device__ __forceinline__ int slot_of(const BlockTableArgs& a, int seq, int pos) {
  const int blk = a.table[(size_t)seq * a.cap + (pos >> a.bt_shift)];
  return (unsigned)blk < (unsigned)a.n_blocks ? (blk << a.bt_shift) + (pos & ((1 << a.bt_shift) - 1)) : 0x7FFFFFFF;
}

// The serial walk that the bookkeeping is defined by - sequences in ascending order give back what they no longer need, highest index first, then
// in ascending order take what they lack - as prefix sums: they say where on the stack each sequence's blocks go and come from.  One workgroup:
// what it puts on the stack it takes from there again behind a barrier.
//   Bound by latency: eight dependent steps of memory, LDS and barriers are 4.5 us for 64 sequences of a row, whose 3 KB are nothing; 960
// sequences that move 8000 ids and look 76000 rows up: 14 us, and 4 for the rows' own launch, where the megabyte would take 0.2.  Which sequence an entry is of is searched
// for in LDS; steps of a fixed number, several searches side by side, came to 14.8.  The walk's parts on several workgroups, which could look the rows up as well, are estimated at three launches of 13 us in
// all against these 18; one workgroup was kept for the few sequences of most steps, and nothing else was built.
__global__ void __launch_bounds__(BT_THREADS) k_block_tables(BlockTableArgs a) {
  __shared__ int gave[BT_MAX_SEQS], took[BT_MAX_SEQS], rowed[BT_MAX_SEQS];
  __shared__ unsigned long long w[48];
  __shared__ int any_bad;
  const int tid = threadIdx.x, B = a.B, F = a.n_free[0];
  int bad = F < 0 || F > a.n_blocks ? ST_BAD : 0;
  unsigned long long sum[3] = {0, 0, 0};                   // blocks given back, blocks taken, rows
  if (tid == 0) any_bad = 0;
#pragma unroll 1
  for (int c = 0; c < B; c += BT_THREADS) {
    const int s = c + tid;
    SeqNeed n = {0, 0, 0, 0, 0};
    if (s < B) n = seq_need(a, s);
    bad |= n.bad;
    unsigned long long v[3] = {(unsigned)max(0, n.have - n.need), (unsigned)max(0, n.need - n.have), (unsigned)max(0, n.rows)};
    block_incl_scan3(v, sum, w);
    if (s < B) { gave[s] = (int)v[0]; took[s] = (int)v[1]; rowed[s] = (int)v[2]; }
  }
  if (sum[2] > (unsigned long long)a.max_rows) bad |= ST_ROWS;
  if (!(bad & ST_BAD)) {
    if (F + sum[0] > (unsigned long long)a.n_blocks) bad |= ST_BAD;
    else if (sum[1] > F + sum[0]) bad |= ST_POOL;
  }
  if (bad) atomicOr(&any_bad, bad);                        // (any_bad was cleared ahead of the scans' barriers)
  __syncthreads();
  bad = any_bad;
  const int G = (int)sum[0], T = (int)sum[1], R = (int)sum[2];
  if (tid == 0) {
    a.status[0] = bad;
    a.n_free_out[0] = bad ? F : F + G - T;
    a.row_start[0] = 0;
  }
  if (bad) {
    for (int s = tid; s < B; s += BT_THREADS) { a.owned_out[s] = a.owned[s]; a.row_start[s + 1] = 0; }
    if (a.max_rows <= BT_ROWS_HERE)
      for (int r = tid; r < a.max_rows; r += BT_THREADS) a.row_seq[r] = a.row_pos[r] = a.row_slot[r] = -1;
    return;
  }
  __syncthreads();
#pragma unroll 1
  for (int i = tid; i < G; i += BT_THREADS) {              // the i-th block given back
    const int s = owner_of(gave, B, i);
    const int first = s ? gave[s - 1] : 0;
    a.stack[F + i] = a.table[(size_t)s * a.cap + (a.shared ? a.shared[s] : 0) + a.owned[s] - 1 - (i - first)];
  }
  __syncthreads();
#pragma unroll 1
  for (int i = tid; i < T; i += BT_THREADS) {              // the i-th block taken
    const int s = owner_of(took, B, i);
    const int first = s ? took[s - 1] : 0;
    a.table[(size_t)s * a.cap + (a.shared ? a.shared[s] : 0) + a.owned[s] + (i - first)] = a.stack[F + G - 1 - i];
  }
  __syncthreads();
  if (a.max_rows <= BT_ROWS_HERE)
#pragma unroll 1
    for (int r = tid; r < a.max_rows; r += BT_THREADS) {
      int seq = -1, pos = -1, slot = -1;
      if (r < R) {
        seq = owner_of(rowed, B, r);
        pos = a.len[seq] + r - (seq ? rowed[seq - 1] : 0);
        slot = slot_of(a, seq, pos);
      }
      a.row_seq[r] = seq; a.row_pos[r] = pos; a.row_slot[r] = slot;
    }
  __syncthreads();                                         // (owned_out may be owned)
  for (int s = tid; s < B; s += BT_THREADS) {
    const int g = gave[s] - (s ? gave[s - 1] : 0), t = took[s] - (s ? took[s - 1] : 0);
    a.owned_out[s] = a.owned[s] - g + t;
    a.row_start[s + 1] = rowed[s];
  }
}

// Sequence, position and slot of every row of a step that has many, behind k_block_tables: one thread per row, whose sequence is searched for first among the
// workgroup's, which stand side by side.  (One workgroup alone takes 81 us for 960 sequences of 76000 rows, with this launch 18; up to
// BT_ROWS_HERE rows, four a thread, the launch costs more than they do.)
__global__ void __launch_bounds__(BLOCK) k_block_table_rows(BlockTableArgs a) {
  const int r = blockIdx.x * BLOCK + threadIdx.x;
  const int all = a.row_start[a.B];                        // (0 if the step could not be)
  int seq = -1, pos = -1, slot = -1;
  const int w = blockIdx.x * BLOCK + (threadIdx.x & ~63);  // the wave's first row
  if (w < all) {                                           // (the whole wave)
    int lo = wave_search(a.B, w, [&](int s) { return a.row_start[s]; });
    int hi = wave_search(a.B, min(w + 63, all - 1), [&](int s) { return a.row_start[s]; });
    if (r < all) {
      while (lo < hi) {                                    // the last of those that begin at or before the row
        const int mid = (lo + hi + 1) >> 1;
        if (a.row_start[mid] <= r) lo = mid; else hi = mid - 1;
      }
      seq = lo;
      pos = a.len[seq] + r - a.row_start[seq];
      slot = slot_of(a, seq, pos);
    }
  }
  if (r < a.max_rows) { a.row_seq[r] = seq; a.row_pos[r] = pos; a.row_slot[r] = slot; }
}

// ---------------------------------------------------------------------------------------------- rotary embedding and append
struct RopeAppendArgs {
  const void *q, *k, *v;
  void* q_out;
  size_t q_stride, k_stride, v_stride, q_out_stride;       // elements from row to row
  const float* rope;                                       // [positions][hd / 2][2] cos, sin; null: nothing is turned
  const int32_t *row_pos, *row_slot;
  int32_t* status;
  Pages p;
  int n_rows, nq, positions;
};

constexpr int RA_HEADS = 4;            // heads of a thread
constexpr int RA_WINDOW = 32;          // rows of a workgroup that puts values

// 16 bytes of a row as floats, and back, rounded once.
template <typename DT>
struct Unit;
template <>
struct Unit<BF16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void get(const u32x4 v, float (&x)[8]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) { x[2 * e] = __uint_as_float(v[e] << 16); x[2 * e + 1] = __uint_as_float(v[e] & 0xFFFF0000u); }
  }
  static __device__ __forceinline__ void put(bf16_t* p, const float (&x)[8]) {
    *(u32x4*)p = u32x4{f2_to_bf16x2(x[0], x[1]), f2_to_bf16x2(x[2], x[3]), f2_to_bf16x2(x[4], x[5]), f2_to_bf16x2(x[6], x[7])};
  }
};
template <>
struct Unit<F32> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void get(const u32x4 v, float (&x)[4]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = __uint_as_float(v[e]);
  }
  static __device__ __forceinline__ void put(float* p, const float (&x)[4]) { *(f32x4*)p = *(const f32x4*)x; }
};

// The first `v_wgs` workgroups put values, the others turn queries and keys.
//   Turning: a thread has 16 bytes of a row's first half of dims, the 16 of the second half that they are paired with, and their angles, for four
// heads in turn.
//   Values lie [dim][token], and a row brings one token of every dim: a workgroup takes 32 rows of a head through LDS and writes, for each dim, the
// eight tokens of an aligned piece at once (16 bytes; fp32 32) where eight rows behind each other fill one, the piece of a row being the business
// of the workgroup that has its first row; what fills no piece goes element by element.
//   Bound by being a launch for small calls (112 rows of the 0.5B heads 5.0 us, 517 of four fp32 heads of 32 4.4).  4099 rows of the 1.5B heads bring and take
// 36 MB in 11.1 us, 3.2 TB/s, where a copy of that size would take 7.5: in the workgroups that put values, of the eight lanes whose rows fill a piece one writes it.  (Values a row at a time, 2 bytes to a
// line: 17.9; windows of 64 rows, heads one by one: 13.4.)
template <typename DT>
__global__ void __launch_bounds__(BLOCK) k_rope_append(RopeAppendArgs a, int v_wgs) {
  typedef typename DT::T T;
  constexpr int N = Unit<DT>::N, PIECE = 8, ROWS = RA_WINDOW + PIECE - 1;
  __shared__ __align__(16) T vals[ROWS][128 + 16 / sizeof(T)];
  __shared__ int slots[PIECE - 1 + ROWS];                  // of rows r0 - 7 ..
  __shared__ int kind[ROWS];                               // 1: first row of a full piece, 2: by itself
  const int hd = a.p.hd, tid = threadIdx.x;
  if ((int)blockIdx.x < v_wgs) {
    const int head = blockIdx.x % a.p.nkv, r0 = blockIdx.x / a.p.nkv * RA_WINDOW;
    const int per = hd / N;
    for (int i = tid; i < ROWS * per; i += BLOCK) {
      const int r = i / per, u = i - r * per;
      if (r0 + r < a.n_rows) *(u32x4*)&vals[r][u * N] = *(const u32x4*)((const T*)a.v + (size_t)(r0 + r) * a.v_stride + head * hd + u * N);
    }
    if (tid < PIECE - 1 + ROWS) {
      const int r = r0 - (PIECE - 1) + tid;
      int s = -1;
      if (r >= 0 && r < a.n_rows) {
        s = a.row_slot[r];
        const int pos = a.row_pos[r];
        const bool out = s >= 0 && (s >> a.p.bt_shift) >= a.p.n_blocks;
        if (out && a.status) atomicOr(a.status, ST_PAGE);
        if (out || pos < 0 || (a.rope && pos >= a.positions)) s = -1;
      }
      slots[tid] = s;
    }
    __syncthreads();
    if (tid < ROWS) {
      const int s = slots[PIECE - 1 + tid], lead = tid - (s & (PIECE - 1));             // the row that would begin the row's piece
      bool full = s >= 0;
      for (int e = 0; e < PIECE; ++e) {
        const int x = lead + e + PIECE - 1;
        full = full && x < PIECE - 1 + ROWS && slots[x] == (s & ~(PIECE - 1)) + e;
      }
      kind[tid] = s < 0 ? 0 : full ? (lead == tid && tid < RA_WINDOW ? 1 : 0) : tid < RA_WINDOW ? 2 : 0;
    }
    __syncthreads();
    // (lanes side by side have the pieces of one dim, which lie side by side in a block)
    for (int i = tid; i < RA_WINDOW * hd; i += BLOCK) {
      const int r = i & (RA_WINDOW - 1), d = i / RA_WINDOW;
      if (kind[r] == 0) continue;
      const int s = slots[PIECE - 1 + r];
      T* dst = (T*)a.p.values + (((size_t)(s >> a.p.bt_shift) * a.p.nkv + head) * hd + d) * a.p.bt + (s & (a.p.bt - 1));
      if (kind[r] == 2) {
        *dst = vals[r][d];
        continue;
      }
      __align__(16) T x[PIECE];
#pragma unroll
      for (int e = 0; e < PIECE; ++e) x[e] = vals[r + e][d];
#pragma unroll
      for (int e = 0; e < PIECE / N; ++e) ((u32x4*)dst)[e] = ((u32x4*)x)[e];
    }
    return;
  }
  const int half = hd >> 1, units = half / N, heads = a.nq + a.p.nkv, groups = (heads + RA_HEADS - 1) / RA_HEADS;
  const long long i = (long long)(blockIdx.x - v_wgs) * BLOCK + tid;
  const int row = (int)(i / (units * groups));
  if (row >= a.n_rows) return;
  const int rest = (int)(i - (long long)row * (units * groups)), group = rest / units, d = (rest - group * units) * N;
  const int pos = a.row_pos[row];
  int slot = a.row_slot[row];
  if (pos < 0) return;
  if (a.rope && pos >= a.positions) {
    if (rest == 0 && a.status) atomicOr(a.status, ST_BAD);
    return;
  }
  if (slot >= 0 && (slot >> a.p.bt_shift) >= a.p.n_blocks) slot = -1;      // (reported with the values)
  float c[N], s[N];
#pragma unroll
  for (int e = 0; e < N; ++e) { c[e] = 1.f; s[e] = 0.f; }
  if (a.rope) {
    const f32x4* cs = (const f32x4*)(a.rope + ((size_t)pos * half + d) * 2);
#pragma unroll
    for (int e = 0; e < N / 2; ++e) {
      const f32x4 v = cs[e];
      c[2 * e] = v[0]; s[2 * e] = v[1]; c[2 * e + 1] = v[2]; s[2 * e + 1] = v[3];
    }
  }
  u32x4 lo[RA_HEADS], hi[RA_HEADS];                        // (all of them requested at once)
#pragma unroll
  for (int k = 0; k < RA_HEADS; ++k) {
    const int h = min(group * RA_HEADS + k, heads - 1);
    const T* src = (h < a.nq ? (const T*)a.q + row * a.q_stride + h * hd : (const T*)a.k + row * a.k_stride + (h - a.nq) * hd) + d;
    lo[k] = *(const u32x4*)src;
    hi[k] = *(const u32x4*)(src + half);
  }
#pragma unroll
  for (int k = 0; k < RA_HEADS; ++k) {
    const int h = group * RA_HEADS + k;
    const bool is_q = h < a.nq;
    if (h >= heads || (!is_q && slot < 0)) break;
    T* dst = (is_q ? (T*)a.q_out + row * a.q_out_stride + h * hd
                   : (T*)a.p.keys + (((size_t)(slot >> a.p.bt_shift) * a.p.nkv + (h - a.nq)) * a.p.bt + (slot & (a.p.bt - 1))) * hd) + d;
    if (!a.rope) {                                         // (as it is: times 1, less 0 times the other, is not the same for infinities)
      *(u32x4*)dst = lo[k];
      *(u32x4*)(dst + half) = hi[k];
      continue;
    }
    float x[N], y[N], u[N], w[N];
    Unit<DT>::get(lo[k], x);
    Unit<DT>::get(hi[k], y);
#pragma unroll
    for (int e = 0; e < N; ++e) {
      u[e] = x[e] * c[e] - y[e] * s[e];
      w[e] = y[e] * c[e] + x[e] * s[e];
    }
    Unit<DT>::put(dst, u);
    Unit<DT>::put(dst + half, w);
  }
}

}  // namespace ssd
