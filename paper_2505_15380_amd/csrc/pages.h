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

// ---------------------------------------------------------------------------------------------- block tables
constexpr int BT_MAX_SEQS = 4096;      // sequences of a call: three prefix sums of them stand in LDS
constexpr int BT_THREADS = 1024;

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

// The serial walk that the bookkeeping is defined by - sequences in ascending order give back what they no longer need, highest index first, then
// in ascending order take what they lack - as prefix sums: they say where on the stack each sequence's blocks go and come from.  One workgroup:
// what it puts on the stack it takes from there again behind a barrier.
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
#pragma unroll 1
  for (int r = tid; r < a.max_rows; r += BT_THREADS) {
    int seq = -1, pos = -1, slot = -1;
    if (r < R) {
      seq = owner_of(rowed, B, r);
      pos = a.len[seq] + r - (seq ? rowed[seq - 1] : 0);
      slot = (a.table[(size_t)seq * a.cap + (pos >> a.bt_shift)] << a.bt_shift) + (pos & ((1 << a.bt_shift) - 1));
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

// One thread per pair of a row's head.
template <typename DT>
__global__ void __launch_bounds__(BLOCK) k_rope_append(RopeAppendArgs a) {
  typedef typename DT::T T;
  const int hd = a.p.hd, half = hd >> 1, heads = a.nq + 2 * a.p.nkv;
  const size_t i = (size_t)blockIdx.x * BLOCK + threadIdx.x;
  const int row = (int)(i / ((size_t)heads * half));
  if (row >= a.n_rows) return;
  const int rest = (int)(i - (size_t)row * heads * half), h = rest / half, d = rest - h * half;
  const int pos = a.row_pos[row], slot = a.row_slot[row];
  const bool is_q = h < a.nq, is_k = !is_q && h < a.nq + a.p.nkv;
  int bad = 0;
  if (a.rope && pos >= a.positions) bad |= ST_BAD;
  if (!is_q && slot >= 0 && (slot >> a.p.bt_shift) >= a.p.n_blocks) bad |= ST_PAGE;
  if (bad) {
    if (d == 0 && a.status) atomicOr(a.status, bad);
    return;
  }
  if (pos < 0 || (!is_q && slot < 0)) return;
  const T* src = is_q ? (const T*)a.q + row * a.q_stride + h * hd
                      : is_k ? (const T*)a.k + row * a.k_stride + (h - a.nq) * hd : (const T*)a.v + row * a.v_stride + (h - a.nq - a.p.nkv) * hd;
  const T x = src[d], y = src[d + half];
  const size_t blk = (size_t)(slot >> a.p.bt_shift);
  const int tok = slot & (a.p.bt - 1);
  if (!is_q && !is_k) {
    T* dst = (T*)a.p.values + (blk * a.p.nkv + (h - a.nq - a.p.nkv)) * hd * a.p.bt + tok;
    dst[(size_t)d * a.p.bt] = x;
    dst[(size_t)(d + half) * a.p.bt] = y;
    return;
  }
  float c = 1.f, s = 0.f;
  if (a.rope) {
    const float* cs = a.rope + ((size_t)pos * half + d) * 2;
    c = cs[0]; s = cs[1];
  }
  const float fx = DT::ld(&x), fy = DT::ld(&y);
  T* dst = is_q ? (T*)a.q_out + row * a.q_out_stride + h * hd : (T*)a.p.keys + ((blk * a.p.nkv + (h - a.nq)) * a.p.bt + tok) * hd;
  DT::st(dst + d, fx * c - fy * s);
  DT::st(dst + d + half, fy * c + fx * s);
}

}  // namespace ssd
