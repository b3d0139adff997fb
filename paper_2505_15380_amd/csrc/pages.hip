// libssd: the paged cache's own steps as calls of their own - block tables from lengths, rotary embedding with the append, and attention over
// pages with a shared prefix.  Host side: checks the arguments and enqueues the kernels on the caller's stream.
#include "../../include/ssd.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "errors.h"
#include "pages.h"
#include "paged_attention.h"

using namespace ssd;

static_assert(ST_POOL == SSD_STATUS_POOL && ST_TABLE == SSD_STATUS_TABLE && ST_ROWS == SSD_STATUS_ROWS && ST_BAD == SSD_STATUS_BATCH && ST_PAGE == SSD_STATUS_PAGE, "");

static inline int cdiv(int a, int b) { return (a + b - 1) / b; }
static int log2_of(int v) {
  int s = 0;
  while ((1 << s) < v) ++s;
  return s;
}
static int check_block_tokens(int bt, int n_blocks) {
  if (bt < 16 || bt > 1024 || (bt & (bt - 1))) return fail(SSD_ENOSUP, "block_tokens = %d: powers of two from 16 to 1024", bt);
  if (n_blocks < 1 || (long long)n_blocks * bt > 0x7FFFFFFFll) return fail(SSD_EINVAL, "n_blocks = %d of %d tokens: slots are 32-bit", n_blocks, bt);
  return SSD_OK;
}
static int check_pages(const ssd_pages* p, Pages& v) {
  if (!p || !p->dev_keys || !p->dev_values) return fail(SSD_EINVAL, "null pages");
  if (p->dtype != SSD_DTYPE_FP32 && p->dtype != SSD_DTYPE_BF16) return fail(SSD_EINVAL, "bad dtype %d", p->dtype);
  if (p->head_dim != 32 && p->head_dim != 64 && p->head_dim != 128) return fail(SSD_ENOSUP, "head_dim %d not in {32,64,128}", p->head_dim);
  if (p->n_kv_heads < 1 || p->n_kv_heads > 1024) return fail(SSD_EINVAL, "n_kv_heads = %d", p->n_kv_heads);
  if (int rc = check_block_tokens(p->block_tokens, p->n_blocks)) return rc;
  if (((uintptr_t)p->dev_keys & 15) || ((uintptr_t)p->dev_values & 15)) return fail(SSD_EINVAL, "pages must be 16-byte aligned");
  v.keys = p->dev_keys; v.values = p->dev_values;
  v.n_blocks = p->n_blocks; v.nkv = p->n_kv_heads; v.bt = p->block_tokens; v.hd = p->head_dim;
  v.bt_shift = log2_of(v.bt);
  return SSD_OK;
}
// Rows of `heads` heads behind each other, read and written 16 bytes at a time.
static int check_rows(const char* what, const void* ptr, size_t stride, int heads, const Pages& p, int dtype) {
  const size_t per16 = dtype == SSD_DTYPE_BF16 ? 8 : 4;
  if (!ptr) return fail(SSD_EINVAL, "%s is null", what);
  if (stride < (size_t)heads * p.hd || stride % per16 || ((uintptr_t)ptr & 15)) return fail(SSD_EINVAL, "%s: rows of %d x %d elements, %zu apart, must not overlap and begin at multiples of 16 bytes", what, heads, p.hd, stride);
  return SSD_OK;
}

extern "C" int ssd_block_tables(int n_seqs, int block_tokens, int n_blocks, int table_cap, int max_rows, const int32_t* dev_len, const int32_t* dev_rows,
                                const int32_t* dev_shared, const int32_t* dev_owned, const int32_t* dev_n_free, int32_t* dev_table, int32_t* dev_free_stack,
                                int32_t* dev_owned_out, int32_t* dev_n_free_out, int32_t* dev_row_start, int32_t* dev_row_seq, int32_t* dev_row_pos,
                                int32_t* dev_row_slot, int32_t* dev_status, void* stream) {
  if (!dev_len || !dev_rows || !dev_owned || !dev_n_free || !dev_table || !dev_free_stack || !dev_owned_out || !dev_n_free_out || !dev_row_start || !dev_row_seq ||
      !dev_row_pos || !dev_row_slot || !dev_status)
    return fail(SSD_EINVAL, "null argument");
  if (n_seqs < 1 || max_rows < 1 || table_cap < 1) return fail(SSD_EINVAL, "bad n_seqs / max_rows / table_cap");
  if (n_seqs > BT_MAX_SEQS) return fail(SSD_ENOSUP, "n_seqs = %d exceeds %d", n_seqs, BT_MAX_SEQS);
  if (int rc = check_block_tokens(block_tokens, n_blocks)) return rc;
  if ((long long)table_cap * block_tokens > (1 << 30) || max_rows > (1 << 30)) return fail(SSD_ENOSUP, "more than 2^30 positions or rows");
  BlockTableArgs a;
  a.len = dev_len; a.rows = dev_rows; a.owned = dev_owned; a.shared = dev_shared; a.n_free = dev_n_free;
  a.table = dev_table; a.stack = dev_free_stack; a.owned_out = dev_owned_out; a.n_free_out = dev_n_free_out; a.row_start = dev_row_start;
  a.row_seq = dev_row_seq; a.row_pos = dev_row_pos; a.row_slot = dev_row_slot; a.status = dev_status;
  a.B = n_seqs; a.bt_shift = log2_of(block_tokens); a.n_blocks = n_blocks; a.cap = table_cap; a.max_rows = max_rows;
  hipLaunchKernelGGL(k_block_tables, dim3(1), dim3(BT_THREADS), 0, (hipStream_t)stream, a);
  LAUNCH_CHECK();
  if (max_rows > BT_ROWS_HERE) {
    hipLaunchKernelGGL(k_block_table_rows, dim3(cdiv(max_rows, BLOCK)), dim3(BLOCK), 0, (hipStream_t)stream, a);
    LAUNCH_CHECK();
  }
  return SSD_OK;
}

extern "C" int ssd_rope_append(const ssd_pages* pages, int n_rows, int n_q_heads, const void* dev_q, size_t q_stride, const void* dev_k, size_t k_stride,
                               const void* dev_v, size_t v_stride, const float* dev_rope, int rope_positions, const int32_t* dev_row_pos,
                               const int32_t* dev_row_slot, void* dev_q_out, size_t q_out_stride, int32_t* dev_status, void* stream) {
  RopeAppendArgs a;
  if (int rc = check_pages(pages, a.p)) return rc;
  if (n_rows < 0 || n_rows > (1 << 24) || n_q_heads < 0 || n_q_heads > 1024) return fail(SSD_EINVAL, "bad n_rows / n_q_heads");
  if (n_rows == 0) return SSD_OK;
  if (!dev_row_pos || !dev_row_slot) return fail(SSD_EINVAL, "null argument");
  if (((uintptr_t)dev_rope & 15)) return fail(SSD_EINVAL, "the table of angles must be 16-byte aligned");
  if (dev_rope && rope_positions < 1) return fail(SSD_EINVAL, "rope_positions = %d", rope_positions);
  if (int rc = check_rows("k", dev_k, k_stride, a.p.nkv, a.p, pages->dtype)) return rc;
  if (int rc = check_rows("v", dev_v, v_stride, a.p.nkv, a.p, pages->dtype)) return rc;
  if (n_q_heads > 0) {
    if (int rc = check_rows("q", dev_q, q_stride, n_q_heads, a.p, pages->dtype)) return rc;
    if (int rc = check_rows("q_out", dev_q_out, q_out_stride, n_q_heads, a.p, pages->dtype)) return rc;
  }
  a.q = dev_q; a.k = dev_k; a.v = dev_v; a.q_out = dev_q_out;
  a.q_stride = q_stride; a.k_stride = k_stride; a.v_stride = v_stride; a.q_out_stride = q_out_stride;
  a.rope = dev_rope; a.row_pos = dev_row_pos; a.row_slot = dev_row_slot; a.status = dev_status;
  a.n_rows = n_rows; a.nq = n_q_heads; a.positions = rope_positions;
  const int per16 = pages->dtype == SSD_DTYPE_BF16 ? 8 : 4;
  const int v_wgs = cdiv(n_rows, RA_WINDOW) * a.p.nkv;
  const long long threads = (long long)n_rows * (a.p.hd / 2 / per16) * cdiv(n_q_heads + a.p.nkv, RA_HEADS);
  const dim3 grid((unsigned)(v_wgs + (threads + BLOCK - 1) / BLOCK));
  if (pages->dtype == SSD_DTYPE_BF16) hipLaunchKernelGGL(k_rope_append<BF16>, grid, dim3(BLOCK), 0, (hipStream_t)stream, a, v_wgs);
  else hipLaunchKernelGGL(k_rope_append<F32>, grid, dim3(BLOCK), 0, (hipStream_t)stream, a, v_wgs);
  LAUNCH_CHECK();
  return SSD_OK;
}

// ------------------------------------------------------------------------------------------------ attention
// How a call is cut.  From sizes that the caller gives alone, so that the workspace's size is known without a device.
struct AttnCut {
  int sh, own;                                             // k_paged_attention's SH and OWN
  bool in_line, by_length;
  int P, P_sh, sh_chunks, own_chunks, sh_slots, own_slots;
};
static AttnCut cut_attention(int dtype, int hd, int nkv, int group, int n_seqs, int n_rows, int max_len, int shared_positions) {
  constexpr int MAX_PARTS = 32;                            // of a source: 64 of a row
  AttnCut c;
  const bool b16 = dtype == SSD_DTYPE_BF16;
  const int packed = n_rows * group, each = cdiv(packed, n_seqs);
  c.own = b16 && each > 64 ? 0 : b16 && each > 32 ? 3 : each <= 16 ? 1 : 2;
  // A prefix is in line with every sequence's own keys where nobody shares it, where a sequence's rows fill tiles of their own, or where reading it again for each costs
  // less than the merge that two sources ask for, 4 us.
  c.in_line = n_seqs == 1 || each >= 256 ||
              (c.own && c.own < 3 && max_len <= 1024 && std::max(shared_positions * 0.0012, (double)n_seqs * shared_positions * nkv * hd * (b16 ? 4 : 8) / 4e6) < 4.0);
  const bool apart = shared_positions > 0 && !c.in_line;
  c.sh = !apart ? 0 : !b16 || packed <= 32 ? 3 : hd < 128 && packed >= 512 ? 2 : 1;
  if (c.sh == 3 && (c.own == 0 || c.own == 3)) c.sh = 1;
  const bool own_tiles = c.own == 0 || c.own == 3;
  const int own_t = c.own == 0 ? 128 : c.own == 3 ? 64 : 16 * c.own, sh_t = c.sh == 3 ? 16 * c.own : 128 * c.sh;
  c.own_slots = packed / own_t + n_seqs;
  c.sh_slots = apart ? cdiv(packed, sh_t) : 0;
  // Chunks of a part: those of the least estimated time.  A workgroup of streams takes 4.5 us and 0.6 for each chunk of a wave, and there is room for 1024 of four waves or 512 of eight.
  // Of tiles, a chunk costs a workgroup of 128 rows `unit` us beside another one on its compute unit, and a workgroup three chunks for being one; 512 have
  // room at a time.  More than one part costs a launch of 4 us, and each part's result is written and read again at 4.7 TB/s.
  const int own_keys = std::max(1, max_len - (apart ? shared_positions : 0)), own_n = cdiv(own_keys, PA_CHUNK), sh_n = cdiv(shared_positions, PA_CHUNK);
  const int own_tile_n = std::max(n_seqs, packed / own_t);
  const double unit = hd == 128 ? 2.2 : hd == 64 ? 1.4 : 1.0, part_us = (double)n_rows * nkv * group * (hd + 2) * 8 / 4.7e6;
  const int waves = own_tiles || c.sh == 1 || c.sh == 2 ? 4 : 8;
  auto stream_chunks = [&](int tiles, int n, bool alone) {
    double best = 1e30;
    int pick = n;
    for (int p = 1; p <= MAX_PARTS; ++p) {
      const int size = cdiv(n, p), parts = cdiv(n, size);
      const double us = (4.5 + 0.6 * cdiv(size, waves)) * std::max(1.0, (double)tiles * nkv * parts / (4096 / waves)) + (parts > 1 && alone ? 4.0 : 0.0) + parts * part_us;
      if (us < best) { best = us; pick = size; }
    }
    return pick;
  };
  c.own_chunks = own_tiles ? 0 : stream_chunks(own_tile_n, own_n, !apart);
  c.sh_chunks = !apart ? 0 : c.sh == 3 ? stream_chunks(c.sh_slots, sh_n, false) : 0;
  if (own_tiles || c.sh == 1 || c.sh == 2) {
    double best = 1e30;
    int pick = 0;
    for (int i = 0; i < 2 * MAX_PARTS; ++i) {              // (one size for both sources: what divides either of them)
      const int n = std::max(4, cdiv(i & 1 ? sh_n : own_n, (i >> 1) + 1));
      const int so = own_tiles ? std::min(n, own_n) : 0, po = so ? cdiv(own_n, so) : 0, ss = apart && c.sh != 3 ? std::min(n, sh_n) : 0, ps = ss ? cdiv(sh_n, ss) : 0;
      if (po > MAX_PARTS || ps > MAX_PARTS) continue;
      const double cost_s = c.sh == 2 ? 1.8 : 1.0, cost_o = c.own == 3 ? 0.6 : 1.0;
      const double load = (double)ps * c.sh_slots * nkv * (ss * cost_s + 3) + (double)po * own_tile_n * nkv * (so * cost_o + 3);
      const double us = unit * std::max({load / 512, ss * cost_s + 3, so * cost_o + 3}) + (po + ps > 1 ? 4 + (po + ps) * part_us : 0);
      if (us < best) { best = us; pick = n; }
    }
    if (own_tiles) c.own_chunks = std::min(pick, own_n);
    if (apart && c.sh != 3) c.sh_chunks = std::min(pick, sh_n);
  }
  const int own_parts = cdiv(own_n, c.own_chunks);
  c.P_sh = apart ? cdiv(sh_n, c.sh_chunks) : 0;
  c.by_length = c.own == 0 && own_parts == 1 && !apart && n_seqs <= 64;
  c.P = c.P_sh + own_parts;
  return c;
}
static int check_attention(const ssd_pages* pages, Pages& p, int n_q_heads, int n_seqs, int n_rows, int max_len, int shared_blocks) {
  if (int rc = check_pages(pages, p)) return rc;
  if (n_q_heads < 1 || n_q_heads % p.nkv || n_q_heads > 1024) return fail(SSD_EINVAL, "%d query heads over %d key/value heads", n_q_heads, p.nkv);
  if (n_seqs < 1 || n_seqs > (1 << 16) || n_rows < 0 || max_len < 1 || max_len > (1 << 30) || shared_blocks < 0) return fail(SSD_EINVAL, "bad n_seqs / n_rows / max_len / shared_blocks");
  if ((long long)n_rows * n_q_heads > (1 << 26)) return fail(SSD_ENOSUP, "n_rows * n_q_heads exceeds 2^26");
  if ((long long)shared_blocks * p.bt > (1 << 30)) return fail(SSD_ENOSUP, "a shared prefix of more than 2^30 positions");
  return SSD_OK;
}
static size_t attention_ws(const AttnCut& c, int n_rows, int nq, int hd) { return c.P > 1 ? (size_t)n_rows * nq * c.P * (hd + 2) * sizeof(float) : 0; }

extern "C" size_t ssd_paged_attention_workspace_bytes(const ssd_pages* pages, int n_q_heads, int n_seqs, int n_rows, int max_len, int shared_blocks) {
  Pages p;
  if (check_attention(pages, p, n_q_heads, n_seqs, n_rows, max_len, shared_blocks)) return (size_t)-1;
  return attention_ws(cut_attention(pages->dtype, p.hd, p.nkv, n_q_heads / p.nkv, n_seqs, n_rows, max_len, shared_blocks * p.bt), n_rows, n_q_heads, p.hd);
}

template <typename DT, int HD, int SH, int OWN>
static int launch_attention(const PagedAttnArgs& a, hipStream_t st) {
  const long long wgs = ((long long)a.sh_slots * a.P_sh + (long long)a.own_slots * (a.P - a.P_sh)) * a.p.nkv;
  if (wgs > 0x7FFFFFFFll) return fail(SSD_ENOSUP, "too many workgroups");
  hipLaunchKernelGGL((k_paged_attention<DT, HD, SH, OWN>), dim3((unsigned)wgs), dim3(PagedShape<SH, OWN>::THREADS), 0, st, a);
  LAUNCH_CHECK();
  if (a.P > 1) {
    hipLaunchKernelGGL((k_paged_attention_merge<DT, HD>), dim3((unsigned)cdiv(a.n_rows * a.nq, BLOCK / WAVE)), dim3(BLOCK), 0, st, a);
    LAUNCH_CHECK();
  }
  return SSD_OK;
}
template <typename DT, int HD, int SH>
static int launch_own(const PagedAttnArgs& a, int own, hipStream_t st) {
  if constexpr (std::is_same<DT, BF16>::value && SH != 3)
    if (own == 0 || own == 3) return own == 0 ? launch_attention<DT, HD, SH, 0>(a, st) : launch_attention<DT, HD, SH, 3>(a, st);
  return own == 1 ? launch_attention<DT, HD, SH, 1>(a, st) : launch_attention<DT, HD, SH, 2>(a, st);
}
template <typename DT, int HD>
static int launch_paged_attention(const PagedAttnArgs& a, const AttnCut& c, hipStream_t st) {
  if (c.sh == 0) return launch_own<DT, HD, 0>(a, c.own, st);
  if (c.sh == 3) return launch_own<DT, HD, 3>(a, c.own, st);
  if constexpr (std::is_same<DT, BF16>::value) {
    if constexpr (HD < 128)
      if (c.sh == 2) return launch_own<DT, HD, 2>(a, c.own, st);
    return launch_own<DT, HD, 1>(a, c.own, st);
  }
  return fail(SSD_ENOSUP, "no kernel");
}

extern "C" int ssd_paged_attention(const ssd_pages* pages, int n_q_heads, float scale, int n_seqs, int n_rows, int max_len, const int32_t* dev_len,
                                   const int32_t* dev_row_start, const int32_t* dev_table, int table_cap, int shared_blocks, const int32_t* dev_shared_table,
                                   const int32_t* dev_shared, const void* dev_q, size_t q_stride, void* dev_out, size_t out_stride, void* dev_ws,
                                   size_t ws_bytes, int32_t* dev_status, void* stream) {
  PagedAttnArgs a;
  if (int rc = check_attention(pages, a.p, n_q_heads, n_seqs, n_rows, max_len, shared_blocks)) return rc;
  if (n_rows == 0) return SSD_OK;
  if (!dev_len || !dev_row_start || !dev_table || (shared_blocks > 0 && !dev_shared_table)) return fail(SSD_EINVAL, "null argument");
  if (table_cap < 1 || (long long)table_cap * a.p.bt > (1 << 30)) return fail(SSD_EINVAL, "table_cap = %d", table_cap);
  if (!std::isfinite(scale)) return fail(SSD_EINVAL, "scale is not finite");
  if (int rc = check_rows("q", dev_q, q_stride, n_q_heads, a.p, pages->dtype)) return rc;
  if (int rc = check_rows("out", dev_out, out_stride, n_q_heads, a.p, pages->dtype)) return rc;
  const AttnCut c = cut_attention(pages->dtype, a.p.hd, a.p.nkv, n_q_heads / a.p.nkv, n_seqs, n_rows, max_len, shared_blocks * a.p.bt);
  const size_t need = attention_ws(c, n_rows, n_q_heads, a.p.hd);
  if (need && (!dev_ws || ((uintptr_t)dev_ws & 15))) return fail(SSD_EINVAL, "workspace is null or not 16-byte aligned");
  if (ws_bytes < need) return fail(SSD_ENOMEM, "attention workspace: need %zu bytes, got %zu", need, ws_bytes);
  a.q = dev_q; a.out = dev_out; a.q_stride = q_stride; a.out_stride = out_stride;
  a.len = dev_len; a.row_start = dev_row_start; a.table = dev_table; a.shared_table = dev_shared_table; a.shared = dev_shared; a.status = dev_status;
  a.o_part = (float*)dev_ws;
  a.ml_part = a.o_part + (size_t)n_rows * n_q_heads * c.P * a.p.hd;
  a.scale2 = scale * 1.44269504088896340736f;
  a.nq = n_q_heads; a.n_seqs = n_seqs; a.n_rows = n_rows; a.cap = table_cap; a.shared_blocks = shared_blocks;
  a.in_line = c.in_line && shared_blocks > 0;
  a.by_length = c.by_length;
  a.P = c.P; a.P_sh = c.P_sh; a.sh_chunks = c.sh_chunks; a.own_chunks = c.own_chunks; a.sh_slots = c.sh_slots; a.own_slots = c.own_slots;
  hipStream_t st = (hipStream_t)stream;
  const bool b16 = pages->dtype == SSD_DTYPE_BF16;
  switch (a.p.hd) {
    case 32: return b16 ? launch_paged_attention<BF16, 32>(a, c, st) : launch_paged_attention<F32, 32>(a, c, st);
    case 64: return b16 ? launch_paged_attention<BF16, 64>(a, c, st) : launch_paged_attention<F32, 64>(a, c, st);
    default: return b16 ? launch_paged_attention<BF16, 128>(a, c, st) : launch_paged_attention<F32, 128>(a, c, st);
  }
}
