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

constexpr long long MOST_THREADS = 0xFFFFFFFFll;           // of a launch

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
    if (dev_q_out == dev_q && q_out_stride != q_stride && n_rows > 1) return fail(SSD_EINVAL, "q_out is q, but its rows are %zu apart, not %zu", q_out_stride, q_stride);
  }
  a.q = dev_q; a.k = dev_k; a.v = dev_v; a.q_out = dev_q_out;
  a.q_stride = q_stride; a.k_stride = k_stride; a.v_stride = v_stride; a.q_out_stride = q_out_stride;
  a.rope = dev_rope; a.row_pos = dev_row_pos; a.row_slot = dev_row_slot; a.status = dev_status;
  a.n_rows = n_rows; a.nq = n_q_heads; a.positions = rope_positions;
  const int per16 = pages->dtype == SSD_DTYPE_BF16 ? 8 : 4;
  const int v_wgs = cdiv(n_rows, RA_WINDOW) * a.p.nkv;
  const long long threads = (long long)n_rows * (a.p.hd / 2 / per16) * cdiv(n_q_heads + a.p.nkv, RA_HEADS);
  const long long wgs = v_wgs + (threads + BLOCK - 1) / BLOCK;
  if (wgs > MOST_THREADS / BLOCK) return fail(SSD_ENOSUP, "n_rows = %d: more threads than a launch has", n_rows);
  const dim3 grid((unsigned)wgs);
  if (pages->dtype == SSD_DTYPE_BF16) hipLaunchKernelGGL(k_rope_append<BF16>, grid, dim3(BLOCK), 0, (hipStream_t)stream, a, v_wgs);
  else hipLaunchKernelGGL(k_rope_append<F32>, grid, dim3(BLOCK), 0, (hipStream_t)stream, a, v_wgs);
  LAUNCH_CHECK();
  return SSD_OK;
}

// ------------------------------------------------------------------------------------------------ attention
// How a call is cut.  From sizes that the caller gives alone, so that the workspace's size is known without a device: the kinds of workgroups and the chunks of a part that have
// the least estimated time,
//     sqrt(longest^2 + load^2) + (3.8 + 0.195 per MB of results for each part, if there are several)  us and what every call takes,
// `longest`: of the workgroups, alone on a compute unit; `load`: of all of them, spread over 256 compute units.  The terms were fitted to 7100 cuts of 126 calls (1 to 256 sequences,
// 1 to 7600 rows, 9 to 16888 positions; bf16 heads of 64 and 128, fp32 heads of 32, with kernels that were up to 8 % slower in some calls), but for the 3.8, of which a graph takes 2.3 and a launch by
// itself more, and for what bf16 heads of 32 and fp32 heads of 64 and 128 have of their own, which were fitted to nothing.  Of 348 other calls with the present kernels (9887 cuts,
// profiles/cuts_paged_attention.txt) the cut that is picked takes 3.0, 2.9 and 4.8 % more time in the mean than the best that was measured with bf16 heads of 32, 64 and 128, and at most 1.38 times
// as long; 7.8, 9.5 and 7.1 % with fp32 ones, and at most 1.73 times.  Rules on the rows of a sequence, measured on the 126, took 24 %, and up to three times.
//   What the parts leave for the merge takes no more than a workspace that grows with rows, length and prefix, so that one for a caller's largest call does for every smaller one:
// rows x heads x parts stay below twice the rows x heads (a shared prefix and own keys) + 2^18, which is 1024 workgroups of 256 rows.  Of 300000 sizes, up to 65536 rows and 512 heads, it
// changes the cut of 1.4 %; by the estimate the mean call then takes 0.03 % longer, and the worst 11 %.
constexpr int PA_PARTS = 32;                               // of a source at most: no more than 64 of a row
static long long partial_rows(long long row_heads, int max_len, int shared_positions) {
  const int parts = std::min(PA_PARTS, cdiv(max_len, PA_CHUNK)) + std::min(PA_PARTS, cdiv(shared_positions, PA_CHUNK));
  return parts < 2 ? 0 : std::min(row_heads * parts, 2 * row_heads + (1 << 18));
}
struct AttnCut {
  int sh, own;                                             // k_paged_attention's SH and OWN
  bool in_line;
  int P, P_sh, sh_chunks, own_chunks, sh_slots, own_slots;
};
static AttnCut cut_attention(int dtype, int hd, int nkv, int group, int n_seqs, int n_rows, int max_len, int shared_positions) {
  constexpr int PARTS[] = {1, 2, 3, 4, 5, 6, 7, 8, 12, 16, PA_PARTS};
  const bool b16 = dtype == SSD_DTYPE_BF16;
  const int most = n_rows ? (int)std::min(2ll + (1 << 18) / ((long long)n_rows * nkv * group), 2ll * PA_PARTS) : 1;        // parts of a row
  const int packed = n_rows * group, each = cdiv(packed, n_seqs), sh_n = cdiv(shared_positions, PA_CHUNK);
  const float part_us = 0.195f * (float)n_rows * nkv * group * (hd + 2) * 8e-6f;
  // A chunk of a workgroup of 128 rows by tiles (bf16), alone and as a share of a full compute unit; a step of a
  // wave of streams, whose keys take 512 bytes of a lane's registers at most.
  const float tile_us = hd == 128 ? 1.13f : hd == 64 ? 0.73f : 0.52f, tile_share = hd == 128 ? 0.60f : hd == 64 ? 0.44f : 0.33f;
  const int steps_a_chunk = std::max(1, PA_CHUNK * hd * (b16 ? 2 : 4) / 8192);
  const float step_us = b16 ? (hd == 32 ? 0.9f : hd == 64 ? 1.5f : 1.68f) : 2.35f;
  struct Source {
    int cuts, best;                                        // (which of them)
    int chunks[11], parts[11];
    float longest[11], load[11];
  };
  // bf16 pages have streams of up to 16 rows (more rows are faster by tiles), fp32 of up to 16 and 32, and those of four waves too: many sequences of few
  // keys are done in fewer rounds of workgroups (243 of up to 335 positions 50.4 -> 31.0 us), few of many keys wait longer (4 behind 3904 positions 56.7, four
  // waves 86.7), and parts are for eight (90 behind 5488 positions 59.2, in parts of four waves 79.1).
  // n: chunks.  kind: 0 tiles of 128 rows, 3 of 64, 4 of 256; 1, 2 streams of up to 16, 32.  `mean`: of the part of the keys that its rows see.
  auto source = [&](Source& x, int kind, int n, int tiles, float mean, int waves, bool whole = false) {
    x.cuts = 0;
    const bool t = kind == 0 || kind >= 3;
    const float size = kind == 4 ? 1.6f : kind == 3 ? 0.78f : 1.f;
    const float share = t ? tile_share * (kind == 3 ? (hd == 128 ? 0.8f : 0.6f) : size) : kind == 1 ? 1.37f : 2.25f;
    for (int p : PARTS) {
      if (whole && p > 1) break;
      const int c = cdiv(n, p), parts = cdiv(n, c), i = x.cuts;
      if (i && c == x.chunks[i - 1]) continue;
      x.chunks[i] = c; x.parts[i] = parts;
      const float seen = parts == 1 ? mean : 1.f;
      const float wgs = (float)tiles * parts * nkv / 256, turns = (wgs + ceilf(wgs)) * 0.5f;
      x.longest[i] = t ? size * tile_us * (c + 1.8f) : 0.9f + step_us * (float)cdiv(c * steps_a_chunk, waves);
      x.load[i] = turns * share * (t ? c * seen + 1.8f : (0.9f + step_us * ceilf(c * steps_a_chunk * seen / waves)) * waves / 8);
      ++x.cuts;
    }
  };
  AttnCut c;
  float best = 1e30f;
  for (int apart = 0; apart <= (shared_positions > 0 && n_seqs > 1); ++apart) {
    const int own_n = cdiv(std::max(1, max_len - (apart ? shared_positions : 0)), PA_CHUNK);
    const float mean = std::max(0.1f, 1.f - (float)n_rows / n_seqs / (2 * PA_CHUNK) / own_n);
    Source shared[3];                                      // by tiles of 128 and 256 rows, by streams
    if (apart && b16) source(shared[0], 0, sh_n, cdiv(packed, 128), 1.f, 4);
    const bool wide = apart && b16 && hd < 128 && packed > 128;
    if (wide) source(shared[1], 4, sh_n, cdiv(packed, 256), 1.f, 4);
    for (int own = b16 ? 0 : 1; own < (b16 ? 4 : 6); ++own) {
      const bool own_tiles = own == 0 || own == 3;
      if (b16 ? own == 2 : own == 3 || (own > 3 && apart)) continue;
      const int rt = own > 3 ? own - 3 : own, own_t = own == 0 ? 128 : own == 3 ? 64 : 16 * rt;
      if ((own == 0 || rt == 2) && each <= own_t / 2) continue;       // (as many workgroups as of the smaller kind)
      Source o;
      const int tiles = n_seqs * cdiv(each, own_t), first_sh = apart ? (b16 ? 1 : 3) : 0;
      source(o, own_tiles ? own : rt, own_n, tiles, mean, own_tiles || (b16 && apart) || own > 3 ? 4 : 8, own > 3);
      for (int sh = first_sh; sh <= (apart ? 3 : 0); ++sh) {
        if ((sh == 3 && own_tiles) || (sh == 2 && !wide)) continue;
        const int sh_slots = sh ? cdiv(packed, sh == 3 ? own_t : 128 * sh) : 0;
        if (sh == 3) {                                     // (eight waves, then, of both)
          if (first_sh != 3) source(o, own, own_n, tiles, mean, 8);
          source(shared[2], own, sh_n, sh_slots, 1.f, 8);
        }
        Source& x = shared[sh ? sh - 1 : 0];
        auto us = [&](int i, int j) {
          const int parts = o.parts[i] + (sh ? x.parts[j] : 0);
          if (parts > most) return 1e30f;
          const float longest = sh ? std::max(o.longest[i], x.longest[j]) : o.longest[i], load = o.load[i] + (sh ? x.load[j] : 0.f);
          return sqrtf(longest * longest + load * load) + (parts > 1 ? 3.8f + parts * part_us : 0.f);
        };
        o.best = x.best = 0;
        float least = 1e30f;
        for (int turn = 0; turn < (sh ? 3 : 1); ++turn) {  // each source's in turn
          Source& y = sh && turn != 1 ? x : o;
          int pick = y.best;
          for (int i = 0; i < y.cuts; ++i) {
            const float t = &y == &o ? us(i, x.best) : us(o.best, i);
            if (t < least) { least = t; pick = i; }
          }
          y.best = pick;
        }
        if (least >= best) continue;
        best = least;
        c.own = own; c.sh = sh; c.in_line = !apart;
        c.own_chunks = o.chunks[o.best];
        c.sh_chunks = sh ? x.chunks[x.best] : 0;
        c.own_slots = packed / own_t + n_seqs;
        c.sh_slots = sh_slots;
        c.P_sh = sh ? x.parts[x.best] : 0;
        c.P = c.P_sh + o.parts[o.best];
      }
    }
  }
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
  return (size_t)partial_rows((long long)n_rows * n_q_heads, max_len, shared_blocks * p.bt) * (p.hd + 2) * sizeof(float);
}

extern "C" int ssd_paged_attention_plan(const ssd_pages* pages, int n_q_heads, int n_seqs, int n_rows, int max_len, int shared_blocks, int plan[4]) {
  Pages p;
  if (int rc = check_attention(pages, p, n_q_heads, n_seqs, n_rows, max_len, shared_blocks)) return rc;
  if (!plan || n_rows < 1) return fail(SSD_EINVAL, plan ? "a call without rows has no plan" : "null argument");
  const AttnCut c = cut_attention(pages->dtype, p.hd, p.nkv, n_q_heads / p.nkv, n_seqs, n_rows, max_len, shared_blocks * p.bt);
  plan[0] = c.sh; plan[1] = c.own; plan[2] = c.P_sh; plan[3] = c.P;
  return SSD_OK;
}

template <typename DT, int HD, int SH, int OWN>
static int launch_attention(const PagedAttnArgs& a, hipStream_t st) {
  const long long wgs = ((long long)a.sh_slots * a.P_sh + (long long)a.own_slots * (a.P - a.P_sh)) * a.p.nkv;
  if (wgs > MOST_THREADS / PagedShape<SH, OWN>::THREADS || (a.P > 1 && (long long)a.n_rows * a.nq > MOST_THREADS / WAVE)) return fail(SSD_ENOSUP, "more threads than a launch has");
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
  if constexpr (std::is_same<DT, BF16>::value) {
    if constexpr (SH != 3)
      if (own != 1) return own == 0 ? launch_attention<DT, HD, SH, 0>(a, st) : launch_attention<DT, HD, SH, 3>(a, st);
  } else {
    if (own == 2) return launch_attention<DT, HD, SH, 2>(a, st);
    if constexpr (SH == 0)
      if (own > 3) return own == 4 ? launch_attention<DT, HD, SH, 4>(a, st) : launch_attention<DT, HD, SH, 5>(a, st);
  }
  return launch_attention<DT, HD, SH, 1>(a, st);
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
  const float scale2 = scale * 1.44269504088896340736f;
  if (!std::isfinite(scale2)) return fail(SSD_EINVAL, "scale, or scale * log2(e), is not finite");
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
  a.scale2 = scale2;
  a.nq = n_q_heads; a.n_seqs = n_seqs; a.n_rows = n_rows; a.cap = table_cap; a.shared_blocks = shared_blocks;
  a.in_line = c.in_line && shared_blocks > 0;
  a.P = c.P; a.P_sh = c.P_sh; a.sh_chunks = c.sh_chunks; a.own_chunks = c.own_chunks; a.sh_slots = c.sh_slots; a.own_slots = c.own_slots;
  hipStream_t st = (hipStream_t)stream;
  const bool b16 = pages->dtype == SSD_DTYPE_BF16;
  switch (a.p.hd) {
    case 32: return b16 ? launch_paged_attention<BF16, 32>(a, c, st) : launch_paged_attention<F32, 32>(a, c, st);
    case 64: return b16 ? launch_paged_attention<BF16, 64>(a, c, st) : launch_paged_attention<F32, 64>(a, c, st);
    default: return b16 ? launch_paged_attention<BF16, 128>(a, c, st) : launch_paged_attention<F32, 128>(a, c, st);
  }
}
