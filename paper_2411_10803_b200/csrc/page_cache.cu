// Decoding-stage cache in pages of 4-bit values: places for tokens (page tables, slots), rows in, rows out.
// The formats and the arithmetic of the values are described in mustdrop.h; the attention that reads
// the pages is in page_attend.cu.
#include <algorithm>

#include "page_internal.h"

namespace mustdrop {

mustdrop_status_t check_page_sizes(const mustdrop_page_config_t* c) {
  if (c == nullptr || c->n_seq <= 0 || c->n_pages <= 0 || (c->flags & ~MUSTDROP_PAGE_FLAG_DEBUG_TIMEOUT) != 0) return MUSTDROP_ERR_INVALID_ARG;
  if (page_log2(c->page) < 0 || c->n_seq > 65535) return MUSTDROP_ERR_UNSUPPORTED;
  if (static_cast<int64_t>(c->n_pages) * c->page > INT32_MAX) return MUSTDROP_ERR_UNSUPPORTED;
  return MUSTDROP_OK;
}

mustdrop_status_t check_page_pool(const mustdrop_page_config_t* c) {
  const mustdrop_status_t st = check_page_sizes(c);
  if (st != MUSTDROP_OK) return st;
  if (c->n_heads <= 0) return MUSTDROP_ERR_INVALID_ARG;
  if ((c->head_dim != 64 && c->head_dim != 128) || c->n_heads > 65535) return MUSTDROP_ERR_UNSUPPORTED;
  return MUSTDROP_OK;
}

mustdrop_status_t check_page_queries(const mustdrop_page_config_t* c) {
  const mustdrop_status_t st = check_page_pool(c);
  if (st != MUSTDROP_OK) return st;
  if (c->q_heads <= 0 || c->n_q <= 0 || c->q_heads % c->n_heads != 0) return MUSTDROP_ERR_INVALID_ARG;
  if (c->n_q > 128 || c->q_heads > 65535 || static_cast<int64_t>(c->q_heads / c->n_heads) * c->n_q > 16384) return MUSTDROP_ERR_UNSUPPORTED;
  return MUSTDROP_OK;
}

namespace {

// ---------------------------------------------------------------------------------------- page tables
//
// A pure function of the lengths: with need[s] = pages sequence s asks for, back[s] = pages it gives back, P the
// sums over the sequences before it, its i-th new page is ring[head + P_need + i] and its i-th returned page goes to
// ring[head + count + P_back + i].  The ring's two ends never meet (count + all of back <= n_pages), so no CTA
// waits for another: each sums need and back over the sequences before its own (two loads per sequence, from L2) and
// handles its own ones.  What the others still read - lengths and state that are updated in place - is written by the CTA that finishes
// last, in a second walk over all of them; one CTA alone, or outputs of their own, need no such order.  Bound: launch and three dependent trips
// to L2 (240 sequences, one token: 4.4 us), for many sequences the sums, which grow with their square, and the walk (2048 sequences, one token:
// 6.4 us with outputs of their own, 10 in place; 65535: 21 and 117).
struct TableParams {
  const int32_t *add, *len, *state;
  int32_t *len_out, *state_out, *ring, *table, *slots;
  int32_t* workspace;
  int32_t n_seq, lg, n_pages, max_pages, rows, per_cta, rows_per_cta;
};

constexpr int kTableThreads = 512;
constexpr int kTableSeqs = kTableThreads;     // most sequences of a CTA
constexpr int kTableBatch = 8, kTableSlots = kTableBatch * kTableThreads;   // most slots of a thread, of a CTA

struct Move {       // what the call does to one sequence
  int32_t cur, grow, need, back, left;   // grow: tokens gained (0 where it shrinks or is refused for its length); left: tokens it then has
  bool bad;
};

__device__ __forceinline__ Move move_of(const TableParams& p, int s) {
  Move m;
  m.cur = p.len[s];
  const int32_t a = p.add[s];
  const int32_t most = p.max_pages << p.lg, mask = (1 << p.lg) - 1;
  const int64_t to = static_cast<int64_t>(m.cur) + a;
  m.grow = m.need = m.back = 0;
  m.left = m.cur;
  m.bad = m.cur < 0 || m.cur > most || a > p.rows || to > most;
  if (m.bad) return m;
  m.left = static_cast<int32_t>(to < 0 ? 0 : to);
  const int32_t had = static_cast<int32_t>((static_cast<uint32_t>(m.cur) + mask) >> p.lg);
  const int32_t pages = static_cast<int32_t>((static_cast<uint32_t>(m.left) + mask) >> p.lg);
  m.grow = max(a, 0);
  m.need = max(pages - had, 0);
  m.back = max(had - pages, 0);
  return m;
}

// Inclusive sums of (x, y) over the CTA's threads (they fit 32 bits: the page table has fewer than 2^31 entries);
// `total` receives the sums over all.
__device__ __forceinline__ int2 scan_pair(int2 v, int2* warp_sums, int2* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int x = __shfl_up_sync(~0u, v.x, d), y = __shfl_up_sync(~0u, v.y, d);
    if (lane >= d) { v.x += x; v.y += y; }
  }
  __syncthreads();
  if (lane == 31) warp_sums[warp] = v;
  __syncthreads();
  int2 all = {0, 0};
#pragma unroll
  for (int w = 0; w < kTableThreads / 32; ++w) {
    const int2 t = warp_sums[w];
    if (w < warp) { v.x += t.x; v.y += t.y; }
    all.x += t.x; all.y += t.y;
  }
  *total = all;
  return v;
}

// Place i (below 2 n_pages) of the ring.
__device__ __forceinline__ int32_t in_ring(const TableParams& p, int32_t i) { return i < p.n_pages ? i : i - p.n_pages; }

__global__ void __launch_bounds__(kTableThreads) page_tables_kernel(TableParams p) {
  __shared__ int2 warp_sums[kTableThreads / 32], sums_before[kTableThreads / 32];
  __shared__ int32_t cur_s[kTableSeqs], grow_s[kTableSeqs], first_s[kTableSeqs];   // first_s: ring offset of the first new page
  __shared__ int32_t back_s[kTableSeqs], back_at_s[kTableSeqs];                    // pages given back, and their place behind the ring's count
  __shared__ int32_t left_s[kTableSeqs];                                           // the new length
  __shared__ int last_s;
  pdl_launch_dependents();
  pdl_wait();
  const int first = blockIdx.x * p.per_cta, n_own = min(p.per_cta, p.n_seq - first);
  int32_t head = p.state[0], count = p.state[1];
  const int32_t given_head = head, given_count = count;
  const bool bad_state = head < 0 || head >= p.n_pages || count < 0 || count > p.n_pages;
  if (bad_state) head = count = 0;   // nothing is free, nothing can be given back
  const bool lead = blockIdx.y == 0;   // of the CTAs that share a range of sequences, the one that reports
  // this CTA's sequences (one per thread) and the sums over those before them, behind one barrier
  int2 before = {0, 0}, total = {0, 0};
  int32_t taken = 0;                   // largest sum of pages asked for that is granted, among this thread's sequences
  {
    const int i = threadIdx.x, s = first + i, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    Move m = {0, 0, 0, 0, 0, false};
    if (i < n_own) m = move_of(p, s);
#pragma unroll 4
    for (int b = threadIdx.x; b < first; b += kTableThreads) {
      const Move x = move_of(p, b);
      before.x += x.need; before.y += x.back;
    }
    int2 upto = {m.need, m.back};
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int x = __shfl_up_sync(~0u, upto.x, d), y = __shfl_up_sync(~0u, upto.y, d);
      if (lane >= d) { upto.x += x; upto.y += y; }
    }
    before.x = __reduce_add_sync(~0u, before.x);
    before.y = __reduce_add_sync(~0u, before.y);
    if (lane == 31) { warp_sums[warp] = upto; sums_before[warp] = before; }
    __syncthreads();
    before = {0, 0};
#pragma unroll
    for (int w = 0; w < kTableThreads / 32; ++w) {
      const int2 own = warp_sums[w], old = sums_before[w];
      before.x += old.x; before.y += old.y;
      total.x += own.x; total.y += own.y;
      if (w < warp) { upto.x += own.x; upto.y += own.y; }
    }
    upto.x += before.x; upto.y += before.y;
    before.x += total.x; before.y += total.y;   // now over all sequences up to the CTA's last
    if (i < n_own) {
      const bool granted = m.need == 0 || upto.x <= count;
      if (granted && m.need > 0) taken = max(taken, upto.x);
      cur_s[i] = m.cur;
      grow_s[i] = granted ? m.grow : 0;
      left_s[i] = granted ? m.left : m.cur;
      first_s[i] = granted && m.need > 0 ? upto.x - m.need : 0;
      if (lead && m.bad) record_status(p.workspace, MUSTDROP_ERR_BAD_LENGTH, s);
      if (lead && !granted) record_status(p.workspace, MUSTDROP_ERR_NO_PAGES, s);
      // what does not fit behind the ring's count was never the pool's
      const int32_t room = bad_state ? 0 : max(p.n_pages - count - (upto.y - m.back), 0);
      if (lead && m.back > room) record_status(p.workspace, MUSTDROP_ERR_BAD_LENGTH, s);
      back_s[i] = min(m.back, room);
      back_at_s[i] = back_s[i] > 0 ? count + (upto.y - m.back) : 0;
    }
  }
  __syncthreads();
  // pages given back: a warp per sequence
  for (int i = threadIdx.x >> 5; lead && i < n_own; i += kTableThreads / 32) {
    const int n = back_s[i];
    if (n == 0) continue;
    const int32_t pages = static_cast<int32_t>((static_cast<uint32_t>(left_s[i]) + (1 << p.lg) - 1) >> p.lg);
    const int32_t* from = p.table + static_cast<size_t>(first + i) * p.max_pages + pages;
    for (int b = threadIdx.x & 31; b < n; b += 32) {
      const int32_t id = from[b];
      if (static_cast<uint32_t>(id) >= static_cast<uint32_t>(p.n_pages)) record_status(p.workspace, MUSTDROP_ERR_BAD_PAGE, first + i);
      p.ring[in_ring(p, in_ring(p, head + back_at_s[i]) + b)] = id;
    }
  }
  // slots, and the table entries of the pages that begin among the new tokens
  const int t0 = blockIdx.y * p.rows_per_cta, n_t = min(p.rows_per_cta, p.rows - t0);
  const int32_t mask = (1 << p.lg) - 1;
  // (a thread's page ids are all asked for before the first is used: one trip to L2 for up to kTableBatch slots)
  const int items = n_own * n_t;                 // at most kTableSlots
  int i = threadIdx.x / n_t, t = threadIdx.x % n_t;
  const int di = kTableThreads / n_t, dt = kTableThreads % n_t;
  int32_t id[kTableBatch], at[kTableBatch];      // at: the slot's place in its page, -1: no slot
#pragma unroll
  for (int k = 0; k < kTableBatch; ++k) {
    id[k] = at[k] = -1;
    if (static_cast<int>(threadIdx.x) + k * kTableThreads < items) {
      const int32_t r = t0 + t;
      if (r < grow_s[i]) {
        const int32_t cur = cur_s[i], pos = cur + r, e = pos >> p.lg;
        const int32_t had = static_cast<int32_t>((static_cast<uint32_t>(cur) + mask) >> p.lg);
        int32_t* const entry = p.table + static_cast<size_t>(first + i) * p.max_pages + e;
        id[k] = e < had ? *entry : p.ring[in_ring(p, head + first_s[i] + (e - had))];
        at[k] = pos & mask;
        if (e >= had && at[k] == 0) *entry = id[k];
      }
      i += di; t += dt;
      if (t >= n_t) { t -= n_t; ++i; }
    }
  }
  i = threadIdx.x / n_t; t = threadIdx.x % n_t;
#pragma unroll
  for (int k = 0; k < kTableBatch; ++k) {
    if (static_cast<int>(threadIdx.x) + k * kTableThreads < items) {
      int32_t slot = -1;
      if (at[k] >= 0) {
        if (static_cast<uint32_t>(id[k]) < static_cast<uint32_t>(p.n_pages)) slot = (id[k] << p.lg) | at[k];
        else record_status(p.workspace, MUSTDROP_ERR_BAD_PAGE, first + i);
      }
      p.slots[static_cast<size_t>(first + i) * p.rows + t0 + t] = slot;
      i += di; t += dt;
      if (t >= n_t) { t -= n_t; ++i; }
    }
  }
  // Lengths and state.  Every CTA has read all of them that lie before its own, so what is updated in place waits for the CTA
  // that finishes last.
  const unsigned all = gridDim.x * gridDim.y;
  const bool in_place = p.len_out == p.len || p.state_out == p.state;
  const bool at_end = first + n_own == p.n_seq;
  bool mine = at_end && lead;          // this CTA writes the state
  if (in_place && all > 1) {
    __syncthreads();
    if (threadIdx.x == 0) {
      __threadfence();
      last_s = atomicInc(reinterpret_cast<unsigned*>(p.workspace) + kTicketWord, all - 1) == all - 1;
      __threadfence();
    }
    __syncthreads();
    if (!last_s) return;
    mine = true;
  } else if (lead) {
    for (int k = threadIdx.x; k < n_own; k += kTableThreads) p.len_out[first + k] = left_s[k];
  }
  if (!mine) return;
  // A second walk over all sequences where this CTA has to write their lengths, or has not seen which were granted.
  if (all > 1 && (in_place || before.x > count)) {
    before = {0, 0};
    taken = 0;
    for (int base = 0; base < p.n_seq; base += kTableThreads) {
      const int s = base + threadIdx.x;
      Move m = {0, 0, 0, 0, 0, false};
      if (s < p.n_seq) m = move_of(p, s);
      int2 upto = scan_pair({m.need, m.back}, warp_sums, &total);
      upto.x += before.x;
      before.x += total.x; before.y += total.y;
      if (s < p.n_seq) {
        const bool granted = m.need == 0 || upto.x <= count;
        if (granted && m.need > 0) taken = max(taken, upto.x);
        if (in_place) p.len_out[s] = granted ? m.left : m.cur;
      }
    }
  }
  if (before.x <= count) {
    taken = before.x;
  } else {
    taken = __reduce_max_sync(~0u, taken);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) warp_sums[threadIdx.x >> 5].x = taken;
    __syncthreads();
    for (int w = 0; w < kTableThreads / 32; ++w) taken = max(taken, warp_sums[w].x);
  }
  if (threadIdx.x == 0) {
    if (bad_state) {
      record_status(p.workspace, MUSTDROP_ERR_BAD_LENGTH, -1);
      p.state_out[0] = given_head;
      p.state_out[1] = given_count;
    } else {
      p.state_out[0] = in_ring(p, head + taken);
      p.state_out[1] = count - taken + min(before.y, p.n_pages - count);
    }
  }
}

// ---------------------------------------------------------------------------------------- rows in, rows out
//
// Store: a lane has one row's group of 32 channels (64 bytes of K and of V), a warp 8 rows of 128 channels or 16 of 64: what a
// group needs once - range, scale, centre, reciprocal - is computed once.  A word of the V codes holds four tokens, so lanes of
// four neighbouring rows exchange theirs and store whole words where their slots are one word's, else single bytes; rows are
// taken so that they are: fours end where slot mod 4 is 3, judged by the sequence's first slot.  With one row per sequence (decoded tokens) a
// warp's rows are heads instead.  Bound: bytes for large calls (64 x 2048 x 8 rows, 705 MB: 123 us, 5.7 TB/s), for those of
// 100 MB neither bytes nor issue alone (32 x 192 x 32 one after the other: 28 us, 4.7 TB/s, issue slots 64 %, ALU pipe 67 %, 39 % of the warps).
//
// Load: 16 lanes hold a row of 128 channels (8 of 64) as 16-byte vectors.  Bound: the bytes written (32 x 608 x 32 rows: 79 us, 4.0 TB/s; a
// plain fill of its buffers runs at 3.9).
// Both: small CTAs, as warps that finish hold their place until the CTA's last one has (256 threads: store 2 to 7 %, load 3 % slower).  And
// no early start of the call that follows: its CTAs would crowd onto the few SMs that are free by then and stay there (with one after 64
// requests' attention, tables, store and attention of the next layer take 79 us, without 71; a store and a load of one token 9.4 against 7.9).
constexpr int kRowThreads = 128;

struct RowParams {
  const int32_t* slots;
  const uint8_t* src[2];   // store: k, v
  uint8_t* dst[2];         // load: k_out, v_out
  uint8_t* pool;
  int32_t* workspace;
  int32_t n_heads, rows, groups, lg;   // groups: store: warps' shares of the rows (TOKENS: of the heads); load: fours of rows
  uint32_t n_slots;        // n_pages * page
  uint32_t warps;          // n_heads (TOKENS: rows) * groups
  int64_t stride[2][3];    // bytes: sequence, head, row
};

template <int D>
__device__ __forceinline__ uint8_t* chunk_of(const RowParams& p, int32_t slot, int head) {
  const int32_t page = slot >> p.lg, chunk = (slot & ((1 << p.lg) - 1)) >> 4;
  return p.pool + (((static_cast<int64_t>(page) * p.n_heads + head) << (p.lg - 4)) + chunk) * Chunk<D>::kBytes;
}

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t to_bf16(float x) {   // round to nearest even; NaN stays NaN
  uint32_t w;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(0.0f), "f"(x));   // (the pair's conversion runs at four times the rate of one)
  return w;
}

__device__ __forceinline__ uint32_t min_bf16x2(uint32_t a, uint32_t b) {   // a NaN stays one
  uint32_t d;
  asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ uint32_t max_bf16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ bool finite_bf16(uint32_t bits) { return (bits & 0x7f80u) != 0x7f80u; }

// (x - z) hi + (x - z) lo + magic for two numbers, each operation rounded.
__device__ __forceinline__ float2 code_pair(float2 x, float minus_z, float hi, float lo, float magic) {
  float2 t;
  asm("{\n\t.reg .b64 d, z, h, l, m, p;\n\t"
      "mov.b64 d, {%2, %3};\n\tmov.b64 z, {%4, %4};\n\tmov.b64 h, {%5, %5};\n\tmov.b64 l, {%6, %6};\n\tmov.b64 m, {%7, %7};\n\t"
      "add.rn.f32x2 d, d, z;\n\tmul.rn.f32x2 p, d, l;\n\tfma.rn.f32x2 p, d, h, p;\n\tadd.rn.f32x2 p, p, m;\n\t"
      "mov.b64 {%0, %1}, p;\n\t}"
      : "=f"(t.x), "=f"(t.y)
      : "f"(x.x), "f"(x.y), "f"(minus_z), "f"(hi), "f"(lo), "f"(magic));
  return t;
}

// Codes of a group's 32 channels as nibbles 0..7 of four words; its scale and centre (bf16 bits).
//
// A code is round((x - z) / s) + 8, ties to even.  With d = x - z (fp32) and the reciprocal of s in two fp32 terms, q = d hi +
// d lo is d / s to 2^-45 before its one rounding.  That decides as the correctly rounded quotient does: a tie s (k + 1/2) has 13
// bits, so another fp32 number d is more than 2^-24 of it away, which q's rounding keeps on its side; a tie itself is kept exactly.
// (|d / s| stays below 32: where the centre's rounding is many steps, so is the spacing of bf16 numbers beside it.)  No division
// and no conversion per channel: both run at a quarter of the rate of what is used here (the 32 x 192 x 32 rows of a pruned prompt: 71
// us with them, 34 without, 31 with two channels to an fp32 instruction).
__device__ __forceinline__ void quantise(const uint4 (&v)[4], uint32_t (&codes)[4], uint32_t* scale, uint32_t* centre) {
  uint32_t lo2 = v[0].x, hi2 = v[0].x;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    lo2 = min_bf16x2(lo2, min_bf16x2(min_bf16x2(v[i].x, v[i].y), min_bf16x2(v[i].z, v[i].w)));
    hi2 = max_bf16x2(hi2, max_bf16x2(max_bf16x2(v[i].x, v[i].y), max_bf16x2(v[i].z, v[i].w)));
  }
  lo2 = min_bf16x2(lo2, lo2 >> 16 | lo2 << 16);
  hi2 = max_bf16x2(hi2, hi2 >> 16 | hi2 << 16);
  // scale: (halves: the difference of two finite numbers may not be one) over 7.5, as below
  const float lo = bf16_lo(lo2), half = __fsub_rn(0.5f * bf16_lo(hi2), 0.5f * lo);
  constexpr float kInv = static_cast<float>(1.0 / 7.5), kInvLow = static_cast<float>(1.0 / 7.5 - static_cast<double>(kInv));
  *scale = to_bf16(__fmaf_rn(half, kInv, __fmul_rn(half, kInvLow)));
  const float s = __uint_as_float(*scale << 16);
  *centre = to_bf16(__fmaf_rn(8.0f, s, lo));
  const float z = __uint_as_float(*centre << 16);
  if (!(s >= 0x1p-100f && s <= 0x1p100f) || !finite_bf16(lo2) || !finite_bf16(hi2)) {
    const bool none = !finite_bf16(lo2) || !finite_bf16(hi2);   // (the centre stays finite: the attention multiplies it by zero for hidden keys)
    if (none) { *scale = 0x7fc0u; *centre = 0; }
#pragma unroll
    for (int i = 0; i < 4; ++i) codes[i] = none ? 0u : 0x88888888u;
    if (none || s == 0.0f) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {                   // a scale whose reciprocal is too large, or has no normal second term
      const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
      uint32_t c8 = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float c = rintf(__fdiv_rn(__fsub_rn((j & 1) ? bf16_hi(w[j >> 1]) : bf16_lo(w[j >> 1]), z), s)) + 8.0f;
        c8 |= static_cast<uint32_t>(fminf(fmaxf(c, 0.0f), 15.0f)) << (4 * j);
      }
      codes[i] = c8;
    }
    return;
  }
  float hi_inv;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(hi_inv) : "f"(s));
  const float lo_inv = __fmul_rn(__fmaf_rn(-s, hi_inv, 1.0f), hi_inv);
  constexpr float kMagic = 12582912.0f;     // 1.5 x 2^23: adding it rounds to a whole number, and its bits plus that number are the sum's
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
    uint32_t c8 = 0;
#pragma unroll
    for (int j = 3; j >= 0; --j) {             // two channels an instruction
      float2 t = make_float2(bf16_lo(w[j]), bf16_hi(w[j]));
      t = code_pair(t, -z, hi_inv, lo_inv, kMagic);
      c8 = c8 * 16u + __float_as_uint(fminf(fmaxf(t.y, kMagic - 8.0f), kMagic + 7.0f));
      c8 = c8 * 16u + __float_as_uint(fminf(fmaxf(t.x, kMagic - 8.0f), kMagic + 7.0f));
    }
    codes[i] = c8 - 0x11111111u * (0x4b400000u - 8u);   // the sum of 16^j (bits of kMagic + c_j - 8): c_j wanted
  }
}

// v[j] = codes[this lane's place] of the j-th of four lanes, STEP apart; `place` is this lane's (mod 4).
template <int STEP>
__device__ __forceinline__ void gather4(const uint32_t (&codes)[4], int place, uint32_t (&v)[4]) {
  const bool b1 = place & 2, b0 = place & 1;
  const uint32_t k0 = b1 ? codes[2] : codes[0], k1 = b1 ? codes[3] : codes[1];
  const uint32_t r0 = __shfl_xor_sync(~0u, b1 ? codes[0] : codes[2], 2 * STEP), r1 = __shfl_xor_sync(~0u, b1 ? codes[1] : codes[3], 2 * STEP);
  const uint32_t own = b0 ? k1 : k0, two = b0 ? r1 : r0;          // of this lane, and of the one two places away
  const uint32_t one = __shfl_xor_sync(~0u, b0 ? k0 : k1, STEP), three = __shfl_xor_sync(~0u, b0 ? r0 : r1, STEP);
  const uint32_t e = b0 ? one : own, o = b0 ? own : one, e2 = b0 ? three : two, o2 = b0 ? two : three;
  v[0] = b1 ? e2 : e; v[1] = b1 ? o2 : o; v[2] = b1 ? e : e2; v[3] = b1 ? o : o2;
}

// Word b of four: byte b of each of four rows' words.
__device__ __forceinline__ void bytes4(const uint32_t (&v)[4], uint32_t (&w)[4]) {
  const uint32_t x0 = __byte_perm(v[0], v[1], 0x5140), x1 = __byte_perm(v[0], v[1], 0x7362);
  const uint32_t y0 = __byte_perm(v[2], v[3], 0x5140), y1 = __byte_perm(v[2], v[3], 0x7362);
  w[0] = __byte_perm(x0, y0, 0x5410); w[1] = __byte_perm(x0, y0, 0x7632);
  w[2] = __byte_perm(x1, y1, 0x5410); w[3] = __byte_perm(x1, y1, 0x7632);
}

// TOKENS: a warp's rows are heads (one row per sequence).
template <int D, bool TOKENS>
__global__ void __launch_bounds__(kRowThreads) page_store_kernel(RowParams p) {
  using C = Chunk<D>;
  constexpr int G = C::kG, kRows = 32 / G;
  pdl_wait();
  const int seq = blockIdx.y, lane = threadIdx.x & 31, at = lane / G, g = lane % G;
  const uint32_t w = blockIdx.x * (kRowThreads / 32) + (threadIdx.x >> 5);
  if (w >= p.warps) return;
  const uint32_t outer = w / static_cast<uint32_t>(p.groups), grp = w - outer * p.groups;
  const int32_t* slots = p.slots + static_cast<int64_t>(seq) * p.rows;
  int head, row;
  if (TOKENS) {
    row = outer;
    head = grp * kRows + at;
  } else {
    head = outer;
    row = kRows * grp - (slots[0] & 3) + at;     // (a negative first slot: any four will do)
  }
  int32_t slot = row >= 0 && row < p.rows && head < p.n_heads ? slots[row] : -1;
  if (slot >= 0 && static_cast<uint32_t>(slot) >= p.n_slots) {
    record_status(p.workspace, MUSTDROP_ERR_BAD_PAGE, seq);
    slot = -1;
  }
  if (__all_sync(~0u, slot < 0)) return;
  uint4 x[2][4];
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
    const uint4* from = reinterpret_cast<const uint4*>(p.src[kv] + seq * p.stride[kv][0] + head * p.stride[kv][1] + row * p.stride[kv][2] + g * 64);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[kv][i] = slot >= 0 ? __ldg(from + i) : make_uint4(0, 0, 0, 0);
  }
  uint8_t* const c = chunk_of<D>(p, max(slot, 0), TOKENS ? min(head, p.n_heads - 1) : head);
  const int r = chunk_row(slot), key = slot & 15;
  uint32_t codes[4], v[4], scale, centre;
  // One token: the lanes of its row exchange words and scales, so that each stores 16 bytes and a sector of L2 is written once
  // (240 sequences, 32 heads: 4.2 us; each its own words: 2 us more).  Many: their rows' words meet in L2 soon, and the exchange costs more.
  quantise(x[0], codes, &scale, &centre);
  if (!TOKENS) {
    if (slot >= 0) {
#pragma unroll
      for (int t = 0; t < 4; ++t) *reinterpret_cast<uint32_t*>(c + C::kK + r * (D / 2) + t * (4 * G) + g * 4) = codes[t];
      uint16_t* const ksz = reinterpret_cast<uint16_t*>(c + C::kKsz) + r * 2 * G + g;
      ksz[0] = static_cast<uint16_t>(scale);
      ksz[G] = static_cast<uint16_t>(centre);
    }
  } else {
    if (G == 4) {
      gather4<1>(codes, g, v);                   // words t = g of the four groups
    } else {
      const uint32_t r0 = __shfl_xor_sync(~0u, g ? codes[0] : codes[2], 1), r1 = __shfl_xor_sync(~0u, g ? codes[1] : codes[3], 1);
      v[0] = g ? r0 : codes[0]; v[1] = g ? codes[2] : r0; v[2] = g ? r1 : codes[1]; v[3] = g ? codes[3] : r1;   // words t = 2 g, 2 g + 1 of both
    }
    const uint32_t own = scale | centre << 16, other = __shfl_xor_sync(~0u, own, 1);
    const uint32_t s2 = __byte_perm(own, other, 0x5410), z2 = __byte_perm(own, other, 0x7632);   // (in even lanes: of groups g, g + 1)
    const uint32_t s4 = __shfl_down_sync(~0u, s2, 2), z4 = __shfl_down_sync(~0u, z2, 2);
    if (slot >= 0) {
      *reinterpret_cast<uint4*>(c + C::kK + r * (D / 2) + g * 16) = make_uint4(v[0], v[1], v[2], v[3]);
      if (g == 0) {
        if (G == 4) *reinterpret_cast<uint4*>(c + C::kKsz + r * 16) = make_uint4(s2, s4, z2, z4);
        else *reinterpret_cast<uint2*>(c + C::kKsz + r * 8) = make_uint2(s2, z2);
      }
    }
  }
  quantise(x[1], codes, &scale, &centre);
  if (!TOKENS) {
    if (slot >= 0) reinterpret_cast<uint16_t*>(c + C::kVs)[r * G + g] = static_cast<uint16_t>(scale);
  } else {
    const uint32_t s2 = __byte_perm(scale, __shfl_xor_sync(~0u, scale, 1), 0x5410), s4 = __shfl_down_sync(~0u, s2, 2);
    if (slot >= 0 && g == 0) {
      if (G == 4) *reinterpret_cast<uint2*>(c + C::kVs + r * 8) = make_uint2(s2, s4);
      else *reinterpret_cast<uint32_t*>(c + C::kVs + r * 4) = s2;
    }
  }
  if (slot >= 0) reinterpret_cast<uint16_t*>(c + C::kVz)[g * 16 + r] = static_cast<uint16_t>(centre);
  // V: byte b of word t is byte (token mod 4) of the word (i = 2 t + b / 2, e = b mod 2) of its group and four tokens
  if (!TOKENS) {
    uint8_t* const words = c + C::kV + ((g >> 1) * 32 + (key >> 2)) * 16 + (g & 1) * 8;
    const int32_t lead = __shfl_sync(~0u, slot, (at & ~3) * G + g);
    const uint32_t fits = __ballot_sync(~0u, slot >= 0 && (lead & 3) == 0 && slot == lead + (at & 3));
    uint32_t of_four = 0;                        // the lanes of this lane's four rows
#pragma unroll
    for (int i = 0; i < 4; ++i) of_four |= 1u << (((at & ~3) + i) * G + g);
    uint32_t word[4];
    gather4<G>(codes, at, v);                    // words t = at mod 4 of the four rows
    bytes4(v, word);
    if ((fits & of_four) == of_four) {
      const int t = at & 3;
      *reinterpret_cast<uint2*>(words + (2 * t) * 64) = make_uint2(word[0], word[1]);
      *reinterpret_cast<uint2*>(words + (2 * t + 1) * 64) = make_uint2(word[2], word[3]);
    } else if (slot >= 0) {
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int b = 0; b < 4; ++b) words[(2 * t + (b >> 1)) * 64 + (b & 1) * 4 + (key & 3)] = static_cast<uint8_t>(codes[t] >> (8 * b));
    }
  } else {
    // one token's bytes: the four of a sector from one instruction (lanes g = 2 h + e; with two groups lanes h, each both e)
    constexpr int kPairs = G / 2;
#pragma unroll
    for (int a = 0; a < kPairs; ++a)
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int h = G == 4 ? g >> 1 : g;
        const uint32_t w = __shfl_sync(~0u, codes[t], at * G + 2 * a + h);
        uint8_t* const to = c + C::kV + ((a * 8 + 2 * t) * 4 + (key >> 2)) * 16 + h * 8 + (key & 3);
        if (slot >= 0) {
          if (G == 4) {
            const uint32_t mine = w >> (8 * (g & 1));
            to[(g & 1) * 4] = static_cast<uint8_t>(mine);
            to[64 + (g & 1) * 4] = static_cast<uint8_t>(mine >> 16);
          } else {
#pragma unroll
            for (int b = 0; b < 4; ++b) to[(b >> 1) * 64 + (b & 1) * 4] = static_cast<uint8_t>(w >> (8 * b));
          }
        }
      }
  }
}

// Eight values z + s (c - 8), rounded to bf16: nibbles j and j + 4 as a bf16 pair 128 + c, less 136, and one fused operation.
__device__ __forceinline__ uint4 values8(uint32_t codes, uint32_t scale, uint32_t centre) {
  const uint32_t s2 = scale | scale << 16, z2 = centre | centre << 16;
  uint32_t v[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    uint32_t y = ((codes >> (4 * j)) & 0x000f000fu) | 0x43004300u;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(y) : "r"(y), "r"(0x43084308u));
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(v[j]) : "r"(y), "r"(s2), "r"(z2));
  }
  return make_uint4(__byte_perm(v[0], v[1], 0x5410), __byte_perm(v[2], v[3], 0x5410), __byte_perm(v[0], v[1], 0x7632), __byte_perm(v[2], v[3], 0x7632));
}

template <int D>
__global__ void __launch_bounds__(kRowThreads) page_load_kernel(RowParams p) {
  constexpr int kLanes = D / 8, kPer = 4 * kLanes / 32;
  using C = Chunk<D>;
  pdl_wait();
  const int seq = blockIdx.y, lane = threadIdx.x & 31;
  const uint32_t w = blockIdx.x * (kRowThreads / 32) + (threadIdx.x >> 5);
  if (w >= p.warps) return;
  const int head = static_cast<int>(w / static_cast<uint32_t>(p.groups)), grp = static_cast<int>(w - static_cast<uint32_t>(head) * p.groups);
  const int c8 = lane % kLanes, sub = lane / kLanes;
  const int g = c8 >> 2, t4 = c8 & 3, a = g >> 1, h = g & 1;
#pragma unroll
  for (int u = 0; u < kPer; ++u) {
    const int row = 4 * grp + sub + u * (32 / kLanes);
    if (row >= p.rows) continue;
    const int32_t slot = p.slots[static_cast<int64_t>(seq) * p.rows + row];
    if (slot < 0) continue;
    if (static_cast<uint32_t>(slot) >= p.n_slots) {
      record_status(p.workspace, MUSTDROP_ERR_BAD_PAGE, seq);
      continue;
    }
    const uint8_t* const c = chunk_of<D>(p, slot, head);
    const int r = chunk_row(slot), key = slot & 15;
    const int64_t at = ((static_cast<int64_t>(seq) * p.n_heads + head) * p.rows + row) * (2 * D) + c8 * 16;
    if (p.dst[0] != nullptr) {
      const uint32_t codes = *reinterpret_cast<const uint32_t*>(c + C::kK + r * (D / 2) + t4 * (4 * C::kG) + g * 4);
      const uint16_t* const ksz = reinterpret_cast<const uint16_t*>(c + C::kKsz) + r * 2 * C::kG + g;
      *reinterpret_cast<uint4*>(p.dst[0] + at) = values8(codes, ksz[0], ksz[C::kG]);
    }
    if (p.dst[1] != nullptr) {
      uint32_t codes = 0;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const uint2 e = *reinterpret_cast<const uint2*>(c + C::kV + (((a * 8 + 2 * t4 + j) * 4 + (key >> 2)) * 4 + h * 2) * 4);
        codes |= ((e.x >> (8 * (key & 3))) & 0xffu) << (16 * j) | ((e.y >> (8 * (key & 3))) & 0xffu) << (16 * j + 8);
      }
      *reinterpret_cast<uint4*>(p.dst[1] + at) =
          values8(codes, reinterpret_cast<const uint16_t*>(c + C::kVs)[r * C::kG + g], reinterpret_cast<const uint16_t*>(c + C::kVz)[g * 16 + r]);
    }
  }
}

mustdrop_status_t done(cudaError_t e) {
  if (e == cudaSuccess) return MUSTDROP_OK;
  set_last_cuda_error(e);
  return MUSTDROP_ERR_CUDA;
}

// Byte strides of [n_seq, n_heads, rows, head_dim] from the configuration's (0: contiguous); false where one is odd.
bool row_strides(const mustdrop_page_config_t* c, int64_t ss, int64_t sh, int64_t sr, int64_t out[3]) {
  if (ss % 8 != 0 || sh % 8 != 0 || sr % 8 != 0) return false;
  out[2] = 2 * (sr != 0 ? sr : c->head_dim);
  out[1] = 2 * (sh != 0 ? sh : static_cast<int64_t>(c->rows) * c->head_dim);
  out[0] = 2 * (ss != 0 ? ss : static_cast<int64_t>(c->n_heads) * c->rows * c->head_dim);
  return true;
}

}  // namespace
}  // namespace mustdrop

extern "C" {

size_t mustdrop_page_pool_bytes(const mustdrop_page_config_t* c) {
  if (mustdrop::check_page_pool(c) != MUSTDROP_OK) return 0;
  return static_cast<size_t>(c->n_pages) * c->n_heads * (c->page / mustdrop::kChunkTokens) * (20 * c->head_dim);
}

size_t mustdrop_page_workspace_bytes(const mustdrop_page_config_t* c) {
  // (a size is only given where the attention would take the query rows: what it writes has to lie in it)
  if ((c != nullptr && c->n_q != 0 ? mustdrop::check_page_queries(c) : mustdrop::check_page_sizes(c)) != MUSTDROP_OK) return 0;
  return mustdrop::kWsStatusBytes + (c->n_q != 0 ? mustdrop::page_attend_partial_bytes(c) : 0);
}

mustdrop_status_t mustdrop_page_tables(const mustdrop_page_config_t* c, const int32_t* add, const int32_t* len,
                                       const int32_t* ring_state, int32_t* len_out, int32_t* ring_state_out, int32_t* ring,
                                       int32_t* page_table, int32_t* slots, void* workspace, void* cuda_stream) {
  using namespace mustdrop;
  const mustdrop_status_t st = check_page_sizes(c);
  if (st != MUSTDROP_OK) return st;
  if (c->rows <= 0 || c->max_pages <= 0) return MUSTDROP_ERR_INVALID_ARG;
  if (static_cast<int64_t>(c->max_pages) * c->page > INT32_MAX || static_cast<int64_t>(c->max_pages) * c->n_seq > INT32_MAX)
    return MUSTDROP_ERR_UNSUPPORTED;
  if (workspace == nullptr) return MUSTDROP_ERR_WORKSPACE;
  const void* ints[] = {add, len, ring_state, len_out, ring_state_out, ring, page_table, slots};
  for (const void* q : ints)
    if (q == nullptr || misaligned(q, 4)) return MUSTDROP_ERR_INVALID_ARG;
  if (misaligned(workspace, 16)) return MUSTDROP_ERR_INVALID_ARG;
  TableParams p;
  p.add = add; p.len = len; p.state = ring_state; p.len_out = len_out; p.state_out = ring_state_out;
  p.ring = ring; p.table = page_table; p.slots = slots; p.workspace = static_cast<int32_t*>(workspace);
  p.n_seq = c->n_seq; p.lg = page_log2(c->page); p.n_pages = c->n_pages; p.max_pages = c->max_pages; p.rows = c->rows;
  // About eight slots a thread: one CTA for the small calls (which then need no ticket), and CTAs that share the rows of long ones.
  p.per_cta = static_cast<int32_t>(std::min<int64_t>(std::min(c->n_seq, kTableSeqs), std::max<int64_t>(1, kTableSlots / c->rows)));
  p.rows_per_cta = std::min(c->rows, kTableSlots);
  dim3 grid(static_cast<unsigned>((c->n_seq + p.per_cta - 1) / p.per_cta), static_cast<unsigned>((static_cast<int64_t>(c->rows) + p.rows_per_cta - 1) / p.rows_per_cta));
  if (grid.y > 65535) return MUSTDROP_ERR_UNSUPPORTED;
  return done(launch_pdl(page_tables_kernel, grid, dim3(kTableThreads), 0, static_cast<cudaStream_t>(cuda_stream), p));
}

mustdrop_status_t mustdrop_page_store(const mustdrop_page_config_t* c, const int32_t* slots, const void* k, const void* v,
                                      void* pool, void* workspace, void* cuda_stream) {
  using namespace mustdrop;
  const mustdrop_status_t st = check_page_pool(c);
  if (st != MUSTDROP_OK) return st;
  if (c->rows <= 0 || slots == nullptr || misaligned(slots, 4)) return MUSTDROP_ERR_INVALID_ARG;
  const void* wide[] = {k, v, pool};
  for (const void* q : wide)
    if (q == nullptr || misaligned(q, 16)) return MUSTDROP_ERR_INVALID_ARG;
  if (misaligned(workspace, 16)) return MUSTDROP_ERR_INVALID_ARG;
  RowParams p = {};
  if (!row_strides(c, c->k_stride_s, c->k_stride_h, c->k_stride_r, p.stride[0]) ||
      !row_strides(c, c->v_stride_s, c->v_stride_h, c->v_stride_r, p.stride[1]))
    return MUSTDROP_ERR_UNSUPPORTED;
  p.slots = slots; p.src[0] = static_cast<const uint8_t*>(k); p.src[1] = static_cast<const uint8_t*>(v);
  p.pool = static_cast<uint8_t*>(pool); p.workspace = static_cast<int32_t*>(workspace);
  p.n_heads = c->n_heads; p.rows = c->rows; p.lg = page_log2(c->page);
  p.n_slots = static_cast<uint32_t>(c->n_pages) << p.lg;
  // A warp's rows are heads where a sequence has one row only and most lanes would have none (32 heads, 240 sequences: 4.2 us against
  // 8.2; two rows: the other way round).
  const int per_warp = 32 / (c->head_dim / kPageGroup);
  const bool tokens = c->rows == 1;
  p.groups = tokens ? (c->n_heads + per_warp - 1) / per_warp
                    : static_cast<int32_t>((static_cast<int64_t>(c->rows) + 3 + per_warp - 1) / per_warp);   // (the first may begin up to three rows before the first)
  const int64_t warps = static_cast<int64_t>(tokens ? c->rows : c->n_heads) * p.groups, blocks = (warps + kRowThreads / 32 - 1) / (kRowThreads / 32);
  if (warps > INT32_MAX) return MUSTDROP_ERR_UNSUPPORTED;
  p.warps = static_cast<uint32_t>(warps);
  const dim3 grid(static_cast<unsigned>(blocks), static_cast<unsigned>(c->n_seq));
  const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  if (c->head_dim == 128)
    return done(tokens ? launch_pdl(page_store_kernel<128, true>, grid, dim3(kRowThreads), 0, stream, p)
                       : launch_pdl(page_store_kernel<128, false>, grid, dim3(kRowThreads), 0, stream, p));
  return done(tokens ? launch_pdl(page_store_kernel<64, true>, grid, dim3(kRowThreads), 0, stream, p)
                     : launch_pdl(page_store_kernel<64, false>, grid, dim3(kRowThreads), 0, stream, p));
}

mustdrop_status_t mustdrop_page_load(const mustdrop_page_config_t* c, const int32_t* slots, const void* pool, void* k_out,
                                     void* v_out, void* workspace, void* cuda_stream) {
  using namespace mustdrop;
  const mustdrop_status_t st = check_page_pool(c);
  if (st != MUSTDROP_OK) return st;
  if (c->rows <= 0 || slots == nullptr || misaligned(slots, 4) || pool == nullptr) return MUSTDROP_ERR_INVALID_ARG;
  const void* wide[] = {pool, k_out, v_out, workspace};
  for (const void* q : wide)
    if (misaligned(q, 16)) return MUSTDROP_ERR_INVALID_ARG;
  if (k_out == nullptr && v_out == nullptr) return MUSTDROP_OK;
  RowParams p = {};
  p.slots = slots; p.dst[0] = static_cast<uint8_t*>(k_out); p.dst[1] = static_cast<uint8_t*>(v_out);
  p.pool = static_cast<uint8_t*>(const_cast<void*>(pool)); p.workspace = static_cast<int32_t*>(workspace);
  p.n_heads = c->n_heads; p.rows = c->rows; p.lg = page_log2(c->page);
  p.n_slots = static_cast<uint32_t>(c->n_pages) << p.lg;
  p.groups = static_cast<int32_t>((static_cast<int64_t>(c->rows) + 3) / 4);
  const int64_t warps = static_cast<int64_t>(c->n_heads) * p.groups, blocks = (warps + kRowThreads / 32 - 1) / (kRowThreads / 32);
  if (warps > INT32_MAX) return MUSTDROP_ERR_UNSUPPORTED;
  p.warps = static_cast<uint32_t>(warps);
  const dim3 grid(static_cast<unsigned>(blocks), static_cast<unsigned>(c->n_seq));
  const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  return done(c->head_dim == 128 ? launch_pdl(page_load_kernel<128>, grid, dim3(kRowThreads), 0, stream, p)
                                 : launch_pdl(page_load_kernel<64>, grid, dim3(kRowThreads), 0, stream, p));
}

}  // extern "C"
