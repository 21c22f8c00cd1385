// Decoding-stage cache in pages of 4-bit values: places for tokens (page tables, slots), rows in, rows out.
// The formats and the arithmetic of the values are described in mustdrop.h; the attention that reads
// the pages is in page_attend.cu.
#include <algorithm>

#include "page_internal.h"

namespace mustdrop {

mustdrop_status_t check_page_sizes(const mustdrop_page_config_t* c) {
  if (c == nullptr || c->n_seq <= 0 || c->n_pages <= 0 || c->flags != 0) return MUSTDROP_ERR_INVALID_ARG;
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

namespace {

// ---------------------------------------------------------------------------------------- page tables
//
// A pure function of the lengths: with need[s] = pages sequence s asks for, back[s] = pages it gives back, P the
// sums over the sequences before it, its i-th new page is ring[head + P_need + i] and its i-th returned page goes to
// ring[head + count + P_back + i].  The ring's two ends never meet (count + all of back <= n_pages), so no CTA
// waits for another: each sums need and back over the sequences before its own (two loads per sequence, from
// L2), handles its own ones, and the CTA that finishes last writes what the others still read - the ring's state and, as
// they may be updated in place, the lengths.  Bound: launch and three dependent trips to L2 for small calls,
// the slots written for large ones.
struct TableParams {
  const int32_t *add, *len, *state;
  int32_t *len_out, *state_out, *ring, *table, *slots;
  int32_t* workspace;
  int32_t n_seq, lg, n_pages, max_pages, rows, per_cta, rows_per_cta;
};

constexpr int kTableThreads = 512;
constexpr int kTableSeqs = 1024;     // most sequences of a CTA

struct Move {       // what the call does to one sequence
  int32_t cur, grow, need, back;   // grow: tokens gained (0 where it shrinks or is refused for its length)
  bool bad;
};

__device__ __forceinline__ Move move_of(const TableParams& p, int s) {
  Move m;
  m.cur = p.len[s];
  const int32_t a = p.add[s];
  const int64_t most = static_cast<int64_t>(p.max_pages) << p.lg;
  const int32_t mask = (1 << p.lg) - 1;
  m.grow = m.need = m.back = 0;
  m.bad = m.cur < 0 || m.cur > most || a > p.rows || m.cur + static_cast<int64_t>(a) > most;
  if (m.bad) return m;
  const int32_t had = static_cast<int32_t>((static_cast<int64_t>(m.cur) + mask) >> p.lg);
  if (a >= 0) {
    m.grow = a;
    m.need = static_cast<int32_t>((static_cast<int64_t>(m.cur) + a + mask) >> p.lg) - had;
  } else {
    const int64_t left = max(static_cast<int64_t>(m.cur) + a, static_cast<int64_t>(0));
    m.back = had - static_cast<int32_t>((left + mask) >> p.lg);
  }
  return m;
}

// Inclusive sums of (x, y) over the CTA's threads; `total` receives the sums over all.  Ends with a barrier passed.
__device__ __forceinline__ longlong2 scan_pair(longlong2 v, longlong2* warp_sums, longlong2* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const long long x = __shfl_up_sync(~0u, v.x, d), y = __shfl_up_sync(~0u, v.y, d);
    if (lane >= d) { v.x += x; v.y += y; }
  }
  __syncthreads();
  if (lane == 31) warp_sums[warp] = v;
  __syncthreads();
  longlong2 all = {0, 0};
#pragma unroll
  for (int w = 0; w < kTableThreads / 32; ++w) {
    const longlong2 t = warp_sums[w];
    if (w < warp) { v.x += t.x; v.y += t.y; }
    all.x += t.x; all.y += t.y;
  }
  *total = all;
  return v;
}

__global__ void __launch_bounds__(kTableThreads) page_tables_kernel(TableParams p) {
  __shared__ longlong2 warp_sums[kTableThreads / 32];
  __shared__ int32_t cur_s[kTableSeqs], grow_s[kTableSeqs], first_s[kTableSeqs];   // first_s: ring offset of the first new page
  __shared__ int32_t back_s[kTableSeqs], back_at_s[kTableSeqs];                    // pages given back, and their place behind the ring's count
  __shared__ int last_s;
  pdl_launch_dependents();
  pdl_wait();
  const int first = blockIdx.x * p.per_cta, n_own = min(p.per_cta, p.n_seq - first);
  int32_t head = p.state[0], count = p.state[1];
  const bool bad_state = head < 0 || head >= p.n_pages || count < 0 || count > p.n_pages;
  if (bad_state) head = count = 0;   // nothing is free, nothing can be given back
  longlong2 before = {0, 0}, total;
  for (int s = threadIdx.x; s < first; s += kTableThreads) {
    const Move m = move_of(p, s);
    before.x += m.need; before.y += m.back;
  }
  if (first > 0) {
    (void)scan_pair(before, warp_sums, &total);
    before = total;
  }
  const bool lead = blockIdx.y == 0;   // of the CTAs that share a range of sequences, the one that reports
  for (int base = 0; base < n_own; base += kTableThreads) {
    const int i = base + threadIdx.x, s = first + i;
    Move m = {0, 0, 0, 0, false};
    if (i < n_own) m = move_of(p, s);
    longlong2 upto = scan_pair({m.need, m.back}, warp_sums, &total);
    upto.x += before.x; upto.y += before.y;
    before.x += total.x; before.y += total.y;
    if (i < n_own) {
      const bool granted = m.need == 0 || upto.x <= count;
      cur_s[i] = m.cur;
      grow_s[i] = granted ? m.grow : 0;
      first_s[i] = granted && m.need > 0 ? static_cast<int32_t>(upto.x - m.need) : 0;
      if (lead && m.bad) record_status(p.workspace, MUSTDROP_ERR_BAD_LENGTH, s);
      if (lead && !granted) record_status(p.workspace, MUSTDROP_ERR_NO_PAGES, s);
      // what does not fit behind the ring's count was never the pool's
      const long long room = bad_state ? 0 : max(static_cast<long long>(p.n_pages) - count - (upto.y - m.back), 0ll);
      if (lead && m.back > room) record_status(p.workspace, MUSTDROP_ERR_BAD_LENGTH, s);
      back_s[i] = static_cast<int32_t>(min(static_cast<long long>(m.back), room));
      back_at_s[i] = static_cast<int32_t>(back_s[i] > 0 ? count + (upto.y - m.back) : 0);
    }
  }
  __syncthreads();
  // pages given back: a warp per sequence
  for (int i = threadIdx.x >> 5; lead && i < n_own; i += kTableThreads / 32) {
    const int n = back_s[i];
    if (n == 0) continue;
    const Move m = move_of(p, first + i);
    const int32_t had = static_cast<int32_t>((static_cast<int64_t>(m.cur) + (1 << p.lg) - 1) >> p.lg);
    const int32_t* from = p.table + static_cast<size_t>(first + i) * p.max_pages + (had - m.back);
    for (int b = threadIdx.x & 31; b < n; b += 32) {
      const int32_t id = from[b];
      if (static_cast<uint32_t>(id) >= static_cast<uint32_t>(p.n_pages)) record_status(p.workspace, MUSTDROP_ERR_BAD_PAGE, first + i);
      p.ring[(static_cast<int64_t>(head) + back_at_s[i] + b) % p.n_pages] = id;
    }
  }
  // slots, and the table entries of the pages that begin among the new tokens
  const int t0 = blockIdx.y * p.rows_per_cta, n_t = min(p.rows_per_cta, p.rows - t0);
  const int32_t mask = (1 << p.lg) - 1;
  const int64_t items = static_cast<int64_t>(n_own) * n_t;
  int i = threadIdx.x / n_t, t = threadIdx.x % n_t;
  const int di = kTableThreads / n_t, dt = kTableThreads % n_t;
  for (int64_t it = threadIdx.x; it < items; it += kTableThreads) {
    const int32_t r = t0 + t;
    int32_t slot = -1;
    if (r < grow_s[i]) {
      int32_t* row = p.table + static_cast<size_t>(first + i) * p.max_pages;
      const int32_t cur = cur_s[i], pos = cur + r, e = pos >> p.lg;
      const int32_t had = static_cast<int32_t>((static_cast<uint32_t>(cur) + mask) >> p.lg);
      const int32_t id = e < had ? row[e] : p.ring[(static_cast<int64_t>(head) + first_s[i] + (e - had)) % p.n_pages];
      if (e >= had && (pos & mask) == 0) row[e] = id;
      if (static_cast<uint32_t>(id) < static_cast<uint32_t>(p.n_pages)) slot = (id << p.lg) | (pos & mask);
      else record_status(p.workspace, MUSTDROP_ERR_BAD_PAGE, first + i);
    }
    p.slots[static_cast<size_t>(first + i) * p.rows + r] = slot;
    i += di; t += dt;
    if (t >= n_t) { t -= n_t; ++i; }
  }
  // the CTA that finishes last: everybody has read what it now overwrites
  __syncthreads();
  if (threadIdx.x == 0) {
    __threadfence();
    const unsigned all = gridDim.x * gridDim.y;
    last_s = all == 1 || atomicInc(reinterpret_cast<unsigned*>(p.workspace) + kTicketWord, all - 1) == all - 1;
    __threadfence();
  }
  __syncthreads();
  if (!last_s) return;
  longlong2 sum = {0, 0};
  long long taken = 0;
  for (int base = 0; base < p.n_seq; base += kTableThreads) {
    const int s = base + threadIdx.x;
    Move m = {0, 0, 0, 0, false};
    int32_t a = 0;
    if (s < p.n_seq) {
      m = move_of(p, s);
      a = p.add[s];
    }
    longlong2 upto = scan_pair({m.need, m.back}, warp_sums, &total);
    upto.x += sum.x;
    sum.x += total.x; sum.y += total.y;
    if (s < p.n_seq) {
      const bool granted = m.need == 0 || upto.x <= count;
      if (granted && m.need > 0) taken = max(taken, upto.x);
      p.len_out[s] = m.bad ? m.cur : a < 0 ? max(m.cur + a, 0) : granted ? m.cur + m.grow : m.cur;
    }
  }
  // the granted needs are those up to the largest sum that fits
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) taken = max(taken, __shfl_xor_sync(~0u, taken, d));
  __syncthreads();
  if ((threadIdx.x & 31) == 0) warp_sums[threadIdx.x >> 5].x = taken;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 0; w < kTableThreads / 32; ++w) taken = max(taken, warp_sums[w].x);
    if (bad_state) {
      record_status(p.workspace, MUSTDROP_ERR_BAD_LENGTH, -1);
      p.state_out[0] = p.state[0];
      p.state_out[1] = p.state[1];
    } else {
      const long long back = min(sum.y, static_cast<long long>(p.n_pages) - count);
      p.state_out[0] = static_cast<int32_t>((head + taken) % p.n_pages);
      p.state_out[1] = static_cast<int32_t>(count - taken + back);
    }
  }
}

// ---------------------------------------------------------------------------------------- rows in, rows out
//
// A warp takes four rows of one head: 16 lanes hold a row of 128 channels (8 of 64) as 16-byte vectors, a lane two
// rows (four).  A lane's eight channels are one word of the K codes; for V a word holds four tokens, so the lanes of
// the four rows exchange their bytes and store whole words where the four slots are neighbours in one word, else single bytes.
// Rows are grouped so that they are: groups of four end where slot mod 4 is 3, judged by the sequence's first slot.  Bound: bytes
// (2 rows of bf16 in, a third as much out, and the reverse).
constexpr int kRowThreads = 256;

struct RowParams {
  const int32_t* slots;
  const uint8_t* src[2];   // store: k, v
  uint8_t* dst[2];         // load: k_out, v_out
  uint8_t* pool;
  int32_t* workspace;
  int32_t n_heads, rows, groups, lg;
  uint32_t n_slots;        // n_pages * page
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
  uint16_t h;
  asm("cvt.rn.bf16.f32 %0, %1;" : "=h"(h) : "f"(x));
  return h;
}

// Codes of eight channels as nibbles 0..7 of a word; scale and centre (bf16 bits) of the group of four lanes.
__device__ __forceinline__ uint32_t quantise8(const uint4& v, uint32_t* scale, uint32_t* centre) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  float x[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) { x[2 * i] = bf16_lo(w[i]); x[2 * i + 1] = bf16_hi(w[i]); }
  float lo = x[0], hi = x[0];
  bool finite = true;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    lo = fminf(lo, x[i]); hi = fmaxf(hi, x[i]);
    finite = finite && (__float_as_uint(x[i]) & 0x7f800000u) != 0x7f800000u;
  }
#pragma unroll
  for (int d = 1; d < 4; d <<= 1) {
    lo = fminf(lo, __shfl_xor_sync(~0u, lo, d));
    hi = fmaxf(hi, __shfl_xor_sync(~0u, hi, d));
    finite = __shfl_xor_sync(~0u, static_cast<int>(finite), d) != 0 && finite;
  }
  *scale = to_bf16(__fdiv_rn(__fsub_rn(0.5f * hi, 0.5f * lo), 7.5f));   // (halves: the difference of two finite numbers may not be one)
  const float s = __uint_as_float(*scale << 16);
  *centre = to_bf16(__fmaf_rn(8.0f, s, lo));
  const float z = __uint_as_float(*centre << 16);
  uint32_t codes = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float c = s > 0.0f ? rintf(__fdiv_rn(__fsub_rn(x[i], z), s)) + 8.0f : 8.0f;
    codes |= static_cast<uint32_t>(fminf(fmaxf(c, 0.0f), 15.0f)) << (4 * i);
  }
  if (!finite) { *scale = 0x7fc0u; *centre = 0; codes = 0; }   // (the centre stays finite: the attention multiplies it by zero for hidden keys)
  return codes;
}

template <int D>
__global__ void __launch_bounds__(kRowThreads) page_store_kernel(RowParams p) {
  constexpr int kLanes = D / 8;              // lanes of a row
  constexpr int kPer = 4 * kLanes / 32;      // rows of a lane: 2, or 1 with 64 channels
  using C = Chunk<D>;
  pdl_launch_dependents();
  pdl_wait();
  const int seq = blockIdx.y, lane = threadIdx.x & 31;
  const int64_t w = static_cast<int64_t>(blockIdx.x) * (kRowThreads / 32) + (threadIdx.x >> 5);
  if (w >= static_cast<int64_t>(p.n_heads) * p.groups) return;
  const int head = static_cast<int>(w / p.groups), grp = static_cast<int>(w % p.groups);
  const int32_t* slots = p.slots + static_cast<int64_t>(seq) * p.rows;
  const int32_t slot0 = slots[0];
  const int row0 = 4 * grp - (slot0 & 3);    // (negative slots: any grouping will do)
  int32_t slot[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = row0 + i;
    slot[i] = r >= 0 && r < p.rows ? slots[r] : -1;
    if (slot[i] >= 0 && static_cast<uint32_t>(slot[i]) >= p.n_slots) {
      if (lane == 0) record_status(p.workspace, MUSTDROP_ERR_BAD_PAGE, seq);
      slot[i] = -1;
    }
  }
  if ((slot[0] & slot[1] & slot[2] & slot[3]) < 0 && slot[0] < 0 && slot[1] < 0 && slot[2] < 0 && slot[3] < 0) return;
  const int c8 = lane % kLanes, sub = lane / kLanes;   // channels 8 c8 .. + 7; rows sub, sub + 32 / kLanes, ..
  const int g = c8 >> 2, t4 = c8 & 3;
  uint4 x[2][kPer];
#pragma unroll
  for (int u = 0; u < kPer; ++u) {
    const int i = sub + u * (32 / kLanes);
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      x[kv][u] = make_uint4(0, 0, 0, 0);
      if (slot[i] >= 0)
        x[kv][u] = __ldg(reinterpret_cast<const uint4*>(p.src[kv] + seq * p.stride[kv][0] + head * p.stride[kv][1] +
                                                        (row0 + i) * p.stride[kv][2] + c8 * 16));
    }
  }
  uint32_t vcodes[kPer];
#pragma unroll
  for (int u = 0; u < kPer; ++u) {
    const int i = sub + u * (32 / kLanes);
    uint32_t s, z, vs, vz;
    const uint32_t kcodes = quantise8(x[0][u], &s, &z);
    vcodes[u] = quantise8(x[1][u], &vs, &vz);
    if (slot[i] >= 0) {
      uint8_t* const c = chunk_of<D>(p, slot[i], head);
      const int r = chunk_row(slot[i]);
      *reinterpret_cast<uint32_t*>(c + C::kK + r * (D / 2) + t4 * (4 * C::kG) + g * 4) = kcodes;
      if (t4 == 0) {
        uint16_t* const ksz = reinterpret_cast<uint16_t*>(c + C::kKsz) + r * 2 * C::kG + g;
        ksz[0] = static_cast<uint16_t>(s);
        ksz[C::kG] = static_cast<uint16_t>(z);
        reinterpret_cast<uint16_t*>(c + C::kVs)[r * C::kG + g] = static_cast<uint16_t>(vs);
        reinterpret_cast<uint16_t*>(c + C::kVz)[g * 16 + r] = static_cast<uint16_t>(vz);
      }
    }
  }
  // V: the four bytes of a lane's codes belong to the words (i = 2 (c8 mod 4) + b / 2, e = b mod 2), b = 0..3, of its group
  const bool whole = slot[0] >= 0 && (slot[0] & 3) == 0 && slot[1] == slot[0] + 1 && slot[2] == slot[0] + 2 && slot[3] == slot[0] + 3;
  uint32_t row_codes[4];                                 // of all four rows, for this lane's channels
#pragma unroll
  for (int i = 0; i < 4; ++i)
    row_codes[i] = __shfl_sync(~0u, vcodes[i / (32 / kLanes)], (i % (32 / kLanes)) * kLanes + c8);
  const int a = g >> 1, h = g & 1;
  auto word_at = [&](uint8_t* c, int r8, int t, int e) { return c + C::kV + (((a * 8 + r8) * 4 + t) * 4 + h * 2 + e) * 4; };
  if (whole) {
    uint8_t* const c = chunk_of<D>(p, slot[0], head);
    const int t = (slot[0] & 15) >> 2;
    for (int j = sub; j < 2; j += 32 / kLanes) {         // the rows of the word table this lane writes: 2 (c8 mod 4) + j
      uint32_t e0 = 0, e1 = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        e0 |= ((row_codes[i] >> (16 * j)) & 0xffu) << (8 * i);
        e1 |= ((row_codes[i] >> (16 * j + 8)) & 0xffu) << (8 * i);
      }
      *reinterpret_cast<uint2*>(word_at(c, 2 * t4 + j, t, 0)) = make_uint2(e0, e1);
    }
  } else {
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
      const int i = sub + u * (32 / kLanes);
      if (slot[i] >= 0) {
        uint8_t* const c = chunk_of<D>(p, slot[i], head);
        const int key = slot[i] & 15;
#pragma unroll
        for (int b = 0; b < 4; ++b) word_at(c, 2 * t4 + (b >> 1), key >> 2, b & 1)[key & 3] = static_cast<uint8_t>(vcodes[u] >> (8 * b));
      }
    }
  }
}

// Eight values z + s (c - 8), rounded to bf16.
__device__ __forceinline__ uint4 values8(uint32_t codes, uint32_t scale, uint32_t centre) {
  const float s = __uint_as_float(scale << 16), z = __uint_as_float(centre << 16);
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float lo = __fmaf_rn(s, static_cast<float>(static_cast<int>((codes >> (8 * i)) & 15u) - 8), z);
    const float hi = __fmaf_rn(s, static_cast<float>(static_cast<int>((codes >> (8 * i + 4)) & 15u) - 8), z);
    w[i] = to_bf16(lo) | (to_bf16(hi) << 16);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

template <int D>
__global__ void __launch_bounds__(kRowThreads) page_load_kernel(RowParams p) {
  constexpr int kLanes = D / 8, kPer = 4 * kLanes / 32;
  using C = Chunk<D>;
  pdl_launch_dependents();
  pdl_wait();
  const int seq = blockIdx.y, lane = threadIdx.x & 31;
  const int64_t w = static_cast<int64_t>(blockIdx.x) * (kRowThreads / 32) + (threadIdx.x >> 5);
  if (w >= static_cast<int64_t>(p.n_heads) * p.groups) return;
  const int head = static_cast<int>(w / p.groups), grp = static_cast<int>(w % p.groups);
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
  if (mustdrop::check_page_sizes(c) != MUSTDROP_OK) return 0;
  return mustdrop::kWsStatusBytes + (c->n_q > 0 ? mustdrop::page_attend_partial_bytes(c) : 0);
}

mustdrop_status_t mustdrop_page_tables(const mustdrop_page_config_t* c, const int32_t* add, const int32_t* len,
                                       const int32_t* ring_state, int32_t* len_out, int32_t* ring_state_out, int32_t* ring,
                                       int32_t* page_table, int32_t* slots, void* workspace, void* cuda_stream) {
  using namespace mustdrop;
  const mustdrop_status_t st = check_page_sizes(c);
  if (st != MUSTDROP_OK) return st;
  if (c->rows <= 0 || c->max_pages <= 0) return MUSTDROP_ERR_INVALID_ARG;
  if (static_cast<int64_t>(c->max_pages) * c->page > INT32_MAX) return MUSTDROP_ERR_UNSUPPORTED;
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
  constexpr int kItems = 8 * kTableThreads;
  p.per_cta = static_cast<int32_t>(std::min<int64_t>(std::min(c->n_seq, kTableSeqs), std::max<int64_t>(1, kItems / c->rows)));
  p.rows_per_cta = std::min(c->rows, kItems);
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
  p.groups = static_cast<int32_t>((static_cast<int64_t>(c->rows) + 3 + 3) / 4);   // (the first group may begin up to three rows before the first)
  const int64_t blocks = (static_cast<int64_t>(c->n_heads) * p.groups + kRowThreads / 32 - 1) / (kRowThreads / 32);
  if (blocks > INT32_MAX) return MUSTDROP_ERR_UNSUPPORTED;
  const dim3 grid(static_cast<unsigned>(blocks), static_cast<unsigned>(c->n_seq));
  const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  return done(c->head_dim == 128 ? launch_pdl(page_store_kernel<128>, grid, dim3(kRowThreads), 0, stream, p)
                                 : launch_pdl(page_store_kernel<64>, grid, dim3(kRowThreads), 0, stream, p));
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
  const int64_t blocks = (static_cast<int64_t>(c->n_heads) * p.groups + kRowThreads / 32 - 1) / (kRowThreads / 32);
  if (blocks > INT32_MAX) return MUSTDROP_ERR_UNSUPPORTED;
  const dim3 grid(static_cast<unsigned>(blocks), static_cast<unsigned>(c->n_seq));
  const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  return done(c->head_dim == 128 ? launch_pdl(page_load_kernel<128>, grid, dim3(kRowThreads), 0, stream, p)
                                 : launch_pdl(page_load_kernel<64>, grid, dim3(kRowThreads), 0, stream, p));
}

}  // extern "C"
