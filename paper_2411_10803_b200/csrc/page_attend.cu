// Attention of the decoded tokens over a cache in pages of 4-bit values (mustdrop_page_attend).
//
//   S[x][q] = scale <K_x, q>,  P = exp(S - m),  out[q] = sum_x P V_x / sum_x P,   K = z + s (c - 8) per group of 32 channels
//
// With C the codes minus 8 (exact in fp16) and Q the query scaled by a power of two into fp16's range (exact):
//   <K_x, q> = sum_g s_xg (sum_{d in g} C_xd Q_d)  +  sum_g z_xg (sum_{d in g} Q_d)
//   out_d    = sum_x (P_x s_xg) C_xd               +  sum_x P_x z_xg
// so the codes go into the matrix instructions as they are, with 16 tokens (K) or 16 channels (V) as the rows and
// the query rows - the query tokens and heads that share a K / V head - as the 8 columns: scales meet fp32 accumulators
// (K) or the probabilities (V), centres are one more instruction each (bf16, the sums over Q in three bf16 terms).
// P s is rounded once, to fp16: 11 bits; a running power of two keeps it in range whatever the scales are.
//
// Bound: HBM.  A token and head is 1.25 D bytes where bf16 has 4 D, and unpacking must keep up with ~23 bytes per
// clock and SM: 9 instructions per 8 codes.  Every warp walks its own range of chunks (16 tokens of one head,
// 20 D contiguous bytes: one bulk copy each) through its own ring in shared memory, without a barrier between warps.  The chunks of
// all (sequence, head, row tile) units form one line that is cut into equal parts, one per warp, whatever
// the lengths are: no host has to know them.  A unit that several warps share is joined by a second kernel from
// partial results (fp32), in the order of the warps: the same call gives the same bits.
#include <algorithm>

#include "page_internal.h"

namespace mustdrop {
namespace {

constexpr int kWarps = 8;             // per CTA
constexpr int kThreads = 32 * kWarps;
constexpr int kMaxSeqs = 4096;
constexpr int kMaxCtas = 320;         // 2 per SM, and some to spare
constexpr int kMinChunks = 2;         // least chunks per warp where there are enough warps: a shorter range is all set-up
constexpr long long kWaitCycles = 200000000ll;   // ~0.1 s: a bulk copy that takes longer will not come

struct AttendParams {
  const uint8_t* q;         // bf16
  const uint8_t* pool;
  const int32_t *table, *len;
  uint16_t* out;
  float* part;              // partial results: [2 * warps][rows][D + 2]
  int32_t* workspace;
  int32_t n_seq, n_heads, group, n_q, rows, tiles;   // rows = n_q * group query rows per unit, in `tiles` row tiles
  int32_t lg, n_pages, max_pages, causal, part_rows;
  int64_t q_ss, q_st, q_sh;   // bytes
  float scale_log2e;
};

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ void mbar_init(uint32_t bar) { asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bar) : "memory"); }
__device__ __forceinline__ bool mbar_try_wait(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.acquire.cta.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity) {   // bounded
  if (mbar_try_wait(bar, parity)) return true;
  const long long t0 = clock64();
  while (!mbar_try_wait(bar, parity))
    if (clock64() - t0 > kWaitCycles) return false;
  return true;
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
  asm volatile("cp.async.bulk.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
               "l"(src), "r"(bytes), "r"(bar)
               : "memory");
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t w;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
  return w;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t w;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
  return w;
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t a) {
  uint32_t d;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
  return d;
}
__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_bf16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Nibbles j and j + 4 of a word as fp16 pairs of codes - 8, for j = 0..3.  A nibble under the bits of 1024 reads 1024 + c
// (bits 0..3) or 1024 + 16 c (bits 4..7); both lose their offset in one exact operation.
__device__ __forceinline__ void unpack8(uint32_t w, uint32_t (&x)[4]) {
  const uint32_t w8 = w >> 8;
  uint32_t y[4];
  asm("lop3.b32 %0, %1, 0x000f000f, 0x64006400, 0xea;" : "=r"(y[0]) : "r"(w));
  asm("lop3.b32 %0, %1, 0x00f000f0, 0x64006400, 0xea;" : "=r"(y[1]) : "r"(w));
  asm("lop3.b32 %0, %1, 0x000f000f, 0x64006400, 0xea;" : "=r"(y[2]) : "r"(w8));
  asm("lop3.b32 %0, %1, 0x00f000f0, 0x64006400, 0xea;" : "=r"(y[3]) : "r"(w8));
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(x[0]) : "r"(y[0]), "r"(0x64086408u));                              // 1032
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(x[1]) : "r"(y[1]), "r"(0x2c002c00u), "r"(0xd480d480u));         // 1/16, -72
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(x[2]) : "r"(y[2]), "r"(0x64086408u));
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(x[3]) : "r"(y[3]), "r"(0x2c002c00u), "r"(0xd480d480u));
}

// The line of chunks: sequence s has heads * tiles units of chunks(s) chunks each.
__device__ __forceinline__ int32_t clamp_len(const AttendParams& p, int s) {
  const int64_t most = static_cast<int64_t>(p.max_pages) << p.lg;
  const int32_t n = p.len[s];
  return n < 0 ? 0 : n > most ? static_cast<int32_t>(most) : n;
}
__device__ __forceinline__ int32_t chunks_of(int32_t len) { return static_cast<int32_t>((static_cast<uint32_t>(len) + kChunkTokens - 1) / kChunkTokens); }

// Equal parts of the line.  With few chunks fewer warps take part, the same number of every CTA.
struct Cut {
  long long total;    // chunks
  int warps;          // that take part, per_cta of each CTA
  int per_cta;
  __device__ __forceinline__ long long begin(int w) const { return total * w / warps; }
  // the warp that has chunk x
  __device__ __forceinline__ int owner(long long x) const { return static_cast<int>(((x + 1) * warps - 1) / total); }
};
__device__ __forceinline__ Cut cut_of(long long total, int ctas) {
  Cut c;
  c.total = total;
  const long long want = (total + kMinChunks - 1) / kMinChunks;
  const long long per = (want + ctas - 1) / ctas;
  c.per_cta = per > kWarps ? kWarps : per < 1 ? 1 : static_cast<int>(per);
  c.warps = static_cast<int>(total < static_cast<long long>(c.per_cta) * ctas ? total : static_cast<long long>(c.per_cta) * ctas);
  return c;
}

// A place on the line.
struct Place {
  int32_t seq, head, tile, chunk, n;   // chunk of n
};
__device__ __forceinline__ void step(const AttendParams& p, Place& x, const int32_t* first) {   // first[s]: chunks (per unit) of the sequences before s
  if (++x.chunk < x.n) return;
  x.chunk = 0;
  if (++x.tile < p.tiles) return;
  x.tile = 0;
  if (++x.head < p.n_heads) return;
  x.head = 0;
  do {
    ++x.seq;
    x.n = x.seq < p.n_seq ? first[x.seq + 1] - first[x.seq] : 1;
  } while (x.n == 0);
}

template <int D, int NT>
struct Shape {
  static constexpr int kG = D / 32, kTiles = D / 16, kRows = 8 * NT;
  // chunks in flight per warp: ~100 KB of ring in each of two CTAs per SM
  static constexpr int kStages = D == 128 ? 5 : 8;
  static constexpr size_t ring = static_cast<size_t>(kWarps) * kStages * Chunk<D>::kBytes;
};

template <int D, int NT>
__global__ void __launch_bounds__(kThreads, NT == 1 ? 2 : 1) page_attend_kernel(const AttendParams p) {
  using S = Shape<D, NT>;
  using C = Chunk<D>;
  constexpr int G = S::kG, kStages = S::kStages;
  extern __shared__ __align__(128) uint8_t ring_all[];
  __shared__ __align__(8) uint64_t bars[kWarps][kStages];
  __shared__ int32_t warp_sum[kWarps];
  int32_t* const first = reinterpret_cast<int32_t*>(ring_all + S::ring);   // [n_seq + 1]
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int r = lane >> 2, t = lane & 3;
  const uint32_t bar0 = smem_u32(&bars[warp][0]);
  const uint8_t* const ring = ring_all + static_cast<size_t>(warp) * kStages * C::kBytes;
  const uint32_t ring0 = smem_u32(ring);
  if (lane == 0) {
    for (int i = 0; i < kStages; ++i) mbar_init(bar0 + 8 * i);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async;" ::: "memory");
  }
  pdl_launch_dependents();
  pdl_wait();

  // chunks (per unit) of the sequences before each one: 32 bits, as the host refuses more; the line has 64
  int32_t carry = 0;
  for (int base = 0; base < p.n_seq; base += kThreads) {
    const int s = base + threadIdx.x;
    int32_t v = s < p.n_seq ? chunks_of(clamp_len(p, s)) : 0;
    if (s < p.n_seq && blockIdx.x == 0 && clamp_len(p, s) != p.len[s]) record_status(p.workspace, MUSTDROP_ERR_BAD_LENGTH, s);
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int32_t u = __shfl_up_sync(~0u, v, d);
      if (lane >= d) v += u;
    }
    __syncthreads();
    if (lane == 31) warp_sum[warp] = v;
    __syncthreads();
    int32_t all = 0;
    for (int w = 0; w < kWarps; ++w) {
      const int32_t u = warp_sum[w];
      if (w < warp) v += u;
      all += u;
    }
    if (s < p.n_seq) first[s + 1] = carry + v;
    carry += all;
  }
  if (threadIdx.x == 0) first[0] = 0;
  __syncthreads();
  const int units_per_seq = p.n_heads * p.tiles;
  const Cut cut = cut_of(static_cast<long long>(carry) * units_per_seq, gridDim.x);
  if (cut.total == 0 || warp >= cut.per_cta) return;
  const int lw = blockIdx.x * cut.per_cta + warp;
  if (lw >= cut.warps) return;
  const long long begin = cut.begin(lw), end = cut.begin(lw + 1);

  Place at;       // where the warp computes
  {
    int lo = 0, hi = p.n_seq - 1;          // the sequence with first[s] * units <= begin < first[s + 1] * units
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (static_cast<long long>(first[mid + 1]) * units_per_seq <= begin) lo = mid + 1; else hi = mid;
    }
    const long long rem = begin - static_cast<long long>(first[lo]) * units_per_seq;
    at.seq = lo;
    at.n = first[lo + 1] - first[lo];
    const int unit = static_cast<int>(rem / at.n);
    at.chunk = static_cast<int>(rem % at.n);
    at.head = unit / p.tiles;
    at.tile = unit % p.tiles;
  }
  const int per_page = p.lg - 4;           // log2 of the chunks per page
  const uint32_t in_page = (1u << per_page) - 1;

  // Copies run kStages chunks ahead of the computation, page ids one chunk further.
  Place ahead = at;
  long long asked = begin;                 // chunks whose page id has been loaded
  int32_t next_id = 0, next_off = 0;
  uint32_t bad = 0;                        // stages whose chunk lies on no page of the pool
  auto ask = [&]() {
    if (asked < end) {
      next_id = __ldg(p.table + static_cast<int64_t>(ahead.seq) * p.max_pages + (ahead.chunk >> per_page));
      next_off = (ahead.head << per_page) + (ahead.chunk & in_page);
      step(p, ahead, first);
    }
    ++asked;
  };
  auto issue = [&](int stage) {
    const bool fine = static_cast<uint32_t>(next_id) < static_cast<uint32_t>(p.n_pages);
    bad = (bad & ~(1u << stage)) | (fine ? 0u : 1u << stage);
    if (lane == 0) {
      if (fine)
        bulk_load(ring0 + stage * C::kBytes, p.pool + (((static_cast<int64_t>(next_id) * p.n_heads) << per_page) + next_off) * C::kBytes,
                  C::kBytes, bar0 + 8 * stage);
      else
        record_status(p.workspace, MUSTDROP_ERR_BAD_PAGE, next_id);
    }
  };
  ask();
  long long issued = begin;
  for (int i = 0; i < kStages && issued < end; ++i, ++issued) {
    issue(i);
    ask();
  }

  uint32_t qf[NT][G][4];                   // Q as the second operand: [g][2 m + {0, 1}]
  uint32_t qz[NT][2];                      // its sums over groups, three bf16 terms
  float cs[NT][2];                         // log2 units per unit of the scaled product, of columns 2t, 2t + 1
  float o[NT][S::kTiles][4], oz[NT][4];    // out (without centres) and the centres' part, rows r, r + 8 and columns 2t, 2t + 1
  float l[NT][2], m[NT][2], thr[NT][2];    // sum (of this lane's tokens), stabiliser, rise of a logit that moves it
  float vs_mul = 1.0f;                     // 2^-E: scales of V in units of 2^E
  bool vs_set = false;
  int32_t lim[NT][2];                      // visible keys of columns 2t, 2t + 1
  int32_t least = 0, len = 0;              // fewest of any column; the sequence's length
  int32_t seg_first = at.chunk;            // first chunk of the segment in hand
  bool fresh = true;

  int stage = 0;
  uint32_t phase = 0;
  bool ok = true;
  for (long long x = begin; x < end; ++x) {
    if (fresh) {
      // ------------------------------------------------------------ a unit begins: its queries
      fresh = false;
      seg_first = at.chunk;
      len = clamp_len(p, at.seq);
      least = len;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const int row = at.tile * S::kRows + nt * 8 + r;
        uint4 w[G];
#pragma unroll
        for (int g = 0; g < G; ++g) w[g] = make_uint4(0, 0, 0, 0);
        if (row < p.rows) {
          const uint8_t* src = p.q + at.seq * p.q_ss + (row / p.group) * p.q_st +
                               (static_cast<int64_t>(at.head) * p.group + row % p.group) * p.q_sh + t * 16;
#pragma unroll
          for (int g = 0; g < G; ++g) w[g] = __ldg(reinterpret_cast<const uint4*>(src + g * 64));
        }
        float top = 0.0f;
#pragma unroll
        for (int g = 0; g < G; ++g) {
          const uint32_t ww[4] = {w[g].x, w[g].y, w[g].z, w[g].w};
#pragma unroll
          for (int i = 0; i < 4; ++i) top = fmaxf(top, fmaxf(fabsf(bf16_lo(ww[i])), fabsf(bf16_hi(ww[i]))));
        }
        top = fmaxf(top, __shfl_xor_sync(~0u, top, 1));
        top = fmaxf(top, __shfl_xor_sync(~0u, top, 2));
        // largest member to [2^14, 2^15)
        const int e = min(max(static_cast<int>((__float_as_uint(top) >> 23) & 0xff) - 127, -98), 127);
        const float up = __uint_as_float(static_cast<uint32_t>(127 + 14 - e) << 23);
        const float back = __uint_as_float(static_cast<uint32_t>(127 - 14 + e) << 23) * p.scale_log2e;
        float sums[G];
#pragma unroll
        for (int g = 0; g < G; ++g) {
          const uint32_t ww[4] = {w[g].x, w[g].y, w[g].z, w[g].w};
          float f[8];
#pragma unroll
          for (int i = 0; i < 4; ++i) { f[2 * i] = bf16_lo(ww[i]) * up; f[2 * i + 1] = bf16_hi(ww[i]) * up; }
#pragma unroll
          for (int i = 0; i < 4; ++i) qf[nt][g][i] = pack_f16(f[i], f[i + 4]);
          float s = ((f[0] + f[1]) + (f[2] + f[3])) + ((f[4] + f[5]) + (f[6] + f[7]));
          s += __shfl_xor_sync(~0u, s, 1);
          s += __shfl_xor_sync(~0u, s, 2);
          sums[g] = s;
        }
        // terms: k slots 4 term + g (two groups: 2 term + g); lane t holds slots 2t, 2t + 1 and 2t + 8, 2t + 9
        const bool odd = (G == 4) && (t & 1);
        float a = odd ? sums[G - 2] : sums[0], b = odd ? sums[G - 1] : sums[1];
        uint32_t term[3];
#pragma unroll
        for (int i = 0; i < 3; ++i) {
          term[i] = pack_bf16(a, b);
          a -= bf16_lo(term[i]);
          b -= bf16_hi(term[i]);
        }
        if (G == 4) {
          qz[nt][0] = t < 2 ? term[0] : term[1];
          qz[nt][1] = t < 2 ? term[2] : 0u;
        } else {
          qz[nt][0] = t == 0 ? term[0] : t == 1 ? term[1] : t == 2 ? term[2] : 0u;
          qz[nt][1] = 0u;
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          cs[nt][j] = __shfl_sync(~0u, back, (2 * t + j) * 4);
          const int col = at.tile * S::kRows + nt * 8 + 2 * t + j;
          lim[nt][j] = p.causal ? min(len, max(0, len - p.n_q + 1 + col / p.group)) : len;
          l[nt][j] = 0.0f; m[nt][j] = 0.0f; thr[nt][j] = -INFINITY;
          if (col < p.rows) least = min(least, lim[nt][j]);
        }
#pragma unroll
        for (int i = 0; i < S::kTiles; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) o[nt][i][j] = 0.0f;
#pragma unroll
        for (int j = 0; j < 4; ++j) oz[nt][j] = 0.0f;
      }
      least = min(least, __shfl_xor_sync(~0u, least, 1));
      least = min(least, __shfl_xor_sync(~0u, least, 2));
      vs_mul = 1.0f;
      vs_set = false;
    }

    // -------------------------------------------------------------- one chunk
    const bool there = ((bad >> stage) & 1u) == 0;
    if (there && !mbar_wait(bar0 + 8 * stage, (phase >> stage) & 1u)) { ok = false; break; }
    if (there) {
      phase ^= 1u << stage;
      const uint8_t* const c = ring + stage * C::kBytes;
      const int key0 = at.chunk * kChunkTokens + 2 * r;    // tokens of this lane's rows: key0 (row r), key0 + 1 (row r + 8)
      const bool edge = at.chunk * kChunkTokens + kChunkTokens > least;

      // logits
      float sacc[NT][4];
      {
        uint32_t kw[2][G];
        float ks[2][G];
        uint32_t kz[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint8_t* const cw = c + C::kK + (r + 8 * h) * (D / 2) + t * (4 * G);
          const uint8_t* const cz = c + C::kKsz + (r + 8 * h) * (4 * G);
          if (G == 4) {
            const uint4 w = *reinterpret_cast<const uint4*>(cw);
            kw[h][0] = w.x; kw[h][1] = w.y; kw[h][G - 2] = w.z; kw[h][G - 1] = w.w;
            const uint4 z = *reinterpret_cast<const uint4*>(cz);
            ks[h][0] = bf16_lo(z.x); ks[h][1] = bf16_hi(z.x); ks[h][G - 2] = bf16_lo(z.y); ks[h][G - 1] = bf16_hi(z.y);
            kz[h] = (t & 1) ? z.w : z.z;
          } else {
            const uint2 w = *reinterpret_cast<const uint2*>(cw);
            kw[h][0] = w.x; kw[h][1] = w.y;
            const uint2 z = *reinterpret_cast<const uint2*>(cz);
            ks[h][0] = bf16_lo(z.x); ks[h][1] = bf16_hi(z.x);
            kz[h] = z.y;
          }
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
          for (int j = 0; j < 4; ++j) sacc[nt][j] = 0.0f;
          mma_bf16(sacc[nt], kz[0], kz[1], kz[0], kz[1], qz[nt][0], qz[nt][1]);
        }
#pragma unroll
        for (int g = 0; g < G; ++g) {
          uint32_t u0[4], u1[4];
          unpack8(kw[0][g], u0);
          unpack8(kw[1][g], u1);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            float a[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            mma_f16(a, u0[0], u1[0], u0[1], u1[1], qf[nt][g][0], qf[nt][g][1]);
            mma_f16(a, u0[2], u1[2], u0[3], u1[3], qf[nt][g][2], qf[nt][g][3]);
            sacc[nt][0] = fmaf(ks[0][g], a[0], sacc[nt][0]);
            sacc[nt][1] = fmaf(ks[0][g], a[1], sacc[nt][1]);
            sacc[nt][2] = fmaf(ks[1][g], a[2], sacc[nt][2]);
            sacc[nt][3] = fmaf(ks[1][g], a[3], sacc[nt][3]);
          }
        }
      }
      // V's scales of this lane's tokens, its centres as a first operand (rows: groups)
      float vs[2][G];
      uint32_t vz[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint8_t* const cv = c + C::kVs + (r + 8 * h) * (2 * G);
        if (G == 4) {
          const uint2 w = *reinterpret_cast<const uint2*>(cv);
          vs[h][0] = bf16_lo(w.x); vs[h][1] = bf16_hi(w.x); vs[h][G - 2] = bf16_lo(w.y); vs[h][G - 1] = bf16_hi(w.y);
        } else {
          const uint32_t w = *reinterpret_cast<const uint32_t*>(cv);
          vs[h][0] = bf16_lo(w); vs[h][1] = bf16_hi(w);
        }
        vz[h] = *reinterpret_cast<const uint32_t*>(c + C::kVz + (r & (G - 1)) * 32 + h * 16 + t * 4);
      }
      if (edge) {
        // hidden keys: logits at -inf, and nothing of bytes that were never written
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (key0 + (j >> 1) >= lim[nt][j & 1]) sacc[nt][j] = -INFINITY;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
          for (int g = 0; g < G; ++g)
            if (key0 + h >= len) vs[h][g] = 0.0f;
          const int kz0 = at.chunk * kChunkTokens + 4 * t + h;   // tokens of the centres' operand: 4t + h, 4t + 2 + h
          if (kz0 >= len) vz[h] &= 0xffff0000u;
          if (kz0 + 2 >= len) vz[h] &= 0x0000ffffu;
        }
      }
      // a logit far above the stabiliser, or a scale far above its unit: move them (rare after the first chunks)
      float rise[NT][4];
      bool move = false;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          rise[nt][j] = fmaf(sacc[nt][j], cs[nt][j & 1], -m[nt][j & 1]);
          move = move || rise[nt][j] > thr[nt][j & 1];
        }
      float vs_top = 0.0f;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int g = 0; g < G; ++g) vs_top = fmaxf(vs_top, vs[h][g]);
      move = move || vs_top * vs_mul > 64.0f || !vs_set;
      if (__any_sync(~0u, move)) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            float top = fmaxf(rise[nt][j], rise[nt][j + 2]);
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
            if (top > thr[nt][j]) {
              const float to = m[nt][j] + top;
              const float f = thr[nt][j] == -INFINITY ? 0.0f : ex2(m[nt][j] - to);   // (nothing summed yet: whatever the factor)
              thr[nt][j] = 8.0f;
              m[nt][j] = to;
              l[nt][j] *= f;
              oz[nt][j] *= f; oz[nt][j + 2] *= f;
#pragma unroll
              for (int i = 0; i < S::kTiles; ++i) { o[nt][i][j] *= f; o[nt][i][j + 2] *= f; }
#pragma unroll
              for (int i = 0; i < 2; ++i) rise[nt][j + 2 * i] = fmaf(sacc[nt][j + 2 * i], cs[nt][j], -m[nt][j]);
            }
          }
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) vs_top = fmaxf(vs_top, __shfl_xor_sync(~0u, vs_top, d));
        if (!vs_set || vs_top * vs_mul > 64.0f) {
          const int e = min(max(static_cast<int>((__float_as_uint(vs_top) >> 23) & 0xff) - 127, -100), 126);
          const float mul = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
          const float f = vs_set ? mul / vs_mul : 1.0f;
          vs_set = true;
          vs_mul = mul;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < S::kTiles; ++i)
#pragma unroll
              for (int j = 0; j < 4; ++j) o[nt][i][j] *= f;
        }
      }
      // probabilities; P and P s, turned into second operands
      uint32_t pz[NT][2], pv[NT][G][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float pr[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) pr[j] = ex2(rise[nt][j]);
        l[nt][0] += pr[0] + pr[2];
        l[nt][1] += pr[1] + pr[3];
        pz[nt][0] = transpose8x8(pack_bf16(pr[0], pr[1]));
        pz[nt][1] = transpose8x8(pack_bf16(pr[2], pr[3]));
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float p0 = pr[2 * h] * vs_mul, p1 = pr[2 * h + 1] * vs_mul;
#pragma unroll
          for (int g = 0; g < G; ++g) {
            float a = p0 * vs[h][g], b = p1 * vs[h][g];
            if (edge) {                        // a hidden key's scale may be a NaN
              if (key0 + h >= lim[nt][0]) a = 0.0f;
              if (key0 + h >= lim[nt][1]) b = 0.0f;
            }
            pv[nt][g][h] = transpose8x8(pack_f16(a, b));
          }
        }
      }
      // out
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) mma_bf16(oz[nt], vz[0], 0u, vz[1], 0u, pz[nt][0], pz[nt][1]);
#pragma unroll
      for (int a = 0; a < S::kTiles / 4; ++a) {
        const uint4 w = *reinterpret_cast<const uint4*>(c + C::kV + (a * 32 + lane) * 16);
        const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t u[4];
          unpack8(ww[i], u);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
            mma_f16(o[nt][4 * a + i], u[0], u[1], u[2], u[3], pv[nt][2 * a + (i >> 1)][0], pv[nt][2 * a + (i >> 1)][1]);
        }
      }
    }
    // the stage is free: the chunk kStages further on
    __syncwarp();
    if (issued < end) {
      issue(stage);
      ask();
      ++issued;
    }
    stage = stage + 1 == kStages ? 0 : stage + 1;

    // -------------------------------------------------------------- the unit, or the range, ends: results out
    const bool unit_ends = at.chunk + 1 == at.n;
    if (unit_ends || x + 1 == end) {
      const bool whole = unit_ends && seg_first == 0;
      const float unit = 1.0f / vs_mul;        // 2^E
      float* const part = p.part + static_cast<size_t>(2 * lw + (seg_first == 0 ? 1 : 0)) * p.part_rows * (D + 2);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          float sum = l[nt][j];
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) sum += __shfl_xor_sync(~0u, sum, d);
          const int in_tile = nt * 8 + 2 * t + j, row = at.tile * S::kRows + in_tile;
          const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
          for (int g = 0; g < G; ++g) {
            const float z = __shfl_sync(~0u, oz[nt][j], g * 4 + t);
            float v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = fmaf(o[nt][2 * g + (i >> 1)][j + 2 * (i & 1)], unit, z);
            if (row < p.rows) {
              const int d0 = 32 * g + 4 * r;
              if (whole) {
                const int tq = row / p.group, j_head = at.head * p.group + row % p.group;
                uint16_t* dst = p.out + ((static_cast<int64_t>(at.seq) * p.n_q + tq) * (static_cast<int64_t>(p.n_heads) * p.group) + j_head) * D + d0;
                *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16(v[0] * inv, v[1] * inv), pack_bf16(v[2] * inv, v[3] * inv));
              } else {
                float* dst = part + in_tile * (D + 2) + 2 + d0;
                *reinterpret_cast<float2*>(dst) = make_float2(v[0], v[1]);
                *reinterpret_cast<float2*>(dst + 2) = make_float2(v[2], v[3]);
              }
            }
          }
          if (!whole && row < p.rows && r == 0)
            *reinterpret_cast<float2*>(part + in_tile * (D + 2)) = make_float2(thr[nt][j] == -INFINITY ? -INFINITY : m[nt][j], sum);
        }
      fresh = true;
    }
    step(p, at, first);
  }
  if (!ok) {
    // gave up: leave only when the copies in flight have landed (bounded)
    if (lane == 0) record_status(p.workspace, MUSTDROP_ERR_TIMEOUT, lw);
    for (int i = 0; i < kStages; ++i)
      if (((bad >> i) & 1u) == 0 && i < end - begin) (void)mbar_wait(bar0 + 8 * i, (phase >> i) & 1u);
  }
}

// Joins the units that several warps share, and writes zeros for sequences without keys.  One CTA per (unit, row).
constexpr int kJoinThreads = 512;

template <int D>
__global__ void __launch_bounds__(kJoinThreads) page_join_kernel(const AttendParams p, int ctas, int kRows) {
  constexpr int kParts = kJoinThreads / D;   // threads of a channel, each joining every kParts-th partial result
  __shared__ long long sums[2][kJoinThreads / 32];
  __shared__ float acc_s[kJoinThreads], l_s[kJoinThreads];
  pdl_launch_dependents();
  const int unit = blockIdx.x, row_in = blockIdx.y;
  const int units_per_seq = p.n_heads * p.tiles;
  const int seq = unit / units_per_seq, u = unit % units_per_seq, head = u / p.tiles, tile = u % p.tiles;
  const int row = tile * kRows + row_in;
  if (row >= p.rows) { pdl_wait(); return; }
  pdl_wait();
  long long before = 0, total = 0;
  for (int s = threadIdx.x; s < p.n_seq; s += kJoinThreads) {
    const int n = chunks_of(clamp_len(p, s));
    total += n;
    if (s < seq) before += n;
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    before += __shfl_xor_sync(~0u, before, d);
    total += __shfl_xor_sync(~0u, total, d);
  }
  if ((threadIdx.x & 31) == 0) { sums[0][threadIdx.x >> 5] = before; sums[1][threadIdx.x >> 5] = total; }
  __syncthreads();
  before = total = 0;
#pragma unroll
  for (int w = 0; w < kJoinThreads / 32; ++w) { before += sums[0][w]; total += sums[1][w]; }
  const int n = chunks_of(clamp_len(p, seq));
  const int d = threadIdx.x % D, part0 = threadIdx.x / D;
  const int tq = row / p.group, j_head = head * p.group + row % p.group;
  uint16_t* const dst = p.out + ((static_cast<int64_t>(seq) * p.n_q + tq) * (static_cast<int64_t>(p.n_heads) * p.group) + j_head) * D + d;
  if (n == 0) {
    if (part0 == 0) *dst = 0;
    return;
  }
  const Cut cut = cut_of(total * units_per_seq, ctas);
  const long long c0 = before * units_per_seq + static_cast<long long>(u) * n;
  const int w0 = cut.owner(c0), w1 = cut.owner(c0 + n - 1);
  if (w0 == w1) return;   // one warp had it all
  // slot 1 of the warp in whose range the unit begins, slot 0 of the others
  auto at = [&](int w) { return p.part + (static_cast<size_t>(2 * w + (w == w0 ? 1 : 0)) * p.part_rows + row_in) * (D + 2); };
  float m = -INFINITY;
  for (int w = w0 + threadIdx.x; w <= w1; w += kJoinThreads) m = fmaxf(m, at(w)[0]);
#pragma unroll
  for (int i = 16; i > 0; i >>= 1) m = fmaxf(m, __shfl_xor_sync(~0u, m, i));
  if ((threadIdx.x & 31) == 0) acc_s[threadIdx.x >> 5] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kJoinThreads / 32; ++i) m = fmaxf(m, acc_s[i]);
  __syncthreads();
  float acc = 0.0f, l = 0.0f;
  for (int w = w0 + part0; w <= w1; w += kParts) {
    const float* const q = at(w);
    const float f = q[0] == -INFINITY ? 0.0f : ex2(q[0] - m);
    l = fmaf(f, q[1], l);
    acc = fmaf(f, q[2 + d], acc);
  }
  acc_s[threadIdx.x] = acc;
  l_s[threadIdx.x] = l;
  __syncthreads();
  if (part0 != 0) return;
#pragma unroll
  for (int i = 1; i < kParts; ++i) { acc += acc_s[i * D + d]; l += l_s[i * D + d]; }
  const float v = l == 0.0f ? 0.0f : acc / l;
  *dst = static_cast<uint16_t>(pack_bf16(v, 0.0f) & 0xffffu);
}

int tiles_of(int rows) { return rows <= 8 ? 1 : 2; }   // column tiles of 8 query rows

template <int D, int NT>
cudaError_t launch_attend(const AttendParams& p, int ctas, cudaStream_t stream) {
  using S = Shape<D, NT>;
  const size_t smem = S::ring + (static_cast<size_t>(p.n_seq) + 1) * sizeof(int32_t);
  cudaError_t e = ensure_kernel_attributes(reinterpret_cast<const void*>(page_attend_kernel<D, NT>), false);
  if (e != cudaSuccess) return e;
  e = launch_pdl(page_attend_kernel<D, NT>, dim3(static_cast<unsigned>(ctas)), dim3(kThreads), smem, stream, p);
  if (e != cudaSuccess) return e;
  const dim3 grid(static_cast<unsigned>(p.n_seq * p.n_heads * p.tiles), static_cast<unsigned>(std::min(p.rows, S::kRows)));
  return launch_pdl(page_join_kernel<D>, grid, dim3(kJoinThreads), 0, stream, p, ctas, S::kRows);
}

}  // namespace

size_t page_attend_partial_bytes(const mustdrop_page_config_t* c) {
  if (c->n_heads <= 0 || c->q_heads <= 0 || c->q_heads % c->n_heads != 0 || c->n_q > 128) return 0;
  const int64_t rows = static_cast<int64_t>(c->q_heads / c->n_heads) * c->n_q;
  const size_t part_rows = static_cast<size_t>(std::min<int64_t>(rows, 8 * tiles_of(static_cast<int>(std::min<int64_t>(rows, 64)))));
  const size_t bytes = static_cast<size_t>(kMaxCtas) * kWarps * 2 * part_rows * (c->head_dim + 2) * sizeof(float);
  return (bytes + 255) / 256 * 256;
}

}  // namespace mustdrop

extern "C" mustdrop_status_t mustdrop_page_attend(const mustdrop_page_config_t* c, const void* q, const void* pool,
                                                  const int32_t* page_table, const int32_t* len, void* out, void* workspace,
                                                  void* cuda_stream) {
  using namespace mustdrop;
  const mustdrop_status_t st = check_page_pool(c);
  if (st != MUSTDROP_OK) return st;
  if (c->q_heads <= 0 || c->n_q <= 0 || c->max_pages <= 0 || c->causal < 0 || c->causal > 1 || c->q_heads % c->n_heads != 0 ||
      !(c->scale >= 0.0f) || c->scale > 3.0e38f)
    return MUSTDROP_ERR_INVALID_ARG;
  if (c->n_q > 128 || c->n_seq > kMaxSeqs || static_cast<int64_t>(c->max_pages) * c->page > INT32_MAX) return MUSTDROP_ERR_UNSUPPORTED;
  const int64_t rows = static_cast<int64_t>(c->q_heads / c->n_heads) * c->n_q;
  if (rows > 16384 || c->q_heads > 65535) return MUSTDROP_ERR_UNSUPPORTED;
  // the line of chunks: sequences' chunks add up in 32 bits, units fit a grid
  const int64_t most = static_cast<int64_t>(c->n_seq) * c->max_pages * (c->page / kChunkTokens);
  if (most > INT32_MAX) return MUSTDROP_ERR_UNSUPPORTED;
  if (workspace == nullptr) return MUSTDROP_ERR_WORKSPACE;
  const void* wide[] = {q, pool, out, workspace};
  for (const void* x : wide)
    if (x == nullptr || misaligned(x, 16)) return MUSTDROP_ERR_INVALID_ARG;
  if (page_table == nullptr || len == nullptr || misaligned(page_table, 4) || misaligned(len, 4)) return MUSTDROP_ERR_INVALID_ARG;
  if (c->q_stride_s % 8 != 0 || c->q_stride_t % 8 != 0 || c->q_stride_h % 8 != 0) return MUSTDROP_ERR_UNSUPPORTED;
  AttendParams p = {};
  p.q = static_cast<const uint8_t*>(q); p.pool = static_cast<const uint8_t*>(pool);
  p.table = page_table; p.len = len; p.out = static_cast<uint16_t*>(out);
  p.part = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + kWsStatusBytes);
  p.workspace = static_cast<int32_t*>(workspace);
  p.n_seq = c->n_seq; p.n_heads = c->n_heads; p.group = c->q_heads / c->n_heads; p.n_q = c->n_q;
  p.rows = static_cast<int32_t>(rows);
  const int nt = tiles_of(p.rows);
  p.tiles = (p.rows + 8 * nt - 1) / (8 * nt);
  p.part_rows = std::min(p.rows, 8 * nt);
  if (static_cast<int64_t>(p.n_seq) * p.n_heads * p.tiles > INT32_MAX ||
      static_cast<int64_t>(p.n_heads) * p.tiles > (1ll << 50) / most)     // (places on the line times warps: 63 bits)
    return MUSTDROP_ERR_UNSUPPORTED;
  p.lg = page_log2(c->page); p.n_pages = c->n_pages; p.max_pages = c->max_pages; p.causal = c->causal;
  p.q_sh = 2 * (c->q_stride_h != 0 ? c->q_stride_h : c->head_dim);
  p.q_st = 2 * (c->q_stride_t != 0 ? c->q_stride_t : static_cast<int64_t>(c->q_heads) * c->head_dim);
  p.q_ss = 2 * (c->q_stride_s != 0 ? c->q_stride_s : static_cast<int64_t>(c->n_q) * c->q_heads * c->head_dim);
  const float scale = c->scale != 0.0f ? c->scale : (c->head_dim == 128 ? 0.08838834764831845f : 0.125f);
  p.scale_log2e = scale * 1.4426950408889634f;
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e == cudaSuccess) {
    const int ctas = std::min(kMaxCtas, sms * (nt == 1 ? 2 : 1));
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (c->head_dim == 128)
      e = nt == 1 ? launch_attend<128, 1>(p, ctas, stream) : launch_attend<128, 2>(p, ctas, stream);
    else
      e = nt == 1 ? launch_attend<64, 1>(p, ctas, stream) : launch_attend<64, 2>(p, ctas, stream);
  }
  if (e == cudaSuccess) return MUSTDROP_OK;
  set_last_cuda_error(e);
  return MUSTDROP_ERR_CUDA;
}
