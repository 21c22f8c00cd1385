// Attention of the decoded tokens over a cache in pages of 4-bit values (mustdrop_page_attend).
//
//   S[x][q] = scale <K_x, q>,  P = exp(S - m),  out[q] = sum_x P V_x / sum_x P,   K = z + s (c - 8) per group of 32 channels
//
//   <K_x, q> = sum_g s_xg (sum_{d in g} C_xd q_d)  +  sum_g z_xg (sum_{d in g} q_d)         C = c - 8
//   out_d    = sum_x (P_x s_xg) C_xd               +  sum_x P_x z_xg
//
// so the codes go into the matrix instructions as they are, with 16 tokens (K) or 16 channels (V) as the rows and the query
// rows - the query tokens and heads that share a K / V head - as the 8 columns.  Scales meet fp32 accumulators (K) or
// the probabilities (V).  Codes are fp16 operands (exact); q is scaled by a power of two into fp16's range (exact but for
// members below 2^-27 of the largest); P s is rounded once, to 11 bits, with a running power of two per query row and group that keeps it
// in fp16's range whatever the scales are.  A word of eight codes is five instructions of bits, and four more where the offset of its operands is
// taken off one by one.  K's is taken off the sums instead (kCodeUnit).  Not V's: the matrix instruction's fp32 sums are cut, not
// rounded, so an offset of 1032 P s in a sum over many tokens leaves a bias (4.5e-3 of the result, 1.6e-3 being bf16's own rounding, over
// 1000 tokens with the offset taken off every 512).  (e4m3 operands, in which a code is a code's own bits, were slower: this GPU runs that
// instruction as two of fp16 behind conversions.)
//
// Bound: HBM where the issue slots keep up: a token and head is 1.25 D bytes where bf16 has 4 D, ~23 bytes per clock and SM, and takes
// some 275 instructions per 16 tokens with one or two query rows, 370 with up to eight.  64 requests of 200 to 1800 keys, 32 heads: 69 us,
// 4.8 TB/s (6.6 TB/s between the first landed chunk and the median warp's last); 2 of 90 to 131 thousand keys, 8 heads of 4 query heads: 72 us,
// 3.9 TB/s.  More query rows than 16 are tiles that each read and unpack all pages again: 16 sequences of 2048 keys with 128 rows 77 us, 15 times
// the products' time.
//
// Every warp walks its own range of chunks (16 tokens of one head, 20 D contiguous bytes, one bulk copy each), two at a
// time, through its own ring in shared memory, without a barrier between warps.  The chunks of all (sequence, head, row tile) units form one
// line that is cut into parts, one per CTA and then one per warp, whatever the lengths are: no host has to know
// them.  A unit that several warps share is joined from partial results (fp32): first those of a CTA, in shared memory
// behind its last barrier, then those of the CTAs, by the CTA that finishes last.  Both add in the order of the line: the same call
// gives the same bits.
#include <algorithm>

#include "page_internal.h"

namespace mustdrop {
namespace {

constexpr int kMaxSeqs = 4096;
constexpr int kMaxCtas = 192;         // one per SM, and some to spare
constexpr size_t kCountBytes = 1024;  // of the workspace: a counter per CTA, zero between calls
constexpr long long kWaitCycles = 200000000ll;   // ~0.1 s: a bulk copy that takes longer will not come

struct AttendParams {
  const uint8_t* q;         // bf16
  const uint8_t* pool;
  const int32_t *table, *len;
  uint16_t* out;
  float* part;              // partial results [CTA][2][part_rows][D + 4]: stabiliser, sum, -, -, D values
  unsigned* joined;         // [CTA]: parts of the unit that begins in this CTA and ends in a later one
  int32_t* workspace;
  int32_t n_seq, n_heads, group, n_q, rows, tiles;   // rows = n_q * group query rows per unit, in `tiles` row tiles
  int32_t lg, n_pages, max_pages, causal, part_rows;
  uint32_t group_magic;       // 2^32 / group, rounded up: a row (below 2^14) over the group is the product's high half
  int64_t q_ss, q_st, q_sh;   // bytes
  float scale_log2e;
  uint32_t give_up;           // lanes of a warp whose waits for copies run out at once (0, but for debugging)
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
  asm volatile("cp.async.bulk.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar)
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
// K's codes are operands as they are, as subnormal numbers: c 2^-24 for even channels, 16 c 2^-24 over a q that is divided by 16 for odd
// ones, so a logit's sums are in units of 2^-24.  What takes 8 off the codes is a sum over q alone.  (An offset of 1024 under the codes, taken off
// the same way, cost seven bits of the sums: 5 % of the result where 8000 nats of products cancel, three and more query rows.  What the unit costs is range at one end and gives at
// the other: keys up to the type's largest, queries up to 2^116 over the scale.)
constexpr float kCodeUnit = 0x1p-24f;
constexpr int kCodeLog2 = 24;
__device__ __forceinline__ uint32_t times_minus8(uint32_t sums) {   // of a bf16 pair
  uint32_t d;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(sums), "r"(0xc100c100u));
  return d;
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
// Nibbles j and j + 4 of a word as fp16 pairs, for j = 0..3: the fields of a word that a mask leaves, as K takes them, ...
struct Consts {   // kept in registers: as literals the compiler loads them again for every word
  uint32_t low, high, magic, sixteenth, minus72;
};
__device__ __forceinline__ uint32_t opaque(uint32_t v) {
  asm volatile("" : "+r"(v));
  return v;
}
__device__ __forceinline__ Consts make_consts() {
  return {opaque(0x000f000fu), opaque(0x00f000f0u), opaque(0x64006400u), opaque(0x2c002c00u), opaque(0xd480d480u)};   // .., 1024, 1/16, -72
}
__device__ __forceinline__ void nibbles8(const Consts& k, uint32_t w, uint32_t (&x)[4]) {
  const uint32_t w8 = w >> 8;
  x[0] = w & k.low; x[1] = w & k.high; x[2] = w8 & k.low; x[3] = w8 & k.high;
}
// ... and less 8, as V does.  (The well-known way from four bits to fp16: a nibble under the bits of 1024 reads 1024 + c, or 1024 + 16 c in bits
// 4..7, and one exact operation a pair takes the rest off.)
__device__ __forceinline__ void codes8(const Consts& k, uint32_t w, uint32_t (&x)[4]) {
  const uint32_t w8 = w >> 8;
  asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(x[0]) : "r"(w), "r"(k.low), "r"(k.magic));
  asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(x[1]) : "r"(w), "r"(k.high), "r"(k.magic));
  asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(x[2]) : "r"(w8), "r"(k.low), "r"(k.magic));
  asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(x[3]) : "r"(w8), "r"(k.high), "r"(k.magic));
  asm("sub.rn.f16x2 %0, %0, %1;" : "+r"(x[0]) : "r"(0x64086408u));                              // 1032
  asm("fma.rn.f16x2 %0, %0, %1, %2;" : "+r"(x[1]) : "r"(k.sixteenth), "r"(k.minus72));
  asm("sub.rn.f16x2 %0, %0, %1;" : "+r"(x[2]) : "r"(0x64086408u));
  asm("fma.rn.f16x2 %0, %0, %1, %2;" : "+r"(x[3]) : "r"(k.sixteenth), "r"(k.minus72));
}

// The line of chunks: sequence s has heads * tiles units of chunks(s) chunks each.
__device__ __forceinline__ int32_t clamp_len(const AttendParams& p, int32_t n) {
  const int32_t most = p.max_pages << p.lg;
  return n < 0 ? 0 : n > most ? most : n;
}
__device__ __forceinline__ int32_t chunks_of(int32_t len) { return static_cast<int32_t>((static_cast<uint32_t>(len) + kChunkTokens - 1) / kChunkTokens); }

// Equal parts of the line, one per CTA: `more` CTAs have per + 1 chunks, the others per.
struct Cut {
  int ctas, per, more;
  __device__ __forceinline__ long long begin(int c) const { return static_cast<long long>(c) * per + min(c, more); }
  // the CTA that has chunk x
  __device__ __forceinline__ int owner(long long x) const {
    const long long big = static_cast<long long>(more) * (per + 1);
    return static_cast<int>(x < big ? divide(x, per + 1) : more + divide(x - big, per));
  }
  static __device__ __noinline__ long long divide(long long a, int b) {   // (a 64-bit division takes some 100 cycles more; one copy, as all that runs once is fetched first)
    return a >> 32 == 0 ? static_cast<uint32_t>(a) / static_cast<uint32_t>(b) : a / b;
  }
};
__device__ __forceinline__ Cut cut_of(long long total, int ctas) {
  Cut c;
  c.ctas = total < ctas ? static_cast<int>(total) : ctas;
  c.per = static_cast<int>(Cut::divide(total, c.ctas));
  c.more = static_cast<int>(total - static_cast<long long>(c.per) * c.ctas);
  return c;
}

// A place in the warp's part of the line: `left` chunks from `chunk` on are of this unit, `rest` chunks come after them.
struct Cursor {
  int32_t seq, head, tile, chunk, left, rest;
};
__device__ __forceinline__ void next_unit(const AttendParams& p, Cursor& x, const int32_t* first) {   // first[s]: chunks (per unit) of the sequences before s
  x.chunk = 0;
  if (++x.tile >= p.tiles) {
    x.tile = 0;
    if (++x.head >= p.n_heads) {
      x.head = 0;
      do {
        ++x.seq;
      } while (x.seq < p.n_seq - 1 && first[x.seq + 1] == first[x.seq]);
    }
  }
  x.left = min(x.rest, first[x.seq + 1] - first[x.seq]);
  x.rest -= x.left;
}

__device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
  return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t a) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a));
  return v;
}
__device__ __forceinline__ uint32_t lds32(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(a));
  return v;
}
__device__ __forceinline__ uint32_t lds16(uint32_t a) {
  uint16_t v;
  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(a));
  return v;
}
// two products an instruction
__device__ __forceinline__ float2 mul_pair(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmul.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
// a where c, else b: as an instruction, so that an array of registers is not made an array in memory
__device__ __forceinline__ float pick(bool c, float a, float b) {
  float d;
  asm("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %3, 0;\n\tselp.f32 %0, %1, %2, p;\n\t}" : "=f"(d) : "f"(a), "f"(b), "r"(static_cast<uint32_t>(c)));
  return d;
}
__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("max.u16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
// Joins `n` partial results of one query row (in order; at(i) gives the i-th) in one warp: lane's channels 4 lane .. + 3.
struct RowSum {
  float m, l;
  float4 v;
};
template <int D, bool OTHERS, typename At>   // OTHERS: parts that other CTAs wrote, past this SM's L1
__device__ __forceinline__ RowSum join_row(int n, At at, int lane) {
  RowSum s = {-INFINITY, 0.0f, make_float4(0.0f, 0.0f, 0.0f, 0.0f)};
  const int c = min(lane, D / 4 - 1);
  constexpr int kBatch = OTHERS ? 8 : 2;   // loads in flight: parts of other CTAs come from L2
  for (int base = 0; base < n; base += kBatch) {
    float2 ml[kBatch];
    float4 x[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      ml[i] = make_float2(-INFINITY, 0.0f);
      x[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      if (base + i < n) {
        const float* const q = at(base + i);
        const float2* const a = reinterpret_cast<const float2*>(q);
        const float4* const b = reinterpret_cast<const float4*>(q + 4) + c;
        ml[i] = OTHERS ? __ldcg(a) : *a;
        x[i] = OTHERS ? __ldcg(b) : *b;
      }
    }
    float m = s.m;
#pragma unroll
    for (int i = 0; i < kBatch; ++i) m = fmaxf(m, ml[i].x);
    const float keep = s.m == -INFINITY ? 0.0f : ex2(s.m - m);
    s.l *= keep; s.v.x *= keep; s.v.y *= keep; s.v.z *= keep; s.v.w *= keep;
    s.m = m;
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const float f = ml[i].x == -INFINITY ? 0.0f : ex2(ml[i].x - m);
      s.l = fmaf(f, ml[i].y, s.l);
      s.v.x = fmaf(f, x[i].x, s.v.x); s.v.y = fmaf(f, x[i].y, s.v.y);
      s.v.z = fmaf(f, x[i].z, s.v.z); s.v.w = fmaf(f, x[i].w, s.v.w);
    }
  }
  return s;
}

// P s goes into fp16 over a unit 2^E of its column and group, as groups' scales may be any powers of two apart: mul = 2^-E, 0 where none is set.
// (One unit for all groups of a column, in the layout for more rows, was 2 to 4 % faster, and rounded a group to nothing beside one 2^24 times it.)
// A unit is set from the pair of chunks that sets the stabiliser - their largest P s, so the tokens that now count are far from both ends of
// fp16 - and again when P s has grown by 2^13, or when the stabiliser moves: whatever set it has then faded.
constexpr float kUnitRoom = 13.0f;
__device__ __forceinline__ int unit_exponent(float mul) { return 127 - static_cast<int>(__float_as_uint(mul) >> 23); }
// log2 of a bf16 scale, from its bits: too small by less than 0.09
__device__ __forceinline__ float scale_log2(uint32_t bits) { return fmaf(static_cast<float>(bits), 1.0f / 128.0f, -127.0f); }
// The unit for a largest P s of 2^size; `f` receives what sums over the old unit are multiplied by.
__device__ __forceinline__ float new_unit(float mul, float size, float* f) {
  int e = min(max(static_cast<int>(ceilf(fmaxf(size, -1000.0f))), -100), 126);
  *f = 1.0f;
  if (mul != 0.0f) {
    const int old = unit_exponent(mul);
    e = max(e, old - 90);                       // (sums stay finite)
    *f = ex2(static_cast<float>(old - e));
  }
  return __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
}

// Query token of a unit's row, and the row's place among the n_q * q_heads rows of its sequence in q and out.
__device__ __forceinline__ int token_of(const AttendParams& p, int row) { return p.group == 1 ? row : static_cast<int>(__umulhi(row, p.group_magic)); }
__device__ __forceinline__ int64_t out_row(const AttendParams& p, int row, int head) {
  const int tq = token_of(p, row);
  return static_cast<int64_t>(tq * p.n_heads + head) * p.group + (row - tq * p.group);
}
__device__ __forceinline__ const uint8_t* q_row(const AttendParams& p, int seq, int head, int row) {
  const int tq = token_of(p, row);
  return p.q + seq * p.q_ss + tq * p.q_st + (static_cast<int64_t>(head) * p.group + (row - tq * p.group)) * p.q_sh;
}

// log2 units of a logit per unit of a product of q over 2^e: a number above zero and finite, as hidden keys' logits are -inf and a zero
// key's are zero (a scale below 2^-37 over a q of zeros would be none: NaN)
__device__ __forceinline__ float log2_per_product(const AttendParams& p, int e) {
  return fminf(fmaxf(ldexpf(p.scale_log2e, e), __uint_as_float(1u)), 3.4e38f);
}

constexpr float kNone = -3.0e38f;   // stabiliser of a column that has seen no key

// What a warp holds of the unit in hand, and its arithmetic, for up to 8 NT query rows: a column each.
template <int D, int NT>
struct Wide {
  using C = Chunk<D>;
  static constexpr int kD = D, G = D / 32, kTiles = D / 16, kRows = 8 * NT;
  // One CTA per SM: 12 warps of up to 168 registers where one column tile needs no more (more warps hide more of a warp's
  // chain copy - logits - probabilities - out), 8 of 255 for two; ~120 KB of ring.
  static constexpr int kWarps = NT == 1 ? 12 : 8;
  static constexpr bool kEarly = false;   // the next unit's queries before this one's results: no registers for it
  static constexpr int kStages = (NT == 1 ? 2 : 3) * (128 / D);

  uint32_t qf[NT][G][4];                   // q as the second operand: [g][2 m + {0, 1}], odd channels over 16
  uint32_t qz[NT][2], qs[NT][2];           // its sums over groups, and those that take the offsets off, in three bf16 terms
  float cs[NT][2];                         // log2 units per unit of the scaled product, of columns 2t, 2t + 1
  float o[NT][kTiles][4], oz[NT][4];    // out (without centres) and the centres' part, rows r, r + 8 and columns 2t, 2t + 1
  float l[NT][2], m[NT][2];                // sum (of this lane's tokens), stabiliser (kNone: no key seen)
  float mul[NT][2][G];                     // 2^-E of columns 2t, 2t + 1 and every group
  uint32_t room[G / 2];                    // 2^15 less the bf16 bits of the P s that the groups' units have room for, two groups to a word
  int32_t least = 0, len = 0;              // fewest visible keys of any column; the sequence's length
  uint4 next_q[NT][G];
  int32_t next_len;

  Consts consts;
  int lane, r, t;

  __device__ __forceinline__ void init() {
    lane = threadIdx.x & 31; r = lane >> 2; t = lane & 3;
    consts = make_consts();
  }

  // asks for a unit's queries and its length: channels 8 t .. + 7 of every group of row r
  __device__ __forceinline__ void fetch(const AttendParams& p, const Cursor& at) {
    next_len = p.len[at.seq];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int row = at.tile * kRows + nt * 8 + r;
#pragma unroll
      for (int g = 0; g < G; ++g) next_q[nt][g] = make_uint4(0, 0, 0, 0);
      if (row < p.rows) {
        const uint8_t* const src = q_row(p, at.seq, at.head, row) + t * 16;
#pragma unroll
        for (int g = 0; g < G; ++g) next_q[nt][g] = __ldg(reinterpret_cast<const uint4*>(src + g * 64));
      }
    }
  }

  __device__ __forceinline__ void begin(const AttendParams& p, const Cursor& at) {
    len = clamp_len(p, next_len);
    least = len;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const uint4(&w)[G] = next_q[nt];
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
      const float back = log2_per_product(p, e - 14 + kCodeLog2);
      float sums[G];
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const uint32_t ww[4] = {w[g].x, w[g].y, w[g].z, w[g].w};
        float f[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) { f[2 * i] = bf16_lo(ww[i]) * up; f[2 * i + 1] = bf16_hi(ww[i]) * up; }
#pragma unroll
        for (int i = 0; i < 4; ++i) qf[nt][g][i] = (i & 1) ? pack_f16(f[i] * 0.0625f, f[i + 4] * 0.0625f) : pack_f16(f[i], f[i + 4]);
        float s = (((f[1] + f[3]) + (f[5] + f[7])) + ((f[0] + f[2]) + (f[4] + f[6]))) * kCodeUnit;
        s += __shfl_xor_sync(~0u, s, 1);
        s += __shfl_xor_sync(~0u, s, 2);
        sums[g] = s;
      }
      // terms of the sums: operand slots 4 term + g (two groups: 2 term + g); lane t holds slots 2t, 2t + 1 and 2t + 8, 2t + 9.
      // (A q that holds an infinity or a NaN has one in its sums: its logits are none either.)
      const bool high = (G == 4) && (t & 1);
      float a = high ? sums[G - 2] : sums[0], b = high ? sums[G - 1] : sums[1];
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
      for (int i = 0; i < 2; ++i) qs[nt][i] = times_minus8(qz[nt][i]);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        cs[nt][j] = __shfl_sync(~0u, back, (2 * t + j) * 4);
        l[nt][j] = 0.0f;
        m[nt][j] = kNone;
#pragma unroll
        for (int g = 0; g < G; ++g) mul[nt][j][g] = 0.0f;
      }
#pragma unroll
      for (int i = 0; i < kTiles; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) o[nt][i][j] = 0.0f;
#pragma unroll
      for (int j = 0; j < 4; ++j) oz[nt][j] = 0.0f;
    }
    if (p.causal) least = max(0, len - p.n_q + 1 + token_of(p, at.tile * kRows));
#pragma unroll
    for (int i = 0; i < G / 2; ++i) room[i] = 0x00010001u;
  }

  __device__ __forceinline__ void pair(const AttendParams& p, const Cursor& at, uint32_t c0, uint32_t gone) {
    const int key0 = at.chunk * kChunkTokens;
    const bool edge = gone != 0 || key0 + 2 * kChunkTokens > least;

    // logits of the tokens 2r (row r) and 2r + 1 (row r + 8) of both chunks
    float sacc[2][NT][4];
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      const uint32_t c = c0 + hf * C::kBytes;
      uint32_t kw[2][G];
      float ks[2][G];
      uint32_t kz[2], kss[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t cw = c + C::kK + (r + 8 * h) * (D / 2) + t * (4 * G);
        const uint32_t cz = c + C::kKsz + (r + 8 * h) * (4 * G);
        if (G == 4) {
          const uint4 w = lds128(cw);
          kw[h][0] = w.x; kw[h][1] = w.y; kw[h][G - 2] = w.z; kw[h][G - 1] = w.w;
          const uint4 z = lds128(cz);
          ks[h][0] = bf16_lo(z.x); ks[h][1] = bf16_hi(z.x); ks[h][G - 2] = bf16_lo(z.y); ks[h][G - 1] = bf16_hi(z.y);
          kss[h] = (t & 1) ? z.y : z.x;
          kz[h] = (t & 1) ? z.w : z.z;
        } else {
          const uint2 w = lds64(cw);
          kw[h][0] = w.x; kw[h][1] = w.y;
          const uint2 z = lds64(cz);
          ks[h][0] = bf16_lo(z.x); ks[h][1] = bf16_hi(z.x);
          kss[h] = z.x;
          kz[h] = z.y;
        }
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int j = 0; j < 4; ++j) sacc[hf][nt][j] = 0.0f;
        mma_bf16(sacc[hf][nt], kz[0], kz[1], kz[0], kz[1], qz[nt][0], qz[nt][1]);
        mma_bf16(sacc[hf][nt], kss[0], kss[1], kss[0], kss[1], qs[nt][0], qs[nt][1]);
      }
#pragma unroll
      for (int g = 0; g < G; ++g) {
        uint32_t u0[4], u1[4];
        nibbles8(consts, kw[0][g], u0);
        nibbles8(consts, kw[1][g], u1);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float a[4] = {0.0f, 0.0f, 0.0f, 0.0f};
          mma_f16(a, u0[0], u1[0], u0[1], u1[1], qf[nt][g][0], qf[nt][g][1]);
          mma_f16(a, u0[2], u1[2], u0[3], u1[3], qf[nt][g][2], qf[nt][g][3]);
          sacc[hf][nt][0] = fmaf(ks[0][g], a[0], sacc[hf][nt][0]);
          sacc[hf][nt][1] = fmaf(ks[0][g], a[1], sacc[hf][nt][1]);
          sacc[hf][nt][2] = fmaf(ks[1][g], a[2], sacc[hf][nt][2]);
          sacc[hf][nt][3] = fmaf(ks[1][g], a[3], sacc[hf][nt][3]);
        }
      }
    }
    // V's scales of this lane's tokens (bf16 pairs of groups), its centres as a first operand (rows: groups)
    uint32_t vsw[2][2][G / 2], vz[2][2];
#pragma unroll
    for (int hf = 0; hf < 2; ++hf)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t c = c0 + hf * C::kBytes;
        if (G == 4) {
          const uint2 w = lds64(c + C::kVs + (r + 8 * h) * (2 * G));
          vsw[hf][h][0] = w.x; vsw[hf][h][G / 2 - 1] = w.y;
        } else {
          vsw[hf][h][0] = lds32(c + C::kVs + (r + 8 * h) * (2 * G));
        }
        vz[hf][h] = lds32(c + C::kVz + (r & (G - 1)) * 32 + h * 16 + t * 4);
      }
    if (edge) {
      // hidden keys: logits at -inf, and nothing of bytes that were never written
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        const int base = key0 + hf * kChunkTokens;
        const int end = (gone >> hf) & 1u ? base : len;        // keys of the chunk that are there end here
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int key = base + 2 * r + h;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              const int col = at.tile * kRows + nt * 8 + 2 * t + j;
              const int lim = p.causal ? min(end, len - p.n_q + 1 + token_of(p, col)) : end;
              if (key >= lim) sacc[hf][nt][2 * h + j] = -INFINITY;
            }
#pragma unroll
          for (int g = 0; g < G / 2; ++g)
            if (key >= end) vsw[hf][h][g] = 0u;
          const int zk = base + 4 * t + h;                     // tokens of the centres' operand: 4t + h, 4t + 2 + h
          if (zk >= end) vz[hf][h] &= 0xffff0000u;
          if (zk + 2 >= end) vz[hf][h] &= 0x0000ffffu;
        }
      }
    }
    // a logit far above the stabiliser, or P s above its unit's room: move them (rare after the first chunks)
    float rise[2][NT][4];
    float high = -INFINITY;
    uint32_t vs_top[G / 2] = {};                 // the largest scales of this lane's tokens, two groups to a word
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          rise[hf][nt][j] = fmaf(sacc[hf][nt][j], cs[nt][j & 1], -m[nt][j & 1]);
          high = fmaxf(high, rise[hf][nt][j]);
        }
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int g = 0; g < G / 2; ++g) vs_top[g] = max_u16x2(vs_top[g], vsw[hf][h][g]);
    }
    // (the largest logit and a group's largest scale, be they of the same token or not; a NaN's bits are above all scales'.  Halves of words
    // are added as they are: no sum of two leaves its 16 bits.)
    uint32_t over = vs_top[0] + room[0], nan = vs_top[0];
    if (G == 4) { over = max_u16x2(over, vs_top[G / 2 - 1] + room[G / 2 - 1]); nan = max_u16x2(nan, vs_top[G / 2 - 1]); }
    over = max(over & 0xffffu, over >> 16);
    if (__any_sync(~0u, high > 8.0f || fmaf(static_cast<float>(over), 1.0f / 128.0f, high) > 256.0f || ((nan + 0x00800080u) & 0x80008000u) != 0)) {
      // A NaN for a scale: NaN in its group's channels (by way of the centres) for the columns that see the key, and the key's
      // scale is zero from here on: a column that does not see it has P = 0, and 0 x NaN would be one.
      uint32_t none = 0;               // bit (nt, j, g)
#pragma unroll
      for (int hf = 0; hf < 2; ++hf)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int g = 0; g < G; ++g) {
            const uint32_t half = (g & 1) ? 0xffff0000u : 0x0000ffffu;
            if ((vsw[hf][h][g >> 1] & half) > (half & 0x7f807f80u)) {
              vsw[hf][h][g >> 1] &= ~half;
#pragma unroll
              for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 2; ++j)
                  if (sacc[hf][nt][2 * h + j] != -INFINITY) none |= 1u << ((nt * 2 + j) * G + g);
            }
          }
#pragma unroll
      for (int d = 4; d < 32; d <<= 1) none |= __shfl_xor_sync(~0u, none, d);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int j = 0; j < 2; ++j)
          if (r < G && ((none >> ((nt * 2 + j) * G + r)) & 1u)) oz[nt][j] = __uint_as_float(0x7fffffffu);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          float top = kNone;
#pragma unroll
          for (int hf = 0; hf < 2; ++hf)
            top = fmaxf(top, fmaxf(sacc[hf][nt][j] * cs[nt][j], sacc[hf][nt][j + 2] * cs[nt][j]));
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
          const bool moves = top > m[nt][j] + 8.0f;
          if (moves) {
            const float f = ex2(m[nt][j] - top);
            m[nt][j] = top;
            l[nt][j] *= f;
            oz[nt][j] *= f; oz[nt][j + 2] *= f;
#pragma unroll
            for (int i = 0; i < kTiles; ++i) { o[nt][i][j] *= f; o[nt][i][j + 2] *= f; }
          }
          // log2 of P s per group, over 1/128 and from -377 on, two groups to a word: a scale's bits are its log2 over 1/128 from -127 on
          uint32_t largest[G / 2] = {};
#pragma unroll
          for (int hf = 0; hf < 2; ++hf)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              rise[hf][nt][j + 2 * h] = fmaf(sacc[hf][nt][j + 2 * h], cs[nt][j], -m[nt][j]);
              const uint32_t up = static_cast<uint32_t>(fmaf(fminf(fmaxf(rise[hf][nt][j + 2 * h], -250.0f), 8.0f), 128.0f, 32000.0f));
#pragma unroll
              for (int i = 0; i < G / 2; ++i) largest[i] = max_u16x2(largest[i], vsw[hf][h][i] + up * 0x10001u);
            }
#pragma unroll
          for (int i = 0; i < G / 2; ++i)
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) largest[i] = max_u16x2(largest[i], __shfl_xor_sync(~0u, largest[i], d));
#pragma unroll
          for (int g = 0; g < G; ++g) {
            const float size = fmaf(static_cast<float>((g & 1) ? largest[g >> 1] >> 16 : largest[g >> 1] & 0xffffu), 1.0f / 128.0f, -377.0f);
            float& unit = mul[nt][j][g];
            if (moves || (unit != 0.0f && size > unit_exponent(unit) + kUnitRoom)) {
              float f;
              unit = new_unit(unit, size, &f);
#pragma unroll
              for (int i = 2 * g; i < 2 * g + 2; ++i) { o[nt][i][j] *= f; o[nt][i][j + 2] *= f; }
            }
          }
        }
#pragma unroll
      for (int i = 0; i < G / 2; ++i) {
        int most[2] = {0x7fff, 0x7fff};      // (a unit's exponent is -100 at least: so is the room, and no half below runs over)
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              const float unit = mul[nt][j][2 * i + e];
              if (unit != 0.0f) most[e] = min(most[e], (unit_exponent(unit) + static_cast<int>(kUnitRoom) + 127) * 128);
            }
        room[i] = 0x80008000u - static_cast<uint32_t>(most[1] << 16 | most[0]);
      }
    }
    // probabilities; P and P s, turned into second operands; out
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      const uint32_t c = c0 + hf * C::kBytes;
      uint32_t pv[NT][G][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float pr[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) pr[j] = ex2(rise[hf][nt][j]);
        l[nt][0] += pr[0] + pr[2];
        l[nt][1] += pr[1] + pr[3];
        // (P in two bf16 terms, 16 bits: far from zero the centres carry the result, and the sum of P beside it is of fp32.  One term was 3 % faster.)
        const uint32_t p0 = pack_bf16(pr[0], pr[1]), p1 = pack_bf16(pr[2], pr[3]);
        mma_bf16(oz[nt], vz[hf][0], 0u, vz[hf][1], 0u, transpose8x8(p0), transpose8x8(p1));
        mma_bf16(oz[nt], vz[hf][0], 0u, vz[hf][1], 0u, transpose8x8(pack_bf16(pr[0] - bf16_lo(p0), pr[1] - bf16_hi(p0))),
                 transpose8x8(pack_bf16(pr[2] - bf16_lo(p1), pr[3] - bf16_hi(p1))));
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
          for (int g = 0; g < G; ++g) {
            const float s = (g & 1) ? bf16_hi(vsw[hf][h][g >> 1]) : bf16_lo(vsw[hf][h][g >> 1]);
            const float2 in_unit = mul_pair(make_float2(pr[2 * h], pr[2 * h + 1]), make_float2(mul[nt][0][g], mul[nt][1][g]));
            const float2 ps = mul_pair(in_unit, make_float2(s, s));
            pv[nt][g][h] = transpose8x8(pack_f16(ps.x, ps.y));
          }
        }
      }
#pragma unroll
      for (int a = 0; a < kTiles / 4; ++a) {
        const uint4 w = lds128(c + C::kV + (a * 32 + lane) * 16);
        const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t u[4];
          codes8(consts, ww[i], u);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
            mma_f16(o[nt][4 * a + i], u[0], u[1], u[2], u[3], pv[nt][2 * a + (i >> 1)][0], pv[nt][2 * a + (i >> 1)][1]);
        }
      }
    }
  }

  __device__ __forceinline__ void end(const AttendParams& p, const Cursor& at, bool whole, float* part) {
    constexpr int kPart = D + 4;
    const int64_t out_seq = static_cast<int64_t>(p.rows) * p.n_heads * D;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float sum = l[nt][j];
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) sum += __shfl_xor_sync(~0u, sum, d);
        const int in_tile = nt * 8 + 2 * t + j, row = at.tile * kRows + in_tile;
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        uint16_t* const dst = p.out + at.seq * out_seq + out_row(p, row, at.head) * D;
#pragma unroll
        for (int g = 0; g < G; ++g) {
          const float z = __shfl_sync(~0u, oz[nt][j], g * 4 + t), unit = mul[nt][j][g] == 0.0f ? 1.0f : 1.0f / mul[nt][j][g];
          float v[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] = fmaf(o[nt][2 * g + (i >> 1)][j + 2 * (i & 1)], unit, z);
          if (row < p.rows) {
            const int d0 = 32 * g + 4 * r;
            if (whole)
              *reinterpret_cast<uint2*>(dst + d0) = make_uint2(pack_bf16(v[0] * inv, v[1] * inv), pack_bf16(v[2] * inv, v[3] * inv));
            else
              *reinterpret_cast<float4*>(part + in_tile * kPart + 4 + d0) = make_float4(v[0], v[1], v[2], v[3]);
          }
        }
        if (!whole && row < p.rows && r == 0)
          *reinterpret_cast<float2*>(part + in_tile * kPart) = make_float2(m[nt][j] == kNone ? -INFINITY : m[nt][j], sum);
      }
  }
};

// The same for one or two query rows (one query token, a K / V head to each query head or two): the 8 columns are the groups of
// 32 channels times two rows, so a lane deals with one group - columns 2t, 2t + 1: group t - and with a quarter of the
// scales, centres and products that the layout above gives every lane.  (64 channels have two groups: the other half of the columns
// is a copy.)  A column's product with another group's channels is zero (logits: its operand is) or not used (out).
template <int D, int R>
struct Narrow {
  using C = Chunk<D>;
  static constexpr int kD = D, G = D / 32, kTiles = D / 16, kRows = R;
  static constexpr bool kEarly = true;
  static constexpr int kWarps = 12, kStages = 2 * (128 / D);   // (16 warps of 128 registers, or three pairs in flight: no faster)

  uint32_t qf[G][4];            // q as the second operand, zero outside the column's group: [2 m + {0, 1}], odd channels over 16
  float qs[R], qo[2];           // sums of q over this lane's group, and those that take the offsets off, of its columns
  float cs[R], m[R], l[R], oz[R];
  float o[kTiles][4];
  float mul[R], most;           // 2^-E of this lane's columns; log2 of the P s that their units have room for
  int32_t least, len;
  uint4 next_q;
  int32_t next_len;
  Consts consts;
  int lane, r, t;

  __device__ __forceinline__ void init() {
    lane = threadIdx.x & 31; r = lane >> 2; t = lane & 3;
    consts = make_consts();
  }

  // asks for a unit's queries and its length, while the one before is finished: this lane's part of the second operand, column
  // n = lane / 4, channels 8 t .. + 7 of its group
  __device__ __forceinline__ void fetch(const AttendParams& p, const Cursor& at) {
    const int n = lane >> 2, group = (n >> 1) & (G - 1);
    next_len = p.len[at.seq];
    next_q = __ldg(reinterpret_cast<const uint4*>(q_row(p, at.seq, at.head, R == 2 ? n & 1 : 0) + group * 64 + t * 16));
  }

  __device__ __forceinline__ void begin(const AttendParams& p, const Cursor& at) {
    len = clamp_len(p, next_len);
    least = p.causal ? max(0, len - p.n_q + 1) : len;
    const int n = lane >> 2, group = (n >> 1) & (G - 1);
    const uint32_t ww[4] = {next_q.x, next_q.y, next_q.z, next_q.w};
    float f[8], top = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = bf16_lo(ww[i]);
      f[2 * i + 1] = bf16_hi(ww[i]);
      top = fmaxf(top, fmaxf(fabsf(f[2 * i]), fabsf(f[2 * i + 1])));
    }
    top = fmaxf(top, __shfl_xor_sync(~0u, top, 1));
    top = fmaxf(top, __shfl_xor_sync(~0u, top, 2));
    top = fmaxf(top, __shfl_xor_sync(~0u, top, 8));
    top = fmaxf(top, __shfl_xor_sync(~0u, top, 16));
    const int e = min(max(static_cast<int>((__float_as_uint(top) >> 23) & 0xff) - 127, -98), 127);   // largest member to [2^14, 2^15)
    const float up = __uint_as_float(static_cast<uint32_t>(127 + 14 - e) << 23);
    const float back = log2_per_product(p, e - 14 + kCodeLog2);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] *= up;
    float sum = (((f[1] + f[3]) + (f[5] + f[7])) + ((f[0] + f[2]) + (f[4] + f[6]))) * kCodeUnit;
    sum += __shfl_xor_sync(~0u, sum, 1);
    sum += __shfl_xor_sync(~0u, sum, 2);
    const float off = -8.0f * sum;
    const bool used = R == 2 || (n & 1) == 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t v = (i & 1) ? pack_f16(f[i] * 0.0625f, f[i + 4] * 0.0625f) : pack_f16(f[i], f[i + 4]);
#pragma unroll
      for (int g = 0; g < G; ++g) qf[g][i] = g == group && used ? v : 0u;
    }
    // to the lanes that own the columns' products
    qo[1] = 0.0f;
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const int from = (2 * t + j) * 4;
      qs[j] = __shfl_sync(~0u, sum, from);
      qo[j] = __shfl_sync(~0u, off, from);
      cs[j] = __shfl_sync(~0u, back, from);
      l[j] = 0.0f; m[j] = kNone; oz[j] = 0.0f; mul[j] = 0.0f;
    }
#pragma unroll
    for (int i = 0; i < kTiles; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) o[i][j] = 0.0f;
    most = INFINITY;
  }

  __device__ __forceinline__ void pair(const AttendParams& p, const Cursor& at, uint32_t c0, uint32_t gone) {
    const int g = t & (G - 1);
    const int key0 = at.chunk * kChunkTokens;
    float s[2][2][R];          // logits of tokens 2r, 2r + 1 of both chunks: this lane's group's part, then the whole
    uint32_t vsb[2][2];        // V scales (bf16 bits) and centres of this lane's tokens and group
    float vz[2][2];
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      const uint32_t c = c0 + hf * C::kBytes;
      float a[4] = {qo[0], qo[1], qo[0], qo[1]};
      uint32_t kw[2][G];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t cw = c + C::kK + (r + 8 * h) * (D / 2) + t * (4 * G);
        if (G == 4) {
          const uint4 w = lds128(cw);
          kw[h][0] = w.x; kw[h][1] = w.y; kw[h][G - 2] = w.z; kw[h][G - 1] = w.w;
        } else {
          const uint2 w = lds64(cw);
          kw[h][0] = w.x; kw[h][1] = w.y;
        }
      }
#pragma unroll
      for (int i = 0; i < G; ++i) {
        uint32_t u0[4], u1[4];
        nibbles8(consts, kw[0][i], u0);
        nibbles8(consts, kw[1][i], u1);
        mma_f16(a, u0[0], u1[0], u0[1], u1[1], qf[i][0], qf[i][1]);
        mma_f16(a, u0[2], u1[2], u0[3], u1[3], qf[i][2], qf[i][3]);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t cz = c + C::kKsz + (r + 8 * h) * (4 * G) + 2 * g;
        const float ks = bf16_lo(lds16(cz)), kz = bf16_lo(lds16(cz + 2 * G));
#pragma unroll
        for (int j = 0; j < R; ++j) {
          s[hf][h][j] = fmaf(ks, a[2 * h + j], kz * qs[j]);
        }
        vsb[hf][h] = lds16(c + C::kVs + (r + 8 * h) * (2 * G) + 2 * g);
        vz[hf][h] = bf16_lo(lds16(c + C::kVz + g * 32 + (r + 8 * h) * 2));
      }
    }
#pragma unroll
    for (int hf = 0; hf < 2; ++hf)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < R; ++j) {
          s[hf][h][j] += __shfl_xor_sync(~0u, s[hf][h][j], 1);
          if (G == 4) s[hf][h][j] += __shfl_xor_sync(~0u, s[hf][h][j], 2);
        }
    if (gone != 0 || key0 + 2 * kChunkTokens > least) {
      // hidden keys: logits at -inf, and nothing of bytes that were never written
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        const int base = key0 + hf * kChunkTokens;
        const int end = (gone >> hf) & 1u ? base : len;        // keys of the chunk that are there end here
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int key = base + 2 * r + h;
#pragma unroll
          for (int j = 0; j < R; ++j)
            if (key >= (p.causal ? min(end, len - p.n_q + 1 + token_of(p, j)) : end)) s[hf][h][j] = -INFINITY;
          if (key >= end) { vsb[hf][h] = 0u; vz[hf][h] = 0.0f; }
        }
      }
    }
    // a logit far above the stabiliser, or P s above its unit's room: move them (rare after the first chunks)
    float high = -INFINITY;
#pragma unroll
    for (int hf = 0; hf < 2; ++hf)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < R; ++j) high = fmaxf(high, fmaf(s[hf][h][j], cs[j], -m[j]));
    uint32_t vs_top = max(max(vsb[0][0], vsb[0][1]), max(vsb[1][0], vsb[1][1]));
    if (__any_sync(~0u, high > 8.0f || high + scale_log2(vs_top) > most || vs_top >= 0x7f80u)) {
      // A NaN for a scale: NaN in its group's channels (by way of the centres) for the rows that see the key, and the key's
      // scale is zero from here on: a row that does not see it has P = 0, and 0 x NaN would be one.
#pragma unroll
      for (int hf = 0; hf < 2; ++hf)
#pragma unroll
        for (int h = 0; h < 2; ++h)
          if (vsb[hf][h] > 0x7f80u) {
            vsb[hf][h] = 0;
#pragma unroll
            for (int j = 0; j < R; ++j)
              if (s[hf][h][j] != -INFINITY) oz[j] = __uint_as_float(0x7fffffffu);
          }
      most = INFINITY;
#pragma unroll
      for (int j = 0; j < R; ++j) {
        float top = fmaxf(fmaxf(s[0][0][j], s[0][1][j]) * cs[j], fmaxf(s[1][0][j], s[1][1][j]) * cs[j]);
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
        const bool moves = top > m[j] + 8.0f;
        if (moves) {
          const float f = ex2(m[j] - top);
          m[j] = top;
          l[j] *= f;
          oz[j] *= f;
#pragma unroll
          for (int i = 0; i < kTiles; ++i) { o[i][j] *= f; o[i][j + 2] *= f; }
        }
        float largest = -INFINITY;     // log2 of P s
#pragma unroll
        for (int hf = 0; hf < 2; ++hf)
#pragma unroll
          for (int h = 0; h < 2; ++h) largest = fmaxf(largest, fmaf(s[hf][h][j], cs[j], -m[j]) + scale_log2(vsb[hf][h]));
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) largest = fmaxf(largest, __shfl_xor_sync(~0u, largest, d));
        if (moves || (mul[j] != 0.0f && largest > unit_exponent(mul[j]) + kUnitRoom)) {
          float f;
          mul[j] = new_unit(mul[j], largest, &f);
#pragma unroll
          for (int i = 0; i < kTiles; ++i) { o[i][j] *= f; o[i][j + 2] *= f; }
        }
        if (mul[j] != 0.0f) most = fminf(most, unit_exponent(mul[j]) + kUnitRoom);
      }
    }
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      const uint32_t c = c0 + hf * C::kBytes;
      uint32_t pv[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float vs = __uint_as_float(vsb[hf][h] << 16);
        float u[2] = {0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < R; ++j) {
          const float pr = ex2(fmaf(s[hf][h][j], cs[j], -m[j]));
          l[j] += pr;
          oz[j] = fmaf(pr, vz[hf][h], oz[j]);
          u[j] = pr * mul[j] * vs;
        }
        pv[h] = transpose8x8(pack_f16(u[0], u[1]));
      }
#pragma unroll
      for (int a = 0; a < kTiles / 4; ++a) {
        const uint4 w = lds128(c + C::kV + (a * 32 + lane) * 16);
        const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t u[4];
          codes8(consts, ww[i], u);
          mma_f16(o[4 * a + i], u[0], u[1], u[2], u[3], pv[0], pv[1]);
        }
      }
    }
  }

  __device__ __forceinline__ void end(const AttendParams& p, const Cursor& at, bool whole, float* part) {
    constexpr int kPart = D + 4;
    const int64_t out_seq = static_cast<int64_t>(p.rows) * p.n_heads * D;
#pragma unroll
    for (int j = 0; j < R; ++j) {
      float sum = l[j], z = oz[j];
#pragma unroll
      for (int d = 4; d < 32; d <<= 1) {
        sum += __shfl_xor_sync(~0u, sum, d);
        z += __shfl_xor_sync(~0u, z, d);
      }
      const float unit = mul[j] == 0.0f ? 1.0f : 1.0f / mul[j];
      float v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[i] = o[i >> 1][j + 2 * (i & 1)];
#pragma unroll
        for (int g = 1; g < G; ++g) v[i] = pick(t == g, o[2 * g + (i >> 1)][j + 2 * (i & 1)], v[i]);
        v[i] = fmaf(v[i], unit, z);
      }
      const int d0 = 32 * t + 4 * r;
      if (whole) {
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        uint16_t* const dst = p.out + at.seq * out_seq + out_row(p, j, at.head) * D;
        if (t < G) *reinterpret_cast<uint2*>(dst + d0) = make_uint2(pack_bf16(v[0] * inv, v[1] * inv), pack_bf16(v[2] * inv, v[3] * inv));
      } else {
        if (t < G) *reinterpret_cast<float4*>(part + j * kPart + 4 + d0) = make_float4(v[0], v[1], v[2], v[3]);
        if (lane == 0) *reinterpret_cast<float2*>(part + j * kPart) = make_float2(m[j] == kNone ? -INFINITY : m[j], sum);
      }
    }
  }
};

template <typename Body>
struct Shared {   // dynamic shared memory of the kernel, from its start
  static constexpr int kPart = Body::kD + 4;    // floats of a partial result's row: stabiliser, sum, -, -, values
  static constexpr int kPair = 2 * Chunk<Body::kD>::kBytes;
  static constexpr int kWarpRing = Body::kStages * kPair;
  static constexpr int kHeadPart = Body::kRows * kPart * 4;             // bytes of a warp's first partial result
  static constexpr int kHeads = Body::kWarps * kWarpRing;
  static constexpr int kFirst = kHeads + Body::kWarps * kHeadPart;      // int32 [n_seq + 1]
  static_assert(Body::kRows * kPart * 4 <= kWarpRing, "a warp's last partial result lies in its ring");
};

template <typename Body>
__global__ void __launch_bounds__(32 * Body::kWarps, 1) page_attend_kernel(const AttendParams p) {
  using Sh = Shared<Body>;
  constexpr int D = Body::kD, kStages = Body::kStages, kWarps = Body::kWarps, kThreads = 32 * kWarps, kRows = Body::kRows;
  constexpr int kPart = Sh::kPart, kPair = Sh::kPair, kBytes = Chunk<D>::kBytes;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ __align__(8) uint64_t bars[kWarps][kStages];
  __shared__ int32_t warp_sum[2][kWarps];
  __shared__ long long ends_s[2];
  __shared__ int split_s[2];                    // CTAs of this CTA's unit (0: cut otherwise), and the first of them
  __shared__ int32_t part_unit[kWarps][2];      // unit of a warp's first / last partial result, -1: none
  __shared__ int join_from[2], join_parts[2];   // units this CTA joins across CTAs: the first CTA, the number of parts (0: not this CTA)
  __shared__ __align__(16) float join_s[kWarps][kPart];
  int32_t* const first = reinterpret_cast<int32_t*>(smem + Sh::kFirst);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t bar0 = smem_u32(&bars[warp][0]);
  const uint32_t ring = smem_u32(smem) + warp * Sh::kWarpRing;
  if (lane == 0) {
    for (int i = 0; i < kStages; ++i) mbar_init(bar0 + 8 * i);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async;" ::: "memory");
  }
  if (lane < 2) part_unit[warp][lane] = -1;
  pdl_wait();     // (and no early start of the call that follows: its CTAs would crowd onto the SMs that finish first)

  // chunks (per unit) of the sequences before each one: 32 bits, as the host refuses more; the line has 64
  int32_t carry = 0, longest = 0;
  for (int base = 0; base < p.n_seq; base += kThreads) {
    const int s = base + threadIdx.x;
    int32_t v = 0;
    if (s < p.n_seq) {
      const int32_t given = p.len[s], n = clamp_len(p, given);
      v = chunks_of(n);
      if (blockIdx.x == 0 && n != given) record_status(p.workspace, MUSTDROP_ERR_BAD_LENGTH, s);
    }
    const int32_t top = __reduce_max_sync(~0u, v);
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int32_t u = __shfl_up_sync(~0u, v, d);
      if (lane >= d) v += u;
    }
    if (base > 0) __syncthreads();
    if (lane == 31) { warp_sum[0][warp] = v; warp_sum[1][warp] = top; }
    __syncthreads();
    int32_t all = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const int32_t u = warp_sum[0][w];
      if (w < warp) v += u;
      all += u;
      longest = max(longest, warp_sum[1][w]);
    }
    if (s < p.n_seq) first[s + 1] = carry + v;
    carry += all;
  }
  if (threadIdx.x == 0) first[0] = 0;
  __syncthreads();
  const int units_per_seq = p.n_heads * p.tiles;
  const int64_t out_seq = static_cast<int64_t>(p.rows) * p.n_heads * D;      // elements of out per sequence

  // ---------------------------------------------------------------- sequences without keys: zeros
  for (int s = blockIdx.x; s < p.n_seq; s += gridDim.x)
    if (first[s + 1] == first[s])
      for (int64_t i = threadIdx.x; i < out_seq / 8; i += kThreads)
        *reinterpret_cast<uint4*>(p.out + s * out_seq + i * 8) = make_uint4(0, 0, 0, 0);
  if (carry == 0) return;

  // This CTA's part of the line: an equal one, except that
  //   - where every unit can have a CTA of its own and no warp then gets more than eight chunks more than with equal parts, it has: nothing is
  //     joined across CTAs (one request, 32 heads, 640 keys: 7.5 us against 12.3);
  //   - where every unit can have a whole number of CTAs and parts get at most 38 chunks longer by that (2 us), they have: a CTA then
  //     has a part of one unit only, and joins are one instead of two in a row.  (One request, 8 heads of 4 query heads, 8192 keys: 13.3 us
  //     against 17.7, 131072 keys: 46.1 against 48.4; one of 32 heads, 4096 keys: 12.6 against 14.7; what it cannot help pays up to 0.4 us.)  No warp gets less than a pair of chunks for it: more
  //     parts are only more to join (2 heads of 4, 3000 keys: 11.6 us; with two pairs at least 13.1).
  //   - where that makes parts at most 72 chunks longer (4 us), their ends move to the nearest unit's, for the same reason: a join across
  //     CTAs takes 3 to 5 us.  (The nearest shape that loses by it would grow by 78 chunks.)  With units of one length, or few of them to a part, a part is then a whole number of the longest; with many
  //     of different lengths it is about half a unit longer.  (64 requests of 200 to 1800 keys, 32 heads: 69.2 against 72.8 us, 9 of 2048 keys:
  //     23.6 against 27.9, 6 of 700: 11.5 against 15.0; but 16 of 1000 to 4000: 55.5 against 49.7.)
  const long long total = static_cast<long long>(carry) * units_per_seq;
  const Cut cut = cut_of(total, gridDim.x);
  const bool few = static_cast<long long>(p.n_seq) * units_per_seq <= gridDim.x;
  int split = 0;                    // CTAs of the unit that this CTA has a part of; 0: one of the other cuts
  long long line0 = 0, line1 = 0;
  if (few && p.n_seq <= 32 && longest > cut.per + 6 * kWarps) {
    // the shortest parts, of 32 lengths, with which that many CTAs do (lane s has sequence s; in quotients that may be one too large)
    const uint32_t n = lane < p.n_seq ? first[lane + 1] - first[lane] : 0, least = max(cut.per, 2 * kWarps), part = least + lane + lane / 4;
    const uint32_t inv = 0xffffffffu / part + 1;
    auto parts_of = [](uint32_t n, uint32_t part, uint32_t inv) { return n == 0 ? 0u : max(1u, __umulhi(n + part - 1, inv)); };
    const uint32_t longest_inv = __shfl_sync(~0u, inv, 31), longest_part = least + 38;
    if (__reduce_add_sync(~0u, parts_of(n, longest_part, longest_inv)) * units_per_seq <= gridDim.x) {
      uint32_t ctas = 0;
#pragma unroll 4
      for (int s = 0; s < p.n_seq; ++s) ctas += parts_of(__shfl_sync(~0u, n, s), part, inv);
      const int fit = __ffs(__ballot_sync(~0u, ctas * units_per_seq <= gridDim.x)) - 1;     // (lane 31's does)
      const uint32_t k = parts_of(n, __shfl_sync(~0u, part, fit), __shfl_sync(~0u, inv, fit));
      uint32_t upto = k * units_per_seq;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const uint32_t u = __shfl_up_sync(~0u, upto, d);
        if (lane >= d) upto += u;
      }
      const int s = __popc(__ballot_sync(~0u, upto <= blockIdx.x));
      if (s >= p.n_seq) return;
      split = __shfl_sync(~0u, k, s);
      const int at = blockIdx.x - (__shfl_sync(~0u, upto, s) - split * units_per_seq), unit = at / split, i = at - unit * split;
      const int chunks = __shfl_sync(~0u, n, s);
      const Cut of_unit = cut_of(chunks, split);
      line0 = static_cast<long long>(first[s]) * units_per_seq + static_cast<long long>(unit) * chunks + of_unit.begin(i);
      line1 = line0 + of_unit.per + (i < of_unit.more ? 1 : 0);
      if (threadIdx.x == 0) { split_s[0] = split; split_s[1] = blockIdx.x - i; }
    }
  }
  const bool own_unit = split == 0 && few && longest <= cut.per + 8 * kWarps;
  const int longer = static_cast<long long>(longest) * p.n_seq == carry || cut.per / 4 < longest ? (cut.per + longest - 1) / longest * longest - cut.per : carry / p.n_seq / 2;
  const bool whole_units = own_unit || (split == 0 && longer <= 72);
  auto unit_begin = [&](int unit, int* n) {
    const int seq = unit / units_per_seq;
    *n = first[seq + 1] - first[seq];
    return static_cast<long long>(first[seq]) * units_per_seq + static_cast<long long>(unit - seq * units_per_seq) * *n;
  };
  // the sequence that has place x of the line (x < total): first[s] * units <= x < first[s + 1] * units
  auto seq_of = [&](long long x) {
    int lo = 0;
    for (int n = p.n_seq; n > 1;) {          // among sequences lo .. lo + n - 1; a step of 32 ways
      const int width = (n + 31) / 32, s = lo + (lane + 1) * width;
      const int past = __popc(__ballot_sync(~0u, (lane + 1) * width < n && static_cast<long long>(first[s]) * units_per_seq <= x));
      lo += past * width;
      n = min(width, n - past * width);
    }
    return lo;
  };
  if (split > 0) {
    // (done)
  } else if (own_unit) {
    if (static_cast<int>(blockIdx.x) >= p.n_seq * units_per_seq) return;
    int n;
    line0 = unit_begin(blockIdx.x, &n);
    line1 = line0 + n;
  } else {
    if (static_cast<int>(blockIdx.x) >= cut.ctas) return;
    line0 = cut.begin(blockIdx.x);
    line1 = cut.begin(blockIdx.x + 1);
    if (whole_units) {
      if (warp < 2) {                            // an end each
        long long x = warp == 0 ? line0 : line1;
        if (x != total) {
          const int s = seq_of(x), n = first[s + 1] - first[s];
          const long long base = static_cast<long long>(first[s]) * units_per_seq;
          x = base + Cut::divide(x - base + n / 2, n) * n;
        }
        if (lane == 0) ends_s[warp] = x;
      }
      __syncthreads();
      line0 = ends_s[0];
      line1 = ends_s[1];
    }
  }
  if (split == 0 && threadIdx.x == 0) split_s[0] = 0;
  if (line0 == line1) return;
  // Its warps share it by pairs of chunks.
  const int pairs = static_cast<int>((line1 - line0 + 1) / 2), n_warps = min(pairs, kWarps);
  const int per_warp = pairs / n_warps, more = pairs - per_warp * n_warps;
  auto warp_begin = [&](int w) { return min(line0 + 2 * (static_cast<long long>(per_warp) * w + min(w, more)), line1); };

  if (warp < n_warps) {
    Cursor at;       // where the warp computes
    {
      const long long begin = warp_begin(warp);
      const int lo = seq_of(begin);
      const long long rem = begin - static_cast<long long>(first[lo]) * units_per_seq;
      const int n = first[lo + 1] - first[lo];
      const int unit = static_cast<int>(Cut::divide(rem, n));
      at.seq = lo;
      at.chunk = static_cast<int>(rem - static_cast<long long>(unit) * n);
      at.head = p.tiles == 1 ? unit : unit / p.tiles;
      at.tile = unit - at.head * p.tiles;
      at.rest = static_cast<int>(warp_begin(warp + 1) - begin);
      at.left = min(at.rest, n - at.chunk);
      at.rest -= at.left;
    }
    const int per_page = p.lg - 4;           // log2 of the chunks per page
    const uint32_t in_page = (1u << per_page) - 1;
    Body body;
    body.init();
    body.fetch(p, at);

    // Copies run kStages pairs of chunks ahead of the computation, page ids one pair further.  Lanes 0 and 1 have a chunk each.
    Cursor ahead = at;
    struct Ask { int32_t id, off, n; };      // page id and place in the page of this lane's chunk, chunks of the pair (0: none is left)
    uint32_t bad = ~0u;                      // two bits per stage: chunks that are on no page of the pool, or none at all
    auto ask = [&]() {
      Ask a = {-1, 0, 0};
      if (ahead.left == 0) {
        if (ahead.rest == 0) return a;
        next_unit(p, ahead, first);
      }
      a.n = min(ahead.left, 2);
      const int c = ahead.chunk + (lane & 1);
      if ((lane & 1) < a.n) a.id = __ldg(p.table + (ahead.seq * p.max_pages + (c >> per_page)));
      a.off = (ahead.head << per_page) + (c & in_page);
      ahead.chunk += a.n;
      ahead.left -= a.n;
      return a;
    };
    auto issue = [&](int stage, const Ask& a) {
      const bool fine = static_cast<uint32_t>(a.id) < static_cast<uint32_t>(p.n_pages);
      const uint32_t have = __ballot_sync(~0u, fine) & 3u;
      bad = (bad & ~(3u << (2 * stage))) | ((have ^ 3u) << (2 * stage));
      const uint32_t bar = bar0 + 8 * stage;
      if (lane == 0 && have != 0)
        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(have == 3u ? kPair : kBytes) : "memory");
      __syncwarp();
      if (lane < a.n) {
        if (fine)
          bulk_load(ring + stage * kPair + lane * kBytes,
                    p.pool + (((static_cast<int64_t>(a.id) * p.n_heads) << per_page) + a.off) * kBytes, kBytes, bar);
        else
          record_status(p.workspace, MUSTDROP_ERR_BAD_PAGE, a.id);
      }
    };
    Ask next;
    {
      Ask begin[kStages];
#pragma unroll
      for (int i = 0; i < kStages; ++i) begin[i] = ask();
      next = ask();
#pragma unroll
      for (int i = 0; i < kStages; ++i)
        if (begin[i].n > 0) issue(i, begin[i]);
    }

    int stage = 0;
    uint32_t phase = 0;
    bool ok = true;
    while (true) {
      const bool from_start = at.chunk == 0;
      body.begin(p, at);
      while (at.left > 0) {
        const uint32_t gone = (bad >> (2 * stage)) & 3u;
        if (gone != 3u) {
          // (one answer for the warp, as what follows needs all its lanes: every lane has a clock of its own to give up by)
          const bool landed = mbar_wait(bar0 + 8 * stage, (phase >> stage) & 1u) && ((p.give_up >> lane) & 1u) == 0;
          if (!__all_sync(~0u, landed)) { ok = false; break; }
          phase ^= 1u << stage;
          body.pair(p, at, ring + stage * kPair, gone);
        }
        const int n = min(at.left, 2);
        at.chunk += n;
        at.left -= n;
        // the stage is free: the pair kStages further on
        __syncwarp();
        if (next.n > 0) {
          issue(stage, next);
          next = ask();
        } else {
          bad |= 3u << (2 * stage);
        }
        stage = stage + 1 == kStages ? 0 : stage + 1;
      }
      if (!ok) break;
      // the unit, or the warp's part, ends: results out
      const Cursor was = at;
      if (at.rest > 0) {
        next_unit(p, at, first);
        if (Body::kEarly) body.fetch(p, at);
      }
      const bool whole = from_start && was.chunk == first[was.seq + 1] - first[was.seq];
      if (!whole && lane == 0) part_unit[warp][from_start] = (was.seq * p.n_heads + was.head) * p.tiles + was.tile;
      // A unit that began before the warp is its first; one that it leaves unfinished is its last: then its ring is idle.
      body.end(p, was, whole, reinterpret_cast<float*>(smem + (from_start ? warp * Sh::kWarpRing : Sh::kHeads + warp * Sh::kHeadPart)));
      if (at.left == 0) break;
      if (!Body::kEarly) body.fetch(p, at);
    }
    if (!ok) {
      // gave up: leave only when the copies in flight have landed (bounded)
      if (lane == 0) record_status(p.workspace, MUSTDROP_ERR_TIMEOUT, blockIdx.x);
      for (int i = 0; i < kStages; ++i)
        if (((bad >> (2 * i)) & 3u) != 3u) (void)mbar_wait(bar0 + 8 * i, (phase >> i) & 1u);
    }
  }

  // ---------------------------------------------------------------- joining
  // Parts of a unit in this CTA: the last one of the warp it begins in (none, if it began before the CTA), then the first ones of
  // the warps that follow.  With few rows a warp joins the unit that begins in it, warp 0 also the one that began before the CTA; with
  // more, or where the CTA has parts of one unit only, the warps share the rows of one unit after the other.  A unit whose parts are all
  // here gets its output; of the others - at most the one the CTA begins in and the one it ends in - the CTA leaves one part for the
  // CTA that comes last.
  __syncthreads();
  auto write_out = [&](int unit, int in_tile, const RowSum& s) {
    const int seq = unit / units_per_seq, u = unit - seq * units_per_seq;
    const int head = p.tiles == 1 ? u : u / p.tiles, row = (u - head * p.tiles) * kRows + in_tile;
    const float inv = s.l == 0.0f ? 0.0f : 1.0f / s.l;
    if (lane < D / 4)
      *reinterpret_cast<uint2*>(p.out + seq * out_seq + out_row(p, row, head) * D + 4 * lane) =
          make_uint2(pack_bf16(s.v.x * inv, s.v.y * inv), pack_bf16(s.v.z * inv, s.v.w * inv));
  };
  auto rows_of = [&](int unit) { return p.tiles == 1 ? p.rows : min(kRows, p.rows - (unit % p.tiles) * kRows); };
  int open[2];                      // units of the parts this CTA leaves: that began before it, that begins in it; -1: none
  {
    const int heads = lane < kWarps ? part_unit[lane][0] : -1, tails = lane < kWarps ? part_unit[lane][1] : -1;
    const uint32_t begun = __ballot_sync(~0u, tails >= 0);         // warps in which a unit begins that they leave unfinished
    open[0] = __shfl_sync(~0u, heads, 0);
    open[1] = begun != 0 ? __shfl_sync(~0u, tails, 31 - __clz(begun)) : -1;
    if (open[1] >= 0) {
      int chunks;
      if (unit_begin(open[1], &chunks) + chunks <= line1) open[1] = -1;
    }
    const bool shared = kRows > 2 || __popc(begun) + (open[0] >= 0 ? 1 : 0) == 1;
    // bit w + 1: join the unit that begins in warp w; bit 0: the one that began before the CTA
    uint32_t mine = (shared ? begun << 1 : begun & (1u << warp) ? 2u << warp : 0u) | ((shared || warp == 0) && open[0] >= 0 ? 1u : 0u);
    for (; mine != 0; mine &= mine - 1) {
      const int w = __ffs(mine) - 2, lead = w >= 0 ? 1 : 0;
      const int unit = lead == 0 ? open[0] : __shfl_sync(~0u, tails, w);
      const uint32_t in = __ballot_sync(~0u, heads == unit);
      const int n = lead + __popc(in), w1 = w + 1;
      const bool leave = unit == open[lead];
      const int rows = rows_of(unit);
      for (int row = shared ? warp : 0; row < rows; row += shared ? kWarps : 1) {
        const RowSum s = join_row<D, false>(n, [&](int k) {
          const int at = k < lead ? w * Sh::kWarpRing : Sh::kHeads + (w1 + k - lead) * Sh::kHeadPart;
          return reinterpret_cast<const float*>(smem + at) + row * kPart;
        }, lane);
        if (!leave) {
          write_out(unit, row, s);
        } else {
          float* const to = p.part + static_cast<size_t>((2 * blockIdx.x + lead) * p.part_rows + row) * kPart;
          if (lane < D / 4) *reinterpret_cast<float4*>(to + 4 + 4 * lane) = s.v;
          if (lane == 0) *reinterpret_cast<float2*>(to) = make_float2(s.m, s.l);
        }
      }
    }
  }
  if (open[0] < 0 && open[1] < 0) return;
  __syncthreads();
  // the counter of a unit is its first CTA's
  if (threadIdx.x < 2) {
    const int unit = open[threadIdx.x];
    int parts = 0;
    if (unit >= 0) {
      int n;
      const long long b = unit_begin(unit, &n);
      const int k = split_s[0], c0 = k > 0 ? split_s[1] : cut.owner(b);
      parts = k > 0 ? k : cut.owner(b + n - 1) - c0 + 1;
      join_from[threadIdx.x] = c0;
      // (release: this CTA's part, ordered before by the barrier; acquire: the others')
      unsigned seen;
      asm volatile("atom.acq_rel.gpu.global.inc.u32 %0, [%1], %2;" : "=r"(seen) : "l"(p.joined + c0), "r"(parts - 1) : "memory");
      if (seen != static_cast<unsigned>(parts - 1)) parts = 0;
    }
    join_parts[threadIdx.x] = parts;
  }
  __syncthreads();
#pragma unroll 1
  for (int k = 0; k < 2; ++k) {
    const int parts = join_parts[k], c0 = join_from[k];
    if (parts == 0) continue;
    const int unit = k == 0 ? open[0] : open[1], rows = rows_of(unit);
    const int share = max(1, min(kWarps / rows, (parts + 7) / 8));   // warps of a row, each joining a run of the parts
    const int run = (parts + share - 1) / share;
    for (int base = 0; base < rows; base += kWarps / share) {
      const int row = base + warp / share, mine = warp % share;
      const bool busy = warp < (kWarps / share) * share && row < rows;
      const int from = min(mine * run, parts), to = min(from + run, parts);
      if (busy) {
        const RowSum s = join_row<D, true>(to - from, [&](int i) {
          const int c = c0 + from + i;
          return p.part + static_cast<size_t>((2 * c + (c == c0 ? 1 : 0)) * p.part_rows + row) * kPart;
        }, lane);
        if (share == 1) {
          write_out(unit, row, s);
        } else {
          if (lane < D / 4) *reinterpret_cast<float4*>(&join_s[warp][4 + 4 * lane]) = s.v;
          if (lane == 0) *reinterpret_cast<float2*>(&join_s[warp][0]) = make_float2(s.m, s.l);
        }
      }
      if (share > 1) {
        __syncthreads();
        if (busy && mine == 0) write_out(unit, row, join_row<D, false>(share, [&](int i) { return &join_s[warp + i][0]; }, lane));
        __syncthreads();
      }
    }
  }
}

// Query rows of a tile for `rows` of a unit.
int tile_rows(int64_t rows) { return rows <= 2 ? static_cast<int>(rows) : rows <= 8 ? 8 : 16; }

template <typename Body>
cudaError_t launch_attend(const AttendParams& p, int sms, cudaStream_t stream) {
  const size_t smem = Shared<Body>::kFirst + (static_cast<size_t>(p.n_seq) + 1) * sizeof(int32_t);
  const cudaError_t e = ensure_kernel_attributes(reinterpret_cast<const void*>(page_attend_kernel<Body>), false);
  if (e != cudaSuccess) return e;
  return launch_pdl(page_attend_kernel<Body>, dim3(static_cast<unsigned>(std::min(kMaxCtas, sms))), dim3(32 * Body::kWarps), smem, stream, p);
}

template <int D>
cudaError_t launch_attend(const AttendParams& p, int tile, int sms, cudaStream_t stream) {
  switch (tile) {
    case 1: return launch_attend<Narrow<D, 1>>(p, sms, stream);
    case 2: return launch_attend<Narrow<D, 2>>(p, sms, stream);
    case 8: return launch_attend<Wide<D, 1>>(p, sms, stream);
    default: return launch_attend<Wide<D, 2>>(p, sms, stream);
  }
}

}  // namespace

size_t page_attend_partial_bytes(const mustdrop_page_config_t* c) {
  const int64_t rows = static_cast<int64_t>(c->q_heads / c->n_heads) * c->n_q;
  const size_t part_rows = static_cast<size_t>(std::min<int64_t>(rows, tile_rows(rows)));
  const size_t bytes = static_cast<size_t>(kMaxCtas) * 2 * part_rows * (c->head_dim + 4) * sizeof(float);
  return kCountBytes + (bytes + 255) / 256 * 256;
}

}  // namespace mustdrop

extern "C" mustdrop_status_t mustdrop_page_attend(const mustdrop_page_config_t* c, const void* q, const void* pool,
                                                  const int32_t* page_table, const int32_t* len, void* out, void* workspace,
                                                  void* cuda_stream) {
  using namespace mustdrop;
  const mustdrop_status_t st = check_page_queries(c);
  if (st != MUSTDROP_OK) return st;
  if (c->max_pages <= 0 || c->causal < 0 || c->causal > 1 || !(c->scale >= 0.0f && c->scale <= 1.0e37f)) return MUSTDROP_ERR_INVALID_ARG;
  if (c->n_seq > kMaxSeqs || static_cast<int64_t>(c->max_pages) * c->page > (1 << 30)) return MUSTDROP_ERR_UNSUPPORTED;   // (token numbers, and a pair of chunks beyond them, in 32 bits)
  const int64_t rows = static_cast<int64_t>(c->q_heads / c->n_heads) * c->n_q;
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
  p.joined = reinterpret_cast<unsigned*>(static_cast<uint8_t*>(workspace) + kWsStatusBytes);
  p.part = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + kWsStatusBytes + kCountBytes);
  p.workspace = static_cast<int32_t*>(workspace);
  p.n_seq = c->n_seq; p.n_heads = c->n_heads; p.group = c->q_heads / c->n_heads; p.n_q = c->n_q;
  p.rows = static_cast<int32_t>(rows);
  p.group_magic = static_cast<uint32_t>((1ull << 32) / static_cast<uint32_t>(p.group)) + 1u;
  const int tile = tile_rows(rows);
  p.tiles = (p.rows + tile - 1) / tile;
  p.part_rows = std::min(p.rows, tile);
  if (static_cast<int64_t>(p.n_seq) * p.n_heads * p.tiles > INT32_MAX ||
      static_cast<int64_t>(p.n_heads) * p.tiles > (1ll << 36) / most)     // (a CTA's part of the line: 31 bits on 64 CTAs)
    return MUSTDROP_ERR_UNSUPPORTED;
  p.lg = page_log2(c->page); p.n_pages = c->n_pages; p.max_pages = c->max_pages; p.causal = c->causal;
  p.q_sh = 2 * (c->q_stride_h != 0 ? c->q_stride_h : c->head_dim);
  p.q_st = 2 * (c->q_stride_t != 0 ? c->q_stride_t : static_cast<int64_t>(c->q_heads) * c->head_dim);
  p.q_ss = 2 * (c->q_stride_s != 0 ? c->q_stride_s : static_cast<int64_t>(c->n_q) * c->q_heads * c->head_dim);
  const float scale = c->scale != 0.0f ? c->scale : (c->head_dim == 128 ? 0.08838834764831845f : 0.125f);
  p.scale_log2e = scale * 1.4426950408889634f;
  p.give_up = (c->flags & MUSTDROP_PAGE_FLAG_DEBUG_TIMEOUT) != 0 ? 0xaaaaaaaau : 0u;
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e == cudaSuccess) {
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    e = c->head_dim == 128 ? launch_attend<128>(p, tile, sms, stream) : launch_attend<64>(p, tile, sms, stream);
  }
  if (e == cudaSuccess) return MUSTDROP_OK;
  set_last_cuda_error(e);
  return MUSTDROP_ERR_CUDA;
}
