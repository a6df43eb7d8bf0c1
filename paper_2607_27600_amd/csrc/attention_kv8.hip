// Attention over a cache in 8 bits: o[i][h] = sum_j softmax_j(scale * q[i][h] . k[j][c]) v[j][c] over the
// entries j that the mask allows, c = h / g, with k and v the values code * 2^e of the cache.
//
// A row is one (query, query head of the group) pair, so the g heads that share a KV head share
// every entry that is read.  Two kernels, by the rows of a sequence and KV head:
//   few (up to FEW_ROWS rows: single tokens, drafts): bound by the bytes of the cache.  Each wave
//     streams entries of its own from memory into MFMA operands, no LDS in the loop.
//   many (chunks of a prompt, the scoring pass): bound by matrix and softmax work.  Blocks of 128
//     rows share tiles of 64 entries, converted once into bf16 tiles in LDS.
// Where few workgroups come of it, the entries of a sequence are cut into pieces and the pieces'
// (maximum, sum, output) are joined by a third kernel, in the pieces' order.
//
// Numbers.  E4M3 has 4 significant bits and the scales are powers of two, so entries become bf16
// exactly wherever it reaches, from 2^-126 to below 2^128 (one conversion instruction for two codes, scale
// included; scales of 2^-100 to 2^119 stay inside, from 2^120 on the largest elements are infinite); products
// accumulate in fp32; a row's maximum and sum are fp32, the reference maximum moving only when it is passed by 2^8
// (numerator and sum share it).  The probabilities are rounded to bf16 for the second product (each by
// up to 2^-8 of itself, independently: what the output's own rounding costs), the sum takes them unrounded.
//
// Masked entries.  Scores are replaced, not added to, so what a masked key holds is lost.  A masked
// value meets a probability of 0, and 0 times NaN or infinity would reach the output: values past the
// sequence are zeroed as they are read, and in tiles that some row sees in part, NaN codes and infinite
// elements are zeroed too and counted by a second product of indicators, by the rows that may see them, whose
// outputs become NaN (the kernel for many marks them instead).
#include <algorithm>

#include "attention_kv8.h"

namespace cc {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// Eight codes (two words) times the scale, in bf16: exact.
__device__ __forceinline__ bf16x8 widen8(uint32_t lo, uint32_t hi, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(int(lo), scale, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(int(lo), scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(int(hi), scale, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(int(hi), scale, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// The same where the two words have scales of their own.
__device__ __forceinline__ bf16x8 widen44(uint32_t lo, uint32_t hi, float slo, float shi) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(int(lo), slo, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(int(lo), slo, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(int(hi), shi, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(int(hi), shi, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// 4 x 4 bytes transposed: word i of the result holds byte i of w[0..3].
__device__ __forceinline__ void transpose4(const uint32_t (&w)[4], uint32_t (&t)[4]) {
  // perm(hi, lo, sel): byte k of the result is byte sel[k] of {lo: 0..3, hi: 4..7}
  const uint32_t a = __builtin_amdgcn_perm(w[1], w[0], 0x05010400u);   // w0.0 w1.0 w0.1 w1.1
  const uint32_t b = __builtin_amdgcn_perm(w[1], w[0], 0x07030602u);   // w0.2 w1.2 w0.3 w1.3
  const uint32_t c = __builtin_amdgcn_perm(w[3], w[2], 0x05010400u);
  const uint32_t d = __builtin_amdgcn_perm(w[3], w[2], 0x07030602u);
  t[0] = __builtin_amdgcn_perm(c, a, 0x05040100u);
  t[1] = __builtin_amdgcn_perm(c, a, 0x07060302u);
  t[2] = __builtin_amdgcn_perm(d, b, 0x05040100u);
  t[3] = __builtin_amdgcn_perm(d, b, 0x07060302u);
}

// A wave-uniform pointer in scalar registers.
__device__ __forceinline__ const char* uniform_ptr(const char* p) {
  const uint64_t u = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = __builtin_amdgcn_readfirstlane(uint32_t(u));
  const uint32_t hi = __builtin_amdgcn_readfirstlane(uint32_t(u >> 32));
  return reinterpret_cast<const char*>((uint64_t(hi) << 32) | lo);
}

// Maximum over the four lanes l % 16 + 16 k.
__device__ __forceinline__ float quad_max(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float quad_sum(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// A plane of the cache: one (sequence, layer, KV head); 16-entry groups lie in one page and one block.
struct Plane {
  const char *k, *v;           // layer and head (contiguous: sequence) part
  const uint8_t *ks, *vs;
  const int32_t* table;        // paged: the sequence's row of the block table
};
__device__ __forceinline__ Plane plane_of(const Kv8Args& a, int b, int h) {
  Plane P;
  const int64_t c = int64_t(a.layer) * a.k.codes.layer_stride + int64_t(h) * a.k.codes.head_stride +
                    (a.k.paged ? 0 : int64_t(b) * a.k.codes.seq_stride);
  const int64_t s = int64_t(a.layer) * a.k.s_layer + int64_t(h) * a.k.s_head + (a.k.paged ? 0 : int64_t(b) * a.k.s_seq);
  P.k = static_cast<const char*>(a.k.codes.base) + c;
  P.v = static_cast<const char*>(a.v.codes.base) + c;
  P.ks = a.k.scale + s;
  P.vs = a.v.scale + s;
  P.table = a.k.codes.block_table + (a.k.paged ? int64_t(b) * a.k.codes.max_pages : 0);
  return P;
}
// Page of the group (contiguous: none), where its codes start, where its scale lies.
__device__ __forceinline__ int group_page(const Kv8Args& a, const Plane& P, int group) {
  return a.k.paged ? P.table[group >> (a.k.codes.page_shift - 4)] : 0;
}
__device__ __forceinline__ int64_t group_codes(const Kv8Args& a, int page, int group) {
  const int slot = a.k.paged ? (group << 4) & a.k.codes.page_mask : group << 4;
  return int64_t(page) * a.k.codes.page_stride + int64_t(slot) * a.k.codes.tok_stride;
}
__device__ __forceinline__ int64_t group_scale(const Kv8Args& a, int page, int group) {
  const int slot = a.k.paged ? (group << 4) & a.k.codes.page_mask : group << 4;
  return int64_t(page) * a.k.s_page + (slot >> a.k.block_shift);
}

// The sequence of a workgroup's item and what its rows may see.
struct Seq {
  int b, q0, m, len, shift;    // shift: cache position of query 0
};
__device__ __forceinline__ Seq seq_of(const Kv8Args& a, int j) {
  Seq s;
  s.b = a.listed ? a.list[j] : j;
  s.q0 = a.cu[s.b];
  s.m = a.cu[s.b + 1] - s.q0;
  s.len = min(max(a.lens[s.b], 0), a.max_len);
  s.shift = s.len - s.m;
  return s;
}
// First and past-the-last entry that query i may see.
__device__ __forceinline__ int first_of(const Kv8Args& a, const Seq& s, int i) {
  return a.mask == CC_MASK_CAUSAL ? 0 : max(0, s.shift + i + (a.inclusive ? 0 : 1));
}
__device__ __forceinline__ int past_of(const Kv8Args& a, const Seq& s, int i) {
  return a.mask == CC_MASK_CAUSAL ? max(0, s.shift + i + 1) : s.len;
}

// Shares of the work of the kernel for few rows.  Lengths are known on the device alone, so every
// workgroup works out its own.  The work is a line of units of 128 entries: the sequences in order, of
// each its KV heads in order, of each its entries.
//   Much work: each of `parts` workgroups takes an equal part of the line, so that a ragged batch keeps
//     every CU busy to the end (64 sequences of 31 to 15987 entries, 4 heads: equal pieces of 2048
//     entries 118 us, of 680 entries 84, shares 76).  A part may hold the end of one (sequence, head),
//     whole ones and the start of another.  Every item takes HEAD units more, without entries, for what
//     it costs to begin one (without them a part of many short sequences is the last: 84 us).
//   Little work (up to LITTLE units for each of two workgroups a CU): the time is that of one chain of
//     round trips, and a second item in a part would double it, so the units become pieces of q units
//     that no two items share, a workgroup each (32 rows, 8 heads, 8000 entries: 23 us, shares 28).
//   A short longest sequence (`direct`): a workgroup for each (sequence, head), nothing to join.
// (Units of 256 entries: that ragged batch 78 us; of 64: those 32 rows 29.)
// An item that is whole in one part is final there; other results are joined.  A result's place is the
// workgroup's index plus that of the (sequence, head): both rise along the line, so no two meet.
constexpr int UNIT = 128;
constexpr int LITTLE = 8;
constexpr int HEAD = 2;
struct Shares {
  int64_t total;     // units of q * 128 entries
  int parts;         // workgroups that have some
  int q;
  int head;          // units without entries at an item's start
  int per;           // sequences of a lane, in order: lane l has [l * per, (l + 1) * per) of the list
  int mine;          // units of one KV head of these
  __device__ __forceinline__ int64_t begin(int w) const { return total * w / parts; }
  // the workgroup whose part unit x is in
  __device__ __forceinline__ int part_of(int64_t x) const { return int(((x + 1) * parts - 1) / total); }
  __device__ __forceinline__ int of(int entry_units) const {
    return entry_units == 0 ? 0 : (entry_units + q - 1) / q + head;
  }
};
__device__ __forceinline__ int entry_units(const Kv8Args& a, int j) {   // of one KV head, 128 entries each
  if (j >= a.n_list) return 0;
  const Seq s = seq_of(a, j);
  const int64_t rows = int64_t(s.m) * a.g;
  return rows == 0 || rows > FEW_ROWS ? 0 : max(1, (s.len + UNIT - 1) / UNIT);
}
// Inclusive sums over the wave (what fits a card's memory has fewer than 2^31 units).
__device__ __forceinline__ int wave_scan(int v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int o = __shfl_up(v, off);
    if (lane >= off) v += o;
  }
  return v;
}
__device__ __forceinline__ int64_t units_in_all(const Kv8Args& a, int mine) {
  return int64_t(a.n_list == 1 ? mine : __builtin_amdgcn_readlane(wave_scan(mine), 63)) * a.hkv;
}
__device__ __forceinline__ Shares shares_of(const Kv8Args& a) {
  Shares s;
  s.q = s.per = 1;
  s.head = 0;
  if (a.direct) {   // a (sequence, head) a workgroup
    s.mine = 1;
    s.total = s.parts = a.n_list * a.hkv;
    return s;
  }
  s.per = (a.n_list + 63) >> 6;
  const int lane = threadIdx.x & 63;
  auto sum = [&](int& n) {
    int v = 0;
    n = 0;
#pragma unroll 4
    for (int c = 0; c < s.per; ++c) {
      const int u = entry_units(a, lane * s.per + c);
      v += s.of(u);
      n += u != 0;
    }
    return v;
  };
  // (one sequence: its length by scalar loads, no sums over the wave; 2 us less of 15)
  int n = 1;
  const int raw = a.n_list == 1 ? entry_units(a, 0) : sum(n);
  s.total = units_in_all(a, raw);
  const int items = a.n_list * a.hkv;
  if (items < a.parts) {
    const int64_t q = max(int64_t(2), (s.total + a.parts - items - 1) / (a.parts - items));
    if (q <= LITTLE) {   // at most total / q + items <= parts pieces
      s.q = int(q);
      s.mine = s.per == 1 ? s.of(raw) : sum(n);
      s.total = units_in_all(a, s.mine);
      s.parts = int(s.total);
      return s;
    }
  }
  s.head = HEAD;
  s.mine = raw + n * HEAD;
  s.total = units_in_all(a, s.mine);
  s.parts = int(min(int64_t(a.parts), s.total));
  return s;
}
struct Item {
  int j, kvh, unit, units;   // sequence of the list, head, unit of its units
};
__device__ __forceinline__ Item item_at(const Kv8Args& a, const Shares& sh, int64_t x) {
  Item it;
  if (a.direct) {
    it.j = int(x) / a.hkv;
    it.kvh = int(x) % a.hkv;
    it.unit = 0;
    it.units = 1;
    return it;
  }
  if (a.n_list == 1) {
    it.j = 0;
    it.units = sh.mine;
    it.kvh = int(x / it.units);
    it.unit = int(x - int64_t(it.kvh) * it.units);
    return it;
  }
  // the lane that has it, then the sequence among the lane's, 64 at a time
  int u = sh.mine, sum = wave_scan(u);
  int l = __builtin_ctzll(__ballot(int64_t(sum) * a.hkv > x));
  it.j = l;
  it.units = __builtin_amdgcn_readlane(u, l);
  int64_t start = int64_t(__builtin_amdgcn_readlane(sum, l) - it.units) * a.hkv;
  if (sh.per > 1) {
    const int j0 = l * sh.per;
    for (int c = 0;; c += 64) {
      const int mine = c + int(threadIdx.x & 63);
      u = mine < sh.per ? sh.of(entry_units(a, j0 + mine)) : 0;
      sum = wave_scan(u);
      const uint64_t past = __ballot(start + int64_t(sum) * a.hkv > x);
      if (past) {
        l = __builtin_ctzll(past);
        it.j = j0 + c + l;
        it.units = __builtin_amdgcn_readlane(u, l);
        start += int64_t(__builtin_amdgcn_readlane(sum, l) - it.units) * a.hkv;
        break;
      }
      start += int64_t(__builtin_amdgcn_readlane(sum, 63)) * a.hkv;
    }
  }
  const int y = int(x - start);
  it.kvh = y / it.units;
  it.unit = y - it.kvh * it.units;
  return it;
}
// First unit of a head of the j-th sequence, and how many it has.
__device__ __forceinline__ void item_of(const Kv8Args& a, const Shares& sh, int j, int64_t& start, int& units) {
  start = 0;
  units = sh.mine;
  if (a.n_list == 1) return;
  int l = j / sh.per;
  int u = sh.mine, sum = wave_scan(u);
  units = __builtin_amdgcn_readlane(u, l);
  start = int64_t(__builtin_amdgcn_readlane(sum, l) - units) * a.hkv;
  if (sh.per == 1) return;
  const int j0 = l * sh.per;
  for (int c = 0;; c += 64) {
    const int mine = c + int(threadIdx.x & 63);
    u = mine < sh.per ? sh.of(entry_units(a, j0 + mine)) : 0;
    sum = wave_scan(u);
    if (j < j0 + c + 64) {
      l = j - j0 - c;
      units = __builtin_amdgcn_readlane(u, l);
      start += int64_t(__builtin_amdgcn_readlane(sum, l) - units) * a.hkv;
      return;
    }
    start += int64_t(__builtin_amdgcn_readlane(sum, 63)) * a.hkv;
  }
}

// ------------------------------------------------------------------ few rows
//
// S^T = K Q^T on 16x16x32 MFMA, entries as its rows, so that a lane holds four entries of one row of
// queries in each 16-entry group, and the two groups of a step are the eight k-slots of its P operand:
// P never moves.  The dims of a product may be taken in any order, so a lane's K operands are whole
// 16-byte pieces of its entry (row l % 16, piece l / 16).  The V operand wants, for one dim, the eight
// entries of the lane's k-slots: a lane loads 8 bytes (head_dim 64: 4) of each of them, 16 lanes
// covering the row, and turns 4 x 4 bytes with eight byte permutations; dim 8 (l % 16) + i is then row
// l % 16 of output block i.
template <int HD, int NR>
__global__ __launch_bounds__(FEW_NT, 2) void attn_few(Kv8Args a) {
  constexpr int NKS = HD / 32;          // k-steps of the first product
  constexpr int NK = HD / 64;           // 16-byte pieces of a lane's entry
  constexpr int NDB = HD / 16;          // 16-dim blocks of the output: also a lane's bytes of a V row
  constexpr int NW = FEW_NT / 64;
  constexpr int ROWS = 16 * NR;
  extern __shared__ float lds[];        // [NW][ROWS][HD] outputs, then [NW][ROWS] (max, sum)
  float2* ml = reinterpret_cast<float2*>(lds + NW * ROWS * HD);
  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Shares sh = shares_of(a);
  if (int(blockIdx.x) >= sh.parts) return;
  int64_t x = sh.begin(blockIdx.x);
  const int64_t x1 = sh.begin(blockIdx.x + 1);
  while (x < x1) {
    int lane = tid & 63;
    asm volatile("" : "+v"(lane));   // what follows from it is made anew for each item, not kept over the loop
    const int grp = lane >> 4, r16 = lane & 15;
    const Item it = item_at(a, sh, x);
    const int j = it.j, kvh = it.kvh;
    const Seq s = seq_of(a, j);
    const int rows = s.m * a.g;
    const int past = it.unit + int(min(int64_t(it.units - it.unit), x1 - x));   // of the item's units
    x += past - it.unit;
    const int u0 = max(0, it.unit - sh.head), u1 = past - sh.head;   // those with entries
    const bool whole = u0 == 0 && past == it.units;
    const int unit = sh.q * UNIT;
    const int c0 = u0 * unit, c1 = a.direct ? s.len : int(min(int64_t(s.len), int64_t(u1) * unit));
    // (another class is met only where every item is a workgroup)
    if (u1 <= u0 || rows == 0 || rows > FEW_ROWS) continue;

    bf16x8 qf[NR][NKS];
    int lo[NR], hi[NR];
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      const int r = min(n * 16 + r16, rows - 1), i = r / a.g;
      lo[n] = first_of(a, s, i);
      hi[n] = past_of(a, s, i);
      const u16* q = a.q + (int64_t(s.q0 + i) * a.hq + kvh * a.g + r % a.g) * HD;
#pragma unroll
      for (int k = 0; k < NKS; ++k)
        qf[n][k] = as_bf16x8(*reinterpret_cast<const uint4*>(q + 64 * (k >> 1) + 16 * grp + 8 * (k & 1)));
    }
    // entries [full0, full1) are seen by every row
    const int full0 = first_of(a, s, s.m - 1), full1 = past_of(a, s, 0);
    // this wave's 16-entry groups: the piece's, in NW runs of whole steps of two
    const int g0 = c0 >> 4, g1 = (c1 + 15) >> 4;
    const int per = ((g1 - g0 + NW - 1) / NW + 1) & ~1;
    int lo_all = first_of(a, s, 0) >> 4, hi_all = (past_of(a, s, s.m - 1) + 15) >> 4;   // nothing to see outside
    int gb = g0 + wave * per, ge = min(g1, gb + per);
    gb = max(gb, lo_all & ~1);
    ge = min(ge, hi_all);
    const Plane P = plane_of(a, s.b, kvh);
    const int last = s.len - 1;

    float m_run[NR], l_run[NR];
    f32x4 acc[NR][NDB];
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      m_run[n] = -INFINITY;
      l_run[n] = 0.f;
#pragma unroll
      for (int d = 0; d < NDB; ++d) acc[n][d] = f32x4{};
    }

    // a lane's places in a whole group: its K row, its four V rows
    const uint32_t ts = uint32_t(a.k.codes.tok_stride);
    const uint32_t ko0 = r16 * ts + 16 * grp;
    const uint32_t vo0[4] = {(4 * grp) * ts + NDB * r16, (4 * grp + 1) * ts + NDB * r16, (4 * grp + 2) * ts + NDB * r16,
                             (4 * grp + 3) * ts + NDB * r16};
    struct Step {
      uint4 k[2][NK];
      uint32_t v[8][NDB / 4];
    };
    // Pages and scales of 64 groups at a time, a lane each.
    for (int sb = gb; sb < ge; sb += 64) {
      const int se = min(ge, sb + 64);
      const int mine = min(sb + lane, se - 1);
      const int page = group_page(a, P, mine);
      const int64_t so = group_scale(a, page, mine);
      const uint32_t sc = uint32_t(P.ks[so]) | (uint32_t(P.vs[so]) << 8);
      auto load = [&](int gr, Step& st) {   // groups gr and gr + 1 (past the end: the last one again)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const int gg = min(gr + t, se - 1);
          const int64_t off = group_codes(a, __builtin_amdgcn_readlane(page, gg - sb), gg);
          const char* kp = uniform_ptr(P.k + off);
          const char* vp = uniform_ptr(P.v + off);
          uint32_t ko = ko0, vo[4] = {vo0[0], vo0[1], vo0[2], vo0[3]};
          const int have = last - (gg << 4);   // the group's last entry; past it: that one again
          if (have < 15) {
            ko = uint32_t(min(r16, have)) * ts + 16 * grp;
#pragma unroll
            for (int e = 0; e < 4; ++e) vo[e] = uint32_t(min(4 * grp + e, have)) * ts + NDB * r16;
          }
#pragma unroll
          for (int k = 0; k < NK; ++k) st.k[t][k] = *reinterpret_cast<const uint4*>(kp + ko + 64 * k);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if constexpr (NDB == 8) {
              const u32x2 w = *reinterpret_cast<const u32x2*>(vp + vo[e]);
              st.v[4 * t + e][0] = w[0];
              st.v[4 * t + e][NDB / 4 - 1] = w[1];
            } else {
              st.v[4 * t + e][0] = *reinterpret_cast<const uint32_t*>(vp + vo[e]);
            }
          }
        }
      };
      auto compute = [&](int gr, Step& st) {
        const uint32_t s0 = __builtin_amdgcn_readlane(sc, gr - sb);
        const uint32_t s1 = __builtin_amdgcn_readlane(sc, min(gr + 1, se - 1) - sb);
        const float ks[2] = {e8m0_scale(s0 & 255u), e8m0_scale(s1 & 255u)};
        const float vs[2] = {e8m0_scale(s0 >> 8), e8m0_scale(s1 >> 8)};
        f32x4 z[NR][2];
#pragma unroll
        for (int n = 0; n < NR; ++n) z[n][0] = z[n][1] = f32x4{};
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int k = 0; k < NKS; ++k) {
            const uint4 w = st.k[t][k >> 1];
            const bf16x8 kf = (k & 1) ? widen8(w.z, w.w, ks[t]) : widen8(w.x, w.y, ks[t]);
#pragma unroll
            for (int n = 0; n < NR; ++n) z[n][t] = mfma16(kf, qf[n][k], z[n][t]);
          }
        const int e0 = gr << 4;
        // past the wave's own groups counts as masked: the last group stands there a second time
        const int stop = min(full1, ge << 4);
        const bool masked = e0 < full0 || e0 + 32 > stop;
        bool nans = false;
        uint32_t hit[NR];
        if (masked) {
          const uint32_t wide[2] = {wide_of(s0 >> 8), wide_of(s1 >> 8)};
#pragma unroll
          for (int n = 0; n < NR; ++n)
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const int key = e0 + 16 * t + 4 * grp + e;
                if (key < lo[n] || key >= min(hi[n], ge << 4)) z[n][t][e] = -INFINITY;
              }
          // values of entries that the sequence does not have
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const bool in = e0 + 16 * t + 4 * grp + e < min(s.len, ge << 4);
#pragma unroll
              for (int i = 0; i < NDB / 4; ++i) {
                if (!in) st.v[4 * t + e][i] = 0;
                nans |= wide_bytes(st.v[4 * t + e][i], wide[t]) != 0;
              }
            }
          nans = __any(nans);
          if (nans) {
            // which outputs of this lane such a value reaches: a product of indicators
#pragma unroll
            for (int n = 0; n < NR; ++n) hit[n] = 0;
            bf16x8 see[NR];
#pragma unroll
            for (int n = 0; n < NR; ++n)
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                const int key = e0 + 16 * (e >> 2) + 4 * grp + (e & 3);
                see[n][e] = (__bf16)(key >= lo[n] && key < min(hi[n], ge << 4) ? 1.f : 0.f);
              }
#pragma unroll
            for (int i = 0; i < NDB / 4; ++i) {
              uint32_t wa[4], wb[4], ta[4], tb[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                wa[e] = whole_bytes(wide_bytes(st.v[e][i], wide[0]));
                wb[e] = whole_bytes(wide_bytes(st.v[4 + e][i], wide[1]));
                st.v[e][i] &= ~wa[e];
                st.v[4 + e][i] &= ~wb[e];
              }
              transpose4(wa, ta);
              transpose4(wb, tb);
#pragma unroll
              for (int d = 0; d < 4; ++d) {
                const bf16x8 one = widen44(ta[d] & 0x38383838u, tb[d] & 0x38383838u, 1.f, 1.f);   // code 0x38: 1
#pragma unroll
                for (int n = 0; n < NR; ++n) {
                  const f32x4 h = mfma16(one, see[n], f32x4{});
#pragma unroll
                  for (int e = 0; e < 4; ++e) hit[n] |= h[e] > 0.f ? 1u << (16 * i + 4 * d + e) : 0u;
                }
              }
            }
          }
        }
        bf16x8 pf[NR];
        bool moved = false;
        float mx[NR];
#pragma unroll
        for (int n = 0; n < NR; ++n) {
          float t = fmaxf(fmaxf(fmaxf(z[n][0][0], z[n][0][1]), fmaxf(z[n][0][2], z[n][0][3])),
                          fmaxf(fmaxf(z[n][1][0], z[n][1][1]), fmaxf(z[n][1][2], z[n][1][3])));
          mx[n] = quad_max(t);
          moved |= mx[n] > m_run[n] + a.room;
        }
        if (__any(moved)) {
#pragma unroll
          for (int n = 0; n < NR; ++n) {
            const bool up = mx[n] > m_run[n] + a.room;
            const float corr = up ? fast_exp2((m_run[n] - mx[n]) * a.c2) : 1.f;   // 0 from -inf
            if (up) m_run[n] = mx[n];
            l_run[n] *= corr;
#pragma unroll
            for (int d = 0; d < NDB; ++d) acc[n][d] *= corr;
          }
        }
#pragma unroll
        for (int n = 0; n < NR; ++n) {
          const float mc = m_run[n] == -INFINITY ? 0.f : m_run[n] * a.c2;
          float p[8], sum = 0.f;
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              p[4 * t + e] = fast_exp2(fmaf(z[n][t][e], a.c2, -mc));
              sum += p[4 * t + e];
            }
          l_run[n] += sum;
          pf[n] = bf16x8{(__bf16)p[0], (__bf16)p[1], (__bf16)p[2], (__bf16)p[3],
                         (__bf16)p[4], (__bf16)p[5], (__bf16)p[6], (__bf16)p[7]};
        }
#pragma unroll
        for (int i = 0; i < NDB / 4; ++i) {
          uint32_t ta[4], tb[4];
          const uint32_t wa[4] = {st.v[0][i], st.v[1][i], st.v[2][i], st.v[3][i]};
          const uint32_t wb[4] = {st.v[4][i], st.v[5][i], st.v[6][i], st.v[7][i]};
          transpose4(wa, ta);
          transpose4(wb, tb);
#pragma unroll
          for (int d = 0; d < 4; ++d) {
            const bf16x8 vf = widen44(ta[d], tb[d], vs[0], vs[1]);
#pragma unroll
            for (int n = 0; n < NR; ++n) acc[n][4 * i + d] = mfma16(vf, pf[n], acc[n][4 * i + d]);
          }
        }
        if (nans) {
#pragma unroll
          for (int n = 0; n < NR; ++n)
#pragma unroll
            for (int i = 0; i < NDB * 4; ++i)
              if (hit[n] >> i & 1u) acc[n][i >> 2][i & 3] = __uint_as_float(0x7fc00000u);
        }
      };
      Step st[2];
      load(sb, st[0]);
      for (int gr = sb; gr < se; gr += 4) {
        if (gr + 2 < se) load(gr + 2, st[1]);
        compute(gr, st[0]);
        if (gr + 2 < se) {
          if (gr + 4 < se) load(gr + 4, st[0]);
          compute(gr + 2, st[1]);
        }
      }
    }

    // The waves' results meet in LDS.
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      const float l = quad_sum(l_run[n]);
      const int row = wave * ROWS + n * 16 + r16;
      if (grp == 0) ml[row] = make_float2(m_run[n], l);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float* o = lds + row * HD + NDB * (4 * grp + e);
#pragma unroll
        for (int d = 0; d < NDB; d += 4)
          *reinterpret_cast<float4*>(o + d) =
              make_float4(acc[n][d][e], acc[n][d + 1][e], acc[n][d + 2][e], acc[n][d + 3][e]);
      }
    }
    __syncthreads();
    constexpr int LPR = HD / 8;   // lanes of a row
    for (int r = tid / LPR; r < rows; r += FEW_NT / LPR) {
      const int d = (tid % LPR) * 8;
      float M = -INFINITY;
#pragma unroll
      for (int w = 0; w < NW; ++w) M = fmaxf(M, ml[w * ROWS + r].x);
      const float ref = M == -INFINITY ? 0.f : M;
      float L = 0.f, o[8] = {};
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const float2 p = ml[w * ROWS + r];
        const float f = fast_exp2((p.x - ref) * a.c2);
        L += p.y * f;
        const float* src = lds + (w * ROWS + r) * HD + d;
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] += src[e] * f;
      }
      if (!whole) {
        const int64_t row = (int64_t(blockIdx.x) + int64_t(j) * a.hkv + kvh) * a.R + r;
        float* po = a.part + row * HD + d;
        *reinterpret_cast<float4*>(po) = make_float4(o[0], o[1], o[2], o[3]);
        *reinterpret_cast<float4*>(po + 4) = make_float4(o[4], o[5], o[6], o[7]);
        if (d == 0) a.part_ml[row] = make_float2(M, L);
      } else {
        // an empty row has L = 0 and outputs 0; a NaN sum stays NaN
        const float inv = L == 0.f ? 0.f : 1.f / L;
        u16* out = a.o + (int64_t(s.q0 + r / a.g) * a.hq + kvh * a.g + r % a.g) * HD + d;
        *reinterpret_cast<uint4*>(out) = make_uint4(pack_bf2(o[0] * inv, o[1] * inv), pack_bf2(o[2] * inv, o[3] * inv),
                                                    pack_bf2(o[4] * inv, o[5] * inv), pack_bf2(o[6] * inv, o[7] * inv));
      }
    }
    __syncthreads();   // the LDS results have been read
  }
}

// ------------------------------------------------------------------ joining pieces

// out = sum_s o_s 2^((m_s - M) c2) / sum_s l_s 2^((m_s - M) c2), M = max m_s.  HD / 4 lanes hold a row.
struct Joined {
  float M, L;
  float4 o;
  // N parts at once, those with in[q] set
  template <int N, class F>
  __device__ __forceinline__ void add(const float2 (&p)[N], F x, const bool (&in)[N], float c2) {
    float t = M;
#pragma unroll
    for (int q = 0; q < N; ++q)
      if (in[q]) t = fmaxf(t, p[q].x);
    const float ref = t == -INFINITY ? 0.f : t, c = fast_exp2((M - ref) * c2);
    M = t;
    L *= c;
    o = make_float4(o.x * c, o.y * c, o.z * c, o.w * c);
#pragma unroll
    for (int q = 0; q < N; ++q) {
      if (!in[q]) continue;
      const float f = fast_exp2((p[q].x - ref) * c2);
      const float4 y = x(q);
      L += p[q].y * f;
      o = make_float4(o.x + y.x * f, o.y + y.y * f, o.z + y.z * f, o.w + y.w * f);
    }
  }
};

// FEW: the pieces are shares of the kernel for few rows, else those of the kernel for many.  A workgroup is
// 256 / (HD / 4) groups of lanes.  With `one`, for up to JOIN_ONE rows in all, it has one row, whose pieces
// the groups share out (128 rows of 64 pieces by a group each, a chain of loads in 16 workgroups: 35 us);
// else a row for each group (finding a row's pieces is half of the work: 1023 sequences, 8 heads of 4
// rows, 352 us with a workgroup for each row), and those of more than JOIN_ALONE pieces are shared out one after
// another (with 8 and with 32: 64 queries of 32 heads on 8, nine pieces, 30 us and 23; one sequence of 131072
// entries among 99 of 20 125 and 118).
constexpr int JOIN_ALONE = 32;
constexpr int JOIN_ONE = 1024;
template <int HD, bool FEW>
__global__ __launch_bounds__(256) void attn_join(Kv8Args a, int one, int64_t group0) {
  constexpr int LPR = HD / 4, NG = 256 / LPR;
  __shared__ float4 po[256];
  __shared__ float2 pm[256];
  __shared__ int sn[NG];
  __shared__ int64_t sslot[NG];
  const int tid = threadIdx.x;
  const int gi = tid / LPR, lane = tid % LPR;
  // few rows: R of each (sequence, head); many: the rows there are, head by head
  const int64_t all = FEW ? int64_t(a.n_list) * a.hkv * a.R : int64_t(a.hkv) * a.all;
  const int64_t row_in = one ? int64_t(blockIdx.x) : (group0 + blockIdx.x) * NG + gi;
  const int d = lane * 4;
  int r, j, kvh, jh = 0;
  if constexpr (FEW) {
    r = int(row_in % a.R);
    jh = int(min(row_in / a.R, int64_t(a.n_list) * a.hkv - 1));
    kvh = jh % a.hkv;
    j = jh / a.hkv;
  } else {
    const int64_t x = min(row_in, all - 1);
    kvh = int(x / a.all);
    r = int(x - int64_t(kvh) * a.all);
    j = 0;
    if (a.listed) {
      for (int i = 1; i < a.n_list; ++i) j += a.first[i] <= r;
      r -= a.first[j];
    } else {   // the last sequence that starts at or before the row's query
      const int query = r / a.g;
      int n = a.n_list;
      while (n > 1) {
        const int half = n >> 1;
        const bool up = a.cu[j + half] <= query;
        j = up ? j + half : j;
        n = up ? n - half : half;
      }
      r -= a.cu[j] * a.g;
    }
  }
  const Seq s = seq_of(a, j);
  const int rows = s.m * a.g;
  bool on = row_in < all && r < rows && (rows <= FEW_ROWS) == FEW;
  // piece i of the row is at slot + i * step
  int64_t slot, step;
  int n;
  if constexpr (FEW) {
    // the rows of a wave lie in one (sequence, head), or the search runs for each in turn
    const Shares sh = shares_of(a);
    const int j0 = __builtin_amdgcn_readfirstlane(j);
    int64_t start;
    int units;
    item_of(a, sh, j0, start, units);
    uint64_t other = __ballot(j != j0);
    while (other) {
      const int jn = __builtin_amdgcn_readlane(j, __builtin_ctzll(other));
      int64_t st;
      int un;
      item_of(a, sh, jn, st, un);
      if (j == jn) {
        start = st;
        units = un;
      }
      other &= ~__ballot(j == jn);
    }
    const int64_t x = start + int64_t(kvh) * units;
    const int wa = sh.part_of(x + sh.head), wb = sh.part_of(x + max(units, 1) - 1);
    n = wb - wa + 1;
    on = on && n > 1;   // a whole one is final
    slot = (int64_t(wa) + jh) * a.R + r;
    step = a.R;
  } else {
    n = min(a.splits, max(1, (s.len + a.piece - 1) / a.piece));
    slot = row_in;
    step = all;
  }
  // pieces first, first + by, ..., four in flight
  auto some = [&](int64_t from, int n, int first, int by) {
    Joined g{-INFINITY, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)};
    for (int i0 = first; i0 < n; i0 += 4 * by) {
      float2 p[4];
      float4 x[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int64_t at = from + min(i0 + q * by, n - 1) * step;
        p[q] = a.part_ml[at];
        x[q] = *reinterpret_cast<const float4*>(a.part + at * HD + d);
      }
      bool in[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) in[q] = i0 + q * by < n;
      g.add(p, [&](int q) { return x[q]; }, in, a.c2);
    }
    return g;
  };
  auto finish = [&](const Joined& g) {
    const float inv = g.L == 0.f ? 0.f : 1.f / g.L;
    u16* out = a.o + (int64_t(s.q0 + r / a.g) * a.hq + kvh * a.g + r % a.g) * HD + d;
    *reinterpret_cast<uint2*>(out) = make_uint2(pack_bf2(g.o.x * inv, g.o.y * inv), pack_bf2(g.o.z * inv, g.o.w * inv));
  };
  auto shared_out = [&](int64_t from, int n, int owner) {
    const Joined mine = some(from, n, gi, NG);
    po[tid] = mine.o;
    pm[tid] = make_float2(mine.M, mine.L);
    __syncthreads();
    if (gi == owner) {
      Joined g{-INFINITY, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)};
      float2 p[NG];
      bool in[NG];
#pragma unroll
      for (int q = 0; q < NG; ++q) {
        p[q] = pm[lane + q * LPR];
        in[q] = true;
      }
      g.add(p, [&](int q) { return po[lane + q * LPR]; }, in, a.c2);
      finish(g);
    }
  };
  if (one) {
    if (on) shared_out(slot, n, 0);   // (alike in the whole workgroup)
    return;
  }
  const bool alone = n <= JOIN_ALONE;
  if (on && alone) finish(some(slot, n, 0, 1));
  if (!__syncthreads_or(on && !alone)) return;
  if (lane == 0) {
    sn[gi] = on && !alone ? n : 0;
    sslot[gi] = slot;
  }
  __syncthreads();
  for (int q = 0; q < NG; ++q) {
    if (sn[q] == 0) continue;
    shared_out(sslot[q], sn[q], q);
    __syncthreads();
  }
}

template <int HD, int NR>
hipError_t few_rows(const Kv8Args& a, hipStream_t s) {
  constexpr int NW = FEW_NT / 64;
  constexpr size_t lds = size_t(NW) * 16 * NR * (HD * 4 + 8);
  if (lds > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(attn_few<HD, NR>),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, int(lds));
    if (e != hipSuccess) return e;
  }
  const int grid = a.direct ? a.n_list * a.hkv : a.parts;
  hipLaunchKernelGGL((attn_few<HD, NR>), dim3(unsigned(grid)), dim3(FEW_NT), lds, s, a);
  return hipGetLastError();
}

template <int HD>
hipError_t launch_dim(const Kv8Args& a, bool few, hipStream_t s) {
  hipError_t e;
  if (few)
    e = a.R <= 16 ? few_rows<HD, 1>(a, s) : few_rows<HD, 2>(a, s);
  else
    e = launch_attn_many(a, s);
  if (e != hipSuccess || !a.part) return e;
  constexpr int NG = 256 / (HD / 4);
  const int one = int64_t(a.n_list) * a.hkv * a.R <= JOIN_ONE;
  const int64_t rows = few ? int64_t(a.n_list) * a.hkv * a.R : int64_t(a.hkv) * a.all;
  const int64_t groups = one ? rows : (rows + NG - 1) / NG;
  for (int64_t group0 = 0; group0 < groups; group0 += MOST_GROUPS) {   // (more than a launch may have: several)
    const dim3 grid(unsigned(std::min(MOST_GROUPS, groups - group0)));
    if (few)
      hipLaunchKernelGGL((attn_join<HD, true>), grid, dim3(256), 0, s, a, one, group0);
    else
      hipLaunchKernelGGL((attn_join<HD, false>), grid, dim3(256), 0, s, a, one, group0);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_attention_kv8(const Kv8Args& a, bool few, hipStream_t s) {
  return a.head_dim == 128 ? launch_dim<128>(a, few, s) : launch_dim<64>(a, few, s);
}

}  // namespace cc
