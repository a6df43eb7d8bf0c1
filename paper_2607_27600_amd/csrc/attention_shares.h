// What the attentions over a cache share, in 8 bits and in bf16: how the work of the kernels for few rows is shared out
// among workgroups, and how results are joined.  A: the arguments of a launch, with the sequences walked (list, listed,
// n_list), their queries and entries (cu, lens, max_len) and heads (hkv, g), and direct and parts; LEAST: units of a piece.
#pragma once

#include "cc_internal.h"

namespace cc {

// Rows (queries times heads of a group) up to which a sequence counts as few: up to two row blocks of 16.  In 8 bits, two
// blocks against the kernel for many, 32 rows, 8000 entries, 8 KV heads of 128: 23.2 us and 24.7, sixteen such
// sequences 83 and 116; four blocks, 64 rows: 41.5 and (68 rows) 31.6, sixteen 328 and 122.
constexpr int FEW_ROWS = 32;

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
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

// The sequence of a workgroup's item and what its rows may see.
struct Seq {
  int b, q0, m, len, shift;    // shift: cache position of query 0
};
template <class A>
__device__ __forceinline__ Seq seq_of(const A& a, int j) {
  Seq s;
  s.b = a.listed ? a.list[j] : j;
  s.q0 = a.cu[s.b];
  s.m = a.cu[s.b + 1] - s.q0;
  s.len = min(max(a.lens[s.b], 0), a.max_len);
  s.shift = s.len - s.m;
  return s;
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
template <class A>
__device__ __forceinline__ int entry_units(const A& a, int j) {   // of one KV head, 128 entries each
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
template <class A>
__device__ __forceinline__ int64_t units_in_all(const A& a, int mine) {
  return int64_t(a.n_list == 1 ? mine : __builtin_amdgcn_readlane(wave_scan(mine), 63)) * a.hkv;
}
template <class A>
__device__ __forceinline__ Shares shares_of(const A& a) {
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
    const int64_t q = max(int64_t(A::LEAST), (s.total + a.parts - items - 1) / (a.parts - items));
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
template <class A>
__device__ __forceinline__ Item item_at(const A& a, const Shares& sh, int64_t x) {
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
template <class A>
__device__ __forceinline__ void item_of(const A& a, const Shares& sh, int j, int64_t& start, int& units) {
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

}  // namespace cc
