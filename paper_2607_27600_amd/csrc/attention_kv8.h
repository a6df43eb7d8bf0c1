// What the kernels of the attention over a cache in 8 bits share with each other and with the planner.
#pragma once

#include "cc_internal.h"

namespace cc {

// Rows (queries times heads of a group) up to which a sequence counts as few: up to two row blocks of 16.  Two
// blocks against the kernel for many, 32 rows, 8000 entries, 8 KV heads of 128: 23.2 us and 24.7, sixteen such
// sequences 83 and 116; four blocks, 64 rows: 41.5 and (68 rows) 31.6, sixteen 328 and 122.
constexpr int FEW_ROWS = 32;
// Few rows: the longest cache of which each (sequence, head) is one workgroup's, with nothing to join.  A
// CU's own loads, some 40 GB/s, are the bound there, so it grows with the workgroups there are, up to where a
// batch of one long sequence among short ones would wait for it.  One token each, heads of 128, that
// against shares of the work:
//   1024: 64 sequences of 1000, 4 heads: 17 us and 27; one of 1024, 8 heads: 13.4 and 14 (of 2048: 19 and 14);
//   2048 from 128 (sequence, head)s: 300 sequences of 1500, 8 heads: 170 and 208; 16 of 2048: 23 and 27 (8 of
//     them 22 and 21; 16, of which four have 2000 entries and the others 20: 22 and 18);
//   not 4096 from 512: 64 sequences, 8 heads: 99 and 107, but 53 and 27 where eight have them and the others 20.
inline int kv8_direct(int64_t items) { return items >= 128 ? 2048 : 1024; }
constexpr int FEW_NT = 256;
constexpr int KV8_LIST = 64;     // sequences of a launch listed by value
constexpr int MANY_ROWS = 128;   // rows of a block of the kernel for many
constexpr int MANY_KEYS = 64;    // entries of its tiles

// Codes that are not finite in bf16: NaN (0x7f), and under scales from 2^120 on those from 2^128 / scale, whose
// codes are (262 - x) * 8 and above for the scale's byte x.  `wide_of(x)` in every byte, added to four codes
// without their signs, raises bit 7 of those that are not.
__device__ __forceinline__ uint32_t wide_of(uint32_t scale_byte) {
  return uint32_t(max(1, 8 * int(min(scale_byte, 254u)) - 1968)) * 0x01010101u;
}
// Bytes 0x80 where a byte of x is such a code.
__device__ __forceinline__ uint32_t wide_bytes(uint32_t x, uint32_t wide) { return ((x & 0x7f7f7f7fu) + wide) & 0x80808080u; }
// Bytes 0xff at bytes 0x80.
__device__ __forceinline__ uint32_t whole_bytes(uint32_t m) { return (m >> 7) * 0xffu; }

// One class of sequences (few or many rows) of a call.
struct Kv8Args {
  const u16* q;
  u16* o;
  Kv8View k, v;                  // alike but for base and scale
  const int32_t *cu, *lens;
  int layer, mask, inclusive, max_len;
  int hq, hkv, g, head_dim;
  float c2;                      // scale * log2(e)
  float room;                    // how far a logit may pass a row's reference maximum: 2^8 in probability
  int R;                         // most rows of a sequence of the class
  int piece, splits;             // many rows: entries of a piece, pieces of the longest sequence
  int nth0;                      // many rows: first row block, in the order of a sequence, of a launch
  int direct, parts;             // few rows: a workgroup for each (sequence, head); else workgroups to share it all
  // Results to be joined (null: none), outputs and (maximum, sum): many rows
  // [splits][Hkv][all], few rows [parts + n_list * Hkv][R].
  float* part;
  float2* part_ml;
  int n_list, listed;            // sequences walked: list[0..n_list), or (listed = 0) all
  int32_t list[KV8_LIST];
  // many rows: rows of the sequences walked one after another, and where each one's start (not listed: all
  // sequences', at their queries times g)
  int32_t all;
  int32_t first[KV8_LIST];
};
hipError_t launch_attention_kv8(const Kv8Args& a, bool few, hipStream_t s);
hipError_t launch_attn_many(const Kv8Args& a, hipStream_t s);

}  // namespace cc
