// What the kernels of the attention over a bf16 cache share with each other and with the planner.
#pragma once

#include "attention_shares.h"

namespace cc {

// One tensor pair of a cache: keys and values alike but for their base, strides in bytes.
struct KvPair {
  KvView at;                   // of the keys
  const void* v;
  int32_t paged;
};

constexpr int KV_ROWS = 128;   // rows of a block of the kernel for many
constexpr int KV_KEYS = 64;    // entries of its tiles
constexpr int KV_LIST = 64;    // sequences of few rows of a launch listed by value
// Few rows: the longest cache of which each (sequence, head) is one workgroup's, with nothing to join.  A CU alone takes
// some 60 GB/s, with four waves half.  That against shares: 16 sequences of 2000, 8 heads, 25 us and 35; 64 of 2000 96 and 103,
// but 40 and 26 where eight have 1900 entries and the others 20; one of 500, 8 heads, 8.8 and 10.9, of 1000 13.2 and 11.0.
inline int kv_direct(int64_t items) { return items < 128 ? 600 : items <= 256 ? 2048 : 1024; }

// Attention of the queries of n_seqs sequences to the entries of a prefix and to their own entries up to their own.
struct KvAttnArgs {
  static constexpr int LEAST = 1;   // (of entries of 16 bits; with two, one sequence of 2048 entries and 8 heads 12.9 us for 11.1)
  const u16* q;
  u16* o;
  float* lse;                  // or null
  KvPair own, pre;
  const int32_t *cu, *lens;    // queries and own entries of the sequences
  const int32_t *pre_first, *pre_lens;   // sequences [pre_first[i], pre_first[i + 1]) are behind prefix i
  int n_seqs, n_prefixes;      // (0: no prefixes)
  int layer, max_len, pre_max;
  int hq, hkv, g, head_dim;
  int N;                       // queries in all
  float scale, c2;             // c2 = scale * log2(e)
  float room;                  // how far a logit may pass a row's reference maximum: 2^8 in probability
  // Few rows: sequences list[0 .. n_list), or (listed = 0) all, those of more than `most` rows left out.
  int n_list, listed, R, most; // R: most rows of one
  static constexpr int direct = 0;   // (short caches have a launch of their own)
  int parts;                   // workgroups that share out the work (attention_shares.h)
  union {
    int32_t list[KV_LIST];
    int32_t few_at[KV_LIST];   // in the arguments of the pass over the prefixes, of the joins and of many rows
  };
  // Rows of a KV head that sequences of few rows have, in all and before the first sequence of each of KV_LIST groups of
  // few_per sequences (few_at; few_before).  Results to be joined lie by them, so that they take no place for the other
  // sequences' rows.
  int few_rows, few_per, mixed;   // mixed: there are others
  // 16 rows a workgroup, behind prefixes (0: rows whole): entries of a piece, pieces of the longest sequence, and where their outputs and
  // (maximum, sum) go, to be joined with the prefixes': [rsplits][few_rows * Hkv], a sequence's [Hkv][rows] together.
  int rpiece, rsplits;
  float* rpart;
  float2* rpart_ml;
  float* fpart;                // [parts + n_list * Hkv][R] outputs and (maximum, sum) to be joined
  float2* fpart_ml;
  int2* fpart_at;              // [n_list * Hkv] first and last workgroup that has some of a (sequence, head)'s entries
  // Many rows.  Row blocks of the sequences of many rows: listed by value, longest first, or (items.n_seqs = 0)
  // sequence b has those from cu[b] g / KV_ROWS + b on, more than its rows need.  Those of up to `few` rows are left out.
  AttnMany items;
  int blocks, few, ends;       // ends: row blocks * Hkv of listed sequences of few rows
  int piece, splits;           // entries of a piece (a multiple of KV_KEYS), pieces of the longest sequence
  // Results to be joined (null: none), outputs and (maximum, sum): [Hkv][places][splits], of the rows from row0 on, or with
  // `skip` of all but those of sequences of few
  int row0, places, skip;
  float* part;
  float2* part_ml;
  // The pass over the prefixes: they stand for sequences, and own, lens and n_seqs are theirs.  Its pieces
  // are sized on the device, by the prefixes' lengths, for `slots` workgroups at the least: a workgroup, and KV_ROWS rows
  // of ppart, for each.  Where prefix i's begin and how many each of its (row block, KV head) has is in pre_at[i].  For the
  // passes over the sequences' own entries ppart and pre_at are what it has left (null: none).
  float* ppart;
  float2* ppart_ml;
  int2* pre_at;
  int slots;
};
// 16 rows a workgroup; with n_prefixes the prefix's entries too.
hipError_t launch_attn_rows(const KvAttnArgs& a, hipStream_t s);
// Workgroups of that, or of the pieces of own entries that go along with the pass over the prefixes.
inline int64_t rows_groups(const KvAttnArgs& a) {
  return (a.listed ? int64_t(a.n_list) * ((a.R + 15) / 16) : int64_t(a.N) * a.g / 16 + a.n_seqs) * a.hkv *
         (a.rpiece ? a.rsplits : 1);
}
// The pass over the prefixes (few_at in its arguments), and with `few` the sequences of few rows, done.
hipError_t launch_attn_prefix(const KvAttnArgs& pass, const KvAttnArgs& own, bool few, hipStream_t s);
// Few rows, work shared out.
hipError_t launch_attn_few(const KvAttnArgs& a, hipStream_t s);
hipError_t launch_attn_kv_many(const KvAttnArgs& a, hipStream_t s);

// What entries receive of the queries' attention, added to what they have.
struct KvWeightsArgs {
  const u16* q;
  const float* lse;            // [N][Hq]
  KvPair own;
  const int32_t *cu, *lens;
  const int32_t* prev_lens;    // or null: every entry has some
  const float* prev;           // or null: none has
  int prev_n;                  // entries that prev holds of a (sequence, KV head)
  float* w;
  int64_t w_seq, w_head, prev_seq, prev_head;
  int n_seqs, layer, max_len, hq, hkv, g, head_dim;
  float c2;
  int R;                       // most rows of a sequence of few
  // Sequences of more than W_FEW_ROWS rows: list[0 .. n_list), or (listed = 0) all there are.
  int n_list, listed;
  int32_t list[KV_LIST];
  int seq0;                    // first sequence (of the list) of a launch
  int chunk, chunks;           // rows of a chunk (a multiple of W_ROWS), chunks of the longest sequence
  float* part;                 // sums of chunks to be added up (null: one chunk): [chunks][n_list][Hkv][max_len]
};
// Rows up to which a sequence's are read by each wave for itself; beyond, in tiles that a workgroup shares.  32 heads on 8, the one
// against the other: 80 rows, 32 sequences of 2000 entries, 47 us and 41; 48 rows 38.8 and 35.8, but eight of 3000 15.5 and 17.0.
constexpr int W_FEW_ROWS = 64;
constexpr int W_KEYS = 256;    // entries of a workgroup
constexpr int W_ROWS = 64;     // rows of a tile
hipError_t launch_weights_few(const KvWeightsArgs& a, hipStream_t s);
hipError_t launch_weights_many(const KvWeightsArgs& a, hipStream_t s);

struct WeightScoresArgs {
  const float* w;
  int64_t w_seq, w_head;
  float* scores;
  const int32_t* cu;
  int n_seqs, hkv, per_head, recent, frozen, longest;
  int seq0;                    // first sequence of a launch
};
hipError_t launch_weight_scores(const WeightScoresArgs& a, hipStream_t s);

struct CompactWeightsArgs {
  float *w, *out;              // out = w: in place
  int64_t w_seq, w_head, out_seq, out_head;
  const int32_t* keep;
  const int32_t* k_h;          // host
  int n_seqs, hkv, per_head;
};
hipError_t launch_compact_weights(const CompactWeightsArgs& a, hipStream_t s);

// ---- shared by the attention kernels

// T at a wave-uniform base and a lane's offset: in the global address space, so that the base stays in scalar registers
// (as generic loads, each with a 64-bit address a lane, the kernel for few rows spilled 45 registers).
template <class T>
__device__ __forceinline__ T load_at(const char* base, uint32_t off) {
  typedef __attribute__((address_space(1))) const char* gptr;
  return *(__attribute__((address_space(1))) const T*)((gptr)(base) + off);
}

// Bits 15 and 31 where the low and the high bf16 of a word are NaN or infinite.
__device__ __forceinline__ uint32_t wide_halves(uint32_t w) { return ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u; }
// 0xffff at bits 15 and 31.
__device__ __forceinline__ uint32_t whole_halves(uint32_t m) { return (m >> 15) * 0xffffu; }

// The log-sum-exp of a row from its reference logit and its sum of 2^((z - ref) c2).
__device__ __forceinline__ float row_lse(float ref, float sum, float scale) {
  return __float_as_uint(sum) == 0u ? -INFINITY : fmaf(ref, scale, __logf(sum));
}
// Its outputs' factor: an empty row has sum 0 and outputs 0, a NaN sum stays NaN.
__device__ __forceinline__ float row_inverse(float sum) { return __float_as_uint(sum) == 0u ? 0.f : 1.f / sum; }

// The last b with start(b) <= x among 0 .. n - 1, start rising from start(0) <= x.
template <class F>
__device__ __forceinline__ int last_at(int n, F start, int64_t x) {
  int b = 0;
  while (n > 1) {
    const int half = n >> 1;
    const bool up = start(b + half) <= x;
    b = up ? b + half : b;
    n = up ? n - half : half;
  }
  return b;
}

// A plane: one (sequence, layer, KV head).  16-entry groups lie in one page.
struct KvPlane {
  const char *k, *v;
  const int32_t* table;
  uint32_t ts;                 // bytes between entries
  int paged, page_shift, page_mask;
  int64_t page_stride;
  __device__ __forceinline__ int page(int group) const { return paged ? table[group >> (page_shift - 4)] : 0; }
  __device__ __forceinline__ int64_t offset(int page, int entry) const {
    return int64_t(page) * page_stride + int64_t(paged ? entry & page_mask : entry) * ts;
  }
};
__device__ __forceinline__ KvPlane kv_plane(const KvPair& p, int b, int layer, int h) {
  const int64_t c = int64_t(layer) * p.at.layer_stride + int64_t(h) * p.at.head_stride + (p.paged ? 0 : int64_t(b) * p.at.seq_stride);
  KvPlane x;
  x.k = static_cast<const char*>(p.at.base) + c;
  x.v = static_cast<const char*>(p.v) + c;
  x.table = p.at.block_table + (p.paged ? int64_t(b) * p.at.max_pages : 0);
  x.ts = uint32_t(p.at.tok_stride);
  x.paged = p.paged;
  x.page_shift = p.at.page_shift;
  x.page_mask = p.at.page_mask;
  x.page_stride = p.at.page_stride;
  return x;
}

// Where the pass over the prefixes has left row `row` of run j's queries, for KV head kvh: rows first, first + KV_ROWS, ... of
// ppart, n of them.
struct PrefixRow {
  int64_t first;
  int n;
};
__device__ __forceinline__ PrefixRow prefix_row(const KvAttnArgs& a, int j, int kvh, int64_t row) {
  const int2 at = a.pre_at[j];
  const int64_t item = row / KV_ROWS * a.hkv + kvh;
  return PrefixRow{(at.x + item * at.y) * KV_ROWS + row % KV_ROWS, at.y};
}

// The rows of a KV head that a sequence has if it is one of few rows.
__device__ __forceinline__ int few_rows_of(const KvAttnArgs& a, int b) {
  const int64_t rows = int64_t(a.cu[b + 1] - a.cu[b]) * a.g;
  return rows > FEW_ROWS ? 0 : int(rows);
}
// Those of the sequences before b, whose queries begin at q0; alike in a wave.  (Without others it is known: 300 tokens behind
// a prefix of 16000, 28 heads on 4, 185 us, counted 190.)
__device__ __forceinline__ int few_before(const KvAttnArgs& a, const int32_t* few_at, int b, int q0) {
  if (!a.mixed) return q0 * a.g;
  const int k = b / a.few_per, lane = threadIdx.x & 63;
  int n = few_at[k];
  for (int i = k * a.few_per; i < b; i += 64)
    n += __builtin_amdgcn_readlane(wave_scan(i + lane < b ? few_rows_of(a, i + lane) : 0), 63);
  return n;
}
// The sequence whose rows of that order row f is among, and its first.
__device__ __forceinline__ int few_at_row(const KvAttnArgs& a, int f, int& first) {
  const int lane = threadIdx.x & 63;
  // (groups past the last sequence begin at few_rows, so a row lies in the last group that begins no later)
  const int k = __builtin_popcountll(__ballot(a.few_at[lane] <= f)) - 1;
  first = a.few_at[k];
  int b = k * a.few_per;
  if (a.few_per == 1) return b;
  for (;; b += 64) {
    const int rows = b + lane < a.n_seqs ? few_rows_of(a, b + lane) : 0, sum = wave_scan(rows);
    const uint64_t past = __ballot(first + sum > f);
    if (past) {
      const int l = __builtin_ctzll(past);
      first += __builtin_amdgcn_readlane(sum, l) - __builtin_amdgcn_readlane(rows, l);
      return b + l;
    }
    first += __builtin_amdgcn_readlane(sum, 63);
  }
}
__device__ __forceinline__ int prefix_of(const KvAttnArgs& a, int b) {
  return last_at(a.n_prefixes, [&](int i) { return int64_t(a.pre_first[i]); }, b);
}

}  // namespace cc
