// Accumulated attention weight: what each cached entry receives of the attention of a call's queries,
//   w[b][c][t] = prev[b][c][t] + sum_{i, h in group c} exp(scale * q[i][h] . k[t][c] - lse[i][h])
// over the queries i that stand at or after entry t, the scores that select by it, and its compaction.
//
// A wave holds 16 KB entries of a (sequence, KV head) as the A operands of 16x16x32 MFMA and takes the rows
// (query, head of the group) that see them 16 at a time.  A lane then holds four entries of one row, so the sum
// over rows stays in its registers until the end, where 16 lanes are added up: no atomics, one order.
// Products and sums are fp32.  Sequences of few rows (single tokens, drafts) are bound by the bytes of their keys, those of
// many by the matrix instructions and exponentials of every (row, entry) pair.
#include <algorithm>
#include <type_traits>

#include "attention_kv.h"

namespace cc {
namespace {

constexpr int NT = 256, NW = NT / 64;

// Over the 16 lanes of an entry.
__device__ __forceinline__ float row_sum(float x) {
#pragma unroll
  for (int off = 1; off < 16; off <<= 1) x += __shfl_xor(x, off);
  return x;
}

// That of element r16 of four, for lanes r16 < 4.
__device__ __forceinline__ float row_sums(const float (&v)[4], int r16) {
  float x = row_sum(v[0]);
#pragma unroll
  for (int e = 1; e < 4; ++e) {
    const float y = row_sum(v[e]);
    x = r16 == e ? y : x;
  }
  return x;
}

// The weights of a (sequence, KV head): what came of a call, added to what entries had.
struct Total {
  float* w;
  const float* prev;
  int had;
  __device__ __forceinline__ Total(const KvWeightsArgs& a, int b, int kvh, int len)
      : w(a.w + int64_t(b) * a.w_seq + int64_t(kvh) * a.w_head),
        prev(a.prev + int64_t(b) * a.prev_seq + int64_t(kvh) * a.prev_head),
        had(a.prev ? min(a.prev_lens ? a.prev_lens[b] : len, a.prev_n) : 0) {}
  __device__ __forceinline__ void put(int t, float x) const { w[t] = t < had ? prev[t] + x : x; }
};

// ------------------------------------------------------------------ few rows

// Each wave for 32 or 64 entries, whose rows it reads for itself.  Bound by the bytes of the keys: 64 sequences of 4000 entries, 28 heads
// on 4, 45 us (5.8 TB/s); eight ragged ones of up to 12001 10 us, a chain of four loads.  With 16 entries a wave (more
// workgroups, rows read twice as often) 51 and 9.7, with 64 51 and 10.6.
template <int HD, int KB>
__global__ __launch_bounds__(NT, 2) void weights_few(KvWeightsArgs a) {
  constexpr int NKS = HD / 32;
  const int tid = threadIdx.x, lane = tid & 63, grp = lane >> 4, r16 = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const unsigned blocks = unsigned(a.max_len + NW * KB * 16 - 1) / (NW * KB * 16);
  const int kvh = int(blockIdx.x % unsigned(a.hkv));
  const unsigned y = blockIdx.x / unsigned(a.hkv);
  const int b = a.seq0 + int(y / blocks), t0 = (int(y % blocks) * NW + wave) * KB * 16;
  const int len = min(max(a.lens[b], 0), a.max_len);
  if (t0 >= len) return;
  const int q0 = a.cu[b], mq = a.cu[b + 1] - q0, rows = mq * a.g, shift = len - mq;
  if (rows > W_FEW_ROWS) return;
  const KvPlane P = kv_plane(a.own, b, a.layer, kvh);

  float sum[KB][4];
#pragma unroll
  for (int k = 0; k < KB; ++k)
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[k][e] = 0.f;
  const Total to(a, b, kvh, len);
  // What the entries have had goes with the keys, a word a lane, as the sums leave (64 sequences of 4000 entries, 28 heads on 4:
  // 44.9 us, 5.8 TB/s; asked for by a lane of 16 for four entries one after another, once the sums were there, 60.8).
  float had[KB];   // of entry 4 grp + r16 of the 16, r16 < 4
  auto take_had = [&] {
#pragma unroll
    for (int k = 0; k < KB; ++k) {
      const int t = t0 + 16 * k + 4 * grp + r16;
      had[k] = r16 < 4 && t < min(len, to.had) ? to.prev[t] : 0.f;
    }
  };
  const int from = min(max(0, t0 - shift), mq) * a.g;   // the first row that sees an entry
  if (from >= rows) {
    take_had();
  } else {
    bf16x8 kf[KB][NKS];
#pragma unroll
    for (int k = 0; k < KB; ++k) {
      const int gg = min((t0 >> 4) + k, (len - 1) >> 4);
      const int t = min(16 * gg + r16, len - 1);
      const char* p = P.k + P.offset(P.page(gg), 16 * gg) + int64_t(t & 15) * P.ts + 16 * grp;
#pragma unroll
      for (int s = 0; s < NKS; ++s) kf[k][s] = as_bf16x8(*reinterpret_cast<const uint4*>(p + 64 * s));
    }
    take_had();
    const int seen = min(max(0, t0 + KB * 16 - 1 - shift), mq) * a.g;   // rows from here on see all of the wave's entries
    int i = (from + r16) / a.g, h = (from + r16) % a.g;
    const int di = 16 / a.g, dh = 16 % a.g;
    for (int r0 = from; r0 < rows; r0 += 16) {
      const bool in = r0 + r16 < rows;
      const int64_t at = int64_t(q0 + (in ? i : mq - 1)) * a.hq + kvh * a.g + (in ? h : 0);
      const float lse = a.lse[at] * kLog2e;
      const u16* q = a.q + at * HD + 8 * grp;
      f32x4 z[KB];
#pragma unroll
      for (int k = 0; k < KB; ++k) z[k] = f32x4{};
#pragma unroll
      for (int s = 0; s < NKS; ++s) {
        const bf16x8 qf = as_bf16x8(*reinterpret_cast<const uint4*>(q + 32 * s));
#pragma unroll
        for (int k = 0; k < KB; ++k) z[k] = mfma16(kf[k][s], qf, z[k]);
      }
      if (r0 < seen || r0 + 16 > rows) {
#pragma unroll
        for (int k = 0; k < KB; ++k)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (in && t0 + 16 * k + 4 * grp + e <= shift + i) sum[k][e] += fast_exp2(fmaf(z[k][e], a.c2, -lse));
      } else {
#pragma unroll
        for (int k = 0; k < KB; ++k)
#pragma unroll
          for (int e = 0; e < 4; ++e) sum[k][e] += fast_exp2(fmaf(z[k][e], a.c2, -lse));
      }
      i += di;
      h += dh;
      if (h >= a.g) {
        h -= a.g;
        ++i;
      }
    }
  }
#pragma unroll
  for (int k = 0; k < KB; ++k) {
    const float x = row_sums(sum[k], r16);
    const int t = t0 + 16 * k + 4 * grp + r16;
    if (r16 < 4 && t < len) to.w[t] = t < to.had ? had[k] + x : x;
  }
}

// ------------------------------------------------------------------ many rows

// 16 and 4 bytes a lane from a scalar base and a lane's offset into LDS at lds + 16 (4) * lane, by the wave; waited for by
// the caller.
__device__ __forceinline__ void dma16(const char* sbase, uint32_t voff, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(voff), "s"(sbase), "s"(lds)
               : "memory", "m0");
}
__device__ __forceinline__ void dma4(const char* sbase, uint32_t voff, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" ::"v"(voff), "s"(sbase), "s"(lds)
               : "memory", "m0");
}
__device__ __forceinline__ uint32_t lds_addr(const void* p) {
  return uint32_t(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) void*)(p)));
}

// One workgroup of eight waves for W_KEYS entries of a (sequence, KV head) and a chunk of the rows: 32 entries a wave, which
// stay in its registers, and tiles of W_ROWS rows that go from memory straight into LDS, two buffers, one barrier a tile.
// A prompt of 16384 tokens, 32 heads on 8: 1.04 to 1.11 ms (1 PFLOP/s).  That is what the card's power allows: at 45% matrix
// use it runs at 2.1 GHz, and 32x32x16 instructions with the exponentials of the rows before between them, in 15% fewer cycles
// (57%), at 1.7, in the same time; as four waves of 64 entries, three buffers, or rows shared in the L2, 1.03 to 1.2 ms.
constexpr int MANY_NT = 512;
template <int HD>
__global__ __launch_bounds__(MANY_NT, 4) void weights_many(KvWeightsArgs a) {
  constexpr int NW = MANY_NT / 64, KB = W_KEYS / 16 / NW, NKS = HD / 32, CPR = HD / 8, ROWB = HD * 2;
  constexpr int RPW = 64 / CPR, NI = W_ROWS / (NW * RPW);   // rows of a wave's load, loads of a wave and tile
  __shared__ __attribute__((aligned(1024))) u16 tile[2][W_ROWS * HD];
  __shared__ __attribute__((aligned(256))) float lse[2][W_ROWS];
  auto swz = [](int r) { return HD == 128 ? r & 15 : (r >> 1) & 7; };
  const int tid = threadIdx.x, lane = tid & 63, grp = lane >> 4, r16 = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const unsigned blocks = unsigned(a.max_len + W_KEYS - 1) / W_KEYS;
  unsigned x = blockIdx.x;
  const int kvh = int(x % unsigned(a.hkv));
  x /= unsigned(a.hkv);
  const int chunk = int(x % unsigned(a.chunks));
  x /= unsigned(a.chunks);
  const int j = a.seq0 + int(x / blocks), b = a.listed ? a.list[j] : j, first = int(x % blocks) * W_KEYS;
  const int len = min(max(a.lens[b], 0), a.max_len);
  const int q0 = a.cu[b], mq = a.cu[b + 1] - q0, rows = mq * a.g, shift = len - mq;
  if (rows <= W_FEW_ROWS || first >= len) return;
  const int from = min(max(0, first - shift), mq) * a.g;          // the first row that sees an entry
  const int r_lo = max(from, chunk * a.chunk) / W_ROWS * W_ROWS;  // this chunk's: whole tiles of the sequence
  const int r_hi = int(min(int64_t(rows), int64_t(chunk + 1) * a.chunk));
  // (a chunk that sees nothing is not added up; the only one writes what there was)
  if (r_lo >= r_hi && a.part) return;
  const int t0 = first + wave * KB * 16;
  const KvPlane P = kv_plane(a.own, b, a.layer, kvh);

  float sum[KB][4];
#pragma unroll
  for (int k = 0; k < KB; ++k)
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[k][e] = 0.f;
  if (r_lo < r_hi) {
    bf16x8 kf[KB][NKS];
#pragma unroll
    for (int k = 0; k < KB; ++k) {
      const int t = min(t0 + 16 * k + r16, len - 1), gg = t >> 4;
      const char* p = P.k + P.offset(P.page(gg), 16 * gg) + int64_t(t & 15) * P.ts + 16 * grp;
#pragma unroll
      for (int s = 0; s < NKS; ++s) kf[k][s] = as_bf16x8(*reinterpret_cast<const uint4*>(p + 64 * s));
    }
    // rows that this wave's entries are seen by begin here, and those that see all of them
    const int mine = min(max(0, t0 - shift), mq) * a.g, all = min(max(0, t0 + KB * 16 - 1 - shift), mq) * a.g;
    // Row r of the sequence is query r / g, head r % g of the group; the g heads of a query lie side by side.  A tile's
    // rows from its first row's query on: x = r % g + (row in the tile) is x / g queries and x % g heads further.
    // (2^24 / g rounded up gives x / g for x g < 2^24; from 64 heads on x is below 2 g.)
    const uint32_t inverse = (1u << 24) / a.g + 1;
    const uint32_t gap = uint32_t(a.hq - a.g);
    auto further = [&](uint32_t x) {   // in rows of q
      return x + (a.g < W_ROWS ? (x * inverse >> 24) * gap : x >= uint32_t(a.g) ? gap : 0);
    };
    const int di = W_ROWS / a.g, dh = W_ROWS % a.g;
    int i0 = r_lo / a.g, h0 = r_lo % a.g;      // the next tile's first row
    uint32_t q_off[NI], lse_off = 0;           // of this lane's loads
    auto offsets = [&](int left) {             // left: rows that there are from the tile on
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const int r = (i * NW + wave) * RPW + lane / CPR;
        q_off[i] = further(h0 + min(r, left - 1)) * ROWB + ((lane % CPR) ^ swz(r)) * 16;
      }
      lse_off = further(h0 + min(lane, left - 1)) * 4;
    };
    auto load = [&](int buf, int r0) {         // tile r0, the next one
      if (r0 == r_lo || dh || r0 + W_ROWS > rows) offsets(rows - r0);
      const int64_t row = int64_t(q0 + i0) * a.hq + kvh * a.g;
      const char* qp = reinterpret_cast<const char*>(a.q) + row * ROWB;
#pragma unroll
      for (int i = 0; i < NI; ++i) dma16(qp, q_off[i], lds_addr(tile[buf] + (i * NW + wave) * RPW * HD));
      if (wave == 0) dma4(reinterpret_cast<const char*>(a.lse + row), lse_off, lds_addr(lse[buf]));
      i0 += di;
      h0 += dh;
      if (h0 >= a.g) {
        h0 -= a.g;
        ++i0;
      }
    };
    load(0, r_lo);
    int buf = 0;
    for (int r0 = r_lo; r0 < r_hi; r0 += W_ROWS, buf ^= 1) {
      __builtin_amdgcn_s_waitcnt(0);   // this wave's part of the tile has landed
      __syncthreads();                 // everyone's, and everyone is done with the other buffer
      if (r0 + W_ROWS < r_hi) load(buf ^ 1, r0 + W_ROWS);
      if (r0 + W_ROWS <= mine) continue;
      // The products of 16 rows with a wave's entries carry the exponentials of the 16 before: one of each takes as
      // long as the other's issue.
      auto take = [&](auto masked) {
        constexpr int NB = W_ROWS / 16;
        f32x4 z[2][KB];
#pragma unroll
        for (int n = 0; n <= NB; ++n) {
          const int r = 16 * n + r16, m = n - 1;
          const char* rowp = reinterpret_cast<const char*>(tile[buf]) + r * ROWB;
          bf16x8 qf[NKS];
          if (n < NB) {
#pragma unroll
            for (int s = 0; s < NKS; ++s) qf[s] = as_bf16x8(*reinterpret_cast<const uint4*>(rowp + (((4 * s + grp) ^ swz(r)) * 16)));
#pragma unroll
            for (int k = 0; k < KB; ++k) z[n & 1][k] = f32x4{};
          }
          const float l2 = n > 0 ? lse[buf][16 * m + r16] * kLog2e : 0.f;
          const bool in = n > 0 && r0 + 16 * m + r16 < r_hi;
          const int last = n > 0 ? shift + (r0 + 16 * m + r16) / a.g : 0;
          // element f of 4 KB: its argument two slots ahead, its power one ahead, its sum
          float arg[4 * KB], p[4 * KB];
          auto argument = [&](int f) { arg[f] = fmaf(z[m & 1][f >> 2][f & 3], a.c2, -l2); };
          auto power = [&](int f) {
            p[f] = fast_exp2(arg[f]);
            if constexpr (decltype(masked)::value) p[f] = in && t0 + 16 * (f >> 2) + 4 * grp + (f & 3) <= last ? p[f] : 0.f;
          };
          if (n > 0) {
            argument(0);
            argument(1);
            power(0);
          }
          constexpr int SLOTS = NKS * KB, PER = 4 * KB / SLOTS;
#pragma unroll
          for (int slot = 0; slot < SLOTS; ++slot) {
            const int s = slot / KB, k = slot % KB;
            if (n < NB) z[n & 1][k] = mfma16(kf[k][s], qf[s], z[n & 1][k]);
            if (n > 0) {
#pragma unroll
              for (int f = slot * PER; f < slot * PER + PER; ++f) {
                if (f + 2 < 4 * KB) argument(f + 2);
                if (f + 1 < 4 * KB) power(f + 1);
                sum[f >> 2][f & 3] += p[f];
                asm volatile("" : "+v"(sum[f >> 2][f & 3]));   // here, between the matrix instructions
              }
            }
            __builtin_amdgcn_sched_barrier(0);
          }
        }
      };
      if (r0 < all || r0 + W_ROWS > r_hi)
        take(std::true_type{});
      else
        take(std::false_type{});
    }
  }
  const Total to(a, b, kvh, len);
  float* part = a.part ? a.part + ((int64_t(chunk) * a.n_list + j) * a.hkv + kvh) * a.max_len : nullptr;
#pragma unroll
  for (int k = 0; k < KB; ++k) {
    const float y = row_sums(sum[k], r16);
    const int t = t0 + 16 * k + 4 * grp + r16;
    if (r16 < 4 && t < len) {
      if (part)
        part[t] = y;
      else
        to.put(t, y);
    }
  }
}

// Adds up the chunks of an entry, in their order.
__global__ __launch_bounds__(NT) void add_chunks(KvWeightsArgs a, int blocks) {
  unsigned x = blockIdx.x;
  const int t = int(x % unsigned(blocks)) * NT + int(threadIdx.x);
  x /= unsigned(blocks);
  const int kvh = int(x % unsigned(a.hkv)), j = a.seq0 + int(x / unsigned(a.hkv)), b = a.listed ? a.list[j] : j;
  const int len = min(max(a.lens[b], 0), a.max_len);
  const int mq = a.cu[b + 1] - a.cu[b], rows = mq * a.g, shift = len - mq;
  if (rows <= W_FEW_ROWS || t >= len) return;
  // what its workgroup's entries are seen by
  const int from = min(max(0, t / W_KEYS * W_KEYS - shift), mq) * a.g;
  const float* part = a.part + (int64_t(j) * a.hkv + kvh) * a.max_len + t;
  const int64_t step = int64_t(a.n_list) * a.hkv * a.max_len;
  float y = 0.f;
  if (from < rows)
    for (int c = from / a.chunk; c <= (rows - 1) / a.chunk; ++c) y += part[c * step];
  Total(a, b, kvh, len).put(t, y);
}

// A score a thread: 768 entries, 4 heads, 2.4 us, the launch and one chain of loads.
__global__ __launch_bounds__(NT) void weight_scores(WeightScoresArgs a, int blocks) {
  const int planes = a.per_head ? a.hkv : 1;
  const int h = int(blockIdx.x % unsigned(planes));
  const unsigned y = blockIdx.x / unsigned(planes);
  const int b = a.seq0 + int(y / unsigned(blocks)), t = int(y % unsigned(blocks)) * NT + int(threadIdx.x);
  const int q0 = a.cu[b], n = a.cu[b + 1] - q0;
  if (t >= n) return;
  const float* w = a.w + int64_t(b) * a.w_seq + t;
  float x = INFINITY;
  if (t >= a.frozen && t < n - a.recent) {
    x = w[int64_t(h) * a.w_head];
    if (!a.per_head)
      for (int k = 1; k < a.hkv; ++k) x += w[int64_t(k) * a.w_head];
  }
  a.scores[(a.per_head ? int64_t(q0) * a.hkv + int64_t(h) * n : int64_t(q0)) + t] = x;
}

// Keep lists of a launch.
struct WeightLists {
  static constexpr int MOST = 64;
  int64_t off[MOST];
  int32_t k[MOST];
};
constexpr int MOVE_NT = 1024, PER = 4;
// A workgroup a plane (in place) or a chunk of one: chunks of 4096 entries.  In place, lists rise, so keep[j] >= j: what
// a chunk writes lies before every later chunk's sources.  4 bytes an entry kept beside the 512 of its keys and values: 512 of 768,
// 4 heads, 2.8 us, the launch and two dependent loads.
__global__ __launch_bounds__(MOVE_NT) void move_weights(CompactWeightsArgs a, WeightLists lists, int first, int chunks, int in_place) {
  const int plane = int(blockIdx.x / unsigned(chunks)), chunk = int(blockIdx.x % unsigned(chunks));
  const int l = a.per_head ? plane : plane / a.hkv;
  const int b = (a.per_head ? (first + plane) / a.hkv : first + l), h = (a.per_head ? first + plane : plane) % a.hkv;
  const int n = lists.k[l];
  const int32_t* keep = a.keep + lists.off[l];
  const float* src = a.w + int64_t(b) * a.w_seq + int64_t(h) * a.w_head;
  float* dst = a.out + int64_t(b) * a.out_seq + int64_t(h) * a.out_head;
  for (int64_t c0 = int64_t(chunk) * MOVE_NT * PER; c0 < n; c0 += int64_t(chunks) * MOVE_NT * PER) {
    float x[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int64_t j = c0 + i * MOVE_NT + int(threadIdx.x);
      x[i] = j < n ? src[keep[j]] : 0.f;
    }
    if (in_place) __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int64_t j = c0 + i * MOVE_NT + int(threadIdx.x);
      if (j < n) dst[j] = x[i];
    }
  }
}

// f(arguments, workgroups) for as many sequences at a time as a launch has workgroups for, `each` of them a sequence (the
// planner refuses more of these than a launch's).
template <class A, class F>
hipError_t by_sequences(A a, int n, int64_t each, F f) {
  if (each > MOST_GROUPS) return hipErrorInvalidValue;
  const int64_t step = MOST_GROUPS / std::max<int64_t>(1, each);
  for (int64_t s = 0; s < n; s += step) {
    a.seq0 = int(s);
    f(a, unsigned(std::min(step, n - s) * each));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
}  // namespace

hipError_t launch_weights_few(const KvWeightsArgs& a, hipStream_t s) {
  auto launch = [&](auto blocks16, auto kernel) {
    constexpr int SPAN = NW * decltype(blocks16)::value * 16;
    return by_sequences(a, a.n_seqs, (int64_t(a.max_len) + SPAN - 1) / SPAN * a.hkv, [&](const KvWeightsArgs& x, unsigned grid) {
      hipLaunchKernelGGL(kernel, dim3(grid), dim3(NT), 0, s, x);
    });
  };
  // Rows of drafts are as many bytes as the entries: 64 of those a wave, so that rows are read half as often, where that
  // leaves workgroups enough (8 sequences of 8 tokens behind 3000 entries, 32 heads on 8, 13.9 us and 15.4, of 16 16.6 and 20.8; but
  // one of 8 behind 1000 6.6 and 5.1, and 16 of 3 behind 4000, 28 heads on 4, 19.7 and 18.6).
  const bool wide = a.R >= 32 && (int64_t(a.max_len) + 255) / 256 * a.hkv * a.n_seqs >= 512;
  using I2 = std::integral_constant<int, 2>;
  using I4 = std::integral_constant<int, 4>;
  if (a.head_dim == 128)
    return wide ? launch(I4{}, weights_few<128, 4>) : launch(I2{}, weights_few<128, 2>);
  return wide ? launch(I4{}, weights_few<64, 4>) : launch(I2{}, weights_few<64, 2>);
}

hipError_t launch_weights_many(const KvWeightsArgs& a, hipStream_t s) {
  const int64_t each = (int64_t(a.max_len) + W_KEYS - 1) / W_KEYS * a.chunks * a.hkv;
  const hipError_t e = by_sequences(a, a.n_list, 2 * each, [&](const KvWeightsArgs& x, unsigned grid) {   // (of 512)
    if (a.head_dim == 128)
      hipLaunchKernelGGL(weights_many<128>, dim3(grid / 2), dim3(MANY_NT), 0, s, x);
    else
      hipLaunchKernelGGL(weights_many<64>, dim3(grid / 2), dim3(MANY_NT), 0, s, x);
  });
  if (e != hipSuccess || !a.part) return e;
  const int blocks = (a.max_len + NT - 1) / NT;
  return by_sequences(a, a.n_list, int64_t(blocks) * a.hkv, [&](const KvWeightsArgs& x, unsigned grid) {
    hipLaunchKernelGGL(add_chunks, dim3(grid), dim3(NT), 0, s, x, blocks);
  });
}

hipError_t launch_weight_scores(const WeightScoresArgs& a, hipStream_t s) {
  const int blocks = (a.longest + NT - 1) / NT;
  return by_sequences(a, a.n_seqs, int64_t(blocks) * (a.per_head ? a.hkv : 1), [&](const WeightScoresArgs& x, unsigned grid) {
    hipLaunchKernelGGL(weight_scores, dim3(grid), dim3(NT), 0, s, x, blocks);
  });
}

hipError_t launch_compact_weights(const CompactWeightsArgs& a, hipStream_t s) {
  const bool in_place = a.out == a.w;
  const int64_t n = int64_t(a.n_seqs) * (a.per_head ? a.hkv : 1);
  int64_t off = 0;
  // the lists of a launch, of fewer than 2^32 threads; planes that leave each a workgroup at the least
  const int64_t planes = a.per_head ? 1 : a.hkv;
  if (planes > MOST_GROUPS / 4) return hipErrorInvalidValue;   // (refused at the entry)
  const int64_t step = std::min<int64_t>(WeightLists::MOST, MOST_GROUPS / 4 / planes);
  for (int64_t first = 0; first < n; first += step) {
    const int here = int(std::min<int64_t>(step, n - first));
    WeightLists lists;
    int most = 0;
    for (int i = 0; i < here; ++i) {
      lists.off[i] = off;
      lists.k[i] = a.k_h[first + i];
      off += lists.k[i];
      most = std::max(most, lists.k[i]);
    }
    if (most == 0) continue;
    const int64_t cut = (int64_t(most) + MOVE_NT * PER - 1) / (MOVE_NT * PER), room = MOST_GROUPS / 4 / (here * planes);
    const int chunks = in_place ? 1 : int(std::min(cut, room));
    const int64_t grid = here * planes * chunks;
    hipLaunchKernelGGL(move_weights, dim3(unsigned(grid)), dim3(MOVE_NT), 0, s, a, lists, int(first), chunks, int(in_place));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace cc
