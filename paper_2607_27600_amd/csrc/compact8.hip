// Compaction of a cache in 8 bits: the kept entries of every cache layer and KV head move to the front
// of their plane, dst[j] = src[keep[j]], and every destination block of entries gets a scale of its
// own.  The entries of a destination block come from several source blocks with scales of their own, so
// its scale is taken from the values that they stand for, and codes whose scale changes are rounded
// again; both scales are powers of two, so only codes that leave the normal range lose bits, and an
// entry whose source has the block's scale is a bit copy.
//
// A workgroup moves chunks of rows, whole blocks: rows in registers, 16 codes a lane; a block's largest
// magnitude by an LDS maximum of whole numbers (order-free); one barrier; the codes.
//   Out of place a chunk of 128 rows (head_dim 64: 256) is a workgroup of 256 threads.  Bound by memory: of
//   four sequences a quarter kept, 8 paged layers, 115 MB in 40 to 49 us (2.9 to 2.3 TB/s; rows of 128 bytes
//   from anywhere: 94% kept reach 4.2, and a mere copy of the codes takes as long).
//   In place one workgroup walks its plane's chunks in rising order: keep is ascending, so the sources of
//   chunk c + 1 lie at or past its first row, beyond everything chunk c writes (codes and scales), and are
//   loaded before chunk c is written; the barrier of chunk c orders its own reads before its writes.
//   Bound by the chain of chunks, a round trip each, so these are four times as long (1024 threads): 15000
//   of 16000 entries, 8 layers of 4 heads, 131 us against 293 with 256 threads; that quarter 47 and 90.
#include <algorithm>

#include "cc_internal.h"

namespace cc {
namespace {

constexpr int U = 4;           // 16-byte row pieces of a thread in a chunk
constexpr int LISTS = COMPACT_INLINE;   // lists of a launch, by value

struct Args {
  Kv8View src[2], dst[2];
  const int32_t* keep;
  int n_layers, n_heads, per_head;
  int chunks, chunk0;          // workgroups of a plane (in place: 1), and the first of the launch
  int id_blocks;
  int32_t* ids[2];
  const int32_t* cu;
  CompactList lists[LISTS];
};

struct Piece {
  uint4 w[U];
  uint32_t sc[U];
};

// ids[cu_b + j] = ids[cu_b + keep[j]], in place: a chunk's reads precede its writes, and later chunks
// read at or past their own first row.
template <int NT>
__device__ __forceinline__ void move_ids(const Args& a, const CompactList& L) {
  const int32_t* keep = a.keep + L.keep_off;
  const int base = a.cu[L.seq];
  for (int j0 = 0; j0 < L.k; j0 += NT * 4) {
    int32_t x[2][4] = {};
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int s = base + keep[min(j0 + u * NT + int(threadIdx.x), L.k - 1)];
      if (a.ids[0]) x[0][u] = a.ids[0][s];
      if (a.ids[1]) x[1][u] = a.ids[1][s];
    }
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int j = j0 + u * NT + threadIdx.x;
      if (j < L.k) {
        if (a.ids[0]) a.ids[0][base + j] = x[0][u];
        if (a.ids[1]) a.ids[1][base + j] = x[1][u];
      }
    }
  }
}

// Largest magnitude of 16 codes times their scale, in the bits of an fp32 number whose exponent goes on past
// 255 (2^127 times 448 has 262; those of numbers rise with them as whole numbers; 0: nothing above 2^-127, far
// below the smallest scale).  Codes without their sign rise with the magnitudes, two to a 32-bit word by packed
// 16-bit maxima; 0x7f is NaN and does not count.
__device__ __forceinline__ uint32_t top_of(const uint4& w, uint32_t sc) {
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  const uint32_t x[4] = {w.x, w.y, w.z, w.w};
  u16x2 m = {0, 0};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, x[i] & 0x007f007fu));
    m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, (x[i] >> 8) & 0x007f007fu));
  }
  uint32_t c = max(uint32_t(m[0]), uint32_t(m[1]));
  if (c == 0x7fu) {
    c = 0;
#pragma unroll 1
    for (int i = 0; i < 16; ++i) {
      const uint32_t b = ((i < 4 ? w.x : i < 8 ? w.y : i < 12 ? w.z : w.w) >> (8 * (i & 3))) & 0x7fu;
      c = max(c, b == 0x7fu ? 0u : b);
    }
  }
  const auto f = __builtin_amdgcn_cvt_pk_f32_fp8(int(c), false);
  const int bits = int(__float_as_uint(f[0]) >> 9);   // (of a code: 9 trailing bits are zeros)
  const int e = int(min(sc, 254u)) - 127;
  return c == 0 ? 0u : uint32_t(max(bits + (e << 14), 0)) << 9;
}

// Codes in the scale 2^(from - 127), in the scale 2^(to - 127).
__device__ __forceinline__ uint4 rescale(const uint4& w, uint32_t from, uint32_t to) {
  // A scale more than 2^18 larger than the block's belongs to zeros and NaN alone; one 2^19 smaller leaves zeros.
  const float f = __uint_as_float(uint32_t(min(max(127 + int(min(from, 254u)) - int(to), 27), 227)) << 23);
  const uint32_t x[4] = {w.x, w.y, w.z, w.w};
  uint32_t y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const auto lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(int(x[i]), f, false);
    const auto hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(int(x[i]), f, true);
    y[i] = e4m3_pack(lo[0], lo[1], hi[0], hi[1]);
  }
  return make_uint4(y[0], y[1], y[2], y[3]);
}

template <int HD, bool INPLACE, int NT>
__global__ __launch_bounds__(NT) void compact8_kernel(Args a) {
  constexpr int LPR = HD / 16, ROWS = NT / LPR, CHUNK = ROWS * U;
  __shared__ uint32_t tops[2][CHUNK / 16];
  const int tid = threadIdx.x;
  if (int(blockIdx.x) < a.id_blocks) {
    move_ids<NT>(a, a.lists[a.per_head ? blockIdx.x * a.n_heads : blockIdx.x]);
    return;
  }
  int i = blockIdx.x - a.id_blocks;
  int c = 0;
  if constexpr (!INPLACE) {
    c = a.chunk0 + i % a.chunks;
    i /= a.chunks;
  }
  const int which = i & 1;
  i >>= 1;
  int head = 0;
  int list = 0;
  head = i % a.n_heads;
  i /= a.n_heads;
  const int layer = i % a.n_layers;
  i /= a.n_layers;
  list = a.per_head ? i * a.n_heads + head : i;
  const CompactList L = a.lists[list];
  const int k = L.k;
  const int nch = (k + CHUNK - 1) / CHUNK;
  if (c >= nch) return;
  const Kv8View sv = which ? a.src[1] : a.src[0], dv = which ? a.dst[1] : a.dst[0];
  const int32_t* keep = a.keep + L.keep_off;
  const int g = tid / LPR, col = (tid % LPR) * 16;
  const int shift = sv.block_shift;
  const char* sb = static_cast<const char*>(sv.codes.base) + int64_t(layer) * sv.codes.layer_stride +
                   int64_t(head) * sv.codes.head_stride + (sv.paged ? 0 : int64_t(L.seq) * sv.codes.seq_stride) + col;
  const uint8_t* ss = sv.scale + int64_t(layer) * sv.s_layer + int64_t(head) * sv.s_head +
                      (sv.paged ? 0 : int64_t(L.seq) * sv.s_seq);
  char* db = static_cast<char*>(const_cast<void*>(dv.codes.base)) + int64_t(layer) * dv.codes.layer_stride +
             int64_t(head) * dv.codes.head_stride + (dv.paged ? 0 : int64_t(L.seq) * dv.codes.seq_stride) + col;
  uint8_t* ds = dv.scale + int64_t(layer) * dv.s_layer + int64_t(head) * dv.s_head +
                (dv.paged ? 0 : int64_t(L.seq) * dv.s_seq);
  const int32_t* sbt = sv.paged ? sv.codes.block_table + int64_t(L.seq) * sv.codes.max_pages : nullptr;
  const int32_t* dbt = dv.paged ? dv.codes.block_table + int64_t(L.seq) * dv.codes.max_pages : nullptr;
  // rows past the list's end repeat its last one; they are neither counted nor written
  auto index = [&](int ch, int (&id)[U]) {
#pragma unroll
    for (int u = 0; u < U; ++u) id[u] = keep[min(ch * CHUNK + u * ROWS + g, k - 1)];
  };
  auto load = [&](const int (&id)[U], Piece& p) {
    int page[U];
#pragma unroll
    for (int u = 0; u < U; ++u) page[u] = sv.paged ? sbt[id[u] >> sv.codes.page_shift] : 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int slot = sv.paged ? id[u] & sv.codes.page_mask : id[u];
      p.w[u] = *reinterpret_cast<const uint4*>(sb + int64_t(page[u]) * sv.codes.page_stride +
                                               int64_t(slot) * sv.codes.tok_stride);
      p.sc[u] = ss[int64_t(page[u]) * sv.s_page + (slot >> shift)];
    }
  };
  int id[U];
  Piece now, next;
  index(c, id);
  load(id, now);
  if (INPLACE && c + 1 < nch) index(c + 1, id);
  if (tid < 2 * (CHUNK / 16)) (&tops[0][0])[tid] = 0;
  __syncthreads();
  const int last = INPLACE ? nch : c + 1;
  for (; c < last; ++c) {
    uint32_t* top = tops[c & 1];
    uint32_t* other = tops[(c & 1) ^ 1];
    int dpage[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int j = min(c * CHUNK + u * ROWS + g, k - 1);
      dpage[u] = dv.paged ? dbt[j >> dv.codes.page_shift] : 0;
    }
    if (INPLACE && c + 1 < nch) {
      load(id, next);
      if (c + 2 < nch) index(c + 2, id);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      uint32_t m = top_of(now.w[u], now.sc[u]);
#pragma unroll
      for (int off = 1; off < LPR; off <<= 1) m = max(m, uint32_t(__shfl_xor(int(m), off)));
      const int r = u * ROWS + g;
      if (col == 0 && c * CHUNK + r < k) atomicMax(&top[r >> shift], m);
    }
    __syncthreads();   // maxima whole; this chunk's rows and scales have all been read
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = u * ROWS + g, j = c * CHUNK + r;
      if (j < k) {
        const uint32_t e = e8m0_of(top[r >> shift]);
        uint4 w = now.w[u];
        if (e != now.sc[u]) w = rescale(w, now.sc[u], e);
        const int slot = dv.paged ? j & dv.codes.page_mask : j;
        *reinterpret_cast<uint4*>(db + int64_t(dpage[u]) * dv.codes.page_stride + int64_t(slot) * dv.codes.tok_stride) = w;
        if (col == 0 && (r & ((1 << shift) - 1)) == 0) ds[int64_t(dpage[u]) * dv.s_page + (slot >> shift)] = uint8_t(e);
      }
    }
    if constexpr (INPLACE) {
      // the other half's maxima were last read before this chunk's barrier; the next chunk's start
      // behind the barrier below
      if (tid < CHUNK / 16) other[tid] = 0;
      __syncthreads();
      now = next;
    }
  }
}

template <int HD>
hipError_t launch_dim(const Compact8Launch& l, hipStream_t s) {
  constexpr int NT = 256, NT_IN = 1024, CHUNK = NT / (HD / 16) * U;
  const int per = l.per_head ? l.n_heads : 1;
  // Sequences of a launch: their lists by value, a workgroup for each plane.  A launch has fewer than 2^32 threads,
  // so long lists out of place take several, each a range of their chunks.
  const int64_t planes = 2 * int64_t(l.n_heads) * l.n_layers;
  const int64_t most = (l.in_place ? MOST_GROUPS * 256 / NT_IN : MOST_GROUPS) - LISTS;   // (workgroups for ids aside)
  if (planes > most) return hipErrorInvalidValue;   // (refused by the caller)
  const int per_launch = int(std::min<int64_t>(LISTS / per, most / planes));
  int64_t off = 0;
  for (int lo = 0; lo < l.n_seqs; lo += per_launch) {
    Args a;
    for (int t = 0; t < 2; ++t) {
      a.src[t] = l.src[t];
      a.dst[t] = l.dst[t];
      a.ids[t] = l.ids[t];
    }
    a.keep = l.keep;
    // the longest lists first: in place a list is one workgroup's, and the last to start should be short
    const int n = std::min(per_launch, l.n_seqs - lo);
    const int32_t* k_h = l.k_h + int64_t(lo) * per;
    int order[LISTS], longest[LISTS];
    int64_t first[LISTS];
    for (int b = 0; b < n; ++b) {
      order[b] = b;
      first[b] = off;
      longest[b] = *std::max_element(k_h + b * per, k_h + (b + 1) * per);
      for (int h = 0; h < per; ++h) off += k_h[b * per + h];
    }
    std::sort(order, order + n, [&](int x, int y) { return longest[x] != longest[y] ? longest[x] > longest[y] : x < y; });
    const int longest_list = longest[order[0]];
    if (longest_list == 0) continue;
    for (int i = 0; i < n; ++i) {
      int64_t at = first[order[i]];
      for (int h = 0; h < per; ++h) {
        const int k = k_h[order[i] * per + h];
        a.lists[i * per + h] = CompactList{at, 0, k, lo + order[i]};
        at += k;
      }
    }
    a.n_layers = l.n_layers;
    a.n_heads = l.n_heads;
    a.per_head = l.per_head;
    a.cu = l.cu_d;
    a.id_blocks = l.ids[0] || l.ids[1] ? n : 0;
    const int chunks = l.in_place ? 1 : (longest_list + CHUNK - 1) / CHUNK;
    const int step = int(std::min<int64_t>(chunks, most / (n * planes)));
    for (a.chunk0 = 0; a.chunk0 < chunks; a.chunk0 += step) {
      a.chunks = std::min(step, chunks - a.chunk0);
      const dim3 grid(unsigned(a.id_blocks + n * planes * a.chunks));
      if (l.in_place)
        hipLaunchKernelGGL((compact8_kernel<HD, true, NT_IN>), grid, dim3(NT_IN), 0, s, a);
      else
        hipLaunchKernelGGL((compact8_kernel<HD, false, NT>), grid, dim3(NT), 0, s, a);
      const hipError_t err = hipGetLastError();
      if (err != hipSuccess) return err;
      a.id_blocks = 0;
    }
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_compact8(const Compact8Launch& l, hipStream_t s) {
  return l.head_dim == 128 ? launch_dim<128>(l, s) : launch_dim<64>(l, s);
}

}  // namespace cc
