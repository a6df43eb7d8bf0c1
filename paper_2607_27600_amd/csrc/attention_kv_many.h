// Attention over a cache in bf16, many rows of a sequence and KV head: prompts and chunks of them, and the
// queries behind one prefix.  The sums, roundings and masks are those of attention_kv.hip.
//
// One workgroup of 4 waves takes 128 rows (32 a wave), a row being a (query, query head of the group)
// pair, and walks tiles of 64 entries up to the last row's.  S^T = K Q^T and O^T = V^T P^T on 32x32x16 MFMA: a lane owns
// one row, its softmax stays in its registers, and its P feeds the second product from them.  Tiles go from memory
// straight into LDS, 16-byte chunks swizzled by bits of the row so that fragment reads hit every bank once; V^T is
// read with transpose reads.  Two K and two V buffers, one barrier a tile.  The matrix instructions of one tile's
// first product carry the exponentials of the tile before, those of the second the packing of P, the row sums and
// the next maximum.
//
// Bound by the clock that the card's power allows: a prompt of 16384, 32 heads on 8, 1.87 to 2.09 ms by card (1.05 to 1.18 PFLOP/s,
// matrix cores busy in 66% of the cycles).  Short prompts are bound by what a block takes to begin and end beside its tiles,
// some 8 us: eight of 1024, 28 heads on 4, 93 us (0.65 PFLOP/s); prompts of 97 to 4001 tokens together 204 to 222 (0.9).  Loads
// are not what a tile waits for: a barrier between the products, so that each has half a step more to land, took 0 to 10% longer.
//
// Where few workgroups come of it, the entries are cut into pieces, whose results a launch of its own joins.
//
// A value in a tile that some rows see in part must not meet their probability of 0 if it is NaN or infinite: the
// waves look such tiles through, and where there is one, they set it to zero in LDS and add it to the outputs of the
// rows that see it.
#pragma once

#include <algorithm>
#include <type_traits>

#include "attention_kv.h"

namespace cc {
namespace many {

constexpr int BN = KV_KEYS;
constexpr int ROWS_W = 32;
constexpr int NWAVES = 4;

typedef short v4i16 __attribute__((ext_vector_type(4)));

template <int HD>
struct Shape {
  static constexpr int TILE = BN * HD;
  static constexpr int ROWB = HD * 2;        // bytes of a tile row
  static constexpr int CPR = HD / 8;         // 16-byte chunks of a row
  static constexpr int RPW = 64 / CPR;       // rows a wave's load fills
  static constexpr int NI = BN / (NWAVES * RPW);   // loads of a wave and tile
  static constexpr int NKS = HD / 16;
  static constexpr int NDB = HD / 32;
  static constexpr int NS = 2 * NKS;
  static constexpr int NPV = 4 * NDB;
  __device__ static constexpr int kswz(int r) { return HD == 128 ? (r & 15) : ((r >> 1) & 7); }
  __device__ static constexpr int vswz(int r) { return HD == 128 ? ((r & 3) << 2) : (((r >> 1) & 1) << 2); }
};

__device__ __forceinline__ v4i16 ds_read_tr(const char* p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4i16*)(p));
}

// 16 bytes a lane into LDS at lds + 16 * lane, by the wave, from a scalar base and a lane's offset or from a lane's
// address.  Through asm, so that the compiler counts LDS reads apart from them; the wait and the barrier at the end
// of every tile order them.
__device__ __forceinline__ void dma16(const char* sbase, uint32_t voff, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(voff), "s"(sbase), "s"(lds)
               : "memory", "m0");
}
__device__ __forceinline__ void dma16(const char* vaddr, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(vaddr), "s"(lds) : "memory", "m0");
}
__device__ __forceinline__ uint32_t lds_addr(const void* p) {
  return uint32_t(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) void*)(p)));
}

// NaN where an operand is, so that a row's maximum needs no look at its operands first: v_maximum3_f32 (a prompt of 16384, 32 heads
// on 8, 1866 us; by fmaxf, whose operands are quieted one by one, 1924).  A NaN maximum moves no reference: its row is NaN anyhow.
__device__ __forceinline__ float maximum(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// Page numbers by scalar loads, waited for at once (vector loads would be waited for behind the tiles' loads).
__device__ __forceinline__ void page_numbers(const int32_t* p0, const int32_t* p1, int& o0, int& o1) {
  asm volatile("s_load_dword %0, %2, 0x0\n\ts_load_dword %1, %3, 0x0\n\ts_waitcnt lgkmcnt(0)"
               : "=&s"(o0), "=&s"(o1) : "s"(p0), "s"(p1) : "memory");
}
__device__ __forceinline__ void page_numbers(const int32_t* p0, const int32_t* p1, const int32_t* p2, const int32_t* p3,
                                             int& o0, int& o1, int& o2, int& o3) {
  asm volatile("s_load_dword %0, %4, 0x0\n\ts_load_dword %1, %5, 0x0\n\t"
               "s_load_dword %2, %6, 0x0\n\ts_load_dword %3, %7, 0x0\n\ts_waitcnt lgkmcnt(0)"
               : "=&s"(o0), "=&s"(o1), "=&s"(o2), "=&s"(o3) : "s"(p0), "s"(p1), "s"(p2), "s"(p3) : "memory");
}

// The pieces of the pass over the prefixes, a workgroup each, prefix by prefix, of each its row blocks, KV heads and pieces in
// order.  All are of as many tiles (TILES at the least) as make no more than `slots` of them, or whole where there are
// more (row block, KV head)s than that.  Lengths are known on the device alone, so every workgroup works it out, and the
// first leaves where each prefix's begin.
struct Piece {
  int j, q0, m, len, item, nth, tiles;   // item: row block * Hkv + KV head; j < 0: none
};
constexpr int TILES = 4;
// Up to that many tiles a workgroup, half as many workgroups: 40 sequences behind 16000 entries, 4 heads of 7 rows, 49.9 us in
// place of 51.4; 64 behind 5000, 8 heads of 4, 28.3 in place of 32.2; but 24 of six tokens behind 30001 and 6000 104 for 90.
constexpr int CHAIN = 16;
__device__ __forceinline__ Piece piece_of(const KvAttnArgs& a, int64_t x) {
  const int lane = threadIdx.x & 63;
  const int64_t items = int64_t(a.blocks) * a.hkv;   // at least those there are
  struct Run {
    int q0, m, len, tiles;
    int64_t items;
  };
  auto run = [&](int i) {   // a lane's
    Run r{0, 0, 0, 0, 0};
    if (i < a.n_seqs) {
      r.q0 = a.cu[a.pre_first[i]];
      r.m = a.cu[a.pre_first[i + 1]] - r.q0;
      r.len = min(max(a.lens[i], 0), a.max_len);
      r.tiles = (r.len + BN - 1) / BN;
      r.items = (int64_t(r.m) * a.g + KV_ROWS - 1) / KV_ROWS * a.hkv;
    }
    return r;
  };
  int tiles = INT32_MAX / BN;
  if (items < a.slots) {   // (fewer than 2^31 tiles, then)
    int64_t all = 0;
    for (int i = 0; i < a.n_seqs; i += 64) {
      const Run r = run(i + lane);
      // lanes' sums of fewer than 512 items of fewer than 2^26 tiles, taken apart at bit 16
      const int64_t mine = r.items * r.tiles;
      all += (int64_t(__builtin_amdgcn_readlane(wave_scan(int(mine >> 16)), 63)) << 16) +
             __builtin_amdgcn_readlane(wave_scan(int(mine & 0xffff)), 63);
    }
    auto per = [&](int64_t groups) { return max(int64_t(TILES), (all + groups - 1) / groups); };
    // (one workgroup a CU, with half the results to pass on, while that is a chain of few tiles)
    const int half = a.slots / 2;
    tiles = int(min(int64_t(tiles), items < half && per(half - items) <= CHAIN ? per(half - items) : per(a.slots - items)));
  }
  Piece p{-1, 0, 0, 0, 0, 0, tiles};
  int64_t start = 0;
  for (int i = 0; i < a.n_seqs; i += 64) {
    const Run r = run(i + lane);
    const int n = max(1, (r.tiles + p.tiles - 1) / p.tiles);
    const int mine = int(r.items) * n;
    const int sum = wave_scan(mine);
    if (x == 0 && threadIdx.x < 64 && i + lane < a.n_seqs) a.pre_at[i + lane] = make_int2(int(start) + sum - mine, n);
    const uint64_t past = __ballot(start + sum > x);
    if (past && p.j < 0) {
      const int l = __builtin_ctzll(past);
      const int at = int(x - start) - (__builtin_amdgcn_readlane(sum, l) - __builtin_amdgcn_readlane(mine, l));
      const int each = __builtin_amdgcn_readlane(n, l);
      p.j = i + l;
      p.q0 = __builtin_amdgcn_readlane(r.q0, l);
      p.m = __builtin_amdgcn_readlane(r.m, l);
      p.len = __builtin_amdgcn_readlane(r.len, l);
      p.item = at / each;
      p.nth = at % each;
      if (x) return p;
    }
    start += __builtin_amdgcn_readlane(sum, 63);
  }
  return p;
}

// Workgroup x of a launch.  SHARED: of the pass over the prefixes.
template <int HD, bool PAGED, bool SHARED>
__device__ __forceinline__ void group(const KvAttnArgs& a, unsigned x, u16* kb0, u16* kb1, u16* vb0, u16* vb1) {
  using SH = Shape<HD>;
  constexpr int TILE = SH::TILE, ROWB = SH::ROWB, CPR = SH::CPR, RPW = SH::RPW, NI = SH::NI;
  constexpr int NKS = SH::NKS, NDB = SH::NDB, NS = SH::NS, NPV = SH::NPV;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hi = lane >> 5, col = lane & 31;

  int b, kvh, rb, q0, m, len, split, piece;
  const unsigned nth = x;
  if constexpr (SHARED) {
    const Piece p = piece_of(a, x);
    if (p.j < 0) return;
    b = p.j;
    q0 = p.q0;
    m = p.m;
    len = p.len;
    split = p.nth;
    rb = p.item / a.hkv;
    kvh = p.item % a.hkv;
    piece = p.tiles * BN;
  } else {
    // Heaviest blocks first: the last rows of the longest sequences, but before them those of sequences of few rows, whose
    // caches may be as long as any (the last ones of the list).
    // Where all are resident at once, two a CU, the second ones begin with the lightest (a prompt of 2048, 32 heads on 8, 47.4 us
    // for 49.9).
    if (gridDim.x <= 512 && x >= 256) x = gridDim.x + 255 - x;
    split = int(x % unsigned(a.splits));
    piece = a.piece;
    x /= unsigned(a.splits);
    if (a.items.n_seqs) {
      const AttnItem w = a.items.item(int(x) < a.ends ? a.blocks * a.hkv - a.ends + int(x) : int(x) - a.ends);
      b = w.seq;
      kvh = w.kvh;
      q0 = w.seq0;
      m = w.n;
      // (the list's items begin with the first blocks)
      rb = int((int64_t(m) * a.g + KV_ROWS - 1) / KV_ROWS) - 1 - w.rb;
    } else {
      // More sequences than are listed: by number, the last rows of the last one first, and a block without rows for each (16
      // prompts of 40 to 2500, 28 heads on 4, 303 us for a floor of 170; 32, which are walked, 447 for 245).
      kvh = int(x % unsigned(a.hkv));
      const int at = a.blocks - 1 - int(x / unsigned(a.hkv));
      auto first_block = [&](int b) { return int64_t(a.cu[b]) * a.g / KV_ROWS + b; };
      b = last_at(a.n_seqs, first_block, at);
      rb = int(at - first_block(b));
      q0 = a.cu[b];
      m = a.cu[b + 1] - q0;
    }
    if (m * a.g <= a.few) return;
    len = min(max(a.lens[b], 0), a.max_len);
  }
  const int rows = m * a.g, row0 = rb * KV_ROWS;
  if (row0 >= rows) return;
  const int shift = len - m;                                                   // entry of query 0
  const int i_lo = row0 / a.g, i_hi = (min(row0 + KV_ROWS, rows) - 1) / a.g;   // the block's queries
  const int c0 = split * piece, c1 = int(min(int64_t(len), int64_t(c0) + piece));
  const int see = SHARED ? c1 : min(c1, max(0, shift + i_hi + 1));     // entries [c0, see) are seen by some row
  const int full = SHARED ? c1 : min(c1, max(0, shift + i_lo + 1));    // those before it by every row
  if (split > 0 && c0 >= see) return;
  const int row = row0 + wave * ROWS_W + col;
  const bool valid = row < rows;
  const int i_row = (valid ? row : rows - 1) / a.g;
  const int past = SHARED ? len : max(0, shift + i_row + 1);           // what the row sees ends here

  bf16x8 qf[NKS];
  {
    const u16* qp = a.q + (int64_t(q0 + i_row) * a.hq + kvh * a.g + (valid ? row : rows - 1) % a.g) * HD + hi * 8;
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) qf[ks] = as_bf16x8(*reinterpret_cast<const uint4*>(qp + ks * 16));
  }

  float m_run = -INFINITY, l_run = 0.f;
  f32x16 acc[NDB];
#pragma unroll
  for (int db = 0; db < NDB; ++db) acc[db] = f32x16{};

  const int tb = c0 / BN, te = (see + BN - 1) / BN;
  if (tb < te) {
    // ---- loads.  Instruction i of wave w fills the RPW tile rows from R = 4 RPW i + RPW w on: lane l the row
    // R + l / CPR at chunk l % CPR, with the row's chunk (l % CPR) ^ swz(row).  The rows lie in one 16-entry slab
    // R / 16, i.e. one page; drow is the lane's row in it.  Rows past the end are the last entry again.
    const int drow = (RPW * NWAVES > 16 ? (wave * RPW) % 16 : wave * RPW) + lane / CPR;
    const int kch = (lane % CPR) ^ SH::kswz(drow), vch = (lane % CPR) ^ SH::vswz(drow);
    const uint32_t ts = uint32_t(a.own.at.tok_stride);
    const uint32_t klane = drow * ts + kch * 16, vlane = drow * ts + vch * 16;
    const KvPlane P = kv_plane(a.own, b, a.layer, kvh);
    const char *kplane = P.k, *vplane = P.v;
    const int last = len - 1, last_page = PAGED ? last >> P.page_shift : 0;
    const uint32_t pstride = uint32_t(P.page_stride);      // a page spans less than 4 GiB
    auto slab_of = [&](int i) { return RPW * NWAVES > 16 ? (RPW * NWAVES / 16) * i + (RPW * wave) / 16 : i; };
    auto load_pages = [&](int t, int (&pg)[NI]) {
      if constexpr (PAGED) {
        const int32_t* pp[NI];
#pragma unroll
        for (int i = 0; i < NI; ++i) pp[i] = P.table + min((t * BN + 16 * slab_of(i)) >> P.page_shift, last_page);
        if constexpr (NI == 4)
          page_numbers(pp[0], pp[1], pp[2], pp[3], pg[0], pg[1], pg[2], pg[3]);
        else
          page_numbers(pp[0], pp[1], pg[0], pg[1]);
      }
    };
    auto load = [&](u16* dst, int t, const char* plane, const char* tile_ptr, uint32_t lane_off, int ch, const int (&pg)[NI]) {
      const int key0 = t * BN;
      u16* to = dst + wave * RPW * HD;
      if (key0 + BN <= len) {
        asm volatile("" : "+v"(lane_off));   // (not widened outside the loop)
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          const int si = slab_of(i);
          const char* base;
          if constexpr (PAGED)
            base = uniform_ptr(plane + (uint64_t(uint32_t(pg[i])) * pstride + uint32_t((key0 + 16 * si) & P.page_mask) * ts));
          else
            base = tile_ptr + int64_t(16 * si) * ts;
          dma16(base, lane_off, lds_addr(to + i * NWAVES * RPW * HD));
        }
      } else {
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          const int key = min(key0 + 16 * slab_of(i) + drow, last);
          const int page = PAGED ? P.table[key >> P.page_shift] : 0;
          dma16(plane + P.offset(page, key) + ch * 16, lds_addr(to + i * NWAVES * RPW * HD));
        }
      }
    };

    // ---- fragments.  K: product j reads row (j & 1) * 32 + col, chunk 2 (j >> 1) + hi.  V^T: product j = (16-entry
    // step j / NDB, dim block j % NDB) wants dim 32 db + col of the entries of the P operand's k-slots, 4 hi + {0..3}
    // and 8 + 4 hi + {0..3} of the step: two transpose reads of 4 entries x 16 dims.
    uint32_t koff[NKS], voff[NDB];
#pragma unroll
    for (int j = 0; j < NKS; ++j) koff[j] = col * ROWB + 16 * ((2 * j + hi) ^ SH::kswz(col));
    {
      const int G = lane >> 4, L = lane & 15, y = L >> 2, r = 4 * (G >> 1) + y;
#pragma unroll
      for (int db = 0; db < NDB; ++db) {
        if constexpr (HD == 128)   // vswz(r) = 4 y: whole 64-byte groups move
          voff[db] = r * ROWB + 64 * (db ^ y) + 32 * (G & 1) + 8 * (L & 3);
        else
          voff[db] = r * ROWB + 16 * ((4 * db + 2 * (G & 1) + ((L & 3) >> 1)) ^ SH::vswz(r)) + 8 * (L & 1);
      }
    }
    auto kfrag = [&](const u16* Kl, int j) {
      return as_bf16x8(*reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(Kl) + koff[j >> 1] + (j & 1) * (32 * ROWB)));
    };
    auto vfrag = [&](const u16* Vl, int j) {
      const char* p = reinterpret_cast<const char*>(Vl) + voff[j % NDB] + (j / NDB) * (16 * ROWB);
      const v4i16 l4 = ds_read_tr(p), h4 = ds_read_tr(p + 8 * ROWB);
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(l4, h4, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    auto half_max = [](float v) {   // over the two lanes of a row
      auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
      return maximum(__uint_as_float(r[0]), __uint_as_float(r[1]));
    };
    auto row_max = [&](const f32x16(&s)[2]) {
      float v = -INFINITY;
#pragma unroll
      for (int mb = 0; mb < 2; ++mb)
#pragma unroll
        for (int e = 0; e < 16; ++e) v = maximum(v, s[mb][e]);
      return half_max(v);
    };
    auto is_masked = [&](int t) { return t * BN + BN > full; };

    // NaN and infinite values in tile t, which rows see in part: zero in LDS, added by the rows that see them.  (Every
    // wave reads the whole tile, so all come to the same answer.)
    auto any_wide = [&](const u16* Vl) {
      uint32_t bits = 0;
#pragma unroll
      for (int q = 0; q < NPV; ++q) {
        const uint4 w = __builtin_bit_cast(uint4, vfrag(Vl, q));
        bits |= wide_halves(w.x) | wide_halves(w.y) | wide_halves(w.z) | wide_halves(w.w);
      }
      return __any(bits != 0);
    };
    auto take_out = [&](u16* Vl, int t) {
      __syncthreads();
      for (int i = tid; i < TILE / 2; i += 256) {
        uint32_t& w = reinterpret_cast<uint32_t*>(Vl)[i];
        w &= ~whole_halves(wide_halves(w));
      }
      __syncthreads();
#pragma unroll 1
      for (int key = t * BN; key < min(t * BN + BN, past); ++key) {
        const int page = PAGED ? P.table[key >> P.page_shift] : 0;
        const u16* v = reinterpret_cast<const u16*>(vplane + P.offset(page, key)) + 4 * hi;
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
          for (int q = 0; q < 16; ++q) {
            const u16 y = v[db * 32 + (q >> 2) * 8 + (q & 3)];
            if ((y & 0x7f80) == 0x7f80) acc[db][q] += bf2f(y);
          }
      }
    };

    const int64_t step_bytes = int64_t(BN) * ts;
    const char* kptr = kplane + int64_t(tb + 2) * step_bytes;   // contiguous: of the next K and V loads
    const char* vptr = vplane + int64_t(tb + 1) * step_bytes;
    int kpg[NI], vpg[NI];   // pages of the tile after next (K), of the next (V), asked for a step ahead
    load_pages(tb, kpg);
    load(kb0, tb, kplane, kplane + int64_t(tb) * step_bytes, klane, kch, kpg);
    load(vb0, tb, vplane, vplane + int64_t(tb) * step_bytes, vlane, vch, kpg);
    load_pages(tb + 1, vpg);
    if (tb + 1 < te) load(kb1, tb + 1, kplane, kplane + int64_t(tb + 1) * step_bytes, klane, kch, vpg);
    if (tb + 2 < te) load_pages(tb + 2, kpg);
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    f32x16 sa[2], sb[2];
    sa[0] = f32x16{};
    sa[1] = f32x16{};
#pragma unroll
    for (int j = 0; j < NS; ++j) sa[j & 1] = mfma32(kfrag(kb0, j), qf[j >> 1], sa[j & 1]);
    if (tb + 2 < te) __syncthreads();   // every wave has read K(tb) before its buffer is refilled
    float mx = row_max(sa);

    // Tile t with parity p: S(t) in sc, its unmasked row maximum in mx; K(t + 1) and V(t) in LDS.  K(t + 2) and
    // V(t + 1) go into the buffers that the tile before has freed.
    auto step = [&](int t, auto par) {
      constexpr int p = decltype(par)::value;
      f32x16(&sc)[2] = p ? sb : sa;
      f32x16(&sn)[2] = p ? sa : sb;
      const u16* Kn = p ? kb0 : kb1;
      u16* Kfree = p ? kb1 : kb0;
      u16* Vc = p ? vb1 : vb0;
      u16* Vfree = p ? vb0 : vb1;
      if (t + 2 < te) load(Kfree, t + 2, kplane, kptr, klane, kch, kpg);
      if (t + 1 < te) load(Vfree, t + 1, vplane, vptr, vlane, vch, vpg);
      kptr += step_bytes;
      vptr += step_bytes;
      bf16x8 kf[4];
      kf[0] = kfrag(Kn, 0);
      kf[1] = kfrag(Kn, 1);
      kf[2] = kfrag(Kn, 2);
      const bool masked = is_masked(t);
      if (masked) {
#pragma unroll
        for (int mb = 0; mb < 2; ++mb)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            sc[mb][e] = t * BN + mb * 32 + (e >> 2) * 8 + hi * 4 + (e & 3) < past ? sc[mb][e] : -INFINITY;
        mx = row_max(sc);
      }
      const bool up = mx > m_run + a.room;
      const float corr = up ? fast_exp2((m_run - mx) * a.c2) : 1.f;   // 0 from -inf
      m_run = up ? mx : m_run;
      const float mc = (m_run == -INFINITY ? 0.f : m_run) * a.c2;
      sn[0] = f32x16{};
      sn[1] = f32x16{};
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_setprio(1);
      constexpr int EPM = 32 / NS;
#pragma unroll
      for (int j = 0; j < NS; ++j) {
        if (j + 3 < NS) kf[(j + 3) & 3] = kfrag(Kn, j + 3);
        sn[j & 1] = mfma32(kf[j & 3], qf[j >> 1], sn[j & 1]);
#pragma unroll
        for (int u = 0; u < EPM; ++u) {
          const int f = EPM * j + u, mb = f >> 4, e = f & 15;
          const float y = fast_exp2(fmaf(sc[mb][e], a.c2, -mc));
          asm volatile("" ::"v"(y));   // here, between the matrix instructions
          sc[mb][e] = y;
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      if (__any(corr != 1.f)) {
#pragma unroll
        for (int db = 0; db < NDB; ++db) acc[db] *= corr;
      }
      if (masked && any_wide(Vc)) take_out(Vc, t);
      bf16x8 pf[4];
      auto pack = [&](int kk) {
#pragma unroll
        for (int e = 0; e < 8; ++e) pf[kk][e] = (__bf16)sc[kk >> 1][(kk & 1) * 8 + e];
      };
      bf16x8 vf[4];
      vf[0] = vfrag(Vc, 0);
      vf[1] = vfrag(Vc, 1);
      vf[2] = vfrag(Vc, 2);
      __builtin_amdgcn_s_setprio(0);
      pack(0);
      float ls0 = 0.f, ls1 = 0.f, m0 = -INFINITY, m1 = -INFINITY;
      constexpr int SPM = 32 / NPV;
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 0; j < NPV; ++j) {
        if (j + 3 < NPV) vf[(j + 3) & 3] = vfrag(Vc, j + 3);
        acc[j % NDB] = mfma32(vf[j & 3], pf[j / NDB], acc[j % NDB]);
        if (j % NDB == NDB - 1 && j < NPV - 1) pack(j / NDB + 1);
#pragma unroll
        for (int u = 0; u < SPM; u += 2) {
          ls0 += sc[(SPM * j + u) >> 4][(SPM * j + u) & 15];
          ls1 += sc[(SPM * j + u + 1) >> 4][(SPM * j + u + 1) & 15];
        }
        asm volatile("" : "+v"(ls0), "+v"(ls1));
        // the row maximum of S(t + 1): 32 entries over the later slots
        constexpr int PER = HD == 64 ? 6 : 3;
        if (j >= 2) {
#pragma unroll
          for (int u = 0; u < PER; ++u) {
            const int f = PER * (j - 2) + u;
            if (f < 16) m0 = maximum(m0, sn[0][f]);
            else if (f < 32) m1 = maximum(m1, sn[1][f - 16]);
          }
          asm volatile("" : "+v"(m0), "+v"(m1));
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      l_run = l_run * corr + (ls0 + ls1);
      mx = half_max(maximum(m0, m1));
      if constexpr (PAGED) {
        // (no LDS read is outstanding here: the scalar loads' wait overlaps the tiles')
#pragma unroll
        for (int i = 0; i < NI; ++i) vpg[i] = kpg[i];
        if (t + 3 < te) load_pages(t + 3, kpg);
      }
      __builtin_amdgcn_s_waitcnt(0);   // this wave's tiles have landed
      __syncthreads();                 // everyone's, and everyone is done with K(t + 1) and V(t)
    };
    using I0 = std::integral_constant<int, 0>;
    using I1 = std::integral_constant<int, 1>;
    for (int t = tb; t < te; t += 2) {
      step(t, I0{});
      if (t + 1 < te) step(t + 1, I1{});
    }
  }

  float l_all = l_run + __shfl_xor(l_run, 32);
  if (a.ppart && !SHARED && split == 0 && valid) {   // a row's first entries go with its prefix
    const int j = prefix_of(a, b);
    const PrefixRow p = prefix_row(a, j, kvh, int64_t(q0 - a.cu[a.pre_first[j]]) * a.g + row);
    for (int s = 0; s < p.n; ++s) {
      const int64_t at = p.first + int64_t(s) * KV_ROWS;
      const float2 ml = a.ppart_ml[at];
      const float top = fmaxf(m_run, ml.x), ref = top == -INFINITY ? 0.f : top;
      const float c = fast_exp2((m_run - ref) * a.c2), f = fast_exp2((ml.x - ref) * a.c2);
      m_run = top;
      l_all = l_all * c + ml.y * f;
#pragma unroll
      for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const f32x4 y = *reinterpret_cast<const f32x4*>(a.ppart + at * HD + db * 32 + q * 8 + 4 * hi);
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[db][q * 4 + e] = acc[db][q * 4 + e] * c + y[e] * f;
        }
    }
  }
  if (a.part || SHARED) {
    const int before = SHARED ? 0 : a.skip ? few_before(a, a.few_at, b, q0) : a.row0;
    if (valid) {
      const int64_t prow = SHARED ? int64_t(nth) * KV_ROWS + wave * ROWS_W + col
                                  : (int64_t(kvh) * a.places + q0 * a.g - before + row) * a.splits + split;
      float* po = (SHARED ? a.ppart : a.part) + prow * HD + 4 * hi;
#pragma unroll
      for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *reinterpret_cast<float4*>(po + db * 32 + q * 8) =
              make_float4(acc[db][q * 4], acc[db][q * 4 + 1], acc[db][q * 4 + 2], acc[db][q * 4 + 3]);
      if (hi == 0) (SHARED ? a.ppart_ml : a.part_ml)[prow] = make_float2(m_run, l_all);
    }
    return;
  }
  const float inv = row_inverse(l_all);
  if (a.lse && valid && hi == 0)
    a.lse[int64_t(q0 + row / a.g) * a.hq + kvh * a.g + row % a.g] = row_lse(m_run, l_all, a.scale);
  // The outputs go out through LDS as whole rows (the K buffers are free), 16 bytes a lane.
  char* stg = reinterpret_cast<char*>(wave < 2 ? kb0 : kb1) + (wave & 1) * (ROWS_W * ROWB);
#pragma unroll
  for (int db = 0; db < NDB; ++db)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      bf16x4 o;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = (__bf16)(acc[db][q * 4 + e] * inv);
      *reinterpret_cast<bf16x4*>(stg + col * ROWB + (((db * 4 + q) ^ SH::kswz(col)) * 16) + hi * 8) = o;
    }
#pragma unroll
  for (int i = 0; i < ROWS_W * CPR / 64; ++i) {
    const int r = RPW * i + lane / CPR, c = lane % CPR;
    const uint4 v = *reinterpret_cast<const uint4*>(stg + r * ROWB + ((c ^ SH::kswz(r)) * 16));
    const int orow = row0 + wave * ROWS_W + r;
    if (orow < rows)
      *reinterpret_cast<uint4*>(a.o + (int64_t(q0 + orow / a.g) * a.hq + kvh * a.g + orow % a.g) * HD + c * 8) = v;
  }
}

}  // namespace many
}  // namespace cc
