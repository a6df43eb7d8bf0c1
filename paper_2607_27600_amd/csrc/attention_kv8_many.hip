// Attention over a cache in 8 bits, many rows of a sequence and KV head: chunks of a prompt (causal) and
// the scoring pass (counter-causal).  The sums, roundings and masks are those of attention_kv8.hip.
//
// One workgroup of 4 waves takes 128 rows (32 a wave), a row being a (query, query head of the group)
// pair, and walks tiles of 64 entries.  S^T = K Q^T and O^T = V^T P^T on 32x32x16 MFMA: a lane owns one
// row, its softmax stays in its registers, and its P feeds the second product from them.
//
// A tile's codes go from memory straight into LDS while the tile before is worked on (each lane reads
// back what its own load brought, so they need no barrier, and no registers for a whole step: with the
// codes held in registers instead the kernel spilled 376 bytes a lane and ran at a fifth of its
// speed), and are turned into bf16 once for the four waves: 32 conversions, 8 LDS writes a wave and
// tile, between the matrix instructions.  (At the end of a step, behind the loads' arrival: 677 us in
// place of 605, 8192 entries scored by 32 heads on 8.)  In LDS a tile is bf16 rows whose 16-byte chunks
// are swizzled by bits of the row so that fragment reads hit every bank once; V^T is read with transpose
// reads.  Two K and two V buffers, one barrier a tile.  Matrix work of one tile is interleaved with the
// exponentials of the tile before.
//
// Bound by the issue of a wave's instructions: 4096 entries scored by 32 heads on 8 in 165 us (830 TFLOP/s),
// against 144 us of cc_attention_cc on bf16 entries.  Counted, a matrix instruction comes with 7.9 vector, 5.6
// scalar and 2.0 LDS ones, there with 5.8, 1.8 and 1.5, and the matrix cores are busy 33% of the time, there 52%.
// (Tests of the last tiles and of the mask between the matrix instructions also cut a step into short basic
// blocks, where that kernel's are half a step long.)
//
// A NaN or infinite value in a tile that some rows see in part becomes the least bf16 number, 2^-133:
// nothing beside fp32 sums, and told from every other value by its last bit (E4M3 values end in zeros).  A
// tile that holds one sends its rows through a loop over its codes, which sets NaN where a row sees it.
#include <algorithm>
#include <type_traits>

#include "attention_kv8.h"

namespace cc {
namespace {

constexpr int BN = MANY_KEYS;
constexpr int ROWS_W = 32;
constexpr int NWAVES = 4;

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short v4i16 __attribute__((ext_vector_type(4)));
typedef short v8i16 __attribute__((ext_vector_type(8)));

template <int HD>
struct Shape {
  static constexpr int TILE = BN * HD;
  static constexpr int ROWB = HD * 2;        // bytes of a tile row in LDS
  static constexpr int CPR = HD / 16;        // 16-code pieces of a row
  static constexpr int RPW = 64 / CPR;       // rows a wave's load covers
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

// 16 bytes a lane from sbase + voff into LDS at lds + 16 * lane, by the wave.  The loads are waited for
// where their bytes are read.
__device__ __forceinline__ void dma16(const char* sbase, uint32_t voff, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(voff), "s"(sbase), "s"(lds)
               : "memory", "m0");
}
__device__ __forceinline__ uint32_t lds_addr(const void* p) {
  return uint32_t(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) void*)(p)));
}
// Sixteen codes times the scale, in bf16.
__device__ __forceinline__ void widen16(const uint4& w, float scale, uint4& lo, uint4& hi) {
  const uint32_t x[4] = {w.x, w.y, w.z, w.w};
  uint32_t y[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    y[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(int(x[i]), scale, false));
    y[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(int(x[i]), scale, true));
  }
  lo = make_uint4(y[0], y[1], y[2], y[3]);
  hi = make_uint4(y[4], y[5], y[6], y[7]);
}

template <int HD>
__global__ __launch_bounds__(256, 2) void attn_many(Kv8Args a) {
  using SH = Shape<HD>;
  constexpr int TILE = SH::TILE, ROWB = SH::ROWB, CPR = SH::CPR, NI = SH::NI;
  constexpr int NKS = SH::NKS, NDB = SH::NDB, NS = SH::NS, NPV = SH::NPV;
  __shared__ __attribute__((aligned(1024))) u16 kb0[TILE];
  __shared__ __attribute__((aligned(1024))) u16 kb1[TILE];
  __shared__ __attribute__((aligned(1024))) u16 vb0[TILE];
  __shared__ __attribute__((aligned(1024))) u16 vb1[TILE];
  // codes on their way: [load][wave][lane][16]
  __shared__ __attribute__((aligned(1024))) char kraw[BN * HD];
  __shared__ __attribute__((aligned(1024))) char vraw[BN * HD];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hi = lane >> 5, col = lane & 31;
  const bool causal = a.mask == CC_MASK_CAUSAL;

  // Heaviest blocks first: the last rows of a causal sequence, the first of a counter-causal one.
  int x = blockIdx.x;
  const int split = x % a.splits;
  x /= a.splits;
  const int kvh = x % a.hkv;
  x /= a.hkv;
  const int j = x % a.n_list, nth = a.nth0 + x / a.n_list;
  const int b = a.listed ? a.list[j] : j;
  const int q0 = a.cu[b], m = a.cu[b + 1] - q0;
  const int rows = m * a.g;
  const int blocks = (rows + MANY_ROWS - 1) / MANY_ROWS;
  if (rows <= FEW_ROWS || nth >= blocks) return;
  const int rb = causal ? blocks - 1 - nth : nth;
  const int len = min(max(a.lens[b], 0), a.max_len);
  const int c0 = split * a.piece, c1 = min(len, c0 + a.piece);
  if (split > 0 && c0 >= len) return;
  const int shift = len - m;     // cache position of query 0

  const int row0 = rb * MANY_ROWS;
  const int row = row0 + wave * ROWS_W + col;
  const bool valid = row < rows;
  const int i_row = (valid ? row : rows - 1) / a.g;
  const int hq = kvh * a.g + (valid ? row : rows - 1) % a.g;
  const int after = a.inclusive ? 0 : 1;
  // entries [lo, hi_) are seen by the row
  const int lo = causal ? 0 : max(0, shift + i_row + after);
  const int past = causal ? max(0, shift + i_row + 1) : len;

  bf16x8 qf[NKS];
  {
    const u16* qp = a.q + (int64_t(q0 + i_row) * a.hq + hq) * HD + hi * 8;
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) qf[ks] = as_bf16x8(*reinterpret_cast<const uint4*>(qp + ks * 16));
  }

  const int i_lo = row0 / a.g, i_hi = (min(row0 + MANY_ROWS, rows) - 1) / a.g;   // the block's queries
  const int see0 = max(c0, causal ? 0 : max(0, shift + i_lo + after));   // entries some row sees
  const int see1 = min(c1, causal ? max(0, shift + i_hi + 1) : len);
  const int full0 = causal ? 0 : max(0, shift + i_hi + after);           // entries every row sees
  const int full1 = causal ? max(0, shift + i_lo + 1) : len;
  const int tb = see0 / BN, te = (see1 + BN - 1) / BN;
  const int stop = min(c1, len);      // (c1 is a multiple of the tile or the sequence's end)

  float m_run = -INFINITY, l_run = 0.f;
  f32x16 acc[NDB];
#pragma unroll
  for (int db = 0; db < NDB; ++db) acc[db] = f32x16{};

  if (see0 < see1) {
    const int64_t cplane = int64_t(a.layer) * a.k.codes.layer_stride + int64_t(kvh) * a.k.codes.head_stride +
                           (a.k.paged ? 0 : int64_t(b) * a.k.codes.seq_stride);
    const int64_t splane = int64_t(a.layer) * a.k.s_layer + int64_t(kvh) * a.k.s_head +
                           (a.k.paged ? 0 : int64_t(b) * a.k.s_seq);
    const char* kplane = static_cast<const char*>(a.k.codes.base) + cplane;
    const char* vplane = static_cast<const char*>(a.v.codes.base) + cplane;
    const uint8_t* kscale = a.k.scale + splane;
    const uint8_t* vscale = a.v.scale + splane;
    const int32_t* table = a.k.paged ? a.k.codes.block_table + int64_t(b) * a.k.codes.max_pages : nullptr;
    const int last = len - 1;

    // Row of the tile and 16-code piece of this lane's load i: rows of one load lie in one 16-entry
    // group, i.e. one page and one scale block.
    const int lrow = (lane / CPR) + wave * SH::RPW;      // + i * NWAVES * RPW
    const int piece = lane % CPR;
    constexpr int RSTEP = NWAVES * SH::RPW;
    // LDS places of the two bf16 chunks: rows i * RSTEP further have the same swizzles.  A write takes eight
    // lanes at a time, and in rows of 256 bytes these should meet eight different chunks modulo 128: half of them
    // write their second chunk first, and read their codes back in that order (0.8%; nothing in rows of 128).
    const int second = HD == 128 ? piece >> 2 : 0;
    uint32_t kst[2], vst[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      kst[h] = lrow * ROWB + (((2 * piece + (h ^ second)) ^ SH::kswz(lrow)) * 16);
      vst[h] = lrow * ROWB + (((2 * piece + (h ^ second)) ^ SH::vswz(lrow)) * 16);
    }
    const uint32_t raw_off = lane * 16 + second * 8;

    // Where a tile's codes lie and their scales (K in byte 0, V in byte 1), for this wave's loads.  Pages
    // and scales are fetched a group a lane, 64 groups (16 tiles) at a time, the next ones in two steps
    // while these are used up.
    struct At {
      int64_t off[NI];
      uint32_t sc[NI];
    };
    const int glast = last >> 4;
    int gbase = tb * 4;
    auto pages_at = [&](int base) { return a.k.paged ? table[min(base + lane, glast) >> (a.k.codes.page_shift - 4)] : 0; };
    auto scales_at = [&](int base, int pg) {
      const int gg = min(base + lane, glast);
      const int slot = a.k.paged ? (gg << 4) & a.k.codes.page_mask : gg << 4;
      const int64_t o = int64_t(pg) * a.k.s_page + (slot >> a.k.block_shift);
      return uint32_t(kscale[o]) | (uint32_t(vscale[o]) << 8);
    };
    int page = pages_at(gbase), page_n = page;
    uint32_t scale = scales_at(gbase, page), scale_n = scale;
    auto look = [&](int t, At& at) {   // every tile once, in order
      const int nth = (t - tb) & 15;
      if (nth == 0 && t > tb) {
        gbase += 64;
        page = page_n;
        scale = scale_n;
      }
      if (nth == 6) page_n = pages_at(gbase + 64);
      if (nth == 11) scale_n = scales_at(gbase + 64, page_n);
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const int gg = min(t * 4 + ((wave * SH::RPW + i * RSTEP) >> 4), glast);
        const int slot = a.k.paged ? (gg << 4) & a.k.codes.page_mask : gg << 4;
        at.off[i] = int64_t(__builtin_amdgcn_readlane(page, gg - gbase)) * a.k.codes.page_stride +
                    int64_t(slot) * a.k.codes.tok_stride;
        at.sc[i] = __builtin_amdgcn_readlane(scale, gg - gbase);
      }
    };
    const uint32_t ts = uint32_t(a.k.codes.tok_stride);
    const uint32_t lane_off = (lrow & 15) * ts + piece * 16;   // (i * RSTEP is a multiple of 16)
    auto load = [&](char* raw, const char* plane, int t, const At& at) {
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        uint32_t off = lane_off;
        if (t * BN + BN > len) {   // past the end: the last entry again
          const int g0 = min(t * 4 + ((wave * SH::RPW + i * RSTEP) >> 4), glast) << 4;
          off = uint32_t(min(lrow & 15, last - g0)) * ts + piece * 16;
        }
        dma16(uniform_ptr(plane + at.off[i]), off, lds_addr(raw + (i * NWAVES + wave) * 1024));
      }
    };
    auto is_masked = [&](int t) { return t * BN < full0 || t * BN + BN > min(full1, stop); };
    auto fetch = [&](const char* raw, int i) {
      const char* p = raw + (i * NWAVES + wave) * 1024;
      const uint2 a8 = *reinterpret_cast<const uint2*>(p + raw_off), b8 = *reinterpret_cast<const uint2*>(p + (raw_off ^ 8));
      return make_uint4(a8.x, a8.y, b8.x, b8.y);
    };
    auto put = [&](u16* dst, int i, const uint4& z, int t, const At& at, auto values) {
      constexpr bool V = decltype(values)::value;
      const uint32_t byte = (at.sc[i] >> (V ? 8 : 0)) & 255u;
      const float f = e8m0_scale(byte);
      uint4 y[2];
      if (V && is_masked(t)) {
        uint32_t w[4] = {z.x, z.y, z.z, z.w}, n[4];
        const bool out = t * BN + lrow + i * RSTEP >= len;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          n[k] = out ? 0 : wide_bytes(w[k], wide_of(byte));
          w[k] = out ? 0 : w[k] & ~whole_bytes(n[k]);
        }
        widen16(make_uint4(w[0], w[1], w[2], w[3]), f, y[0], y[1]);
        auto tag = [](uint32_t& lo, uint32_t& hi, uint32_t m) {
          lo |= ((m >> 7) & 1u) | ((m << 1) & 0x10000u);
          hi |= ((m >> 23) & 1u) | ((m >> 15) & 0x10000u);
        };
        tag(y[0].x, y[0].y, n[0]);
        tag(y[0].z, y[0].w, n[1]);
        tag(y[1].x, y[1].y, n[2]);
        tag(y[1].z, y[1].w, n[3]);
      } else {
        widen16(z, f, y[0], y[1]);
      }
      char* d = reinterpret_cast<char*>(dst) + i * RSTEP * ROWB;
      *reinterpret_cast<uint4*>(d + (V ? vst : kst)[0]) = y[0];
      *reinterpret_cast<uint4*>(d + (V ? vst : kst)[1]) = y[1];
    };
    // the codes that this wave asked for have arrived; but for its latest loads of one tensor
    auto arrived = [] { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); };
    auto arrived_but = [] { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(NI) : "memory"); };
    auto read_back = [] { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); };

    uint32_t koff[NKS];
#pragma unroll
    for (int jj = 0; jj < NKS; ++jj) koff[jj] = col * ROWB + 16 * ((2 * jj + hi) ^ SH::kswz(col));
    uint32_t voff[NDB];
    {
      const int G = lane >> 4, L = lane & 15, y = L >> 2;
      const int r = 4 * (G >> 1) + y;
#pragma unroll
      for (int db = 0; db < NDB; ++db) {
        if constexpr (HD == 128)
          voff[db] = r * ROWB + 64 * (db ^ y) + 32 * (G & 1) + 8 * (L & 3);
        else
          voff[db] = r * ROWB + 16 * ((4 * db + 2 * (G & 1) + ((L & 3) >> 1)) ^ SH::vswz(r)) + 8 * (L & 1);
      }
    }
    auto kfrag = [&](const u16* Kl, int q) {
      return as_bf16x8(*reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(Kl) + koff[q >> 1] +
                                                       (q & 1) * (32 * ROWB)));
    };
    auto vfrag = [&](const u16* Vl, int q) {
      const char* p = reinterpret_cast<const char*>(Vl) + voff[q % NDB] + (q / NDB) * (16 * ROWB);
      const v4i16 l4 = ds_read_tr(p), h4 = ds_read_tr(p + 8 * ROWB);
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(l4, h4, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    auto half_max = [](float v) {
      auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
      return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    };
    auto row_max = [&](const f32x16(&s)[2]) {
      float v = -INFINITY;
#pragma unroll
      for (int mb = 0; mb < 2; ++mb)
#pragma unroll
        for (int e = 0; e < 16; ++e) v = fmaxf(v, s[mb][e]);
      return half_max(v);
    };
    auto seen = [&](int t, int mb, int e) {
      const int key = t * BN + mb * 32 + (e >> 2) * 8 + hi * 4 + (e & 3);
      return key >= lo && key < past;
    };

    using Keys = std::false_type;
    using Values = std::true_type;
    At at1, at2, at3;   // tiles t + 1, t + 2, t + 3
    look(tb, at1);
    load(kraw, kplane, tb, at1);
    load(vraw, vplane, tb, at1);
    arrived();
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      put(kb0, i, fetch(kraw, i), tb, at1, Keys{});
      put(vb0, i, fetch(vraw, i), tb, at1, Values{});
    }
    at2 = at3 = at1;
    if (tb + 1 < te) {
      look(tb + 1, at1);
      read_back();
      load(kraw, kplane, tb + 1, at1);
      arrived();
#pragma unroll
      for (int i = 0; i < NI; ++i) put(kb1, i, fetch(kraw, i), tb + 1, at1, Keys{});
      read_back();
      if (tb + 2 < te) {
        look(tb + 2, at2);
        load(kraw, kplane, tb + 2, at2);
      }
      load(vraw, vplane, tb + 1, at1);
      if (tb + 3 < te) look(tb + 3, at3);
    }
    __syncthreads();
    f32x16 sa[2], sb[2];
    sa[0] = f32x16{};
    sa[1] = f32x16{};
#pragma unroll
    for (int q = 0; q < NS; ++q) sa[q & 1] = mfma32(kfrag(kb0, q), qf[q >> 1], sa[q & 1]);
    if (tb + 2 < te) __syncthreads();   // every wave has read K(tb) before its buffer is refilled
    float mx = row_max(sa);

    // NaN into the outputs of rows that see a NaN or infinite value in tile t.
    auto poison = [&](int t) {
#pragma unroll 1
      for (int key = max(t * BN, lo); key < min(t * BN + BN, past); ++key) {
        const int gg = key >> 4;
        const int pg = a.k.paged ? table[gg >> (a.k.codes.page_shift - 4)] : 0;
        const int slot = a.k.paged ? key & a.k.codes.page_mask : key;
        const char* v = vplane + int64_t(pg) * a.k.codes.page_stride + int64_t(slot) * a.k.codes.tok_stride + 4 * hi;
        const uint32_t wide = wide_of(vscale[int64_t(pg) * a.k.s_page + (slot >> a.k.block_shift)]);
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const uint32_t n = wide_bytes(*reinterpret_cast<const uint32_t*>(v + db * 32 + q * 8), wide);
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if ((n >> (8 * e)) & 0x80u) acc[db][q * 4 + e] = __uint_as_float(0x7fc00000u);
          }
      }
    };

    // Tile t with parity P: S(t) in sc, its unmasked row maximum in mx; K(t+1) and V(t) in LDS; the codes
    // of K(t+2) and V(t+1) on their way since the step before.  K(t+2) is turned into bf16 between the
    // matrix instructions of S(t+1), V(t+1) between those of P V, into buffers that the tile before has freed,
    // and the codes of the next tile are asked for right behind.
    auto step = [&](int t, auto par) {
      constexpr int P = decltype(par)::value;
      f32x16(&sc)[2] = P ? sb : sa;
      f32x16(&sn)[2] = P ? sa : sb;
      const u16* Kn = P ? kb0 : kb1;
      u16* Kfree = P ? kb1 : kb0;
      const u16* Vc = P ? vb1 : vb0;
      u16* Vfree = P ? vb0 : vb1;
      const bool more_k = t + 2 < te, more_v = t + 1 < te;
      const bool masked = is_masked(t);
      bf16x8 kf[4];
      kf[0] = kfrag(Kn, 0);
      kf[1] = kfrag(Kn, 1);
      kf[2] = kfrag(Kn, 2);
      if (masked) {
#pragma unroll
        for (int mb = 0; mb < 2; ++mb)
#pragma unroll
          for (int e = 0; e < 16; ++e) sc[mb][e] = seen(t, mb, e) ? sc[mb][e] : -INFINITY;
        mx = row_max(sc);
      }
      const bool up = mx > m_run + a.room;
      const float corr = up ? fast_exp2((m_run - mx) * a.c2) : 1.f;
      m_run = up ? mx : m_run;
      const float mc = (m_run == -INFINITY ? 0.f : m_run) * a.c2;
      sn[0] = f32x16{};
      sn[1] = f32x16{};
      if (more_k) arrived_but();   // (V(t+1) was asked for behind K(t+2))
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_setprio(1);
      constexpr int EPM = 32 / NS;
      uint4 raw[NI];
#pragma unroll
      for (int q = 0; q < NS; ++q) {
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          if (q == 1 + 6 * i && more_k) raw[i] = fetch(kraw, i);
          if (q == 5 + 6 * i && more_k) put(Kfree, i, raw[i], t + 2, at2, Keys{});
        }
        if (q + 3 < NS) kf[(q + 3) & 3] = kfrag(Kn, q + 3);
        sn[q & 1] = mfma32(kf[q & 3], qf[q >> 1], sn[q & 1]);
#pragma unroll
        for (int u = 0; u < EPM; ++u) {
          const int f = EPM * q + u, mb = f >> 4, e = f & 15;
          const float p = fast_exp2(fmaf(sc[mb][e], a.c2, -mc));
          asm volatile("" ::"v"(p));
          sc[mb][e] = p;
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      if (t + 3 < te) load(kraw, kplane, t + 3, at3);
      if (__any(corr != 1.f)) {
#pragma unroll
        for (int db = 0; db < NDB; ++db) acc[db] *= corr;
      }
      bool tagged = false;
      if (masked) {
        uint32_t bits = 0;
#pragma unroll
        for (int q = 0; q < NPV; ++q) {
          const uint4 w = __builtin_bit_cast(uint4, vfrag(Vc, q));
          bits |= w.x | w.y | w.z | w.w;
        }
        tagged = __any((bits & 0x00010001u) != 0);
      }
      bf16x8 pf[4];
      auto pack = [&](int kk) {
#pragma unroll
        for (int e = 0; e < 8; ++e) pf[kk][e] = (__bf16)sc[kk >> 1][(kk & 1) * 8 + e];
      };
      __builtin_amdgcn_s_setprio(0);
      float ls0 = 0.f, ls1 = 0.f, m0 = -INFINITY, m1 = -INFINITY;
      bf16x8 vf[4];
      vf[0] = vfrag(Vc, 0);
      vf[1] = vfrag(Vc, 1);
      vf[2] = vfrag(Vc, 2);
      pack(0);
      constexpr int SPM = 32 / NPV;
      if (more_v) {
        if (t + 3 < te)
          arrived_but();
        else
          arrived();
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int q = 0; q < NPV; ++q) {
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          if (q == 1 + 6 * i && more_v) raw[i] = fetch(vraw, i);
          if (q == 5 + 6 * i && more_v) put(Vfree, i, raw[i], t + 1, at1, Values{});
        }
        if (q + 3 < NPV) vf[(q + 3) & 3] = vfrag(Vc, q + 3);
        acc[q % NDB] = mfma32(vf[q & 3], pf[q / NDB], acc[q % NDB]);
        if (q % NDB == NDB - 1 && q < NPV - 1) pack(q / NDB + 1);
#pragma unroll
        for (int u = 0; u < SPM; u += 2) {
          ls0 += sc[(SPM * q + u) >> 4][(SPM * q + u) & 15];
          ls1 += sc[(SPM * q + u + 1) >> 4][(SPM * q + u + 1) & 15];
        }
        asm volatile("" : "+v"(ls0), "+v"(ls1));
        // the row maximum of S(t+1): 32 entries over the later slots
        constexpr int PER = (32 + NPV - 3) / (NPV - 2);
        if (q >= 2) {
#pragma unroll
          for (int u = 0; u < PER; ++u) {
            const int f = PER * (q - 2) + u;
            if (f < 16) m0 = fmaxf(m0, sn[0][f]);
            else if (f < 32) m1 = fmaxf(m1, sn[1][f - 16]);
          }
          asm volatile("" : "+v"(m0), "+v"(m1));
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      if (masked && tagged) poison(t);
      l_run = l_run * corr + (ls0 + ls1);
      mx = half_max(fmaxf(m0, m1));
      if (more_k) load(vraw, vplane, t + 2, at2);
      at1 = at2;
      at2 = at3;
      if (t + 4 < te) look(t + 4, at3);
      __syncthreads();
    };
    using I0 = std::integral_constant<int, 0>;
    using I1 = std::integral_constant<int, 1>;
    for (int t = tb; t < te; t += 2) {
      step(t, I0{});
      if (t + 1 < te) step(t + 1, I1{});
    }
  }

  const float l_all = l_run + __shfl_xor(l_run, 32);
  if (a.splits > 1) {
    if (valid) {
      const int64_t prow = (int64_t(split) * a.hkv + kvh) * a.all + (a.listed ? a.first[j] : q0 * a.g) + row;
      float* po = a.part + prow * HD + 4 * hi;
#pragma unroll
      for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *reinterpret_cast<float4*>(po + db * 32 + q * 8) =
              make_float4(acc[db][q * 4], acc[db][q * 4 + 1], acc[db][q * 4 + 2], acc[db][q * 4 + 3]);
      if (hi == 0) a.part_ml[prow] = make_float2(m_run, l_all);
    }
    return;
  }
  const float inv = l_all == 0.f ? 0.f : 1.f / l_all;   // an empty row gives 0, a NaN sum NaN
  // The outputs go out through LDS as whole rows (the K buffers are free), 16 bytes a lane.
  char* stg = reinterpret_cast<char*>(wave < 2 ? kb0 : kb1) + (wave & 1) * (ROWS_W * ROWB);
  constexpr int OCPR = HD / 8;
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
  for (int i = 0; i < ROWS_W * OCPR / 64; ++i) {
    const int r = (64 / OCPR) * i + lane / OCPR, c = lane % OCPR;
    const uint4 v = *reinterpret_cast<const uint4*>(stg + r * ROWB + ((c ^ SH::kswz(r)) * 16));
    const int orow = row0 + wave * ROWS_W + r;
    if (orow < rows)
      *reinterpret_cast<uint4*>(a.o + (int64_t(q0 + orow / a.g) * a.hq + kvh * a.g + orow % a.g) * HD + c * 8) = v;
  }
}

}  // namespace

hipError_t launch_attn_many(const Kv8Args& args, hipStream_t s) {
  // A workgroup for each row block of the longest sequence, sequence, head and piece.  A long sequence among many
  // short ones makes more of these than one launch may have: row blocks are shared out over launches.
  const int blocks = int((int64_t(args.R) + MANY_ROWS - 1) / MANY_ROWS);
  const int64_t each = int64_t(args.n_list) * args.hkv * args.splits;
  if (each > MOST_GROUPS) return hipErrorInvalidValue;   // (refused by the planner)
  const int most = int(MOST_GROUPS / each);
  Kv8Args a = args;
  for (a.nth0 = 0; a.nth0 < blocks; a.nth0 += most) {
    const dim3 grid(unsigned(each * std::min(most, blocks - a.nth0)));
    if (a.head_dim == 128)
      hipLaunchKernelGGL(attn_many<128>, grid, dim3(256), 0, s, a);
    else
      hipLaunchKernelGGL(attn_many<64>, grid, dim3(256), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace cc
