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
// exactly (one conversion instruction for two codes, scale included); products accumulate in
// fp32; a row's maximum and sum are fp32, the reference maximum moving only when it is passed by 2^8
// (numerator and sum share it).  The probabilities are rounded to bf16 for the second product (off
// by 2^-9 each, independently), the sum takes them unrounded.
//
// Masked entries.  Scores are replaced, not added to, so what a masked key holds is lost.  A masked
// value meets a probability of 0, and 0 * NaN would reach the output: values past the sequence are
// zeroed as they are read, and in tiles that some row sees in part, NaN codes are zeroed too and
// counted by a second product of indicators, by the rows that may see them.
#include <algorithm>

#include "attention_kv8.h"

namespace cc {
namespace {

constexpr float kRescale = 8.f;   // log2 headroom before the reference maximum moves

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

// Bytes 0x80 where a byte of x is a NaN code (0x7f or 0xff).
__device__ __forceinline__ uint32_t nan_bytes(uint32_t x) { return ((x & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }
// x without its NaN codes; ones (code 0x38) in their places.
__device__ __forceinline__ uint32_t nan_mask(uint32_t x) { return (nan_bytes(x) >> 7) * 0xffu; }

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
__global__ __launch_bounds__(FEW_NT) void attn_few(Kv8Args a) {
  constexpr int NKS = HD / 32;          // k-steps of the first product
  constexpr int NK = HD / 64;           // 16-byte pieces of a lane's entry
  constexpr int NDB = HD / 16;          // 16-dim blocks of the output: also a lane's bytes of a V row
  constexpr int NW = FEW_NT / 64;
  constexpr int ROWS = 16 * NR;
  extern __shared__ float lds[];        // [NW][ROWS][HD] outputs, then [NW][ROWS] (max, sum)
  float2* ml = reinterpret_cast<float2*>(lds + NW * ROWS * HD);
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int grp = lane >> 4, r16 = lane & 15;
  int x = blockIdx.x;
  const int kvh = x % a.hkv;
  x /= a.hkv;
  const int split = x % a.splits, j = x / a.splits;
  const Seq s = seq_of(a, j);
  const int rows = s.m * a.g;
  if (rows == 0 || rows > FEW_ROWS) return;
  const int c0 = split * a.piece, c1 = min(s.len, c0 + a.piece);
  if (split > 0 && c0 >= s.len) return;   // the join does not read this piece

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
        const int e0 = gg << 4;
        {
          const char* p = P.k + off + int64_t(min(r16, last - e0)) * a.k.codes.tok_stride + 16 * grp;
#pragma unroll
          for (int k = 0; k < NK; ++k) st.k[t][k] = *reinterpret_cast<const uint4*>(p + 64 * k);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const char* p = P.v + off + int64_t(min(4 * grp + e, last - e0)) * a.v.codes.tok_stride + NDB * r16;
          if constexpr (NDB == 8) {
            const u32x2 w = *reinterpret_cast<const u32x2*>(p);
            st.v[4 * t + e][0] = w[0];
            st.v[4 * t + e][NDB / 4 - 1] = w[1];
          } else {
            st.v[4 * t + e][0] = *reinterpret_cast<const uint32_t*>(p);
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
      if (masked) {
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
              nans |= nan_bytes(st.v[4 * t + e][i]) != 0;
            }
          }
        nans = __any(nans);
      }
      bf16x8 pf[NR];
      bool moved = false;
      float mx[NR];
#pragma unroll
      for (int n = 0; n < NR; ++n) {
        float t = fmaxf(fmaxf(fmaxf(z[n][0][0], z[n][0][1]), fmaxf(z[n][0][2], z[n][0][3])),
                        fmaxf(fmaxf(z[n][1][0], z[n][1][1]), fmaxf(z[n][1][2], z[n][1][3])));
        mx[n] = quad_max(t);
        moved |= mx[n] > m_run[n] + kRescale / a.c2;
      }
      if (__any(moved)) {
#pragma unroll
        for (int n = 0; n < NR; ++n) {
          const bool up = mx[n] > m_run[n] + kRescale / a.c2;
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
        if (!nans) {
#pragma unroll
          for (int d = 0; d < 4; ++d) {
            const bf16x8 vf = widen44(ta[d], tb[d], vs[0], vs[1]);
#pragma unroll
            for (int n = 0; n < NR; ++n) acc[n][4 * i + d] = mfma16(vf, pf[n], acc[n][4 * i + d]);
          }
        } else {
#pragma unroll
          for (int d = 0; d < 4; ++d) {
            const uint32_t na = nan_mask(ta[d]), nb = nan_mask(tb[d]);
            const bf16x8 vf = widen44(ta[d] & ~na, tb[d] & ~nb, vs[0], vs[1]);
            const bf16x8 one = widen44(na & 0x38383838u, nb & 0x38383838u, 1.f, 1.f);
#pragma unroll
            for (int n = 0; n < NR; ++n) {
              bf16x8 see;
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                const int key = e0 + 16 * (e >> 2) + 4 * grp + (e & 3);
                see[e] = (__bf16)(key >= lo[n] && key < min(hi[n], ge << 4) ? 1.f : 0.f);
              }
              const f32x4 hits = mfma16(one, see, f32x4{});
              f32x4 o = mfma16(vf, pf[n], acc[n][4 * i + d]);
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (hits[e] > 0.f) o[e] = __uint_as_float(0x7fc00000u);
              acc[n][4 * i + d] = o;
            }
          }
        }
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
    if (a.splits > 1) {
      const int64_t row = (int64_t(split) * a.n_list * a.hkv + int64_t(j) * a.hkv + kvh) * a.R + r;
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
}

// ------------------------------------------------------------------ joining pieces

// out = sum_s o_s 2^((m_s - M) c2) / sum_s l_s 2^((m_s - M) c2), M = max m_s.  HD / 4 lanes take a row, G
// groups of them its pieces in turn, four in flight; the groups meet in LDS.  G = 8 from 8 pieces on
// (128 rows of 64 pieces: 35 us with G = 1, a chain of loads in 16 workgroups).
template <int HD, int G>
__global__ __launch_bounds__(256) void attn_join(Kv8Args a, int few) {
  constexpr int LPR = HD / 4, PER = 256 / (LPR * G);
  __shared__ float4 po[G > 1 ? 256 : 1];
  __shared__ float2 pm[G > 1 ? 256 : 1];
  const int tid = threadIdx.x;
  const int gi = tid / LPR % G, lane = tid % LPR;
  const int row_in = blockIdx.x * PER + tid / (LPR * G);
  const int d = lane * 4;
  const int64_t step = int64_t(a.n_list) * a.hkv * a.R;
  bool on = row_in < step;
  const int r = row_in % a.R, jh = on ? row_in / a.R : 0;
  const int kvh = jh % a.hkv;
  const Seq s = seq_of(a, jh / a.hkv);
  const int rows = s.m * a.g;
  on = on && r < rows && (rows <= FEW_ROWS) == (few != 0);
  const int n = min(a.splits, max(1, (s.len + a.piece - 1) / a.piece));
  float M = -INFINITY, L = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  if (on) {
    for (int i0 = gi; i0 < n; i0 += 4 * G) {
      float2 p[4];
      float4 x[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int64_t at = min(i0 + q * G, n - 1) * step + row_in;
        p[q] = a.part_ml[at];
        x[q] = *reinterpret_cast<const float4*>(a.part + at * HD + d);
      }
      float t = M;
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (i0 + q * G < n) t = fmaxf(t, p[q].x);
      const float ref = t == -INFINITY ? 0.f : t;
      const float c = fast_exp2((M - ref) * a.c2);
      M = t;
      L *= c;
      o = make_float4(o.x * c, o.y * c, o.z * c, o.w * c);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (i0 + q * G >= n) continue;
        const float f = fast_exp2((p[q].x - ref) * a.c2);
        L += p[q].y * f;
        o.x += x[q].x * f;
        o.y += x[q].y * f;
        o.z += x[q].z * f;
        o.w += x[q].w * f;
      }
    }
  }
  if constexpr (G > 1) {
    po[tid] = o;
    pm[tid] = make_float2(M, L);
    __syncthreads();
    if (gi != 0) return;
    M = -INFINITY;
#pragma unroll
    for (int q = 0; q < G; ++q) M = fmaxf(M, pm[tid + q * LPR].x);
    const float ref = M == -INFINITY ? 0.f : M;
    L = 0.f;
    o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int q = 0; q < G; ++q) {
      const float2 p = pm[tid + q * LPR];
      const float4 x = po[tid + q * LPR];
      const float f = fast_exp2((p.x - ref) * a.c2);
      L += p.y * f;
      o.x += x.x * f;
      o.y += x.y * f;
      o.z += x.z * f;
      o.w += x.w * f;
    }
  }
  if (!on) return;
  const float inv = L == 0.f ? 0.f : 1.f / L;
  u16* out = a.o + (int64_t(s.q0 + r / a.g) * a.hq + kvh * a.g + r % a.g) * HD + d;
  *reinterpret_cast<uint2*>(out) = make_uint2(pack_bf2(o.x * inv, o.y * inv), pack_bf2(o.z * inv, o.w * inv));
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
  const int64_t grid = int64_t(a.n_list) * a.splits * a.hkv;
  if (grid > INT32_MAX) return hipErrorInvalidValue;
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
  if (e != hipSuccess || a.splits == 1) return e;
  const int64_t rows = int64_t(a.n_list) * a.hkv * a.R;
  if (a.splits >= 8) {
    constexpr int PER = 256 / (HD / 4 * 8);
    hipLaunchKernelGGL((attn_join<HD, 8>), dim3(unsigned((rows + PER - 1) / PER)), dim3(256), 0, s, a, few ? 1 : 0);
  } else {
    constexpr int PER = 256 / (HD / 4);
    hipLaunchKernelGGL((attn_join<HD, 1>), dim3(unsigned((rows + PER - 1) / PER)), dim3(256), 0, s, a, few ? 1 : 0);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attention_kv8(const Kv8Args& a, bool few, hipStream_t s) {
  return a.head_dim == 128 ? launch_dim<128>(a, few, s) : launch_dim<64>(a, few, s);
}

}  // namespace cc
