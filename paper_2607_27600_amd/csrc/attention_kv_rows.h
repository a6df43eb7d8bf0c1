// Attention over a cache in bf16: o[i][h] = sum_j softmax_j(scale * q[i][h] . k[j][c]) v[j][c] over the entries of
// the query's prefix and its sequence's own up to the query's, c = h / g, and the log-sum-exp of each row.
//
// A row is one (query, query head of the group) pair, so the g heads that share a KV head share every entry
// that is read.  A wave streams entries from memory into MFMA operands, no LDS in the loop: few rows are bound by the bytes of
// their entries, which pass once, and a step's 16 KB in registers are what a wave keeps in flight.
//
// S^T = K Q^T on 16x16x32 MFMA, entries as its rows, so that a lane holds four entries of one row of
// queries in each 16-entry group, and the two groups of a step are the eight k-slots of its P operand:
// P never moves.  The V operand wants, for one dim, the eight entries of the lane's k-slots: a lane loads 16
// bytes (head_dim 64: 8) of each of them, 16 lanes covering the row, and turns them with byte permutations;
// dim NDB (l % 16) + i is then row l % 16 of output block i.
//
// Numbers.  Products accumulate in fp32; a row's maximum and sum are fp32, the reference maximum moving only when
// it is passed by 2^8 (numerator and sum share it).  The probabilities are rounded to bf16 for the second product
// (each by up to 2^-8 of itself, independently: what the output's own rounding costs), the sum takes them
// unrounded.
//
// Masked entries.  Scores are replaced, not added to, so what a masked key holds is lost.  A masked
// value meets a probability of 0, and 0 times NaN or infinity would reach the output: values past the
// sequence are zeroed as they are read, and in steps that some row sees in part, NaN and infinite elements are
// zeroed too and added by the rows that see them.
#pragma once

#include <algorithm>
#include <type_traits>

#include "attention_kv.h"

namespace cc {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// NR blocks of 16 rows, in a wave: queries, running maximum and sum, outputs.
template <int HD, int NR>
struct Rows {
  static constexpr int NKS = HD / 32;   // k-steps of the first product: 16-byte pieces of a lane's entry
  static constexpr int NDB = HD / 16;   // 16-dim blocks of the output: also a lane's elements of a V row
  static constexpr int VW = NDB / 2;    // words of these
  bf16x8 qf[NR][NKS];
  float m[NR], l[NR];
  f32x4 acc[NR][NDB];
  typedef uint32_t Words __attribute__((ext_vector_type(VW)));
  // a step: two groups of 16 entries
  struct Keys {
    u32x4 k[2][NKS];
  };
  struct Values {
    Words v[8];
  };

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      m[n] = -INFINITY;
      l[n] = 0.f;
#pragma unroll
      for (int d = 0; d < NDB; ++d) acc[n][d] = f32x4{};
    }
  }

  // 16-entry groups [gb, ge) of a plane of len entries, of which row block n's rows (one a lane) see those before
  // past[n], and every row those before full.
  template <bool LONG>
  __device__ __forceinline__ void run(const KvAttnArgs& a, const KvPlane& P, int gb, int ge, int len, const int (&past)[NR],
                                      int full) {
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));   // what follows from it is made anew for each item, not kept over a loop of them
    const int grp = lane >> 4, r16 = lane & 15;
    const int last = len - 1;
    const uint32_t ts = P.ts;
    // Steps before group `mid` are seen by every row.  (Past the wave's own groups counts as masked: the last group
    // stands there a second time.)
    const int stop = min(ge << 4, len);
    const int mid = gb + max(0, min(full, stop) - (gb << 4)) / 32 * 2;
    // Pages of 64 groups at a time, a lane each.
    for (int sb = gb; sb < ge; sb += 64) {
      const int se = min(ge, sb + 64);
      const int page = P.page(min(sb + lane, se - 1));
      auto base = [&](int gg) { return P.offset(__builtin_amdgcn_readlane(page, gg - sb), gg << 4); };
      // of groups gr and gr + 1 (past the end: the last one again; past a group's last entry: that one again)
      auto load_keys = [&](int gr, Keys& st) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const int gg = min(gr + t, se - 1);
          const char* kp = uniform_ptr(P.k + base(gg));
          const uint32_t ko = uint32_t(min(r16, last - (gg << 4))) * ts + 16 * grp;
#pragma unroll
          for (int k = 0; k < NKS; ++k) st.k[t][k] = load_at<u32x4>(kp, ko + 64 * k);
        }
      };
      auto load_values = [&](int gr, Values& st) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const int gg = min(gr + t, se - 1);
          const char* vp = uniform_ptr(P.v + base(gg));
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t vo = uint32_t(min(4 * grp + e, last - (gg << 4))) * ts + 2 * NDB * r16;
            st.v[4 * t + e] = load_at<Words>(vp, vo);
          }
        }
      };
      // The probabilities of a step, as far as the running maximum goes.
      auto scores = [&](int gr, const Keys& st, bf16x8(&pf)[NR], auto masked) {
        f32x4 z[NR][2];
#pragma unroll
        for (int n = 0; n < NR; ++n) z[n][0] = z[n][1] = f32x4{};
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int k = 0; k < NKS; ++k)
#pragma unroll
            for (int n = 0; n < NR; ++n) z[n][t] = mfma16(__builtin_bit_cast(bf16x8, st.k[t][k]), qf[n][k], z[n][t]);
        const int e0 = gr << 4;
        if constexpr (decltype(masked)::value) {
#pragma unroll
          for (int n = 0; n < NR; ++n)
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (e0 + 16 * t + 4 * grp + e >= min(past[n], stop)) z[n][t][e] = -INFINITY;
        }
        float mx[NR];
        bool moved = false;
#pragma unroll
        for (int n = 0; n < NR; ++n) {
          mx[n] = quad_max(fmaxf(fmaxf(fmaxf(z[n][0][0], z[n][0][1]), fmaxf(z[n][0][2], z[n][0][3])),
                                 fmaxf(fmaxf(z[n][1][0], z[n][1][1]), fmaxf(z[n][1][2], z[n][1][3]))));
          moved |= mx[n] > m[n] + a.room;
        }
        if (__any(moved)) {
#pragma unroll
          for (int n = 0; n < NR; ++n) {
            const bool up = mx[n] > m[n] + a.room;
            const float corr = up ? fast_exp2((m[n] - mx[n]) * a.c2) : 1.f;   // 0 from -inf
            if (up) m[n] = mx[n];
            l[n] *= corr;
#pragma unroll
            for (int d = 0; d < NDB; ++d) acc[n][d] *= corr;
          }
        }
#pragma unroll
        for (int n = 0; n < NR; ++n) {
          const float mc = m[n] == -INFINITY ? 0.f : m[n] * a.c2;
          float sum = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float p = fast_exp2(fmaf(z[n][e >> 2][e & 3], a.c2, -mc));
            sum += p;
            pf[n][e] = (__bf16)p;
          }
          l[n] += sum;
        }
      };
      auto values = [&](int gr, Values& st, const bf16x8(&pf)[NR], auto masked) {
        const int e0 = gr << 4;
        bool wide = false;
        if constexpr (decltype(masked)::value) {
          uint32_t bits = 0;
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
              for (int i = 0; i < VW; ++i) {
                if (e0 + 16 * t + 4 * grp + e >= stop) st.v[4 * t + e][i] = 0;   // values that the sequence does not have
                bits |= wide_halves(st.v[4 * t + e][i]);
              }
          wide = __any(bits != 0);
          if (wide) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
#pragma unroll
              for (int i = 0; i < VW; ++i) st.v[e][i] &= ~whole_halves(wide_halves(st.v[e][i]));
          }
        }
#pragma unroll
        for (int i = 0; i < VW; ++i)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            // perm(hi, lo, sel): byte k of the result is byte sel[k] of {lo: 0..3, hi: 4..7}
            const uint32_t sel = h ? 0x07060302u : 0x05040100u;
            const uint4 w = make_uint4(
                __builtin_amdgcn_perm(st.v[1][i], st.v[0][i], sel), __builtin_amdgcn_perm(st.v[3][i], st.v[2][i], sel),
                __builtin_amdgcn_perm(st.v[5][i], st.v[4][i], sel), __builtin_amdgcn_perm(st.v[7][i], st.v[6][i], sel));
#pragma unroll
            for (int n = 0; n < NR; ++n) acc[n][2 * i + h] = mfma16(as_bf16x8(w), pf[n], acc[n][2 * i + h]);
          }
        if (wide) {   // the NaN and infinite elements, for the rows that see them
#pragma unroll 1
          for (int key = e0; key < min(e0 + 32, stop); ++key) {
            const char* v = P.v + base(key >> 4) + int64_t(key & 15) * ts + 2 * NDB * 4 * grp;
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
              for (int d = 0; d < NDB; ++d) {
                const float x = bf2f(reinterpret_cast<const u16*>(v)[NDB * e + d]);
                if ((__float_as_uint(x) & 0x7f800000u) == 0x7f800000u) {
#pragma unroll
                  for (int n = 0; n < NR; ++n)
                    if (key < past[n]) acc[n][d][e] += x;
                }
              }
          }
        }
      };
      // In flight: the keys of the next step during a step's first product, its values during the second (the fences
      // keep loads from being hoisted, which takes twice the registers).  In long runs the last step asks for itself again:
      // loads under a condition are waited for as if they might not be there, which costs drafts of 8 tokens (8000
      // entries, 16 sequences, 32 heads on 8) 37 of 165 us; in short ones asking again costs more (500 entries, 8 heads, one
      // token: 10.7 us for 9.0).
      Keys k[2];
      Values v[2];
      bf16x8 pf[NR];
      const int sm = min(se, mid), end = sm - 2;
      auto step = [&](int gr, Keys& k0, Keys& k1, Values& v0, Values& v1) {
        const int next = min(gr + 2, end);
        const bool more = LONG || gr + 2 < sm;
        if (more) load_keys(next, k1);
        scores(gr, k0, pf, std::false_type{});
        __builtin_amdgcn_sched_barrier(0);
        if (more) load_values(next, v1);
        __builtin_amdgcn_sched_barrier(0);
        values(gr, v0, pf, std::false_type{});
        __builtin_amdgcn_sched_barrier(0);
      };
      if (sb < sm) {
        load_keys(sb, k[0]);
        load_values(sb, v[0]);
        int gr = sb;
        for (; gr + 2 < sm; gr += 4) {
          step(gr, k[0], k[1], v[0], v[1]);
          step(gr + 2, k[1], k[0], v[1], v[0]);
        }
        if (gr < sm) {   // (its loads are the last ones asked for)
          scores(gr, k[0], pf, std::false_type{});
          values(gr, v[0], pf, std::false_type{});
        }
      }
#pragma unroll 1
      for (int gr = max(sb, mid); gr < se; gr += 2) {   // the last ones
        load_keys(gr, k[0]);
        load_values(gr, v[0]);
        scores(gr, k[0], pf, std::true_type{});
        values(gr, v[0], pf, std::true_type{});
      }
    }
  }
};

// The waves' results of rows [row0, rows) of a (sequence, KV head) meet in LDS, [NW][ROWS][HD] outputs and [NW][ROWS] (max, sum);
// done(r, d, M, L, o) gets the eight outputs of row row0 + r from d on.
template <int HD, int NR, int NW, class F>
__device__ __forceinline__ void meet(const KvAttnArgs& a, const Rows<HD, NR>& st, float* lds, float2* ml, int rows, F done) {
  constexpr int ROWS = 16 * NR, LPR = HD / 8, NDB = HD / 16;
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));
  const int lane = tid & 63, grp = lane >> 4, r16 = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    const float l = quad_sum(st.l[n]);
    const int row = wave * ROWS + n * 16 + r16;
    if (grp == 0) ml[row] = make_float2(st.m[n], l);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float* o = lds + row * HD + NDB * (4 * grp + e);
#pragma unroll
      for (int d = 0; d < NDB; d += 4)
        *reinterpret_cast<float4*>(o + d) = make_float4(st.acc[n][d][e], st.acc[n][d + 1][e], st.acc[n][d + 2][e], st.acc[n][d + 3][e]);
    }
  }
  __syncthreads();
  for (int r = tid / LPR; r < rows; r += NW * 64 / LPR) {
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
    float4 x[2] = {make_float4(o[0], o[1], o[2], o[3]), make_float4(o[4], o[5], o[6], o[7])};
    done(r, d, M, L, x);
  }
}

// The final result of row r of the sequence of query q0, eight outputs from d on.
template <int HD>
__device__ __forceinline__ void finish(const KvAttnArgs& a, int q0, int kvh, int r, int d, float M, float L, const float4 (&o)[2]) {
  const float inv = row_inverse(L);
  const int64_t out = int64_t(q0 + r / a.g) * a.hq + kvh * a.g + r % a.g;
  *reinterpret_cast<uint4*>(a.o + out * HD + d) =
      make_uint4(pack_bf2(o[0].x * inv, o[0].y * inv), pack_bf2(o[0].z * inv, o[0].w * inv), pack_bf2(o[1].x * inv, o[1].y * inv),
                 pack_bf2(o[1].z * inv, o[1].w * inv));
  if (a.lse && d == 0) a.lse[out] = row_lse(M, L, a.scale);
}

// Rows' queries; row block n has rows row0 + 16 n ...
template <int HD, int NR>
__device__ __forceinline__ void load_queries(const KvAttnArgs& a, Rows<HD, NR>& st, int q0, int kvh, int row0, int rows, int (&i)[NR]) {
  int lane = threadIdx.x & 63;
  asm volatile("" : "+v"(lane));
  const int grp = lane >> 4, r16 = lane & 15;
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    const int row = min(row0 + 16 * n + r16, rows - 1);
    i[n] = row / a.g;
    const u16* q = a.q + (int64_t(q0 + i[n]) * a.hq + kvh * a.g + row % a.g) * HD + 8 * grp;
#pragma unroll
    for (int k = 0; k < HD / 32; ++k) st.qf[n][k] = as_bf16x8(*reinterpret_cast<const uint4*>(q + 32 * k));
  }
}

// ------------------------------------------------------------------ whole rows

// What the last of the 16 rows from row0 on sees of its mq queries' len entries.
__device__ __forceinline__ int rows_see(const KvAttnArgs& a, int mq, int len, int row0) {
  return max(0, len - mq + (min(row0 + 16, mq * a.g) - 1) / a.g + 1);
}

// One workgroup for 16 rows of a (sequence, KV head): its NW waves share out the entries, the prefix's and the sequence's, or
// (PIECES) a piece of the sequence's, to be joined.  lds: [NW][16][HD] outputs, ml: [NW][16] (max, sum).
template <int HD, int NW, bool PIECES>
__device__ __forceinline__ void rows_group(const KvAttnArgs& a, unsigned group, float* lds, float2* ml,
                                           const int32_t* few_at = nullptr) {
  constexpr int ROWS = 16;
  const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
  const int kvh = int(group % unsigned(a.hkv));
  int64_t x = group / unsigned(a.hkv);
  int split = 0;
  if constexpr (PIECES) {
    split = int(x % a.rsplits);
    x /= a.rsplits;
  }
  int b, row0;
  if (a.listed) {
    const int each = (a.R + ROWS - 1) / ROWS;
    b = a.list[int(x) / each];
    row0 = int(x) % each * ROWS;
  } else {
    // sequence b has the blocks from cu[b] g / 16 + b on, more than its rows need
    auto first_block = [&](int b) { return int64_t(a.cu[b]) * a.g / ROWS + b; };
    b = last_at(a.n_seqs, first_block, x);
    row0 = int(x - first_block(b)) * ROWS;
  }
  const int q0 = a.cu[b], mq = a.cu[b + 1] - q0, rows = mq * a.g;
  if (row0 >= rows || rows > a.most) return;
  const int len = min(max(a.lens[b], 0), a.max_len), shift = len - mq;
  const int most = rows_see(a, mq, len, row0);
  if (PIECES && split > 0 && split * a.rpiece >= most) return;
  Rows<HD, 1> st;
  int i[1];
  load_queries(a, st, q0, kvh, row0, rows, i);
  st.clear();
  auto part = [&](int g0, int g1, int& gb, int& ge) {   // this wave's, in whole steps of two
    const int per = ((g1 - g0 + NW - 1) / NW + 1) & ~1;
    gb = g0 + wave * per;
    ge = min(g1, gb + per);
  };
  int gb, ge;
  if (!PIECES && a.n_prefixes) {
    const int j = prefix_of(a, b);
    const int n = min(max(a.pre_lens[j], 0), a.pre_max);
    const int past[1] = {n};
    part(0, (n + 15) >> 4, gb, ge);
    st.template run<false>(a, kv_plane(a.pre, j, a.layer, kvh), gb, ge, n, past, n);
  }
  const int past[1] = {max(0, shift + i[0] + 1)};
  part(PIECES ? split * a.rpiece >> 4 : 0, (PIECES ? min(most, (split + 1) * a.rpiece) + 15 : most + 15) >> 4, gb, ge);
  st.template run<false>(a, kv_plane(a.own, b, a.layer, kvh), gb, ge, len, past, max(0, shift + row0 / a.g + 1));
  const int64_t place =
      PIECES ? (int64_t(split) * a.few_rows + few_before(a, few_at, b, q0)) * a.hkv + int64_t(kvh) * rows + row0 : 0;
  meet<HD, 1, NW>(a, st, lds, ml, min(ROWS, rows - row0), [&](int r, int d, float M, float L, float4(&o)[2]) {
    if constexpr (!PIECES) return finish<HD>(a, q0, kvh, row0 + r, d, M, L, o);
    const int64_t at = place + r;
    float* po = a.rpart + at * HD + d;
    *reinterpret_cast<float4*>(po) = o[0];
    *reinterpret_cast<float4*>(po + 4) = o[1];
    if (d == 0) a.rpart_ml[at] = make_float2(M, L);
  });
}

}  // namespace cc
