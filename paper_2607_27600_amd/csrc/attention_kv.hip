// Attention over a cache in bf16: o[i][h] = sum_j softmax_j(scale * q[i][h] . k[j][c]) v[j][c] over the entries of
// the query's prefix and its sequence's own up to the query's, c = h / g, and the log-sum-exp of each row.
//
// A row is one (query, query head of the group) pair, so the g heads that share a KV head share every entry
// that is read.  A wave streams entries from memory into MFMA operands, no LDS in the loop.
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
#include "attention_kv.h"

namespace cc {
namespace {

constexpr int NT = 256, NW = NT / 64;

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// Maximum and sum over the four lanes l % 16 + 16 k.
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

// NR blocks of 16 rows, in a wave: queries, running maximum and sum, outputs.
template <int HD, int NR>
struct Rows {
  static constexpr int NKS = HD / 32;   // k-steps of the first product: 16-byte pieces of a lane's entry
  static constexpr int NDB = HD / 16;   // 16-dim blocks of the output: also a lane's elements of a V row
  static constexpr int VW = NDB / 2;    // words of these
  bf16x8 qf[NR][NKS];
  float m[NR], l[NR];
  f32x4 acc[NR][NDB];
  struct Step {                         // two groups of 16 entries
    uint4 k[2][NKS];
    uint32_t v[8][VW];
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
  __device__ __forceinline__ void run(const KvAttnArgs& a, const KvPlane& P, int gb, int ge, int len, const int (&past)[NR],
                                      int full) {
    const int lane = threadIdx.x & 63, grp = lane >> 4, r16 = lane & 15;
    const int last = len - 1;
    const uint32_t ts = P.ts;
    // Pages of 64 groups at a time, a lane each.
    for (int sb = gb; sb < ge; sb += 64) {
      const int se = min(ge, sb + 64);
      const int page = P.page(min(sb + lane, se - 1));
      auto base = [&](int gg) { return P.offset(__builtin_amdgcn_readlane(page, gg - sb), gg << 4); };
      auto load = [&](int gr, Step& st) {   // groups gr and gr + 1 (past the end: the last one again)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const int gg = min(gr + t, se - 1);
          const int64_t off = base(gg);
          const char* kp = uniform_ptr(P.k + off);
          const char* vp = uniform_ptr(P.v + off);
          const int have = last - (gg << 4);   // the group's last entry; past it: that one again
          const uint32_t ko = uint32_t(min(r16, have)) * ts + 16 * grp;
#pragma unroll
          for (int k = 0; k < NKS; ++k) st.k[t][k] = *reinterpret_cast<const uint4*>(kp + ko + 64 * k);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const char* x = vp + uint32_t(min(4 * grp + e, have)) * ts + 2 * NDB * r16;
            if constexpr (VW == 4) {
              const uint4 w = *reinterpret_cast<const uint4*>(x);
              st.v[4 * t + e][0] = w.x;
              st.v[4 * t + e][1] = w.y;
              st.v[4 * t + e][VW - 2] = w.z;
              st.v[4 * t + e][VW - 1] = w.w;
            } else {
              const uint2 w = *reinterpret_cast<const uint2*>(x);
              st.v[4 * t + e][0] = w.x;
              st.v[4 * t + e][1] = w.y;
            }
          }
        }
      };
      auto compute = [&](int gr, Step& st) {
        f32x4 z[NR][2];
#pragma unroll
        for (int n = 0; n < NR; ++n) z[n][0] = z[n][1] = f32x4{};
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int k = 0; k < NKS; ++k)
#pragma unroll
            for (int n = 0; n < NR; ++n) z[n][t] = mfma16(as_bf16x8(st.k[t][k]), qf[n][k], z[n][t]);
        const int e0 = gr << 4;
        // past the wave's own groups counts as masked: the last group stands there a second time
        const int stop = min(ge << 4, len);
        const bool masked = e0 + 32 > min(full, stop);
        bool wide = false;
        if (masked) {
#pragma unroll
          for (int n = 0; n < NR; ++n)
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (e0 + 16 * t + 4 * grp + e >= min(past[n], stop)) z[n][t][e] = -INFINITY;
          uint32_t bits = 0;
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
              for (int i = 0; i < VW; ++i) {
                uint32_t& w = st.v[4 * t + e][i];
                if (e0 + 16 * t + 4 * grp + e >= stop) w = 0;   // values that the sequence does not have
                bits |= wide_halves(w);
              }
          wide = __any(bits != 0);
          if (wide) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
#pragma unroll
              for (int i = 0; i < VW; ++i) st.v[e][i] &= ~whole_halves(wide_halves(st.v[e][i]));
          }
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
        bf16x8 pf[NR];
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
                if (!(fabsf(x) < INFINITY)) {
#pragma unroll
                  for (int n = 0; n < NR; ++n)
                    if (key < past[n]) acc[n][d][e] += x;
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
  }
};

// One workgroup for 16 rows of a (sequence, KV head): its waves share out the entries, the prefix's and the
// sequence's, and their results meet in LDS.
template <int HD>
__global__ __launch_bounds__(NT, 2) void attn_rows(KvAttnArgs a) {
  constexpr int ROWS = 16, LPR = HD / 8;
  using R = Rows<HD, 1>;
  constexpr int NDB = R::NDB;
  __shared__ float lds[NW * ROWS * HD];
  __shared__ float2 ml[NW * ROWS];
  const int tid = threadIdx.x, lane = tid & 63, grp = lane >> 4, r16 = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kvh = int(blockIdx.x % unsigned(a.hkv));
  const int64_t x = blockIdx.x / unsigned(a.hkv);
  // sequence b has the blocks from cu[b] g / 16 + b on, more than its rows need
  auto first_block = [&](int b) { return int64_t(a.cu[b]) * a.g / ROWS + b; };
  const int b = last_at(a.n_seqs, first_block, x);
  const int q0 = a.cu[b], mq = a.cu[b + 1] - q0, rows = mq * a.g;
  const int row0 = int(x - first_block(b)) * ROWS;
  if (row0 >= rows || (!a.n_prefixes && rows > KV_FEW_ROWS)) return;
  const int len = min(max(a.lens[b], 0), a.max_len), shift = len - mq;
  const int row = min(row0 + r16, rows - 1), i = row / a.g;
  R st;
  {
    const u16* q = a.q + (int64_t(q0 + i) * a.hq + kvh * a.g + row % a.g) * HD + 8 * grp;
#pragma unroll
    for (int k = 0; k < R::NKS; ++k) st.qf[0][k] = as_bf16x8(*reinterpret_cast<const uint4*>(q + 32 * k));
  }
  st.clear();
  auto part = [&](int groups, int& gb, int& ge) {   // this wave's, in whole steps of two
    const int per = ((groups + NW - 1) / NW + 1) & ~1;
    gb = wave * per;
    ge = min(groups, gb + per);
  };
  int gb, ge;
  if (a.n_prefixes) {
    const int j = last_at(a.n_prefixes, [&](int i) { return int64_t(a.pre_first[i]); }, b);
    const int n = min(max(a.pre_lens[j], 0), a.pre_max);
    const int past[1] = {n};
    part((n + 15) >> 4, gb, ge);
    st.run(a, kv_plane(a.pre, j, a.layer, kvh), gb, ge, n, past, n);
  }
  const int past[1] = {max(0, shift + i + 1)};
  const int most = max(0, shift + (min(row0 + ROWS, rows) - 1) / a.g + 1);   // what the last row sees
  part((most + 15) >> 4, gb, ge);
  st.run(a, kv_plane(a.own, b, a.layer, kvh), gb, ge, len, past, max(0, shift + row0 / a.g + 1));

  const float l = quad_sum(st.l[0]);
  if (grp == 0) ml[wave * ROWS + r16] = make_float2(st.m[0], l);
#pragma unroll
  for (int e = 0; e < 4; ++e)
#pragma unroll
    for (int d = 0; d < NDB; ++d) lds[(wave * ROWS + r16) * HD + NDB * (4 * grp + e) + d] = st.acc[0][d][e];
  __syncthreads();
  for (int r = tid / LPR; r < min(ROWS, rows - row0); r += NT / LPR) {
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
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] += lds[(w * ROWS + r) * HD + d + e] * f;
    }
    // an empty row has L = 0 and outputs 0; a NaN sum stays NaN
    const float inv = L == 0.f ? 0.f : 1.f / L;
    const int64_t out = int64_t(q0 + (row0 + r) / a.g) * a.hq + kvh * a.g + (row0 + r) % a.g;
    *reinterpret_cast<uint4*>(a.o + out * HD + d) = make_uint4(pack_bf2(o[0] * inv, o[1] * inv), pack_bf2(o[2] * inv, o[3] * inv),
                                                               pack_bf2(o[4] * inv, o[5] * inv), pack_bf2(o[6] * inv, o[7] * inv));
    if (a.lse && d == 0) a.lse[out] = row_lse(ref, L, a.scale);
  }
}

}  // namespace

hipError_t launch_attn_rows(const KvAttnArgs& a, hipStream_t s) {
  const int64_t blocks = (int64_t(a.N) * a.g / 16 + a.n_seqs) * a.hkv;
  if (blocks > MOST_GROUPS) return hipErrorInvalidValue;
  if (a.head_dim == 128)
    hipLaunchKernelGGL(attn_rows<128>, dim3(unsigned(blocks)), dim3(NT), 0, s, a);
  else
    hipLaunchKernelGGL(attn_rows<64>, dim3(unsigned(blocks)), dim3(NT), 0, s, a);
  return hipGetLastError();
}

}  // namespace cc
