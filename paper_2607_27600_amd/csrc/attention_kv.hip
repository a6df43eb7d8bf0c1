// Attention over a cache in bf16, few rows of a sequence and KV head (single tokens, drafts) and short prompts: whole rows,
// and rows whose entries are shared out among workgroups and joined.
#include <algorithm>

#include "attention_kv_rows.h"

namespace cc {
namespace {

// ------------------------------------------------------------------ whole rows

// A workgroup's waves share out the entries of 16 rows and meet in LDS: one launch, nothing to join.  Bound by the chain of loads:
// a prompt of 200 tokens, 32 heads on 8, 8.1 us (400 workgroups); four tokens behind 900 entries each 13.4, 32 workgroups, each
// of 460 KB at some 60 GB/s.
template <int HD, int NW>
__global__ __launch_bounds__(64 * NW, 2) void attn_rows(KvAttnArgs a) {
  __shared__ float lds[NW * 16 * HD];
  __shared__ float2 ml[NW * 16];
  rows_group<HD, NW, false>(a, blockIdx.x, lds, ml);
}

// ------------------------------------------------------------------ few rows, work shared out

// Single tokens and drafts over long caches: every workgroup takes an equal share of all (sequence, head)s' entries, two workgroups
// a CU.  Bound by the bytes of the cache: 48 ragged sequences of up to 15987 entries, 28 heads on 4, 94 us (5.2 TB/s) and 6 for
// the join; one of 2048, 32 heads on 8, is a chain of loads, 8 us and 4.
constexpr int FEW_NT = 256;
template <int HD, int NR>
__global__ __launch_bounds__(FEW_NT, 2) void attn_few(KvAttnArgs a) {
  constexpr int NW = FEW_NT / 64, ROWS = 16 * NR;
  extern __shared__ float lds[];        // [NW][ROWS][HD] outputs, then [NW][ROWS] (max, sum)
  float2* ml = reinterpret_cast<float2*>(lds + NW * ROWS * HD);
  const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
  const Shares sh = shares_of(a);
  if (int(blockIdx.x) >= sh.parts) return;
  int64_t x = sh.begin(blockIdx.x);
  const int64_t x1 = sh.begin(blockIdx.x + 1);
  while (x < x1) {
    const Item it = item_at(a, sh, x);
    const int j = it.j, kvh = it.kvh;
    const Seq s = seq_of(a, j);
    const int rows = s.m * a.g;
    const int past_unit = it.unit + int(min(int64_t(it.units - it.unit), x1 - x));   // of the item's units
    x += past_unit - it.unit;
    const int u0 = max(0, it.unit - sh.head), u1 = past_unit - sh.head;   // those with entries
    const bool whole = u0 == 0 && past_unit == it.units;
    if (u1 <= u0) continue;
    if (threadIdx.x == 0) {
      int2* at = a.fpart_at + int64_t(j) * a.hkv + kvh;
      if (u0 == 0) at->x = int(blockIdx.x);
      if (past_unit == it.units) at->y = int(blockIdx.x);
    }
    const int unit = sh.q * UNIT;
    const int c0 = u0 * unit, c1 = int(min(int64_t(s.len), int64_t(u1) * unit));
    Rows<HD, NR> st;
    int i[NR], past[NR];
    load_queries(a, st, s.q0, kvh, 0, rows, i);
    st.clear();
#pragma unroll
    for (int n = 0; n < NR; ++n) past[n] = max(0, s.shift + i[n] + 1);
    // this wave's 16-entry groups: the piece's, in NW runs of whole steps of two
    const int g0 = c0 >> 4, g1 = (c1 + 15) >> 4;
    const int per = ((g1 - g0 + NW - 1) / NW + 1) & ~1;
    const int gb = g0 + wave * per, ge = min(g1, gb + per);
    st.template run<true>(a, kv_plane(a.own, s.b, a.layer, kvh), gb, ge, s.len, past, max(0, s.shift + 1));
    meet<HD, NR, NW>(a, st, lds, ml, rows, [&](int r, int d, float M, float L, float4(&o)[2]) {
      if (whole) return finish<HD>(a, s.q0, kvh, r, d, M, L, o);
      const int64_t row = (int64_t(blockIdx.x) + int64_t(j) * a.hkv + kvh) * a.R + r;
      float* po = a.fpart + row * HD + d;
      *reinterpret_cast<float4*>(po) = o[0];
      *reinterpret_cast<float4*>(po + 4) = o[1];
      if (d == 0) a.fpart_ml[row] = make_float2(M, L);
    });
    __syncthreads();   // the LDS results have been read
  }
}

// Joins the pieces of rows that are cut between shares.  A workgroup has NG groups of HD / 8 lanes.  With `one`, for up
// to JOIN_ONE rows in all, they share out one row's pieces; else a row each.
constexpr int JOIN_ONE = 1024;
template <int HD>
__global__ __launch_bounds__(256) void attn_few_join(KvAttnArgs a, int one, int64_t group0) {
  constexpr int LPR = HD / 8, NG = 256 / LPR;
  __shared__ float4 po[2][256];
  __shared__ float2 pm[256];
  const int tid = threadIdx.x, gi = tid / LPR, lane = tid % LPR, d = lane * 8;
  const int64_t all = int64_t(a.n_list) * a.hkv * a.R;
  const int64_t row_in = one ? int64_t(blockIdx.x) : (group0 + blockIdx.x) * NG + gi;
  const int r = int(row_in % a.R), jh = int(min(row_in / a.R, int64_t(a.n_list) * a.hkv - 1));
  const int kvh = jh % a.hkv, j = jh / a.hkv;
  const Seq s = seq_of(a, j);
  const int rows = s.m * a.g;
  bool on = row_in < all && r < rows && rows <= FEW_ROWS;
  const int2 parts = on ? a.fpart_at[jh] : make_int2(0, 0);
  const int wa = parts.x, n = parts.y - wa + 1;
  on = on && n > 1;   // a whole one is final
  const int64_t slot = (int64_t(wa) + jh) * a.R + r;   // piece i at slot + i R
  Joined g[2] = {{-INFINITY, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)}, {-INFINITY, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)}};
  if (on) {
    const int first = one ? gi : 0, by = one ? NG : 1;
    for (int i0 = first; i0 < n; i0 += 4 * by) {   // four in flight
      float2 p[4];
      float4 y[2][4];
      bool in[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int64_t at = slot + int64_t(min(i0 + q * by, n - 1)) * a.R;
        in[q] = i0 + q * by < n;
        p[q] = a.fpart_ml[at];
        y[0][q] = *reinterpret_cast<const float4*>(a.fpart + at * HD + d);
        y[1][q] = *reinterpret_cast<const float4*>(a.fpart + at * HD + d + 4);
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) g[k].add(p, [&](int q) { return y[k][q]; }, in, a.c2);
    }
  }
  if (one) {   // (alike in the whole workgroup)
    if (!on) return;
    po[0][tid] = g[0].o;
    po[1][tid] = g[1].o;
    pm[tid] = make_float2(g[0].M, g[0].L);
    __syncthreads();
    if (gi) return;
    float2 p[NG];
    bool in[NG];
#pragma unroll
    for (int q = 0; q < NG; ++q) {
      p[q] = pm[lane + q * LPR];
      in[q] = true;
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      g[k] = {-INFINITY, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)};
      g[k].add(p, [&](int q) { return po[k][lane + q * LPR]; }, in, a.c2);
    }
  }
  if (!on) return;
  float4 o[2] = {g[0].o, g[1].o};
  finish<HD>(a, s.q0, kvh, r, d, g[0].M, g[0].L, o);
}

template <int HD, int NR>
hipError_t few_rows(const KvAttnArgs& a, hipStream_t s) {
  constexpr int NW = FEW_NT / 64;
  constexpr size_t lds = size_t(NW) * 16 * NR * (HD * 4 + 8);
  if (lds > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(attn_few<HD, NR>),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, int(lds));
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((attn_few<HD, NR>), dim3(unsigned(a.parts)), dim3(FEW_NT), lds, s, a);
  return hipGetLastError();
}

template <int HD>
hipError_t few_dim(const KvAttnArgs& a, hipStream_t s) {
  hipError_t e = a.R <= 16 ? few_rows<HD, 1>(a, s) : few_rows<HD, 2>(a, s);
  if (e != hipSuccess) return e;
  constexpr int NG = 256 / (HD / 8);
  const int64_t rows = int64_t(a.n_list) * a.hkv * a.R;
  const int one = rows <= JOIN_ONE;
  const int64_t groups = one ? rows : (rows + NG - 1) / NG;
  for (int64_t g0 = 0; g0 < groups; g0 += MOST_GROUPS) {   // (more than a launch may have: several)
    hipLaunchKernelGGL((attn_few_join<HD>), dim3(unsigned(std::min(MOST_GROUPS, groups - g0))), dim3(256), 0, s, a, one, g0);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_attn_few(const KvAttnArgs& a, hipStream_t s) { return a.head_dim == 128 ? few_dim<128>(a, s) : few_dim<64>(a, s); }

hipError_t launch_attn_rows(const KvAttnArgs& a, hipStream_t s) {
  const int64_t blocks = rows_groups(a);
  if (blocks > MOST_GROUPS / 2) return hipErrorInvalidValue;   // (refused by the planner)
  // Eight waves where there is a CU for every workgroup, so that a wave's chain of loads is short.
  const bool wide = blocks <= 256;
  auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(unsigned(blocks)), dim3(wide ? 512 : 256), 0, s, a); };
  if (a.head_dim == 128)
    wide ? launch(attn_rows<128, 8>) : launch(attn_rows<128, 4>);
  else
    wide ? launch(attn_rows<64, 8>) : launch(attn_rows<64, 4>);
  return hipGetLastError();
}

}  // namespace cc
