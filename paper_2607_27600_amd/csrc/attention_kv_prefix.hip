// The pass over the prefixes that runs of sequences share, and with it, in the same launch, over the own entries of the
// sequences of few rows, in pieces of rpiece; a second launch joins the two.  A prefix is read for 128 rows of its run at a time,
// whatever their sequences, so what the run's sequences would each read is read some once.
//
// 40 sequences of one token behind 16000 entries, 28 heads on 4: 32 us and 7 for the join (one after the other the two passes take 24
// and 25, either with half of the card's slots empty); 24 of six tokens behind 30001 and 6000, 32 heads on 8, 80 and 10.  Bound by
// what comes beside the tiles: their load before the first, and outputs in fp32 that go out to be joined (14 and 37 MB).
#include <algorithm>

#include "attention_kv_many.h"
#include "attention_kv_rows.h"

namespace cc {
namespace {

template <int HD, bool PAGED>
__global__ __launch_bounds__(256, 2) void attn_prefix(KvAttnArgs pass, KvAttnArgs own, unsigned groups) {
  constexpr int TILE = KV_KEYS * HD;
  __shared__ __attribute__((aligned(1024))) u16 lds[4 * TILE];
  if (blockIdx.x < groups)
    many::group<HD, PAGED, true>(pass, blockIdx.x, lds, lds + TILE, lds + 2 * TILE, lds + 3 * TILE);
  else
    rows_group<HD, 4, true>(own, blockIdx.x - groups, reinterpret_cast<float*>(lds), reinterpret_cast<float2*>(lds + 2 * TILE),
                                pass.few_at);
}

// Joins what the pass over the prefixes has of a row with its own pieces: a wave a row, whose groups of HD / 8 lanes share out
// the pieces, the prefix's first, four in flight each.
template <int HD>
__global__ __launch_bounds__(256) void attn_rows_join(KvAttnArgs a, int64_t group0) {
  constexpr int LPR = HD / 8, NG = 64 / LPR;
  const int lane = threadIdx.x & 63, gi = lane / LPR, d = (lane % LPR) * 8;
  const int64_t x = (group0 + blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
  const int64_t all = int64_t(a.few_rows) * a.hkv;
  if (x >= all) return;
  int first;
  const int b = few_at_row(a, int(x / a.hkv), first);
  const int q0 = a.cu[b], mq = a.cu[b + 1] - q0, rows = mq * a.g;
  const int at_b = int(x - int64_t(first) * a.hkv), kvh = at_b / rows, row = at_b % rows;
  const int own = max(rows_see(a, mq, min(max(a.lens[b], 0), a.max_len), row & ~15) - 1, 0) / a.rpiece + 1;
  const int j = prefix_of(a, b);
  const PrefixRow p = prefix_row(a, j, kvh, int64_t(q0 - a.cu[a.pre_first[j]]) * a.g + row);
  const int n = p.n + own;
  Joined g[2] = {{-INFINITY, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)}, {-INFINITY, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)}};
  for (int i0 = gi; i0 < n; i0 += 4 * NG) {
    float2 ml[4];
    float4 y[2][4];
    bool in[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int i = min(i0 + q * NG, n - 1);
      const bool pre = i < p.n;
      const int64_t at = pre ? p.first + int64_t(i) * KV_ROWS : int64_t(i - p.n) * all + x;
      const float* from = (pre ? a.ppart : a.rpart) + at * HD + d;
      in[q] = i0 + q * NG < n;
      ml[q] = (pre ? a.ppart_ml : a.rpart_ml)[at];
      y[0][q] = *reinterpret_cast<const float4*>(from);
      y[1][q] = *reinterpret_cast<const float4*>(from + 4);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) g[k].add(ml, [&](int q) { return y[k][q]; }, in, a.c2);
  }
  // the groups' results, pairs first
#pragma unroll
  for (int off = LPR; off < 64; off <<= 1) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const float2 ml[1] = {make_float2(__shfl_xor(g[k].M, off), __shfl_xor(g[k].L, off))};
      const float4 o = make_float4(__shfl_xor(g[k].o.x, off), __shfl_xor(g[k].o.y, off), __shfl_xor(g[k].o.z, off),
                                   __shfl_xor(g[k].o.w, off));
      const bool in[1] = {true};
      g[k].add(ml, [&](int) { return o; }, in, a.c2);
    }
  }
  if (gi) return;
  const float4 o[2] = {g[0].o, g[1].o};
  finish<HD>(a, q0, kvh, row, d, g[0].M, g[0].L, o);
}

}  // namespace

hipError_t launch_attn_prefix(const KvAttnArgs& pass, const KvAttnArgs& own, bool few, hipStream_t s) {
  const int64_t groups = std::max<int64_t>(pass.slots, int64_t(pass.blocks) * pass.hkv), rows = few ? rows_groups(own) : 0;
  if (groups + rows > MOST_GROUPS) return hipErrorInvalidValue;   // (refused by the planner)
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(unsigned(groups + rows)), dim3(256), 0, s, pass, own, unsigned(groups));
  };
  if (pass.head_dim == 128)
    pass.own.paged ? launch(attn_prefix<128, true>) : launch(attn_prefix<128, false>);
  else
    pass.own.paged ? launch(attn_prefix<64, true>) : launch(attn_prefix<64, false>);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !few) return e;
  KvAttnArgs join = own;
  std::copy_n(pass.few_at, KV_LIST, join.few_at);
  const int64_t waves = (int64_t(own.few_rows) * own.hkv + 3) / 4;
  for (int64_t g0 = 0; g0 < waves; g0 += MOST_GROUPS) {
    const dim3 grid(unsigned(std::min(MOST_GROUPS, waves - g0)));
    if (own.head_dim == 128)
      hipLaunchKernelGGL(attn_rows_join<128>, grid, dim3(256), 0, s, join, g0);
    else
      hipLaunchKernelGGL(attn_rows_join<64>, grid, dim3(256), 0, s, join, g0);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace cc
