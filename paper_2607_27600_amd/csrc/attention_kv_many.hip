// Attention over a cache in bf16, many rows of a sequence and KV head: prompts and chunks of them.
#include <algorithm>

#include "attention_kv_many.h"

namespace cc {
namespace {

// (Two K and two V buffers as distinct objects: what fills one and what reads another are told apart.)
template <int HD, bool PAGED>
__global__ __launch_bounds__(256, 2) void attn_many(KvAttnArgs a) {
  constexpr int TILE = KV_KEYS * HD;
  __shared__ __attribute__((aligned(1024))) u16 kb0[TILE];
  __shared__ __attribute__((aligned(1024))) u16 kb1[TILE];
  __shared__ __attribute__((aligned(1024))) u16 vb0[TILE];
  __shared__ __attribute__((aligned(1024))) u16 vb1[TILE];
  many::group<HD, PAGED, false>(a, blockIdx.x, kb0, kb1, vb0, vb1);
}

// Joins a row's pieces, in their order.  They lie one behind the other (all of a piece together: 128 tokens and a chunk of 16
// behind 16000 entries 97.5 us, so 96.0).
template <int HD, bool SKIP>
__global__ __launch_bounds__(256) void attn_join(KvAttnArgs a, int64_t group0) {
  constexpr int LPR = HD / 4, NG = 256 / LPR;
  const int gi = threadIdx.x / LPR, d = (threadIdx.x % LPR) * 4;
  const int64_t all = int64_t(a.N) * a.g, x = (group0 + blockIdx.x) * NG + gi;
  if (x >= all * a.hkv) return;
  const int kvh = int(x / all);
  const int64_t r = x - int64_t(kvh) * all;
  const int query = int(r / a.g);
  const int b = last_at(a.n_seqs, [&](int i) { return int64_t(a.cu[i]); }, query);
  const int q0 = a.cu[b], m = a.cu[b + 1] - q0, rows = m * a.g;
  if (rows <= a.few) return;
  const int len = min(max(a.lens[b], 0), a.max_len);
  // the pieces that the row's block has
  const int block = int(r - int64_t(q0) * a.g) / KV_ROWS;
  const int see = min(len, max(0, len - m + (min((block + 1) * KV_ROWS, rows) - 1) / a.g + 1));
  const int n = max(see - 1, 0) / a.piece + 1;
  int before = a.row0;
  if constexpr (SKIP) {   // (one by one: b differs in a wave)
    const int k = b / a.few_per;
    before = a.few_at[k];
    for (int i = k * a.few_per; i < b; ++i) before += few_rows_of(a, i);
  }
  const int64_t first = (int64_t(kvh) * a.places + r - before) * a.splits;
  Joined j{-INFINITY, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)};
  for (int i0 = 0; i0 < n; i0 += 4) {   // four in flight
    float2 p[4];
    float4 y[4];
    bool in[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int64_t at = first + min(i0 + q, n - 1);
      in[q] = i0 + q < n;
      p[q] = a.part_ml[at];
      y[q] = *reinterpret_cast<const float4*>(a.part + at * HD + d);
    }
    j.add(p, [&](int q) { return y[q]; }, in, a.c2);
  }
  const float inv = row_inverse(j.L);
  const int64_t at = int64_t(query) * a.hq + kvh * a.g + r % a.g;
  *reinterpret_cast<uint2*>(a.o + at * HD + d) = make_uint2(pack_bf2(j.o.x * inv, j.o.y * inv), pack_bf2(j.o.z * inv, j.o.w * inv));
  if (a.lse && d == 0) a.lse[at] = row_lse(j.M, j.L, a.scale);
}

template <int HD>
hipError_t launch_dim(const KvAttnArgs& a, hipStream_t s) {
  const int64_t each = int64_t(a.blocks) * a.hkv;
  const dim3 grid(unsigned(each * a.splits));
  if (a.own.paged)
    hipLaunchKernelGGL((attn_many<HD, true>), grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((attn_many<HD, false>), grid, dim3(256), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.part) return e;
  constexpr int NG = 256 / (HD / 4);
  const int64_t groups = (int64_t(a.N) * a.g * a.hkv + NG - 1) / NG;
  for (int64_t g0 = 0; g0 < groups; g0 += MOST_GROUPS) {
    const dim3 here(unsigned(std::min(MOST_GROUPS, groups - g0)));
    if (a.skip)
      hipLaunchKernelGGL((attn_join<HD, true>), here, dim3(256), 0, s, a, g0);
    else
      hipLaunchKernelGGL((attn_join<HD, false>), here, dim3(256), 0, s, a, g0);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_attn_kv_many(const KvAttnArgs& a, hipStream_t s) {
  return a.head_dim == 128 ? launch_dim<128>(a, s) : launch_dim<64>(a, s);
}

}  // namespace cc
