// Log-probabilities, entropies and alternatives from the LM head: z = W_lm u for every row, and of z the
// logit of a given word, logsumexp, the entropy log S - sum e^(z-M) (z-M) / S with S = sum e^(z-M), and
// the largest logits with their words.  The contraction is that of gemm_tile.h, and everything is taken
// from its accumulators: the [N][V] logits never leave registers.
//
// Per (row, 256-word tile) the epilogue writes (max, S, sum e^(z-max) (z-max)) against the tile's own
// maximum, in log2 units; per (row, 128 words of a wave) it writes the words that may be among the
// largest, in falling order.  A second kernel joins both, a wave a row.
//
// Logits are ranked as whole numbers: a key that rises with the logit, 1 for NaN, 0 for none.
#include <algorithm>

#include "gemm_tile.h"

namespace cc {
namespace {

constexpr int VT = 256;          // words of a tile (MB = 8)
constexpr int SLAB = 2048;       // rows worked on at a time: bounds the workspace
constexpr int NE = 16;           // rows of a block of the tables below

// Tables of one slab, in blocks of 16 rows: [row / 16][tile or half tile][..][row % 16].
struct Tables {
  float4* part;      // [tile]: (max, S, T, -) in log2 units
  uint8_t* count;    // [half tile]: candidates
  uint2* cand;       // [half tile][top]: (key, word), falling
  float* target;     // [row]
};

__device__ __forceinline__ uint32_t key_of(float z) {
  const uint32_t u = __float_as_uint(z + 0.f);   // -0 ranks as +0
  const uint32_t k = u ^ (uint32_t(int32_t(u) >> 31) | 0x80000000u);
  return z != z ? 1u : k;
}
__device__ __forceinline__ float logit_of(uint32_t key) {
  return key == 1u ? __uint_as_float(0x7fc00000u) : __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key);
}

// (M, S, T) += (m, s, t): S = sum 2^(x-M), T = sum 2^(x-M) (x-M) over the logits x in log2 units.
__device__ __forceinline__ void fold3(float& M, float& S, float& T, float m, float s, float t) {
  const float n = fmaxf(M, m);
  const float ref = n == -INFINITY ? 0.f : n;
  const float a = exp2f(M - ref), b = exp2f(m - ref);
  // an empty part has S = T = 0 and M = -inf: its difference is not taken
  const float dM = M == -INFINITY ? 0.f : M - ref, dm = m == -INFINITY ? 0.f : m - ref;
  T = a * fmaf(S, dM, T) + b * fmaf(s, dm, t);
  S = S * a + s * b;
  M = n;
}

template <int NB>
struct EpiLogprobs {
  static constexpr int MB = VT / 32;
  Tables tb;
  const int32_t* ids;   // [rows of the slab] or null
  int tiles, top;

  __device__ void operator()(f32x4 (&acc)[MB][NB], const TileArgs& g, int tm, int, int m0w, int n0w, int lane,
                             char* lds) const {
    const int grp = lane >> 4, c16 = lane & 15;
    const int wave = threadIdx.x >> 6, wm = wave >> 2, wn = wave & 3;
    float* red = reinterpret_cast<float*>(lds);   // [2][64 NB][3]
    const int rows = g.M - m0w;                   // words of this wave that exist
    int rt[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) rt[b] = ids ? ids[min(n0w + b * 16 + c16, g.N - 1)] - m0w : -1;
    float mx[NB], sm[NB], tt[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      mx[b] = -INFINITY;
#pragma unroll
      for (int a = 0; a < MB; ++a)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (a * 16 + 4 * grp + e < rows) mx[b] = fmaxf(mx[b], acc[a][b][e]);
      mx[b] *= kLog2e;
      const float mc = mx[b] == -INFINITY ? 0.f : mx[b];
      sm[b] = tt[b] = 0.f;
#pragma unroll
      for (int a = 0; a < MB; ++a)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          // -inf logits weigh nothing, and 0 * -inf must not be taken
          const float x = fmaxf(fmaf(acc[a][b][e], kLog2e, -mc), -1e30f);
          const float p = fast_exp2(x);
          if (a * 16 + 4 * grp + e < rows) {
            sm[b] += acc[a][b][e] != acc[a][b][e] ? acc[a][b][e] : p;   // (the maximum above drops a NaN)
            tt[b] = fmaf(p, x, tt[b]);
          }
        }
    }
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int r = rt[b];
      const bool own = n0w + b * 16 + c16 < g.N && uint32_t(r) < uint32_t(16 * MB) && ((r >> 2) & 3) == grp;
      if (__any(own)) {
        const int idx = (r >> 4) * 4 + (r & 3);
        float z = 0.f;
#pragma unroll
        for (int a = 0; a < MB; ++a)
#pragma unroll
          for (int e = 0; e < 4; ++e) z = idx == a * 4 + e ? acc[a][b][e] : z;
        if (own) tb.target[n0w + b * 16 + c16] = z;
      }
    }
#pragma unroll
    for (int b = 0; b < NB; ++b) {
#pragma unroll
      for (int off = 16; off < 64; off <<= 1) {
        const float m2 = __shfl_xor(mx[b], off), s2 = __shfl_xor(sm[b], off), t2 = __shfl_xor(tt[b], off);
        fold3(mx[b], sm[b], tt[b], m2, s2, t2);
      }
      if (grp == 0) {
        float* r = red + ((wm * 4 + wn) * 16 * NB + b * 16 + c16) * 3;
        r[0] = mx[b];
        r[1] = sm[b];
        r[2] = tt[b];
      }
    }
    __syncthreads();
    {
      const int t = threadIdx.x, n = n0w - wn * 16 * NB + t;   // tile column t
      if (t < 64 * NB && n < g.N) {
        const float* p = red + t * 3;
        const float* q = red + (64 * NB + t) * 3;
        float M = p[0], S = p[1], T = p[2];
        fold3(M, S, T, q[0], q[1], q[2]);
        tb.part[(int64_t(n / NE) * tiles + tm) * NE + n % NE] = make_float4(M, S, T, 0.f);
      }
    }
    if (top == 0) return;
    // Candidates: the largest first, a round at a time.  A lane looks for its largest (the lowest word of
    // equal ones: its words rise with a and e), four lanes agree on the row's, and its owner drops it.
    const int tw = tm * 2 + wm;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int n = n0w + b * 16 + c16;
      uint32_t key[MB * 4];
#pragma unroll
      for (int a = 0; a < MB; ++a)
#pragma unroll
        for (int e = 0; e < 4; ++e) key[a * 4 + e] = a * 16 + 4 * grp + e < rows ? key_of(acc[a][b][e]) : 0u;
      const int64_t at = (int64_t(min(n, g.N - 1) / NE) * 2 * tiles + tw) * NE + n % NE;
      int c = 0;
      for (int round = 0; round < top; ++round) {
        uint32_t best = 0;
        int word = 0;
#pragma unroll
        for (int i = 0; i < MB * 4; ++i) {
          const bool up = key[i] > best;
          best = up ? key[i] : best;
          word = up ? (i >> 2) * 16 + 4 * grp + (i & 3) : word;
        }
        uint32_t K = best;
        int W = word;
#pragma unroll
        for (int off = 16; off < 64; off <<= 1) {
          const uint32_t k2 = __shfl_xor(K, off);
          const int w2 = __shfl_xor(W, off);
          const bool up = k2 > K || (k2 == K && w2 < W);
          K = up ? k2 : K;
          W = up ? w2 : W;
        }
        const bool more = K != 0;
        if (!__any(more)) break;
        if (more && grp == 0 && n < g.N)
          tb.cand[((at / NE) * top + round) * NE + n % NE] = make_uint2(K, uint32_t(m0w + W));
        c += more;
        const int drop = more && W == word && K == best && ((W >> 2) & 3) == grp ? (W >> 4) * 4 + (W & 3) : -1;
#pragma unroll
        for (int i = 0; i < MB * 4; ++i) key[i] = drop == i ? 0u : key[i];
      }
      if (grp == 0 && n < g.N) tb.count[at] = uint8_t(c);
    }
  }
};

struct JoinArgs {
  Tables tb;
  int tiles, top, N;
  const int32_t* ids;
  float *logprob, *entropy, *top_logprob;
  int32_t* top_ids;
};

// One wave a row, 16 rows a workgroup (they share the lines of the tables).
__global__ __launch_bounds__(1024) void logprobs_join(JoinArgs a) {
  const int lane = threadIdx.x & 63, e = threadIdx.x >> 6;
  const int blk = blockIdx.x, n = blk * NE + e;
  if (n >= a.N) return;
  float M = -INFINITY, S = 0.f, T = 0.f;
  for (int t0 = lane; t0 < a.tiles; t0 += 8 * 64) {
    float4 p[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const int t = t0 + q * 64;
      p[q] = t < a.tiles ? a.tb.part[(int64_t(blk) * a.tiles + t) * NE + e] : make_float4(-INFINITY, 0.f, 0.f, 0.f);
    }
#pragma unroll
    for (int q = 0; q < 8; ++q) fold3(M, S, T, p[q].x, p[q].y, p[q].z);
  }
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const float m2 = __shfl_xor(M, off), s2 = __shfl_xor(S, off), t2 = __shfl_xor(T, off);
    fold3(M, S, T, m2, s2, t2);
  }
  const float lse = kLn2 * (M + log2f(S));
  if (lane == 0) {
    // log P <= 0 and entropy >= 0: rounding may take either a few ulps past
    if (a.logprob) {
      const float d = a.tb.target[n] - lse;
      a.logprob[n] = d > 0.f ? 0.f : d;
    }
    if (a.entropy) {
      const float h = kLn2 * (log2f(S) - T / S);
      a.entropy[n] = h < 0.f ? 0.f : h;
    }
  }
  const int top = a.top;
  if (top == 0) return;
  // The largest so far, lane r the r-th.  (key, word): larger keys first, then lower words.
  uint32_t key = 0;
  int word = INT32_MAX;
  const int halves = 2 * a.tiles;
  for (int t0 = 0; t0 < halves; t0 += 64) {
    const int t = t0 + lane;
    const int64_t at = (int64_t(blk) * halves + min(t, halves - 1)) * NE + e;
    const int c = t < halves ? a.tb.count[at] : 0;
    for (int r = 0; r < top; ++r) {
      uint2 x = make_uint2(0, 0);
      if (r < c) x = a.tb.cand[((at / NE) * top + r) * NE + e];
      const uint32_t kth = __shfl(key, top - 1);
      const int kw = __shfl(word, top - 1);
      uint64_t in = __ballot(x.x != 0 && (x.x > kth || (x.x == kth && int(x.y) < kw)));
      if (in == 0) break;   // lists fall: nothing further of them passes either
      while (in) {
        const int l = __builtin_ctzll(in);
        in &= in - 1;
        const uint32_t K = __shfl(x.x, l);
        const int W = __shfl(int(x.y), l);
        const int pos = __popcll(__ballot(lane < top && (key > K || (key == K && word < W))));
        const uint32_t ku = __shfl_up(key, 1);
        const int wu = __shfl_up(word, 1);
        key = lane > pos ? ku : lane == pos ? K : key;
        word = lane > pos ? wu : lane == pos ? W : word;
      }
    }
  }
  if (lane < top) {
    const float d = logit_of(key) - lse;
    a.top_ids[int64_t(n) * top + lane] = word;
    a.top_logprob[int64_t(n) * top + lane] = d > 0.f ? 0.f : d;
  }
}

size_t up256(size_t x) { return (x + 255) & ~size_t(255); }

struct Layout {
  size_t part, count, cand, target, total;
};
Layout layout(int N, int V, int top) {
  const size_t rows = (size_t(std::min(N, SLAB)) + NE - 1) / NE * NE, tiles = (size_t(V) + VT - 1) / VT;
  Layout L;
  L.part = 0;
  L.count = L.part + up256(tiles * rows * sizeof(float4));
  L.cand = L.count + up256(top ? 2 * tiles * rows : 0);
  L.target = L.cand + up256(2 * tiles * rows * top * sizeof(uint2));
  L.total = N ? L.target + up256(rows * sizeof(float)) : 0;
  return L;
}

template <int AM>
hipError_t launch_tiles(const TileArgs& g, const Tables& tb, const int32_t* ids, int tiles, int top, hipStream_t s) {
  if (g.K >= kWideRow) return launch_tile<8, 3, 3, 2, AM, true>(g, EpiLogprobs<3>{tb, ids, tiles, top}, 1, s);
  switch (lmhead_tile_width(g.M, g.N, g.K)) {
    case 1: return launch_tile<8, 1, 4, 4, AM>(g, EpiLogprobs<1>{tb, ids, tiles, top}, 1, s);
    case 2: return launch_tile<8, 2, 3, 3, AM>(g, EpiLogprobs<2>{tb, ids, tiles, top}, 1, s);
    case 3: return launch_tile<8, 3, 3, 2, AM>(g, EpiLogprobs<3>{tb, ids, tiles, top}, 1, s);
    default: return launch_tile<8, 4, 3, 2, AM>(g, EpiLogprobs<4>{tb, ids, tiles, top}, 1, s);
  }
}

}  // namespace

size_t logprobs_ws_bytes(int N, int V, int top) { return layout(N, V, top).total; }

hipError_t launch_logprobs(const LogprobsLaunch& l, hipStream_t s) {
  const Layout L = layout(l.N, l.V, l.top);
  char* ws = static_cast<char*>(l.ws);
  Tables tb;
  tb.part = reinterpret_cast<float4*>(ws + L.part);
  tb.count = reinterpret_cast<uint8_t*>(ws + L.count);
  tb.cand = reinterpret_cast<uint2*>(ws + L.cand);
  tb.target = reinterpret_cast<float*>(ws + L.target);
  const int tiles = int((int64_t(l.V) + VT - 1) / VT);
  for (int lo = 0; lo < l.N; lo += SLAB) {
    TileArgs g{};
    g.A = static_cast<const u16*>(l.w);
    g.B = l.u + int64_t(lo) * l.D;
    g.M = l.V;
    g.N = std::min(SLAB, l.N - lo);
    g.K = l.D;
    const int32_t* ids = l.ids ? l.ids + lo : nullptr;
    hipError_t err = l.packed ? launch_tiles<A_PACKED>(g, tb, ids, tiles, l.top, s)
                              : launch_tiles<A_ROWS>(g, tb, ids, tiles, l.top, s);
    if (err != hipSuccess) return err;
    JoinArgs j;
    j.tb = tb;
    j.tiles = tiles;
    j.top = l.top;
    j.N = g.N;
    j.ids = ids;
    j.logprob = l.ids ? l.logprob + lo : nullptr;
    j.entropy = l.entropy ? l.entropy + lo : nullptr;
    j.top_ids = l.top ? l.top_ids + int64_t(lo) * l.top : nullptr;
    j.top_logprob = l.top ? l.top_logprob + int64_t(lo) * l.top : nullptr;
    hipLaunchKernelGGL(logprobs_join, dim3((g.N + NE - 1) / NE), dim3(1024), 0, s, j);
    err = hipGetLastError();
    if (err != hipSuccess) return err;
  }
  return hipSuccess;
}

}  // namespace cc
