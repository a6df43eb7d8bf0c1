// Log-probabilities, entropies and alternatives from the LM head: z = W_lm u for every row, and of z the
// logit of a given word, logsumexp, the entropy log S - sum e^(z-M) (z-M) / S with S = sum e^(z-M), and
// the largest logits with their words.  The contraction is that of gemm_tile.h, and everything is taken
// from its accumulators: the [N][V] logits never leave registers.
//
// Per (row, 256-word tile) the epilogue writes (max, S, sum e^(z-max) (z-max)) against the tile's own
// maximum, in log2 units; per (row, 128 words of a wave) it lists the words that may be among the
// largest.  A second kernel joins both, a wave a row.
//
// Logits are ranked as whole numbers: a key that rises with the logit, 1 for NaN, 0 for none.
//
// What may be among the largest.  Every row has 32 slots; a half tile that finds a candidate raises
// slot (half tile % 32) to its largest key, so the slots hold 32 different words of the row and the
// top-th largest of them is a bound that at least `top` words reach.  Words below the bound as a
// workgroup happens to read it are dropped: the candidates depend on the order in which workgroups run,
// the words that come of them do not.  A tenth of the vocabulary in, few half tiles find any.  (Without
// the bound every half tile lists its `top` largest: 2000 rows of 3584, 152064 words, five
// alternatives 1896 us, 1702 with it; cc_lmhead_score_packed on the same rows 1580.)
#include <algorithm>

#include "gemm_tile.h"

namespace cc {
namespace {

constexpr int VT = 256;          // words of a tile (MB = 8)
constexpr int SLAB = 2048;       // rows worked on at a time: bounds the workspace

// Tables of one slab.  A row's numbers lie together for the wave that joins them: 16 rows side by side, as
// the tiles write them, let every load of the join touch 64 lines (64 rows 30 us; now 15, some ten round trips).
struct Tables {
  float4* part;      // [row][tile]: (max, S, T, -) in log2 units
  uint8_t* count;    // [row][half tile]: candidates
  uint2* cand;       // [row][half tile][top]: (key, word)
  float* target;     // [row]
  uint32_t* slots;   // [row][32]: keys; null: no bound
  uint32_t* bound;   // [row]: a key that at least `top` words of the row reach (0: not known)
};
// Whole numbers that other XCDs write: past this one's own cache.
__device__ __forceinline__ uint32_t load_shared(const uint32_t* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Bounds from slots, for `rows` rows from n0 on: two at a time, a half of the lanes each, and the slots of
// eight rows on their way together.
__device__ __forceinline__ void raise_bounds(const Tables& tb, int top, int n0, int rows) {
  const int lane = threadIdx.x & 63, half = lane & 32;
#pragma unroll 1
  for (int r = 0; r < rows; r += 8) {
    uint32_t v[4];
#pragma unroll
    for (int q = 0; q < 4; ++q)
      v[q] = load_shared(tb.slots + int64_t(n0 + min(r + 2 * q + (half >> 5), rows - 1)) * 32 + (lane & 31));
#pragma unroll 1
    for (int q = 0; q < 4; ++q) {
      const uint32_t w = q == 0 ? v[0] : q == 1 ? v[1] : q == 2 ? v[2] : v[3];
      int rank = 0;
#pragma unroll
      for (int j = 0; j < 32; ++j) {
        const uint32_t o = __shfl(w, half + j);
        rank += o > w || (o == w && j < (lane & 31));
      }
      if (rank == top - 1 && w > 1u) atomicMax(tb.bound + n0 + min(r + 2 * q + (half >> 5), rows - 1), w);
    }
  }
}

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

  // Per row: largest logit, and of the lane's words (max, S, T) in log2 units.  Only workgroups on the
  // vocabulary's edge ask whether a word exists.
  template <bool EDGE>
  __device__ __forceinline__ void sums(const f32x4 (&acc)[MB][NB], int rows, int grp, float (&mx)[NB], float (&sm)[NB],
                                       float (&tt)[NB], float (&zmax)[NB]) const {
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      float m = -INFINITY;
#pragma unroll
      for (int a = 0; a < MB; ++a)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (!EDGE || a * 16 + 4 * grp + e < rows) m = fmaxf(m, acc[a][b][e]);
      zmax[b] = m;
      mx[b] = m * kLog2e;
      const float mc = m == -INFINITY ? 0.f : mx[b];
      float s = 0.f, t = 0.f;
#pragma unroll
      for (int a = 0; a < MB; ++a)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          // A logit of -inf weighs nothing, and 0 * -inf must not be taken; a NaN (which the maxima pass
          // over) stays in S.
          const float x = fmaf(acc[a][b][e], kLog2e, -mc), p = fast_exp2(x);
          if (!EDGE || a * 16 + 4 * grp + e < rows) {
            s += p;
            t = fmaf(p, fmaxf(x, -1e30f), t);
          }
        }
      sm[b] = s;
      tt[b] = t;
    }
  }

  // (inlined: as a function, which it becomes where two kernels call it, it takes the accumulators through
  // memory, and the main loop loses its scalar registers)
  __device__ __forceinline__ void operator()(f32x4 (&acc)[MB][NB], const TileArgs& g, int tm, int, int m0w, int n0w, int lane,
                             char* lds) const {
    const int grp = lane >> 4, c16 = lane & 15;
    const int wave = threadIdx.x >> 6, wm = wave >> 2, wn = wave & 3;
    float* red = reinterpret_cast<float*>(lds);   // [2][64 NB][3]
    const int rows = g.M - m0w;                   // words of this wave that exist
    int rt[NB];
    uint32_t bound[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b)   // read ahead of the sums, which hide it
      bound[b] = tb.bound ? load_shared(tb.bound + min(n0w + b * 16 + c16, g.N - 1)) : 0u;
#pragma unroll
    for (int b = 0; b < NB; ++b) rt[b] = ids ? int(uint32_t(ids[min(n0w + b * 16 + c16, g.N - 1)]) - uint32_t(m0w)) : -1;
    float mx[NB], sm[NB], tt[NB], zmax[NB];
    if (rows >= 16 * MB)
      sums<false>(acc, rows, grp, mx, sm, tt, zmax);
    else
      sums<true>(acc, rows, grp, mx, sm, tt, zmax);
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
        tb.part[int64_t(n) * tiles + tm] = make_float4(M, S, T, 0.f);
      }
    }
    if (top == 0) return;
    // Candidates.
    const int tw = tm * 2 + wm;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int n = n0w + b * 16 + c16;
      bound[b] = __shfl(bound[b], c16);   // the row's four lanes go by one reading of it
      const int64_t at = int64_t(min(n, g.N - 1)) * 2 * tiles + tw;
      // (NaN logits are passed over by the maximum; they count only while there is no bound)
      if (!__any(bound[b] == 0u || key_of(zmax[b]) >= bound[b])) {
        if (grp == 0 && n < g.N) tb.count[at] = 0;
        continue;
      }
      int c = 0;             // of the row, in lanes of group 0
      uint32_t first = 0;    // its largest
      bool listed = false;
      if (!__any(bound[b] == 0u)) {
        // Few words reach a known bound: listed as they are met, if every row has room for its own.
        const float least = logit_of(bound[b]);
        auto reaches = [&](int i) {
          return acc[i >> 2][b][i & 3] >= least && (i >> 2) * 16 + 4 * grp + (i & 3) < rows;
        };
        int own = 0;
#pragma unroll
        for (int i = 0; i < MB * 4; ++i) own += reaches(i);
        int before = 0;
        c = own;
#pragma unroll
        for (int off = 16; off < 64; off <<= 1) {
          const int o = __shfl_xor(c, off);
          before += (grp & (off >> 4)) ? o : 0;
          c += o;
        }
        listed = !__any(c > top);
        if (listed) {
#pragma unroll
          for (int i = 0; i < MB * 4; ++i)
            if (reaches(i)) {
              const uint32_t k = key_of(acc[i >> 2][b][i & 3]);
              first = max(first, k);
              if (n < g.N)
                tb.cand[at * top + before] =
                    make_uint2(k, uint32_t(m0w + (i >> 2) * 16 + 4 * grp + (i & 3)));
              ++before;
            }
#pragma unroll
          for (int off = 16; off < 64; off <<= 1) first = max(first, uint32_t(__shfl_xor(int(first), off)));
        }
      }
      if (!listed) {
        // The largest first, a round at a time.  A lane looks for its largest (the lowest word of equal
        // ones: its words rise with a and e), four lanes agree on the row's, and its owner drops it.
        uint32_t key[MB * 4];
#pragma unroll
        for (int i = 0; i < MB * 4; ++i)
          key[i] = (i >> 2) * 16 + 4 * grp + (i & 3) < rows ? key_of(acc[i >> 2][b][i & 3]) : 0u;
        c = 0;
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
          const bool more = K != 0 && K >= bound[b];
          if (!__any(more)) break;
          if (round == 0) first = more ? K : 0u;
          if (more && grp == 0 && n < g.N)
            tb.cand[at * top + round] = make_uint2(K, uint32_t(m0w + W));
          c += more;
          const int drop = more && W == word && K == best && ((W >> 2) & 3) == grp ? (W >> 4) * 4 + (W & 3) : -1;
#pragma unroll
          for (int i = 0; i < MB * 4; ++i) key[i] = drop == i ? 0u : key[i];
        }
      }
      if (grp == 0 && n < g.N) tb.count[at] = uint8_t(c);
      if (tb.slots && grp == 0 && n < g.N && first > 1u) atomicMax(tb.slots + int64_t(n) * 32 + (tw & 31), first);
    }
    // Now and then a half tile turns the slots of its rows into bounds, for all the others: at the end of the
    // first round of workgroups (which reach half tile 63), then once in 128.  It holds up its workgroup by
    // some 40 us.  (2000 rows of 3584, 152064 words, one and five alternatives: 1669 and 1702 us, once in 64
    // 1695 and 1730, once in 32 1740 and 1765; a bound made by whoever finds a candidate held up nearly
    // all workgroups by 6 us, 1700 and 1746.)
    if (tb.slots && (tw == 63 || (tw & 127) == 127)) raise_bounds(tb, top, n0w, min(16 * NB, g.N - n0w));
  }
};

__global__ __launch_bounds__(256) void clear_kernel(uint32_t* p, int n) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i < n) p[i] = 0;
}

struct JoinArgs {
  Tables tb;
  const int32_t* ids;
  int V;
  int tiles, top;
  int falling;       // candidates are listed the largest first
  float *logprob, *entropy, *top_logprob;
  int32_t* top_ids;
};

// One wave a row and workgroup.
__global__ __launch_bounds__(64) void logprobs_join(JoinArgs a) {
  const int lane = threadIdx.x, n = blockIdx.x;
  const Tables& tb = a.tb;
  float M = -INFINITY, S = 0.f, T = 0.f;
  for (int t0 = lane; t0 < a.tiles; t0 += 8 * 64) {
    float4 p[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const int t = t0 + q * 64;
      p[q] = t < a.tiles ? tb.part[int64_t(n) * a.tiles + t] : make_float4(-INFINITY, 0.f, 0.f, 0.f);
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
      // (no tile has written the logit of a word that is not there)
      const bool there = uint32_t(a.ids[n]) < uint32_t(a.V);
      const float d = there ? tb.target[n] - lse : __uint_as_float(0x7fc00000u);
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
  auto passes = [&](uint32_t k, int w, uint32_t kth, int kw) { return k != 0 && (k > kth || (k == kth && w < kw)); };
  auto take = [&](uint2 x) {   // whatever of the lanes' candidates is among the largest
    uint64_t in = __ballot(passes(x.x, int(x.y), __shfl(key, top - 1), __shfl(word, top - 1)));
    while (in) {
      const int l = __builtin_ctzll(in);
      in &= in - 1;
      const uint32_t K = __builtin_amdgcn_readlane(x.x, l);
      const int W = __builtin_amdgcn_readlane(int(x.y), l);
      const int pos = __popcll(__ballot(lane < top && (key > K || (key == K && word < W))));
      const uint32_t ku = __shfl_up(key, 1);
      const int wu = __shfl_up(word, 1);
      key = lane > pos ? ku : lane == pos ? K : key;
      word = lane > pos ? wu : lane == pos ? W : word;
    }
  };
  // Eight half tiles a lane at a time: their counts and first candidates are loaded together.
  constexpr int H = 8;
  uint32_t bound = 0;
  for (int t0 = 0; t0 < halves; t0 += 64 * H) {
    int c[H];
    uint2 x[H];
    int64_t at[H];
#pragma unroll
    for (int q = 0; q < H; ++q) {
      const int t = t0 + q * 64 + lane;
      at[q] = int64_t(n) * halves + min(t, halves - 1);
      c[q] = t < halves ? tb.count[at[q]] : 0;
    }
#pragma unroll
    for (int q = 0; q < H; ++q) x[q] = c[q] ? tb.cand[at[q] * top] : make_uint2(0, 0);
    uint32_t best = 0;
#pragma unroll
    for (int q = 0; q < H; ++q) best = max(best, x[q].x);
    // a bound that `top` of the lanes reach, bit by bit: fewer candidates are put in their place one by one
    uint32_t reach = 0;
#pragma unroll
    for (int bit = 31; bit >= 0; --bit) {
      const uint32_t next = reach | (1u << bit);
      if (__popcll(__ballot(best >= next)) >= top) reach = next;
    }
    bound = max(bound, reach);
#pragma unroll
    for (int q = 0; q < H; ++q) {
      bool more = x[q].x >= bound;
      take(more ? x[q] : make_uint2(0, 0));
      if (!a.falling) more = true;
      for (int r = 1;; ++r) {
        more = more && r < c[q];
        if (!__any(more)) break;
        uint2 y = make_uint2(0, 0);
        if (more) y = tb.cand[at[q] * top + r];
        if (a.falling) more = y.x >= bound;
        take(y.x >= bound ? y : make_uint2(0, 0));
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
  size_t count, cand, target, slots, bound, total;   // the partial sums first
};
// The first round of workgroups knows no bound, so it is kept from two rounds of 256-row tiles on (it costs
// a launch that clears it).  1000 rows of 2048, 40000 words, three rounds, 5 and 20 alternatives: 221 and
// 364 us without, 204 and 265 with it; 300 rows of 4096, 128256 words, 398 and 546, 389 and 477.  A tile of up
// to 64 rows is soon looked through, and waiting for a bound never paid: 64 rows of 3584, 152064 words, 5 and 20
// alternatives, with it 250 and 318 us, without 240 and 288; of 2048, 300000 words, 268 and 336, 269 and 341.
bool bounded(int N, int V, int top) {
  return top > 0 && N > 64 && (int64_t(V) + VT - 1) / VT * ((std::min(N, SLAB) + 255) / 256) >= 2 * 256;
}
Layout layout(int N, int V, int top) {
  const size_t rows = size_t(std::min(N, SLAB)), tiles = (size_t(V) + VT - 1) / VT;
  Layout L;
  L.count = up256(tiles * rows * sizeof(float4));
  L.cand = L.count + up256(top ? 2 * tiles * rows : 0);
  L.target = L.cand + up256(2 * tiles * rows * top * sizeof(uint2));
  L.slots = L.target + up256(rows * sizeof(float));
  const bool b = bounded(N, V, top);
  L.bound = L.slots + up256(b ? rows * 32 * sizeof(uint32_t) : 0);
  L.total = N ? L.bound + up256(b ? rows * sizeof(uint32_t) : 0) : 0;
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
  tb.part = reinterpret_cast<float4*>(ws);
  tb.count = reinterpret_cast<uint8_t*>(ws + L.count);
  tb.cand = reinterpret_cast<uint2*>(ws + L.cand);
  tb.target = reinterpret_cast<float*>(ws + L.target);
  const bool bound = bounded(l.N, l.V, l.top);
  tb.slots = bound ? reinterpret_cast<uint32_t*>(ws + L.slots) : nullptr;
  tb.bound = bound ? reinterpret_cast<uint32_t*>(ws + L.bound) : nullptr;
  const int tiles = int((int64_t(l.V) + VT - 1) / VT);
  for (int lo = 0; lo < l.N; lo += SLAB) {
    TileArgs g{};
    g.A = static_cast<const u16*>(l.w);
    g.B = l.u + int64_t(lo) * l.D;
    g.M = l.V;
    g.N = std::min(SLAB, l.N - lo);
    g.K = l.D;
    const int32_t* ids = l.ids ? l.ids + lo : nullptr;
    if (bound) {
      const int n = int((L.total - L.slots) / sizeof(uint32_t));
      hipLaunchKernelGGL(clear_kernel, dim3((n + 255) / 256), dim3(256), 0, s, tb.slots, n);
    }
    hipError_t err = l.packed ? launch_tiles<A_PACKED>(g, tb, ids, tiles, l.top, s)
                              : launch_tiles<A_ROWS>(g, tb, ids, tiles, l.top, s);
    if (err != hipSuccess) return err;
    JoinArgs j;
    j.tb = tb;
    j.ids = ids;
    j.V = l.V;
    j.tiles = tiles;
    j.top = l.top;
    j.falling = !bound;
    j.logprob = l.ids ? l.logprob + lo : nullptr;
    j.entropy = l.entropy ? l.entropy + lo : nullptr;
    j.top_ids = l.top ? l.top_ids + int64_t(lo) * l.top : nullptr;
    j.top_logprob = l.top ? l.top_logprob + int64_t(lo) * l.top : nullptr;
    hipLaunchKernelGGL(logprobs_join, dim3(g.N), dim3(64), 0, s, j);
    err = hipGetLastError();
    if (err != hipSuccess) return err;
  }
  return hipSuccess;
}

}  // namespace cc
