// Appending new tokens to the cache: keys rotated to their positions on the way, values as they
// are, into rows of the cache's type or into E4M3 codes with a power-of-two scale for each block of
// entries and head; the queries of the same tokens are rotated in the same launch.
//
// Rotation: elements e and e + d/2 of a row turn by the angle pos * theta^(-2e/d).  The angle is
// taken in fp64, in revolutions and less its whole ones (a position of 2^20 keeps 2^-33 of a
// revolution), its sine and cosine in fp32; a workgroup computes those of its tokens once, in LDS,
// for all its heads.
//
// 8 bits: a workgroup owns a whole scale block (a block's entries lie in one page), so its scale
// needs no second pass: rows in registers, the largest magnitude of a head by shuffles and one LDS
// maximum (order-free: the same bits whatever the order), then the codes.  Scales are powers of two,
// so a block whose scale grows with a later token keeps its entries exactly, but for codes that
// fall below the normal range, and products with scales are exact wherever they are taken.
//
// Bound by memory for chunks of a prompt (8192 tokens, 32 heads on 8, into 8 bits: 185 MB in 42 us, 4.4 TB/s, and in 33
// where the last-level cache still holds the cache's pages; 3166 ragged tokens into bf16 pages: 78 MB in 15.0 us,
// 5.2 TB/s; a large copy reaches 4.9) and by the round trips to lengths, then rows, for single tokens (eight:
// 6 us); a row is read 16 elements a lane (e .. e + 7 and their partners), 16 bytes a load.
#include <algorithm>
#include <cmath>

#include "cc_internal.h"

namespace cc {
namespace {

constexpr int NT = 256;
// Tokens of a query unit (1, 4 and 16: 8192 tokens of 32 heads 48.6, 44.9 and 54.5 us, one token each of 256
// sequences 6.7, 8.3 and 15.8, 64 of them 5.3, 5.5 and 12.9).
constexpr int QT = 4;
constexpr int PLAIN_SHIFT = 4; // tokens of a unit of a 16/32-bit cache: 16

template <int HD>
struct AppendArgs {
  cc_rows k, v, q;
  void* q_out;
  const int32_t *cached, *pos, *cu;
  Kv8View kc, vc;
  int n_seqs, M, layer, hq, hkv, capacity, rotate;
  int shift;                 // log2 of the tokens of a key/value unit (a scale block)
  int each;                  // new tokens of every sequence, or -1: they differ
  int splits, heads;         // head ranges of a unit, heads of a range
  int units_kv, units_q, units;   // per layer: key/value units, query units, workgroups
  double freq[HD / 2];       // revolutions per position
};

// The last b with start(b) <= x, start rising: 64 candidates at a time, one round trip for up to 64
// sequences where a binary search takes six.
template <class F>
__device__ __forceinline__ int find_last(int n, int x, F start) {
  const int lane = threadIdx.x & 63;
  int lo = 0;
  while (n > 1) {
    const int step = (n + 63) >> 6;
    const int b = lo + lane * step;
    const bool le = lane * step < n && start(b) <= x;
    const int c = __popcll(__ballot(le));   // start(lo) <= x always
    lo += (c - 1) * step;
    n = min(step, n - (c - 1) * step);
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

struct Eight {
  float v[8];
};
__device__ __forceinline__ Eight load8(const u16* p) {
  const uint4 u = *reinterpret_cast<const uint4*>(p);
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
  Eight r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    r.v[2 * i] = __uint_as_float(w[i] << 16);
    r.v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
  return r;
}
__device__ __forceinline__ Eight load8(const float* p) {
  const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
  return Eight{{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
}
__device__ __forceinline__ void store8(u16* p, const float* x) {
  *reinterpret_cast<uint4*>(p) =
      make_uint4(pack_bf2(x[0], x[1]), pack_bf2(x[2], x[3]), pack_bf2(x[4], x[5]), pack_bf2(x[6], x[7]));
}
__device__ __forceinline__ void store8(float* p, const float* x) {
  *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
  *reinterpret_cast<float4*>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
}

// (cos, sin) of position pos for pair e.
__device__ __forceinline__ float2 turn(int pos, double freq) {
  double r = double(pos) * freq;
  r -= rint(r);
  float s, c;
  sincospif(2.f * float(r), &s, &c);
  return make_float2(c, s);
}

// x[0..7] and x[8..15] hold the pairs whose (cos, sin) are cs[0..7].
__device__ __forceinline__ void rotate16(float (&x)[16], const float2* cs) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float2 t = cs[i];
    const float lo = x[i], hi = x[8 + i];
    x[i] = lo * t.x - hi * t.y;
    x[8 + i] = hi * t.x + lo * t.y;
  }
}

template <class T, int HD, bool F8>
__global__ __launch_bounds__(NT) void append_kernel(AppendArgs<HD> a) {
  constexpr int LPR = HD / 16;        // lanes of a row
  constexpr int ROWS = NT / LPR;      // rows of a pass
  constexpr int MAXP = F8 ? (128 + ROWS - 1) / ROWS : 1;
  extern __shared__ float2 table[];   // [tokens][HD / 2]
  __shared__ uint32_t amax[64];
  const int tid = threadIdx.x;
  const int g = tid / LPR, c = tid % LPR;   // row of the pass, chunk of the row
  const int li = blockIdx.x / a.units;
  int u = blockIdx.x - li * a.units;
  if (u >= a.units_kv) {   // queries: QT tokens, all heads
    u -= a.units_kv;
    const int i0 = u * QT, nt = min(QT, a.M - i0);
    if (a.rotate) {
      for (int x = tid; x < QT * (HD / 2); x += NT) {
        const int i = x / (HD / 2);   // HD / 2 is at least a half wave: the search below runs in whole waves
        const int tok = i0 + min(i, nt - 1);
        int pos;
        if (a.pos) {
          pos = a.pos[tok];
        } else {
          int b = tok;
          if (a.each < 0) {
            if constexpr (HD == 128)
              b = find_last(a.n_seqs, tok, [&](int y) { return a.cu[y]; });
            else {   // two tokens a wave: the lower half's, then the upper half's
              const int t0 = __builtin_amdgcn_readlane(tok, 0), t1 = __builtin_amdgcn_readlane(tok, 63);
              const int b0 = find_last(a.n_seqs, t0, [&](int y) { return a.cu[y]; });
              const int b1 = find_last(a.n_seqs, t1, [&](int y) { return a.cu[y]; });
              b = tok == t0 ? b0 : b1;
            }
          } else {
            b = tok / a.each;
          }
          pos = max(a.cached[b], 0) + tok - a.cu[b];
        }
        table[x] = turn(pos, a.freq[x % (HD / 2)]);
      }
      __syncthreads();
    }
    for (int r = g; r < nt * a.hq; r += ROWS) {
      const int i = r / a.hq, h = r % a.hq;
      const T* src = static_cast<const T*>(a.q.base) + int64_t(i0 + i) * a.q.tok_stride + int64_t(h) * a.q.head_stride;
      const Eight lo = load8(src + c * 8), hi = load8(src + HD / 2 + c * 8);
      float x[16];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[e] = lo.v[e];
        x[8 + e] = hi.v[e];
      }
      if (a.rotate) rotate16(x, table + i * (HD / 2) + c * 8);
      T* dst = static_cast<T*>(a.q_out) + (int64_t(i0 + i) * a.hq + h) * HD;
      store8(dst + c * 8, x);
      store8(dst + HD / 2 + c * 8, x + 8);
    }
    return;
  }
  const bool keys = (u & 1) == 0;
  u >>= 1;
  const int split = u % a.splits;
  u /= a.splits;
  // Units of a sequence: its tokens may touch one block more than they fill.  Sequence b's first unit
  // is cu[b] / block + 2 b, which leaves every one enough.
  int b, j;
  if (a.each >= 0) {
    const int per = (a.each + 2 * (1 << a.shift) - 2) >> a.shift;
    b = u / per;
    j = u - b * per;
  } else {
    auto start = [&](int y) { return (a.cu[y] >> a.shift) + 2 * y; };
    b = find_last(a.n_seqs, u, start);
    j = u - start(b);
  }
  const int first = a.cu[b], m = a.cu[b + 1] - first;
  const int was = max(a.cached[b], 0);
  const int blk = (was >> a.shift) + j;
  const int64_t b0 = int64_t(blk) << a.shift;   // the block's first entry
  const int64_t end = min(int64_t(was) + m, int64_t(a.capacity));
  const int t0 = int(max(b0, int64_t(was))), t1 = int(min(b0 + (1 << a.shift), end));
  if (m <= 0 || b0 >= end || t0 >= t1) return;
  const Kv8View& kv = keys ? a.kc : a.vc;
  const cc_rows& in = keys ? a.k : a.v;
  const int layer = a.layer + li;
  int64_t dst0;        // the block's first row, head 0
  int64_t sc0 = 0;     // its scale, head 0
  if (kv.paged) {
    const int page = kv.codes.block_table[int64_t(b) * kv.codes.max_pages + (b0 >> kv.codes.page_shift)];
    if (page < 0) return;
    const int slot = int(b0) & kv.codes.page_mask;
    dst0 = int64_t(layer) * kv.codes.layer_stride + int64_t(page) * kv.codes.page_stride + slot * kv.codes.tok_stride;
    sc0 = int64_t(layer) * kv.s_layer + int64_t(page) * kv.s_page + (slot >> a.shift);
  } else {
    dst0 = int64_t(b) * kv.codes.seq_stride + int64_t(layer) * kv.codes.layer_stride + b0 * kv.codes.tok_stride;
    sc0 = int64_t(b) * kv.s_seq + int64_t(layer) * kv.s_layer + blk;
  }
  const int nt = t1 - t0, i0 = first + (t0 - was);
  const int h_lo = split * a.heads, h_hi = min(a.hkv, h_lo + a.heads);
  const bool rot = keys && a.rotate;
  if (F8 && tid < 64) amax[tid] = 0;
  if (rot)
    for (int x = tid; x < nt * (HD / 2); x += NT) {
      const int i = x / (HD / 2);
      table[x] = turn(a.pos ? a.pos[i0 + i] : t0 + i, a.freq[x % (HD / 2)]);
    }
  if (F8 || rot) __syncthreads();
  // Rows of a pass: TS tokens of ROWS / TS heads.
  int ts_log = 0;
  while ((1 << ts_log) < nt && (1 << ts_log) < ROWS) ++ts_log;
  const int TS = 1 << ts_log, HS = ROWS >> ts_log;
  const int ti = g & (TS - 1);
  char* base = static_cast<char*>(const_cast<void*>(kv.codes.base));
  for (int hb = h_lo; hb < h_hi; hb += HS) {
    const int h = hb + (g >> ts_log);
    const bool on = h < h_hi;
    const T* src = static_cast<const T*>(in.base) + int64_t(li) * in.layer_stride + int64_t(i0) * in.tok_stride +
                   int64_t(on ? h : h_lo) * in.head_stride;
    char* rows = base + dst0 + int64_t(on ? h : h_lo) * kv.codes.head_stride;
    uint8_t* sc = kv.scale + sc0 + int64_t(on ? h : h_lo) * kv.s_head;
    float x[MAXP][16];
    float top = 0.f;
#pragma unroll
    for (int p = 0; p < MAXP; ++p) {
      const int i = ti + p * TS;
      if (on && i < nt) {
        const Eight lo = load8(src + int64_t(i) * in.tok_stride + c * 8);
        const Eight hi = load8(src + int64_t(i) * in.tok_stride + HD / 2 + c * 8);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          x[p][e] = lo.v[e];
          x[p][8 + e] = hi.v[e];
        }
        if (rot) rotate16(x[p], table + i * (HD / 2) + c * 8);
        if constexpr (F8) {
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float y = fabsf(x[p][e]);
            if (y <= 3.402823466e38f) top = fmaxf(top, y);   // finite
          }
        } else {
          T* dst = reinterpret_cast<T*>(rows + (t0 + i - b0) * kv.codes.tok_stride);
          store8(dst + c * 8, x[p]);
          store8(dst + HD / 2 + c * 8, x[p] + 8);
        }
      }
    }
    if constexpr (F8) {
#pragma unroll
      for (int off = 1; off < LPR; off <<= 1) top = fmaxf(top, __shfl_xor(top, off));
      if (on && c == 0) atomicMax(&amax[h - h_lo], __float_as_uint(top));
      const bool held = on && t0 > b0;   // entries before the new ones share the block
      const uint32_t old = held ? *sc : 0;
      __syncthreads();   // the maxima are whole, and every old scale is read before any is written
      if (!on) continue;
      const uint32_t fresh = e8m0_of(amax[h - h_lo]);
      const uint32_t e = max(fresh, held ? min(old, 254u) : 0u);
      const float inv = e8m0_inverse(e);
#pragma unroll
      for (int p = 0; p < MAXP; ++p) {
        const int i = ti + p * TS;
        if (i < nt) {
#pragma unroll
          for (int k = 0; k < 16; ++k) {
            const float y = x[p][k];
            x[p][k] = fabsf(y) <= 3.402823466e38f ? y * inv : __uint_as_float(0x7fc00000u);
          }
          char* dst = rows + (t0 + i - b0) * kv.codes.tok_stride;
          *reinterpret_cast<uint2*>(dst + c * 8) = make_uint2(e4m3_pack(x[p][0], x[p][1], x[p][2], x[p][3]),
                                                              e4m3_pack(x[p][4], x[p][5], x[p][6], x[p][7]));
          *reinterpret_cast<uint2*>(dst + HD / 2 + c * 8) =
              make_uint2(e4m3_pack(x[p][8], x[p][9], x[p][10], x[p][11]),
                         e4m3_pack(x[p][12], x[p][13], x[p][14], x[p][15]));
        }
      }
      if (ti == 0 && c == 0) *sc = uint8_t(e);
      if (held && e > old) {   // the entries before, in the grown scale
        const float f = e8m0_scale(old) * inv;
        for (int64_t t = b0 + ti; t < t0; t += TS) {
          uint4* w = reinterpret_cast<uint4*>(rows + (t - b0) * kv.codes.tok_stride + c * 16);
          const uint4 o = *w;
          const uint32_t in4[4] = {o.x, o.y, o.z, o.w};
          uint32_t n4[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(int(in4[k]), false);
            const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8(int(in4[k]), true);
            n4[k] = e4m3_pack(lo[0] * f, lo[1] * f, hi[0] * f, hi[1] * f);
          }
          *w = make_uint4(n4[0], n4[1], n4[2], n4[3]);
        }
      }
    }
  }
}

template <class T, int HD, bool F8>
hipError_t launch_typed(const AppendLaunch& l, hipStream_t s) {
  AppendArgs<HD> a;
  a.k = l.k;   // (bases and first layer below)
  a.v = l.v;
  a.q = l.q;
  a.q_out = l.q_out;
  a.cached = l.cached;
  a.pos = l.pos;
  a.cu = l.cu_d;
  a.kc = l.kc;
  a.vc = l.vc;
  a.n_seqs = l.n_seqs;
  a.M = l.cu_h[l.n_seqs];
  a.hq = l.n_heads_q;
  a.hkv = l.n_heads_kv;
  a.capacity = l.capacity;
  a.rotate = l.rotate;
  a.shift = F8 ? l.kc.block_shift : PLAIN_SHIFT;
  const int B = 1 << a.shift;
  a.each = l.cu_h[1];
  for (int b = 1; b < l.n_seqs && a.each >= 0; ++b)
    if (l.cu_h[b + 1] - l.cu_h[b] != a.each) a.each = -1;
  const int64_t blocks = a.each >= 0 ? int64_t(l.n_seqs) * ((a.each + 2 * B - 2) / B) : a.M / B + 2 * int64_t(l.n_seqs);
  // Heads are shared out until there are some 640 workgroups, one head each at the most.  (8 heads of 128,
  // up to 256, 640 and 1024 workgroups: two sequences' chunks of 500 8.7, 7.4 and 7.4 us, one of 2000 10.6,
  // 10.0 and 13.8, one token each of 256 sequences 5.8, 5.8 and 8.3; 8192 tokens in blocks of 64
  // 51.7, 43.9 and 45.0.)
  a.splits = int(std::min<int64_t>(a.hkv, std::max<int64_t>(1, 640 / (2 * blocks * l.n_layers))));
  a.splits = std::max(a.splits, (a.hkv + 63) / 64);
  a.heads = (a.hkv + a.splits - 1) / a.splits;
  a.splits = (a.hkv + a.heads - 1) / a.heads;
  const int64_t kv = 2 * blocks * a.splits, q = l.q.base ? (a.M + QT - 1) / QT : 0;
  if (kv + q > MOST_GROUPS) return hipErrorInvalidValue;   // (refused by the caller)
  a.units_kv = int(kv);
  a.units_q = int(q);
  a.units = int(kv + q);
  if (l.rotate) {
    const double step = -2.0 / HD * std::log(l.theta);
    for (int e = 0; e < HD / 2; ++e) a.freq[e] = std::exp(e * step) / 6.283185307179586476925;
  }
  const int most = a.each >= 0 ? std::min(B, a.each) : B;
  const size_t lds = l.rotate ? size_t(std::max(most, QT)) * (HD / 2) * sizeof(float2) : 0;
  // layers past one launch's workgroups go into further launches
  const int step = int(MOST_GROUPS / a.units);
  for (int lo = 0; lo < l.n_layers; lo += step) {
    a.layer = l.layer + lo;
    a.k.base = static_cast<const T*>(l.k.base) + lo * l.k.layer_stride;
    a.v.base = static_cast<const T*>(l.v.base) + lo * l.v.layer_stride;
    hipLaunchKernelGGL((append_kernel<T, HD, F8>), dim3(unsigned(a.units * std::min(step, l.n_layers - lo))), dim3(NT), lds, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <class T>
hipError_t launch_of(const AppendLaunch& l, hipStream_t s) {
  if (l.head_dim == 128) return l.f8 ? launch_typed<T, 128, true>(l, s) : launch_typed<T, 128, false>(l, s);
  return l.f8 ? launch_typed<T, 64, true>(l, s) : launch_typed<T, 64, false>(l, s);
}

}  // namespace

hipError_t launch_append(const AppendLaunch& l, hipStream_t s) {
  if (l.cu_h[l.n_seqs] == 0) return hipSuccess;
  return l.dtype == CC_BF16 ? launch_of<u16>(l, s) : launch_of<float>(l, s);
}

}  // namespace cc
