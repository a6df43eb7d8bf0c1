// C ABI of libcc: argument validation, planning (grids, work lists, workspace layout)
// and kernel launches for the refresh-scoring pass.  Host code only; every kernel lives
// in its own translation unit behind the launchers declared in cc_internal.h.
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstring>
#include <mutex>
#include <vector>

#include "attention_kv.h"
#include "attention_kv8.h"
#include "cc_internal.h"

using namespace cc;

namespace {

constexpr size_t kAlign = 256;

size_t align_up(size_t x) { return (x + kAlign - 1) & ~(kAlign - 1); }
int esize(int dtype) { return dtype == CC_BF16 ? 2 : 4; }
bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool is_pow2(int x) { return x > 0 && (x & (x - 1)) == 0; }

#define CC_TRY(x)                       \
  do {                                  \
    cc_status _st = (x);                \
    if (_st != CC_OK) return _st;       \
  } while (0)

#define CC_HIP(x)                                   \
  do {                                              \
    if ((x) != hipSuccess) return CC_ERR_HIP;       \
  } while (0)

cc_status check_problem(const cc_problem* p) {
  if (!p) return CC_ERR_ARG;
  if (p->dtype != CC_F32 && p->dtype != CC_BF16) return CC_ERR_DTYPE;
  if (p->mode != CC_MODE_LAST_LAYER && p->mode != CC_MODE_FULL &&
      p->mode != CC_MODE_LAST_LAYER_H && p->mode != CC_MODE_LAST_LAYER_FUSED)
    return CC_ERR_ARG;
  if (p->diag != CC_DIAG_STRICT && p->diag != CC_DIAG_INCLUSIVE) return CC_ERR_ARG;
  if (p->n_seqs < 1 || !p->cu_seqlens_h || !p->cu_seqlens_d) return CC_ERR_ARG;
  if (p->cu_seqlens_h[0] != 0) return CC_ERR_SHAPE;
  for (int b = 0; b < p->n_seqs; ++b)
    if (p->cu_seqlens_h[b + 1] < p->cu_seqlens_h[b]) return CC_ERR_SHAPE;
  if (p->n_heads_q < 1 || p->n_heads_kv < 1) return CC_ERR_SHAPE;
  if (p->n_heads_q % p->n_heads_kv != 0) return CC_ERR_SHAPE;
  if (p->head_dim < 1 || p->hidden < 1 || p->vocab < 1) return CC_ERR_SHAPE;
  if (p->n_frozen < 0) return CC_ERR_ARG;
  if (!std::isfinite(p->softmax_scale) || p->softmax_scale < 0.f) return CC_ERR_ARG;
  if (p->head_dim != 64 && p->head_dim != 128) return CC_ERR_UNSUPPORTED;
  // bf16 projections and the LM head step K in 64-element tiles
  if (p->dtype == CC_BF16 && p->hidden % 64 != 0) return CC_ERR_UNSUPPORTED;
  if (p->mode == CC_MODE_FULL || p->mode == CC_MODE_LAST_LAYER_H) {
    if ((p->mode == CC_MODE_FULL && p->n_layers < 1) || p->ffn < 1) return CC_ERR_SHAPE;
    if (p->dtype != CC_BF16) return CC_ERR_UNSUPPORTED;
    // the W_q epilogue rotates pairs 64 rows apart, the halves of a 128-wide head
    if (p->head_dim != 128) return CC_ERR_UNSUPPORTED;
    if (p->ffn % 64 != 0) return CC_ERR_UNSUPPORTED;
    if (!(p->rope_theta > 0.f) || !(p->rms_eps >= 0.f)) return CC_ERR_ARG;
  }
  if (p->lmhead_packed != 0 && p->lmhead_packed != 1) return CC_ERR_ARG;
  if (p->lmhead_packed && p->dtype != CC_BF16) return CC_ERR_UNSUPPORTED;
  return CC_OK;
}

int n_tokens(const cc_problem* p) { return p->cu_seqlens_h[p->n_seqs]; }
int max_len(const cc_problem* p) {
  int m = 0;
  for (int b = 0; b < p->n_seqs; ++b) m = std::max(m, p->cu_seqlens_h[b + 1] - p->cu_seqlens_h[b]);
  return m;
}

// es: bytes of a cache element; longest: entries that a sequence's block-table row must reach (-1: the
// problem's longest sequence).
cc_status check_kv(const cc_problem* p, const cc_kv* kv, int min_layers, int es = 0, int longest = -1) {
  if (!kv || !kv->k || !kv->v) return CC_ERR_ARG;
  if (kv->layout != CC_KV_CONTIGUOUS && kv->layout != CC_KV_PAGED) return CC_ERR_ARG;
  if (kv->n_layers < min_layers) return CC_ERR_SHAPE;
  if (kv->layer_stride < 0 || kv->head_stride < 0 || kv->tok_stride < p->head_dim)
    return CC_ERR_SHAPE;
  if (es == 0) es = esize(p->dtype);
  if (!aligned16(kv->k) || !aligned16(kv->v)) return CC_ERR_ARG;
  auto str_ok = [&](int64_t s) { return (s * es) % 16 == 0; };
  if (!str_ok(kv->layer_stride) || !str_ok(kv->head_stride) || !str_ok(kv->tok_stride))
    return CC_ERR_UNSUPPORTED;
  if (kv->layout == CC_KV_PAGED) {
    if (!kv->block_table || !is_pow2(kv->page_size) || kv->page_size < 16) return CC_ERR_ARG;
    if (kv->page_stride < 0 || !str_ok(kv->page_stride)) return CC_ERR_UNSUPPORTED;
    // in-page byte offsets are 32-bit in the kernels
    constexpr int64_t kPageLimit = int64_t(1) << 32;
    if (kv->page_stride * es >= kPageLimit || int64_t(kv->page_size) * kv->tok_stride * es >= kPageLimit)
      return CC_ERR_UNSUPPORTED;
    const int64_t len = longest >= 0 ? longest : max_len(p);
    if (kv->max_pages < (len + kv->page_size - 1) / kv->page_size) return CC_ERR_SHAPE;
  } else {
    if (kv->seq_stride < 0 || !str_ok(kv->seq_stride)) return CC_ERR_UNSUPPORTED;
  }
  return CC_OK;
}

// Address view for kernels; byte_strides = true multiplies strides by the element size.
KvView make_view(const cc_kv* kv, const void* base, int es_mult) {
  KvView v;
  v.base = base;
  v.seq_stride = kv->seq_stride * es_mult;
  v.layer_stride = kv->layer_stride * es_mult;
  v.head_stride = kv->head_stride * es_mult;
  v.tok_stride = kv->tok_stride * es_mult;
  v.page_stride = kv->page_stride * es_mult;
  v.block_table = kv->block_table;
  int shift = 0;
  if (kv->layout == CC_KV_PAGED)
    while ((1 << shift) < kv->page_size) ++shift;
  v.page_shift = shift;
  v.page_mask = kv->layout == CC_KV_PAGED ? kv->page_size - 1 : 0;
  v.max_pages = kv->max_pages;
  v.pad = 0;
  return v;
}

float softmax_scale(const cc_problem* p) {
  return p->softmax_scale > 0.f ? p->softmax_scale : 1.f / std::sqrt(float(p->head_dim));
}

// Attention work items, heaviest first: an item's cost is the number of keys its first
// row may attend to, n_b - first position.
std::vector<int4> attention_work(const cc_problem* p) {
  const int rows_item = attention_rows_per_item(p->dtype, p->head_dim);
  const int g = p->n_heads_q / p->n_heads_kv;
  std::vector<int4> items;
  std::vector<int64_t> cost;
  for (int b = 0; b < p->n_seqs; ++b) {
    const int n = p->cu_seqlens_h[b + 1] - p->cu_seqlens_h[b];
    const int64_t rows = int64_t(n) * g;
    const int nrb = int((rows + rows_item - 1) / rows_item);
    for (int rb = 0; rb < nrb; ++rb)
      for (int h = 0; h < p->n_heads_kv; ++h) {
        items.push_back(make_int4(b, h, rb, 0));
        cost.push_back(n - int64_t(rb) * rows_item / g);
      }
  }
  std::vector<int> idx(items.size());
  for (size_t i = 0; i < idx.size(); ++i) idx[i] = int(i);
  std::stable_sort(idx.begin(), idx.end(), [&](int a, int c) { return cost[a] > cost[c]; });
  std::vector<int4> out(items.size());
  for (size_t i = 0; i < idx.size(); ++i) out[i] = items[idx[i]];
  return out;
}

size_t attention_ws_bytes(const cc_problem* p) {
  const int rows_item = attention_rows_per_item(p->dtype, p->head_dim);
  const int g = p->n_heads_q / p->n_heads_kv;
  size_t items = 0;
  for (int b = 0; b < p->n_seqs; ++b) {
    const int64_t n = p->cu_seqlens_h[b + 1] - p->cu_seqlens_h[b];
    items += size_t((n * g + rows_item - 1) / rows_item) * p->n_heads_kv;
  }
  return align_up(items * sizeof(int4));
}

// Input width of the LM head: the model width, or Hq*d for the W_o-folded weight.
int lmhead_k(const cc_problem* p) {
  return p->mode == CC_MODE_LAST_LAYER_FUSED ? p->n_heads_q * p->head_dim : p->hidden;
}

// What an LM head call needs: per-(vocabulary tile, entry) partials and target logits.
size_t lmhead_ws_bytes(const cc_problem* p) {
  const size_t N = n_tokens(p);
  const int vt = lmhead_vocab_tile(p->dtype);
  const size_t n_vt = (p->vocab + vt - 1) / vt;
  return align_up(n_vt * N * sizeof(float2)) + align_up(N * sizeof(float));
}

struct ScoreLayout {
  size_t attn, o, u, lm, total;
};

struct FullLayout {
  size_t attn, rot, h, a, q, o, act, lm, part, total;
};

FullLayout full_layout(const cc_problem* p) {
  FullLayout L;
  const size_t N = n_tokens(p);
  const size_t HD = size_t(p->n_heads_q) * p->head_dim;
  size_t off = 0;
  L.attn = off;
  off += attention_ws_bytes(p);
  L.rot = off;
  off += align_up(N * (p->head_dim / 2) * sizeof(float2));
  L.h = off;
  off += align_up(N * p->hidden * sizeof(float));
  L.a = off;
  off += align_up(N * p->hidden * 2);
  L.q = off;
  off += align_up(N * HD * 2);
  L.o = off;
  off += align_up(N * HD * 2);
  L.act = off;
  off += align_up(N * size_t(p->ffn) * 2);
  L.lm = off;
  off += lmhead_ws_bytes(p);
  // split-K partial sums of the projections whose tiles underfill the chip (small N)
  const int D = p->hidden, F = p->ffn, hd = int(HD);
  size_t part = 0;
  auto need = [&](int M, int Nn, int K) {
    const int S = gemm_split_slices(M, Nn, K);
    if (S > 1) part = std::max(part, size_t(S) * size_t(M) * size_t(Nn) * sizeof(float));
  };
  need(int(N), D, hd);   // W_o
  need(int(N), D, F);    // W_down
  L.part = off;
  off += align_up(part);
  L.total = off;
  return L;
}

ScoreLayout score_layout(const cc_problem* p) {
  ScoreLayout L;
  const size_t N = n_tokens(p), es = esize(p->dtype);
  size_t off = 0;
  L.attn = off;
  off += attention_ws_bytes(p);
  L.o = off;
  off += align_up(N * p->n_heads_q * p->head_dim * es);
  L.u = off;
  if (p->mode != CC_MODE_LAST_LAYER_FUSED) off += align_up(N * p->hidden * es);
  L.lm = off;
  off += lmhead_ws_bytes(p);
  L.total = off;
  return L;
}

char* at(void* ws, size_t off) { return static_cast<char*>(ws) + off; }

// Attention over cache layer `layer`.  The work list is uploaded into `ws` unless an earlier
// call of the same cc_score already did (upload = false).
cc_status run_attention(const cc_problem* p, const void* q, const cc_kv* kv, int layer, void* o,
                        void* ws, hipStream_t s, bool upload = true) {
  AttnLaunch a;
  a.table = AttnTable{nullptr, p->cu_seqlens_d};
  a.items.nkv = p->n_heads_kv;
  a.items.n_seqs = 0;
  if (p->n_seqs <= ATTN_INLINE) {
    const int rows_item = attention_rows_per_item(p->dtype, p->head_dim);
    const int g = p->n_heads_q / p->n_heads_kv;
    int64_t blocks = 0;
    for (int b = 0; b < p->n_seqs; ++b) {
      const int seq0 = p->cu_seqlens_h[b], n = p->cu_seqlens_h[b + 1] - seq0;
      const int nb = int((int64_t(n) * g + rows_item - 1) / rows_item);
      a.items.seqs[a.items.n_seqs++] = AttnSeq{b, seq0, n, nb};
      blocks += nb;
    }
    std::stable_sort(a.items.seqs, a.items.seqs + a.items.n_seqs,
                     [](const AttnSeq& x, const AttnSeq& y) { return x.blocks > y.blocks; });
    a.n_work = int(blocks * p->n_heads_kv);
  } else {
    const std::vector<int4> work = attention_work(p);
    if (upload && !work.empty())
      CC_HIP(hipMemcpyAsync(ws, work.data(), work.size() * sizeof(int4), hipMemcpyHostToDevice, s));
    a.table.table = static_cast<const int4*>(ws);
    a.n_work = int(work.size());
  }
  if (a.n_work == 0) return CC_OK;
  a.dtype = p->dtype;
  a.q = q;
  a.o = o;
  a.k = make_view(kv, kv->k, 1);
  a.v = make_view(kv, kv->v, 1);
  a.paged = kv->layout == CC_KV_PAGED;
  a.layer = layer;
  a.n_heads_q = p->n_heads_q;
  a.n_heads_kv = p->n_heads_kv;
  a.head_dim = p->head_dim;
  a.scale = softmax_scale(p);
  a.inclusive = p->diag == CC_DIAG_INCLUSIVE;
  CC_HIP(launch_attention(a, s));
  return CC_OK;
}

// LM head over rows u [N][D]; D is the model width unless given (the fused weight's
// input width Hq*d).
cc_status run_lmhead(const cc_problem* p, const void* u, const void* w_lm, const int32_t* ids,
                     float* scores, float* lse, void* ws, hipStream_t s, int D = 0,
                     const void* w_packed = nullptr) {
  const int N = n_tokens(p);
  const int vt = lmhead_vocab_tile(p->dtype);
  const size_t n_vt = (p->vocab + vt - 1) / vt;
  LmHeadLaunch a;
  a.dtype = p->dtype;
  a.u = u;
  a.w_lm = w_lm;
  a.ids = ids;
  a.scores = scores;
  a.lse = lse;
  a.partial = reinterpret_cast<float2*>(ws);
  a.target = reinterpret_cast<float*>(at(ws, align_up(n_vt * N * sizeof(float2))));
  a.cu_d = p->cu_seqlens_d;
  a.n_seqs = p->n_seqs;
  a.N = N;
  a.D = D > 0 ? D : p->hidden;
  a.V = p->vocab;
  a.n_frozen = p->n_frozen;
  if (p->lmhead_packed) {
    if (!w_packed) return CC_ERR_ARG;
    a.w_packed = w_packed;
  }
  CC_HIP(launch_lmhead(a, s));
  return CC_OK;
}

// The row-major LM head weight, needed unless the packed one is used.
bool lm_weight_ok(const cc_problem* p, const void* w_lm) {
  return p->lmhead_packed || (w_lm && aligned16(w_lm));
}

// The packed LM head needs its weight (checked before anything is launched).
cc_status check_packed(const cc_problem* p, const void* w_packed) {
  if (!p->lmhead_packed || n_tokens(p) == 0) return CC_OK;
  if (!w_packed || !aligned16(w_packed)) return CC_ERR_ARG;
  return CC_OK;
}

cc_status check_ws(void* ws, size_t have, size_t need) {
  if (have < need) return CC_ERR_WORKSPACE;
  if (need > 0 && !ws) return CC_ERR_ARG;
  if (need > 0 && (reinterpret_cast<uintptr_t>(ws) % kAlign) != 0) return CC_ERR_ARG;
  return CC_OK;
}

// Full L-layer pass (Sec. 3.1): h = E[x]; per layer a = RMSNorm(h), q = RoPE(W_q a),
// o = counter-causal attention on the stored K_l, V_l, h += W_o o, b = RMSNorm(h),
// h += W_down (silu(W_gate b) * W_up b); then u = RMSNorm(h) and the LM head.
cc_status score_full(const cc_problem* p, const cc_inputs* in, float* scores, void* ws,
                     size_t ws_bytes, void* stream) {
  CC_TRY(check_kv(p, &in->kv, p->n_layers));
  const int N = n_tokens(p);
  if (N > 0 && (!in->embed || !in->layers_h || !in->final_norm || !in->token_ids || !scores))
    return CC_ERR_ARG;
  if (N > 0) {
    if (!aligned16(in->embed) || !lm_weight_ok(p, in->w_lm) || !aligned16(in->final_norm))
      return CC_ERR_ARG;
    for (int l = 0; l < p->n_layers; ++l) {
      const cc_layer_weights& W = in->layers_h[l];
      const void* ptrs[7] = {W.attn_norm, W.wq, W.wo, W.mlp_norm, W.w_gate, W.w_up, W.w_down};
      for (const void* q : ptrs)
        if (!q || !aligned16(q)) return CC_ERR_ARG;
    }
  }
  CC_TRY(check_packed(p, in->w_lm_packed));
  const FullLayout L = full_layout(p);
  CC_TRY(check_ws(ws, ws_bytes, L.total));
  if (N == 0) return CC_OK;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int D = p->hidden, F = p->ffn, HD = p->n_heads_q * p->head_dim;
  float2* rot = reinterpret_cast<float2*>(at(ws, L.rot));
  float* h = reinterpret_cast<float*>(at(ws, L.h));
  void* a = at(ws, L.a);
  void* q = at(ws, L.q);
  void* o = at(ws, L.o);
  void* act = at(ws, L.act);
  float* part = reinterpret_cast<float*>(at(ws, L.part));
  CC_HIP(launch_enter(in->embed, in->token_ids, in->pos_ids, p->cu_seqlens_d, p->n_seqs, rot, h,
                      in->layers_h[0].attn_norm, a, N, D, p->head_dim, double(p->rope_theta), p->rms_eps, s));
  for (int l = 0; l < p->n_layers; ++l) {
    const cc_layer_weights& W = in->layers_h[l];
    const void* next = l + 1 < p->n_layers ? in->layers_h[l + 1].attn_norm : in->final_norm;
    CC_HIP(launch_qproj_rope(W.wq, a, q, rot, N, D, HD, s));
    CC_TRY(run_attention(p, q, &in->kv, l, o, at(ws, L.attn), s, l == 0));
    CC_HIP(launch_linear_residual_norm(o, W.wo, h, W.mlp_norm, a, N, D, HD, p->rms_eps, part, s));
    CC_HIP(launch_gate_up_swiglu(W.w_gate, W.w_up, a, act, N, D, F, s));
    CC_HIP(launch_linear_residual_norm(act, W.w_down, h, next, a, N, D, F, p->rms_eps, part, s));
  }
  return run_lmhead(p, a, in->w_lm, in->token_ids, scores, nullptr, at(ws, L.lm), s, 0,
                    in->w_lm_packed);
}

// The exact fast variant (Sec. 3.1, fast single-layer approximation): one layer of the
// full pass, entered with the stored activations H instead of the embedding stack, on
// the cache's last layer.
cc_status score_last_h(const cc_problem* p, const cc_inputs* in, float* scores, void* ws,
                       size_t ws_bytes, void* stream) {
  CC_TRY(check_kv(p, &in->kv, 1));
  const int N = n_tokens(p);
  if (N > 0 && (!in->h_last || !in->layers_h || !in->final_norm || !in->token_ids || !scores))
    return CC_ERR_ARG;
  if (N > 0) {
    if (!aligned16(in->h_last) || !lm_weight_ok(p, in->w_lm) || !aligned16(in->final_norm))
      return CC_ERR_ARG;
    const cc_layer_weights& W = in->layers_h[0];
    const void* ptrs[7] = {W.attn_norm, W.wq, W.wo, W.mlp_norm, W.w_gate, W.w_up, W.w_down};
    for (const void* q : ptrs)
      if (!q || !aligned16(q)) return CC_ERR_ARG;
  }
  CC_TRY(check_packed(p, in->w_lm_packed));
  const FullLayout L = full_layout(p);
  CC_TRY(check_ws(ws, ws_bytes, L.total));
  if (N == 0) return CC_OK;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int D = p->hidden, F = p->ffn, HD = p->n_heads_q * p->head_dim;
  float2* rot = reinterpret_cast<float2*>(at(ws, L.rot));
  float* h = reinterpret_cast<float*>(at(ws, L.h));
  void* a = at(ws, L.a);
  void* q = at(ws, L.q);
  void* o = at(ws, L.o);
  void* act = at(ws, L.act);
  float* part = reinterpret_cast<float*>(at(ws, L.part));
  const cc_layer_weights& W = in->layers_h[0];
  // H widens to the fp32 stream
  CC_HIP(launch_enter(in->h_last, nullptr, in->pos_ids, p->cu_seqlens_d, p->n_seqs, rot, h, W.attn_norm, a, N,
                      D, p->head_dim, double(p->rope_theta), p->rms_eps, s));
  CC_HIP(launch_qproj_rope(W.wq, a, q, rot, N, D, HD, s));
  CC_TRY(run_attention(p, q, &in->kv, in->kv.n_layers - 1, o, at(ws, L.attn), s));
  CC_HIP(launch_linear_residual_norm(o, W.wo, h, W.mlp_norm, a, N, D, HD, p->rms_eps, part, s));
  CC_HIP(launch_gate_up_swiglu(W.w_gate, W.w_up, a, act, N, D, F, s));
  CC_HIP(launch_linear_residual_norm(act, W.w_down, h, in->final_norm, a, N, D, F, p->rms_eps, part, s));
  return run_lmhead(p, a, in->w_lm, in->token_ids, scores, nullptr, at(ws, L.lm), s, 0,
                    in->w_lm_packed);
}

}  // namespace

extern "C" {

const char* cc_status_str(cc_status s) {
  switch (s) {
    case CC_OK: return "CC_OK";
    case CC_ERR_ARG: return "CC_ERR_ARG: invalid argument";
    case CC_ERR_SHAPE: return "CC_ERR_SHAPE: inconsistent sizes";
    case CC_ERR_DTYPE: return "CC_ERR_DTYPE: unsupported dtype for this call";
    case CC_ERR_WORKSPACE: return "CC_ERR_WORKSPACE: workspace too small";
    case CC_ERR_UNSUPPORTED: return "CC_ERR_UNSUPPORTED: no kernel for this shape";
    case CC_ERR_HIP: return "CC_ERR_HIP: HIP runtime error";
    case CC_ERR_SCRATCH: return "CC_ERR_SCRATCH: larger than the static scratch of the allocation-free entry point";
  }
  return "unknown cc_status";
}

const char* cc_version(void) { return "libcc gfx950 " __DATE__; }

cc_status cc_attention_workspace(const cc_problem* p, size_t* bytes) {
  if (!bytes) return CC_ERR_ARG;
  CC_TRY(check_problem(p));
  *bytes = attention_ws_bytes(p);
  return CC_OK;
}

cc_status cc_attention_cc(const cc_problem* p, const void* q, const cc_kv* kv, int32_t layer,
                          void* o, void* ws, size_t ws_bytes, void* stream) {
  CC_TRY(check_problem(p));
  CC_TRY(check_kv(p, kv, 1));
  if (layer < 0 || layer >= kv->n_layers) return CC_ERR_ARG;
  if (n_tokens(p) > 0 && (!q || !o)) return CC_ERR_ARG;
  if (p->dtype == CC_BF16 && (!aligned16(q) || !aligned16(o))) return CC_ERR_ARG;
  CC_TRY(check_ws(ws, ws_bytes, attention_ws_bytes(p)));
  return run_attention(p, q, kv, layer, o, ws, static_cast<hipStream_t>(stream));
}

cc_status cc_lmhead_workspace(const cc_problem* p, size_t* bytes) {
  if (!bytes) return CC_ERR_ARG;
  CC_TRY(check_problem(p));
  *bytes = lmhead_ws_bytes(p);
  // Of a packed problem the query has always covered a packed copy of the entry rows as well.  The
  // calls need no more than the above, and cc_score_workspace asks for no more.
  if (p->lmhead_packed) *bytes += align_up(packed_rows_bytes(n_tokens(p), lmhead_k(p)));
  return CC_OK;
}

cc_status cc_lmhead_score(const cc_problem* p, const void* u, const void* w_lm,
                          const int32_t* token_ids, float* scores, float* lse, void* ws,
                          size_t ws_bytes, void* stream) {
  CC_TRY(check_problem(p));
  if (n_tokens(p) > 0 && (!u || !w_lm || !token_ids || !scores)) return CC_ERR_ARG;
  if (p->dtype == CC_BF16 && (!aligned16(u) || !aligned16(w_lm))) return CC_ERR_ARG;
  if (p->lmhead_packed && n_tokens(p) > 0) return CC_ERR_ARG;   // cc_lmhead_score_packed
  CC_TRY(check_ws(ws, ws_bytes, lmhead_ws_bytes(p)));
  return run_lmhead(p, u, w_lm, token_ids, scores, lse, ws, static_cast<hipStream_t>(stream));
}

}  // extern "C"

// ------------------------------------------------------------------ allocation-free LM head
// The scratch of cc_lmhead_score_noalloc: a file-scope device array, one per GPU.  In host
// code its name is a host-side stand-in, not a device address, so it is never passed to a
// kernel or a copy; the device address comes from hipGetSymbolAddress, taken once per
// device with that device current and kept here.
namespace {
static __device__ __align__(256) unsigned char scratch[CC_NOALLOC_SCRATCH_BYTES];

constexpr int kMaxDevices = 64;
std::mutex g_scratch_mu;
void* g_scratch_ptr[kMaxDevices] = {};

// The scratch's device address on the current device (looked up on its first use there).
cc_status scratch_address(void** out) {
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess) return CC_ERR_HIP;
  if (dev < 0 || dev >= kMaxDevices) return CC_ERR_UNSUPPORTED;
  std::lock_guard<std::mutex> lock(g_scratch_mu);
  if (!g_scratch_ptr[dev]) {
    void* ptr = nullptr;
    if (hipGetSymbolAddress(&ptr, HIP_SYMBOL(scratch)) != hipSuccess || !ptr) return CC_ERR_HIP;
    g_scratch_ptr[dev] = ptr;
  }
  *out = g_scratch_ptr[dev];
  return CC_OK;
}
}  // namespace

extern "C" {

cc_status cc_lmhead_score_noalloc(const cc_problem* p, const void* u, const void* w_lm,
                                  const int32_t* token_ids, float* scores, float* lse,
                                  void* stream) {
  CC_TRY(check_problem(p));
  if (p->lmhead_packed) return CC_ERR_ARG;
  if (n_tokens(p) > 0 && (!u || !w_lm || !token_ids || !scores)) return CC_ERR_ARG;
  if (p->dtype == CC_BF16 && (!aligned16(u) || !aligned16(w_lm))) return CC_ERR_ARG;
  const size_t need = lmhead_ws_bytes(p);
  if (need > CC_NOALLOC_SCRATCH_BYTES) return CC_ERR_SCRATCH;
  if (n_tokens(p) == 0) return CC_OK;
  void* ws = nullptr;
  CC_TRY(scratch_address(&ws));
  return run_lmhead(p, u, w_lm, token_ids, scores, lse, ws, static_cast<hipStream_t>(stream));
}

cc_status cc_lmhead_score_packed(const cc_problem* p, const void* u, const void* w_packed,
                                 const int32_t* token_ids, float* scores, float* lse, void* ws,
                                 size_t ws_bytes, void* stream) {
  CC_TRY(check_problem(p));
  if (!p->lmhead_packed) return CC_ERR_ARG;
  if (n_tokens(p) > 0 && (!u || !token_ids || !scores)) return CC_ERR_ARG;
  if (!aligned16(u)) return CC_ERR_ARG;
  CC_TRY(check_packed(p, w_packed));
  CC_TRY(check_ws(ws, ws_bytes, lmhead_ws_bytes(p)));
  return run_lmhead(p, u, nullptr, token_ids, scores, lse, ws, static_cast<hipStream_t>(stream),
                    0, w_packed);
}

cc_status cc_pack_lmhead_bytes(int64_t rows, int32_t cols, size_t* bytes) {
  if (!bytes || rows < 0 || cols < 1 || cols % 32 != 0) return CC_ERR_ARG;
  *bytes = packed_rows_bytes(rows, cols);
  return CC_OK;
}

cc_status cc_pack_lmhead(const void* x, int64_t rows, int32_t cols, void* out,
                         size_t out_bytes, void* stream) {
  size_t need = 0;
  CC_TRY(cc_pack_lmhead_bytes(rows, cols, &need));
  if (rows == 0) return CC_OK;
  if (!x || !out || !aligned16(x) || !aligned16(out)) return CC_ERR_ARG;
  if (out_bytes < need) return CC_ERR_WORKSPACE;
  const char* xb = static_cast<const char*>(x);
  const char* ob = static_cast<const char*>(out);
  if (ob < xb + size_t(rows) * cols * 2 && xb < ob + need) return CC_ERR_ARG;   // overlap
  CC_HIP(launch_pack_rows(x, rows, cols, cols, out, static_cast<hipStream_t>(stream)));
  return CC_OK;
}

cc_status cc_linear(int32_t dtype, const void* x, const void* w, void* y, int32_t M, int32_t N,
                    int32_t K, void* stream) {
  if (dtype != CC_F32 && dtype != CC_BF16) return CC_ERR_DTYPE;
  if (M < 0 || N < 0 || K < 1) return CC_ERR_SHAPE;
  if (M > 0 && N > 0 && (!x || !w || !y)) return CC_ERR_ARG;
  if (dtype == CC_BF16) {
    if (K % 64 != 0) return CC_ERR_UNSUPPORTED;
    if (!aligned16(x) || !aligned16(w)) return CC_ERR_ARG;
  }
  CC_HIP(launch_linear(dtype, x, w, y, M, N, K, static_cast<hipStream_t>(stream)));
  return CC_OK;
}

cc_status cc_score_workspace(const cc_problem* p, size_t* bytes) {
  if (!bytes) return CC_ERR_ARG;
  CC_TRY(check_problem(p));
  const bool last = p->mode == CC_MODE_LAST_LAYER || p->mode == CC_MODE_LAST_LAYER_FUSED;
  *bytes = last ? score_layout(p).total : full_layout(p).total;
  return CC_OK;
}

cc_status cc_score(const cc_problem* p, const cc_inputs* in, float* scores, void* ws,
                   size_t ws_bytes, void* stream) {
  CC_TRY(check_problem(p));
  if (!in) return CC_ERR_ARG;
  if (p->mode == CC_MODE_FULL) return score_full(p, in, scores, ws, ws_bytes, stream);
  if (p->mode == CC_MODE_LAST_LAYER_H) return score_last_h(p, in, scores, ws, ws_bytes, stream);
  CC_TRY(check_kv(p, &in->kv, 1));
  const int N = n_tokens(p);
  const bool fused = p->mode == CC_MODE_LAST_LAYER_FUSED;
  if (N > 0 && (!in->q || (!fused && !in->w_o) || !in->token_ids || !scores)) return CC_ERR_ARG;
  if (N > 0 && !p->lmhead_packed && !in->w_lm) return CC_ERR_ARG;
  if (p->dtype == CC_BF16 &&
      (!aligned16(in->q) || (!fused && !aligned16(in->w_o)) || !lm_weight_ok(p, in->w_lm)))
    return CC_ERR_ARG;
  CC_TRY(check_packed(p, in->w_lm_packed));
  const ScoreLayout L = score_layout(p);
  CC_TRY(check_ws(ws, ws_bytes, L.total));
  if (N == 0) return CC_OK;
  hipStream_t s = static_cast<hipStream_t>(stream);
  void* o = at(ws, L.o);
  void* u = at(ws, L.u);
  CC_TRY(run_attention(p, in->q, &in->kv, in->kv.n_layers - 1, o, at(ws, L.attn), s));
  const int qdim = p->n_heads_q * p->head_dim;
  if (fused)   // z = (W_lm W_o) y straight from the attention rows
    return run_lmhead(p, o, in->w_lm, in->token_ids, scores, nullptr, at(ws, L.lm), s, qdim,
                      in->w_lm_packed);
  CC_HIP(launch_linear(p->dtype, o, in->w_o, u, N, p->hidden, qdim, s));
  return run_lmhead(p, u, in->w_lm, in->token_ids, scores, nullptr, at(ws, L.lm), s, 0,
                    in->w_lm_packed);
}

// ------------------------------------------------------------------ fused LM-head weight

cc_status cc_fuse_wo_lmhead_workspace(int32_t dtype, int32_t hidden, int32_t qdim,
                                      size_t* bytes) {
  if (!bytes) return CC_ERR_ARG;
  if (dtype != CC_F32 && dtype != CC_BF16) return CC_ERR_DTYPE;
  if (hidden < 1 || qdim < 1) return CC_ERR_SHAPE;
  *bytes = align_up(size_t(hidden) * qdim * esize(dtype));
  return CC_OK;
}

cc_status cc_fuse_wo_lmhead(int32_t dtype, const void* w_lm, const void* w_o, void* out,
                            int32_t vocab, int32_t hidden, int32_t qdim, void* ws,
                            size_t ws_bytes, void* stream) {
  if (dtype != CC_F32 && dtype != CC_BF16) return CC_ERR_DTYPE;
  if (vocab < 1 || hidden < 1 || qdim < 1) return CC_ERR_SHAPE;
  if (!w_lm || !w_o || !out) return CC_ERR_ARG;
  if (dtype == CC_BF16) {
    if (hidden % 64 != 0) return CC_ERR_UNSUPPORTED;
    if (!aligned16(w_lm) || !aligned16(w_o) || !aligned16(out)) return CC_ERR_ARG;
  }
  CC_TRY(check_ws(ws, ws_bytes, align_up(size_t(hidden) * qdim * esize(dtype))));
  hipStream_t s = static_cast<hipStream_t>(stream);
  // W_o [hidden][qdim] -> W_o^T [qdim][hidden] (K-contiguous), then out = W_lm (W_o^T)^T
  CC_HIP(launch_transpose(dtype, w_o, ws, hidden, qdim, s));
  CC_HIP(launch_linear(dtype, w_lm, ws, out, vocab, qdim, hidden, s));
  return CC_OK;
}

// ------------------------------------------------------------------ FP8 LM head

cc_status cc_quantize_fp8_workspace(int64_t rows, size_t* bytes) {
  if (!bytes || rows < 0) return CC_ERR_ARG;
  *bytes = align_up(size_t(rows + 1) * sizeof(float));
  return CC_OK;
}

cc_status cc_quantize_fp8(int32_t dtype, const void* x, int64_t rows, int32_t cols,
                          int32_t per_row, uint8_t* codes, float* scale, void* ws,
                          size_t ws_bytes, void* stream) {
  if (dtype != CC_F32 && dtype != CC_BF16) return CC_ERR_DTYPE;
  if (rows < 0 || rows > INT32_MAX || cols < 4 || cols % 4 != 0) return CC_ERR_SHAPE;
  if (per_row != 0 && per_row != 1) return CC_ERR_ARG;
  if (rows == 0) return CC_OK;
  if (!x || !codes || !scale) return CC_ERR_ARG;
  if ((reinterpret_cast<uintptr_t>(codes) & 3u) != 0) return CC_ERR_ARG;
  if ((reinterpret_cast<uintptr_t>(x) & uintptr_t(4 * esize(dtype) - 1)) != 0) return CC_ERR_ARG;
  CC_TRY(check_ws(ws, ws_bytes, align_up(size_t(rows + 1) * sizeof(float))));
  CC_HIP(launch_quantize_e4m3(dtype, x, rows, cols, per_row, codes, scale,
                              static_cast<float*>(ws), static_cast<hipStream_t>(stream)));
  return CC_OK;
}

namespace {
struct Fp8Layout {
  size_t uq, su, amax, partial, target, total;
};
Fp8Layout fp8_layout(const cc_problem* p) {
  Fp8Layout L;
  const size_t N = n_tokens(p), D = p->hidden;
  const size_t n_vt = (p->vocab + 255) / 256;
  size_t off = 0;
  L.uq = off;
  off += align_up(N * D);
  L.su = off;
  off += align_up(N * sizeof(float));
  L.amax = off;
  off += align_up((N + 1) * sizeof(float));
  L.partial = off;
  off += align_up(n_vt * N * sizeof(float2));
  L.target = off;
  off += align_up(N * sizeof(float));
  L.total = off;
  return L;
}
}  // namespace

cc_status cc_lmhead_fp8_workspace(const cc_problem* p, size_t* bytes) {
  if (!bytes) return CC_ERR_ARG;
  CC_TRY(check_problem(p));
  *bytes = fp8_layout(p).total;
  return CC_OK;
}

cc_status cc_lmhead_score_fp8(const cc_problem* p, const void* u, const uint8_t* w_codes,
                              const float* w_scale, const int32_t* token_ids, float* scores,
                              float* lse, void* ws, size_t ws_bytes, void* stream) {
  CC_TRY(check_problem(p));
  if (p->hidden % 128 != 0) return CC_ERR_UNSUPPORTED;
  const int N = n_tokens(p);
  if (N > 0 && (!u || !w_codes || !w_scale || !token_ids || !scores)) return CC_ERR_ARG;
  if (N > 0 && !aligned16(w_codes)) return CC_ERR_ARG;
  if (N > 0 && (reinterpret_cast<uintptr_t>(u) & uintptr_t(4 * esize(p->dtype) - 1)) != 0)
    return CC_ERR_ARG;
  const Fp8Layout L = fp8_layout(p);
  CC_TRY(check_ws(ws, ws_bytes, L.total));
  if (N == 0) return CC_OK;
  LmHeadFp8Launch a;
  a.dtype = p->dtype;
  a.u = u;
  a.wq = w_codes;
  a.sw = w_scale;
  a.ids = token_ids;
  a.scores = scores;
  a.lse = lse;
  a.uq = reinterpret_cast<uint8_t*>(at(ws, L.uq));
  a.su = reinterpret_cast<float*>(at(ws, L.su));
  a.amax_ws = reinterpret_cast<float*>(at(ws, L.amax));
  a.partial = reinterpret_cast<float2*>(at(ws, L.partial));
  a.target = reinterpret_cast<float*>(at(ws, L.target));
  a.cu_d = p->cu_seqlens_d;
  a.n_seqs = p->n_seqs;
  a.N = N;
  a.D = p->hidden;
  a.V = p->vocab;
  a.n_frozen = p->n_frozen;
  CC_HIP(launch_lmhead_fp8(a, static_cast<hipStream_t>(stream)));
  return CC_OK;
}

// ------------------------------------------------------------------ selection

cc_status cc_select_workspace(int32_t n_segs, size_t* bytes) {
  if (!bytes || n_segs < 0) return CC_ERR_ARG;
  *bytes = align_up(size_t(n_segs) * sizeof(SelSeg));
  return CC_OK;
}

cc_status cc_select_keep(const float* scores, int32_t n_segs, const int64_t* seg_start_h,
                         const int32_t* seg_len_h, const int32_t* k_h, int32_t* keep_idx,
                         void* ws, size_t ws_bytes, void* stream) {
  if (n_segs < 0) return CC_ERR_ARG;
  if (n_segs == 0) return CC_OK;
  if (!seg_start_h || !seg_len_h || !k_h) return CC_ERR_ARG;
  std::vector<SelSeg> segs(n_segs);
  int64_t out = 0;
  int mx = 0;
  bool any_len = false;
  for (int i = 0; i < n_segs; ++i) {
    if (seg_len_h[i] < 0 || seg_start_h[i] < 0) return CC_ERR_SHAPE;
    if (k_h[i] < 0 || k_h[i] > seg_len_h[i]) return CC_ERR_SHAPE;
    segs[i].start = seg_start_h[i];
    segs[i].len = seg_len_h[i];
    segs[i].k = k_h[i];
    segs[i].out = out;
    out += k_h[i];
    mx = std::max(mx, seg_len_h[i]);
    any_len = any_len || (k_h[i] > 0);
  }
  if (any_len && (!scores || !keep_idx)) return CC_ERR_ARG;
  CC_TRY(check_ws(ws, ws_bytes, align_up(size_t(n_segs) * sizeof(SelSeg))));
  hipStream_t s = static_cast<hipStream_t>(stream);
  // a few descriptors travel in the kernel arguments, regular layouts as a formula; others
  // are copied into the workspace
  if (n_segs > SEL_INLINE && !select_regular(segs.data(), n_segs))
    CC_HIP(hipMemcpyAsync(ws, segs.data(), segs.size() * sizeof(SelSeg), hipMemcpyHostToDevice, s));
  CC_HIP(launch_select(scores, segs.data(), static_cast<const SelSeg*>(ws), n_segs, mx, keep_idx, s));
  return CC_OK;
}

// ------------------------------------------------------------------ compaction

namespace {
// Room for the keep lists, which are uploaded when they do not fit the kernel arguments.
size_t compact_ws_bytes(size_t n_lists) { return align_up(n_lists * sizeof(CompactList)); }

// The lists of a compaction in the order the kernels want: sequences by falling budget (of
// the longest list of each), heads in order.  per: lists a sequence; take: lists kept of them
// (per, or 1: the first).  Checks the budgets; off: kept entries in all.
cc_status compact_lists(const cc_problem* p, const int32_t* k_h, int per, int take, bool flat,
                        std::vector<CompactList>& lists, int& max_k, int64_t& off) {
  const int B = p->n_seqs;
  std::vector<CompactList> raw(size_t(B) * take);
  std::vector<int> most(B, 0), order(B);
  off = 0;
  max_k = 0;
  for (int b = 0; b < B; ++b) {
    const int n = p->cu_seqlens_h[b + 1] - p->cu_seqlens_h[b];
    order[b] = b;
    for (int h = 0; h < per; ++h) {
      const int k = k_h[int64_t(b) * per + h];
      if (k < 0 || k > n) return CC_ERR_SHAPE;
      if (h < take) {
        raw[size_t(b) * take + h] = CompactList{off, flat ? p->cu_seqlens_h[b] : 0, k, b};
        most[b] = std::max(most[b], k);
      }
      off += k;
    }
    max_k = std::max(max_k, most[b]);
  }
  std::stable_sort(order.begin(), order.end(), [&](int x, int y) { return most[x] > most[y]; });
  lists.resize(raw.size());
  for (int i = 0; i < B; ++i)
    std::copy_n(raw.begin() + size_t(order[i]) * take, take, lists.begin() + size_t(i) * take);
  return CC_OK;
}

// The lists by value with the launch, or uploaded into the workspace.
cc_status compact_run(CompactLaunch& c, const std::vector<CompactList>& lists, void* ws, hipStream_t s) {
  c.lists_h = lists.data();
  c.lists_d = nullptr;
  if (lists.size() > size_t(COMPACT_INLINE)) {
    CC_HIP(hipMemcpyAsync(ws, lists.data(), lists.size() * sizeof(CompactList), hipMemcpyHostToDevice, s));
    c.lists_d = static_cast<const CompactList*>(ws);
  }
  CC_HIP(launch_compact(c, s));
  return CC_OK;
}
}  // namespace

cc_status cc_compact_workspace(const cc_problem* p, int32_t cache_layers, int32_t per_head,
                               size_t* bytes) {
  if (!bytes) return CC_ERR_ARG;
  CC_TRY(check_problem(p));
  if (per_head != 0 && per_head != 1) return CC_ERR_ARG;
  if (cache_layers < 1) return CC_ERR_ARG;
  *bytes = compact_ws_bytes(size_t(p->n_seqs) * (per_head ? p->n_heads_kv : 1));
  return CC_OK;
}

cc_status cc_compact_kv(const cc_problem* p, const cc_kv* kv, const int32_t* keep_idx,
                        const int32_t* k_h, int32_t per_head, int32_t* token_ids,
                        int32_t* pos_ids, const cc_kv* out, void* ws, size_t ws_bytes,
                        void* stream) {
  CC_TRY(check_problem(p));
  CC_TRY(check_kv(p, kv, 1));
  if (per_head != 0 && per_head != 1) return CC_ERR_ARG;
  if (!k_h) return CC_ERR_ARG;
  if (out) {
    CC_TRY(check_kv(p, out, kv->n_layers));
    if (out->layout != kv->layout) return CC_ERR_ARG;
  }
  const int es = esize(p->dtype);
  const int row_bytes = p->head_dim * es;
  if (row_bytes % 16 != 0 || !is_pow2(row_bytes / 16) || row_bytes / 16 > 256)
    return CC_ERR_UNSUPPORTED;
  const int hkv = p->n_heads_kv, per = per_head ? hkv : 1;
  std::vector<CompactList> lists;
  int max_k = 0;
  int64_t off = 0;
  CC_TRY(compact_lists(p, k_h, per, per, false, lists, max_k, off));
  if (off > 0 && !keep_idx) return CC_ERR_ARG;
  CC_TRY(check_ws(ws, ws_bytes, compact_ws_bytes(lists.size())));
  hipStream_t s = static_cast<hipStream_t>(stream);
  CompactLaunch c;
  c.n_tensors = 2;
  const cc_kv* dst = out ? out : kv;
  c.src[0] = make_view(kv, kv->k, es);
  c.src[1] = make_view(kv, kv->v, es);
  c.dst[0] = make_view(dst, dst->k, es);
  c.dst[1] = make_view(dst, dst->v, es);
  c.paged = kv->layout == CC_KV_PAGED;
  c.row_bytes = row_bytes;
  c.keep = keep_idx;
  c.n_seqs = p->n_seqs;
  c.n_layers = kv->n_layers;
  c.n_heads = hkv;
  c.per_head = per_head;
  c.max_k = max_k;
  c.in_place = out == nullptr;
  c.ids[0] = token_ids;
  c.ids[1] = pos_ids;
  c.cu_d = p->cu_seqlens_d;
  return compact_run(c, lists, ws, s);
}

// Token-major per-entry rows (e.g. the stored activations H) follow the keep lists of
// the cache.  The rows are cut into column slabs of up to 256 bytes; each (sequence, slab)
// is one plane of the compaction kernels, addressed through a flat view whose planes
// start at the sequence's first row.
namespace {
int rows_slab_bytes(int row_bytes) {
  int slab = 256;
  while (slab > 16 && row_bytes % slab != 0) slab >>= 1;
  return slab;
}
}  // namespace

cc_status cc_compact_rows_workspace(const cc_problem* p, int32_t row_bytes, int32_t per_head,
                                    size_t* bytes) {
  if (!bytes) return CC_ERR_ARG;
  CC_TRY(check_problem(p));
  if (per_head != 0 && per_head != 1) return CC_ERR_ARG;
  if (row_bytes < 16 || row_bytes % 16 != 0) return CC_ERR_UNSUPPORTED;
  *bytes = compact_ws_bytes(p->n_seqs);
  return CC_OK;
}

cc_status cc_compact_rows(const cc_problem* p, void* rows, int32_t row_bytes,
                          const int32_t* keep_idx, const int32_t* k_h, int32_t per_head,
                          void* out_rows, void* ws, size_t ws_bytes, void* stream) {
  CC_TRY(check_problem(p));
  if (per_head != 0 && per_head != 1) return CC_ERR_ARG;
  if (row_bytes < 16 || row_bytes % 16 != 0) return CC_ERR_UNSUPPORTED;
  if (!k_h) return CC_ERR_ARG;
  const int hkv = p->n_heads_kv;
  const int slab = rows_slab_bytes(row_bytes), n_slabs = row_bytes / slab;
  std::vector<CompactList> lists;
  int max_k = 0;
  int64_t off = 0;
  CC_TRY(compact_lists(p, k_h, per_head ? hkv : 1, 1, true, lists, max_k, off));
  if (off > 0 && (!keep_idx || !rows)) return CC_ERR_ARG;
  if ((rows && !aligned16(rows)) || (out_rows && !aligned16(out_rows))) return CC_ERR_ARG;
  CC_TRY(check_ws(ws, ws_bytes, compact_ws_bytes(lists.size())));
  if (max_k == 0) return CC_OK;
  hipStream_t s = static_cast<hipStream_t>(stream);
  auto view = [&](void* base) {
    KvView v{};
    v.base = base;
    v.head_stride = slab;      // bytes: column slab h
    v.tok_stride = row_bytes;  // bytes: one entry
    return v;
  };
  CompactLaunch c;
  c.n_tensors = 1;
  c.src[0] = c.src[1] = view(rows);
  c.dst[0] = c.dst[1] = view(out_rows ? out_rows : rows);
  c.paged = false;
  c.row_bytes = slab;
  c.keep = keep_idx;
  c.n_seqs = p->n_seqs;
  c.n_layers = 1;
  c.n_heads = n_slabs;   // a column slab is a "head" of the flat view
  c.per_head = 0;
  c.max_k = max_k;
  c.in_place = out_rows == nullptr;
  c.ids[0] = c.ids[1] = nullptr;
  c.cu_d = p->cu_seqlens_d;
  return compact_run(c, lists, ws, s);
}

}  // extern "C"

// ------------------------------------------------------------------ cache in 8 bits

namespace {

cc_status check_kv8(const cc_problem* p, const cc_kv8* kv, int min_layers, int longest) {
  if (!kv) return CC_ERR_ARG;
  CC_TRY(check_kv(p, &kv->codes, min_layers, 1, longest));
  if (!kv->k_scale || !kv->v_scale) return CC_ERR_ARG;
  if (!is_pow2(kv->scale_block) || kv->scale_block < 16 || kv->scale_block > 128) return CC_ERR_UNSUPPORTED;
  if (kv->scale_layer_stride < 0 || kv->scale_head_stride < 0) return CC_ERR_SHAPE;
  if (kv->codes.layout == CC_KV_PAGED) {
    if (kv->scale_page_stride < 0 || kv->scale_block > kv->codes.page_size) return CC_ERR_SHAPE;
  } else if (kv->scale_seq_stride < 0) {
    return CC_ERR_SHAPE;
  }
  return CC_OK;
}

Kv8View make_view8(const cc_kv8* kv, const void* base, uint8_t* scale) {
  Kv8View v;
  v.codes = make_view(&kv->codes, base, 1);
  v.scale = scale;
  v.s_seq = kv->scale_seq_stride;
  v.s_layer = kv->scale_layer_stride;
  v.s_head = kv->scale_head_stride;
  v.s_page = kv->scale_page_stride;
  v.block_shift = 0;
  while ((1 << v.block_shift) < kv->scale_block) ++v.block_shift;
  v.paged = kv->codes.layout == CC_KV_PAGED;
  return v;
}

cc_status check_rows(const cc_problem* p, const cc_rows& r) {
  const int es = esize(p->dtype);
  if (!r.base || !aligned16(r.base)) return CC_ERR_ARG;
  if (r.layer_stride < 0 || r.tok_stride < 0 || r.head_stride < 0) return CC_ERR_SHAPE;
  if (r.layer_stride * es % 16 || r.tok_stride * es % 16 || r.head_stride * es % 16) return CC_ERR_UNSUPPORTED;
  return CC_OK;
}

// The checks of both appends but the cache's own, and the launch's sizes.
cc_status plan_append(const cc_problem* p, const cc_append* a, const cc_kv* kv, AppendLaunch& l) {
  if (a->n_layers < 1 || a->layer < 0 || a->layer > kv->n_layers - a->n_layers) return CC_ERR_SHAPE;
  if (a->rotate != 0 && a->rotate != 1) return CC_ERR_ARG;
  if (a->rotate && !(p->rope_theta > 0.f && std::isfinite(p->rope_theta))) return CC_ERR_ARG;
  if (a->capacity < 0) return CC_ERR_SHAPE;
  const int64_t room = kv->layout == CC_KV_PAGED ? int64_t(kv->max_pages) * kv->page_size : INT32_MAX;
  if (a->capacity == 0 && kv->layout != CC_KV_PAGED) return CC_ERR_ARG;
  l.capacity = int(std::min<int64_t>({a->capacity ? a->capacity : room, room, INT32_MAX - 128}));
  // one layer's workgroups: units of 16 tokens or more in ranges of up to 64 heads, of four tokens for queries
  const int64_t M = n_tokens(p), ranges = (p->n_heads_kv + 63) / 64;
  if (2 * (M / 16 + 2 * int64_t(p->n_seqs)) * ranges + M / 4 + 640 > MOST_GROUPS) return CC_ERR_UNSUPPORTED;
  if (M > 0) {
    CC_TRY(check_rows(p, a->k));
    CC_TRY(check_rows(p, a->v));
    if (!a->cached) return CC_ERR_ARG;
    if (a->q.base) {
      if (a->n_layers != 1) return CC_ERR_UNSUPPORTED;
      CC_TRY(check_rows(p, a->q));
      if (!a->q_out || !aligned16(a->q_out)) return CC_ERR_ARG;
    }
  }
  l.dtype = p->dtype;
  l.k = a->k;
  l.v = a->v;
  l.q = a->q;
  l.q_out = a->q_out;
  l.cached = a->cached;
  l.pos = a->pos_ids;
  l.cu_d = p->cu_seqlens_d;
  l.cu_h = p->cu_seqlens_h;
  l.n_seqs = p->n_seqs;
  l.layer = a->layer;
  l.n_layers = a->n_layers;
  l.n_heads_q = p->n_heads_q;
  l.n_heads_kv = p->n_heads_kv;
  l.head_dim = p->head_dim;
  l.rotate = a->rotate;
  l.theta = p->rope_theta;
  return CC_OK;
}

}  // namespace

extern "C" {

cc_status cc_append_kv(const cc_problem* p, const cc_append* a, const cc_kv* kv, void* stream) {
  CC_TRY(check_problem(p));
  if (!a) return CC_ERR_ARG;
  CC_TRY(check_kv(p, kv, 1));
  AppendLaunch l;
  CC_TRY(plan_append(p, a, kv, l));
  const int es = esize(p->dtype);
  l.f8 = false;
  l.kc = Kv8View{};
  l.kc.codes = make_view(kv, kv->k, es);
  l.kc.paged = kv->layout == CC_KV_PAGED;
  l.vc = l.kc;
  l.vc.codes = make_view(kv, kv->v, es);
  CC_HIP(launch_append(l, static_cast<hipStream_t>(stream)));
  return CC_OK;
}

cc_status cc_append_kv8(const cc_problem* p, const cc_append* a, const cc_kv8* kv, void* stream) {
  CC_TRY(check_problem(p));
  if (!a) return CC_ERR_ARG;
  CC_TRY(check_kv8(p, kv, 1, -1));
  AppendLaunch l;
  CC_TRY(plan_append(p, a, &kv->codes, l));
  l.f8 = true;
  l.kc = make_view8(kv, kv->codes.k, kv->k_scale);
  l.vc = make_view8(kv, kv->codes.v, kv->v_scale);
  CC_HIP(launch_append(l, static_cast<hipStream_t>(stream)));
  return CC_OK;
}

cc_status cc_compact_kv8(const cc_problem* p, const cc_kv8* kv, const int32_t* keep_idx,
                         const int32_t* k_h, int32_t per_head, int32_t* token_ids,
                         int32_t* pos_ids, const cc_kv8* out, void* stream) {
  CC_TRY(check_problem(p));
  CC_TRY(check_kv8(p, kv, 1, -1));
  if (per_head != 0 && per_head != 1) return CC_ERR_ARG;
  if (!k_h) return CC_ERR_ARG;
  if (out) {
    CC_TRY(check_kv8(p, out, kv->codes.n_layers, -1));
    if (out->codes.layout != kv->codes.layout || out->scale_block != kv->scale_block) return CC_ERR_ARG;
  }
  const int hkv = p->n_heads_kv, per = per_head ? hkv : 1;
  if (per > COMPACT_INLINE) return CC_ERR_UNSUPPORTED;   // the lists of a sequence travel with one launch
  if (int64_t(hkv) * kv->codes.n_layers >= 1 << 20) return CC_ERR_UNSUPPORTED;   // as do its planes
  int64_t off = 0;
  for (int64_t i = 0; i < int64_t(p->n_seqs) * per; ++i) {
    const int b = int(i / per);
    if (k_h[i] < 0 || k_h[i] > p->cu_seqlens_h[b + 1] - p->cu_seqlens_h[b]) return CC_ERR_SHAPE;
    off += k_h[i];
  }
  if (off == 0) return CC_OK;
  if (!keep_idx) return CC_ERR_ARG;
  const cc_kv8* dst = out ? out : kv;
  Compact8Launch c;
  c.src[0] = make_view8(kv, kv->codes.k, kv->k_scale);
  c.src[1] = make_view8(kv, kv->codes.v, kv->v_scale);
  c.dst[0] = make_view8(dst, dst->codes.k, dst->k_scale);
  c.dst[1] = make_view8(dst, dst->codes.v, dst->v_scale);
  c.keep = keep_idx;
  c.k_h = k_h;
  c.n_seqs = p->n_seqs;
  c.n_layers = kv->codes.n_layers;
  c.n_heads = hkv;
  c.per_head = per_head;
  c.head_dim = p->head_dim;
  c.in_place = out == nullptr;
  c.ids[0] = token_ids;
  c.ids[1] = pos_ids;
  c.cu_d = p->cu_seqlens_d;
  CC_HIP(launch_compact8(c, static_cast<hipStream_t>(stream)));
  return CC_OK;
}

}  // extern "C"

namespace {

// One class of sequences of a call, few or many rows: which they are, and how their entries are cut.
// Sizes only, so that the workspace query and the call agree.
struct Kv8Class {
  int n = 0;               // sequences of the class
  int n_list = 0, listed = 0;
  int32_t list[KV8_LIST], first[KV8_LIST];   // first: rows of the class before the sequence's
  int64_t all = 0;         // rows walked
  int R = 0, piece = 0, splits = 1, direct = 0, parts = 0;
  size_t part = 0, total = 0;   // workspace: (maximum, sum) pairs behind the outputs
};

constexpr int kCus = 256;

Kv8Class kv8_class(const cc_problem* p, int max_len, bool few) {
  Kv8Class c;
  const int g = p->n_heads_q / p->n_heads_kv;
  int64_t blocks = 0;
  for (int b = 0; b < p->n_seqs; ++b) {
    const int64_t rows = int64_t(p->cu_seqlens_h[b + 1] - p->cu_seqlens_h[b]) * g;
    if (rows == 0 || (rows <= FEW_ROWS) != few) continue;
    if (c.n < KV8_LIST) {
      c.list[c.n] = b;
      c.first[c.n] = int32_t(c.all);
    }
    ++c.n;
    c.all += rows;
    c.R = int(std::max<int64_t>(c.R, rows));
    blocks += few ? 1 : (rows + MANY_ROWS - 1) / MANY_ROWS;
  }
  if (c.n == 0) return c;
  c.listed = c.n <= KV8_LIST;
  c.n_list = c.listed ? c.n : p->n_seqs;
  if (!c.listed) c.all = int64_t(n_tokens(p)) * g;
  const int64_t items = blocks * p->n_heads_kv;   // workgroups without a cut
  size_t rows = 0;                                // partial results
  if (few) {
    // Short caches: a workgroup for each (sequence, head), nothing to join.  Else the work is shared out
    // among two workgroups a CU, all that fit at a time (eight a CU where there are as many (sequence,
    // head)s: 1023 sequences of 200 to 4000 entries 683 us, with two 652; 600 of 50 to 9000 503 and 466).
    c.direct = max_len <= kv8_direct(items);
    c.parts = 2 * kCus;
    if (!c.direct) rows = (size_t(c.parts) + size_t(c.n_list) * p->n_heads_kv) * c.R;
  } else {
    // As many pieces as leave no more than two workgroups a CU, what is resident (512 queries of 32 heads on 8
    // at 8000 entries 110 us, half as many pieces 142, twice 125; rounded up, 600 queries at 30000 500 us for
    // 365 and 24 sequences of 64 at 3000 157 for 130, 18 ragged ones 90 for 100), of 256 entries at the least
    // (128 queries of 8 heads on one at 4000 21 us, of 512 27, of 128 24).
    // And no more than leave a launch a row block (MOST_GROUPS).
    const int64_t want = std::max<int64_t>(1, std::min<int64_t>({2 * kCus / items, (int64_t(max_len) + 255) / 256,
                                                                 MOST_GROUPS / (int64_t(c.n_list) * p->n_heads_kv)}));
    c.piece = int(((int64_t(max_len) + want - 1) / want + MANY_KEYS - 1) / MANY_KEYS * MANY_KEYS);
    c.piece = std::max(c.piece, MANY_KEYS);
    c.splits = std::max(1, int((int64_t(max_len) + c.piece - 1) / c.piece));
    if (c.splits > 1) rows = size_t(c.splits) * p->n_heads_kv * c.all;
  }
  if (rows) {
    c.part = align_up(rows * p->head_dim * sizeof(float));
    c.total = c.part + align_up(rows * sizeof(float2));
  }
  return c;
}

// Both classes of a call, few rows first.
cc_status kv8_plan(const cc_problem* p, int max_len, Kv8Class (&c)[2]) {
  for (int i = 0; i < 2; ++i) {
    c[i] = kv8_class(p, max_len, i == 0);
    // what every launch of a class has a workgroup for
    if (int64_t(c[i].n_list) * p->n_heads_kv * c[i].splits > MOST_GROUPS) return CC_ERR_UNSUPPORTED;
  }
  return CC_OK;
}

cc_status check_attention8(const cc_problem* p, int32_t mask, int32_t max_len) {
  CC_TRY(check_problem(p));
  if (mask != CC_MASK_CAUSAL && mask != CC_MASK_COUNTER_CAUSAL) return CC_ERR_ARG;
  if (max_len < 0 || max_len > INT32_MAX - 4096) return CC_ERR_SHAPE;
  if (p->dtype != CC_BF16) return CC_ERR_UNSUPPORTED;
  if (int64_t(n_tokens(p)) * (p->n_heads_q / p->n_heads_kv) > INT32_MAX) return CC_ERR_UNSUPPORTED;
  return CC_OK;
}

}  // namespace

extern "C" {

cc_status cc_attention_kv8_workspace(const cc_problem* p, int32_t mask, int32_t max_kv_len, size_t* bytes) {
  if (!bytes) return CC_ERR_ARG;
  CC_TRY(check_attention8(p, mask, max_kv_len));
  Kv8Class classes[2];
  CC_TRY(kv8_plan(p, max_kv_len, classes));
  *bytes = classes[0].total + classes[1].total;
  return CC_OK;
}

cc_status cc_attention_kv8(const cc_problem* p, const void* q, const cc_kv8* kv, int32_t layer, int32_t mask,
                           const int32_t* kv_lens, int32_t max_kv_len, void* o, void* ws, size_t ws_bytes,
                           void* stream) {
  CC_TRY(check_attention8(p, mask, max_kv_len));
  CC_TRY(check_kv8(p, kv, 1, max_kv_len));
  if (layer < 0 || layer >= kv->codes.n_layers) return CC_ERR_ARG;
  if (kv->codes.tok_stride >= int64_t(1) << 28) return CC_ERR_UNSUPPORTED;   // 16 entries by 32-bit offsets
  const int N = n_tokens(p);
  if (N > 0 && (!q || !o || !kv_lens || !aligned16(q) || !aligned16(o))) return CC_ERR_ARG;
  Kv8Class classes[2];
  CC_TRY(kv8_plan(p, max_kv_len, classes));
  CC_TRY(check_ws(ws, ws_bytes, classes[0].total + classes[1].total));
  if (N == 0) return CC_OK;
  size_t off = 0;
  for (int i = 0; i < 2; ++i) {
    const Kv8Class& c = classes[i];
    if (c.n == 0) continue;
    Kv8Args a;
    a.q = static_cast<const u16*>(q);
    a.o = static_cast<u16*>(o);
    a.k = make_view8(kv, kv->codes.k, kv->k_scale);
    a.v = make_view8(kv, kv->codes.v, kv->v_scale);
    a.cu = p->cu_seqlens_d;
    a.lens = kv_lens;
    a.layer = layer;
    a.mask = mask;
    a.inclusive = p->diag == CC_DIAG_INCLUSIVE;
    a.max_len = max_kv_len;
    a.hq = p->n_heads_q;
    a.hkv = p->n_heads_kv;
    a.g = p->n_heads_q / p->n_heads_kv;
    a.head_dim = p->head_dim;
    a.c2 = softmax_scale(p) * kLog2e;
    a.room = std::min(8.f / a.c2, FLT_MAX);   // (finite: a first logit passes -inf by more)
    a.R = c.R;
    a.piece = c.piece;
    a.splits = c.splits;
    a.nth0 = 0;
    a.direct = c.direct;
    a.parts = c.parts;
    a.part = c.total ? reinterpret_cast<float*>(at(ws, off)) : nullptr;
    a.part_ml = c.total ? reinterpret_cast<float2*>(at(ws, off + c.part)) : nullptr;
    a.n_list = c.n_list;
    a.listed = c.listed;
    std::copy_n(c.list, c.listed ? c.n : 0, a.list);
    a.all = int32_t(c.all);
    std::copy_n(c.first, c.listed ? c.n : 0, a.first);
    CC_HIP(launch_attention_kv8(a, i == 0, static_cast<hipStream_t>(stream)));
    off += c.total;
  }
  return CC_OK;
}

}  // extern "C"

// ------------------------------------------------------------------ attention over a bf16 cache

namespace {

cc_status check_attention_kv(const cc_problem* p, int32_t max_len) {
  CC_TRY(check_problem(p));
  if (max_len < 0 || max_len > INT32_MAX - 4096) return CC_ERR_SHAPE;
  if (p->dtype != CC_BF16) return CC_ERR_UNSUPPORTED;
  if (int64_t(n_tokens(p)) * (p->n_heads_q / p->n_heads_kv) > INT32_MAX - 4096) return CC_ERR_UNSUPPORTED;
  // what a launch has workgroups for, at the least
  if (int64_t(p->n_seqs) * p->n_heads_kv > MOST_GROUPS / 2) return CC_ERR_UNSUPPORTED;
  return CC_OK;
}

cc_status check_view16(const cc_problem* p, const cc_kv* kv, int32_t layer, int32_t max_len) {
  CC_TRY(check_kv(p, kv, 1, 0, max_len));
  if (layer < 0 || layer >= kv->n_layers) return CC_ERR_ARG;
  if (kv->tok_stride >= int64_t(1) << 27) return CC_ERR_UNSUPPORTED;   // 16 entries by 32-bit offsets
  return CC_OK;
}

cc_status check_prefix(const cc_problem* p, const cc_prefix* x) {
  if (!x || x->n_prefixes < 1 || !x->first_seq_h) return CC_ERR_ARG;
  if (x->max_len < 0 || x->max_len > INT32_MAX - 4096) return CC_ERR_SHAPE;
  if (x->first_seq_h[0] != 0 || x->first_seq_h[x->n_prefixes] != p->n_seqs) return CC_ERR_SHAPE;
  for (int i = 0; i < x->n_prefixes; ++i)
    if (x->first_seq_h[i + 1] < x->first_seq_h[i]) return CC_ERR_SHAPE;
  if (int64_t(x->n_prefixes) * p->n_heads_kv > MOST_GROUPS / 2) return CC_ERR_UNSUPPORTED;
  return CC_OK;
}

// Row blocks of the kernel for many and how their entries are cut.
struct KvMany {
  AttnMany items;              // up to ATTN_INLINE sequences; else all are walked
  int n = 0;
  int64_t blocks = 0;
  int piece = KV_KEYS, splits = 1;
  int64_t rows = 0;            // of a KV head
  int row0 = 0, places = 0, skip = 0;   // which of the call's rows have a place among the results to be joined
  size_t part = 0, total = 0;  // workspace: (maximum, sum) pairs behind the outputs
  void add(int seq, int seq0, int m, int g) {
    if (n == 0) row0 = seq0 * g;
    places = (seq0 + m) * g - row0;
    rows += int64_t(m) * g;
    const int nb = int((int64_t(m) * g + KV_ROWS - 1) / KV_ROWS);
    if (n < ATTN_INLINE) items.seqs[n] = AttnSeq{seq, seq0, m, nb};
    ++n;
    blocks += nb;
  }
  // walked: sequences there are
  cc_status cut(const cc_problem* p, int walked, int max_len) {
    items.nkv = p->n_heads_kv;
    items.n_seqs = n <= ATTN_INLINE ? n : 0;
    std::stable_sort(items.seqs, items.seqs + items.n_seqs, [](const AttnSeq& x, const AttnSeq& y) { return x.n > y.n; });
    if (n == 0) return CC_OK;
    const int64_t each = blocks * p->n_heads_kv;
    if (!items.n_seqs) blocks = int64_t(n_tokens(p)) * (p->n_heads_q / p->n_heads_kv) / KV_ROWS + walked;
    if (blocks * p->n_heads_kv > MOST_GROUPS) return CC_ERR_UNSUPPORTED;
    // As many pieces as leave no more than two workgroups a CU, what is resident, of 256 entries at the least; but only
    // where they take some 12 tiles off a workgroup's chain, what the join costs.
    int64_t want = std::max<int64_t>(1, std::min<int64_t>({2 * kCus / each, (int64_t(max_len) + 255) / 256,
                                                           MOST_GROUPS / (blocks * p->n_heads_kv)}));
    if ((int64_t(max_len) - max_len / want) / KV_KEYS <= 12) want = 1;
    piece = std::max(KV_KEYS, int(((int64_t(max_len) + want - 1) / want + KV_KEYS - 1) / KV_KEYS * KV_KEYS));
    splits = std::max(1, int((int64_t(max_len) + piece - 1) / piece));
    if (splits > 1) {
      // From the first row to the last; where more of these than not are of sequences of few, those are left out: to find a
      // row takes some 2 us more then (128 tokens between two chunks of 16 behind 16000 entries, 32 heads on 8, 107.2 us and
      // 104.8, but 17 MB in place of 85).
      skip = places > 2 * rows;
      if (skip) {
        row0 = 0;
        places = int(rows);
      }
      const size_t out = size_t(splits) * p->n_heads_kv * places;
      part = align_up(out * p->head_dim * sizeof(float));
      total = part + align_up(out * sizeof(float2));
    }
    return CC_OK;
  }
};

// How a call's sequences are taken.  Sizes only, so that the workspace query and the call agree.
struct KvPlan {
  bool rows = false;           // all by 16 rows a workgroup
  bool inside = false;         // which takes the prefix's entries too
  bool along = false;          // few rows: with the others
  int ends = 0;                // those that are
  int n_few = 0, n_list = 0, listed = 0, R = 0, parts = 0;
  bool direct = false;         // few rows: by 16 rows a workgroup
  int32_t list[KV_LIST];
  int few_rows = 0, few_per = 1;   // of a KV head, and where groups of few_per sequences begin among them
  int32_t few_at[KV_LIST];
  int rpiece = 0, rsplits = 1; // behind prefixes: entries of a piece of those (0: whole)
  size_t fpart = 0, fat = 0, ftotal = 0;
  KvMany many;
  int64_t pre_blocks = 0;      // row blocks of the pass over the prefixes (0: none)
  size_t pre_at = 0, ppart = 0, ptotal = 0;   // its workspace: where its pieces are, outputs, (maximum, sum) pairs
  size_t total() const { return ptotal + ftotal + many.total; }
};

// Prompts, chunks and sequences behind a prefix: up to that many entries, and that many workgroups of 16 rows, each has its
// own, with nothing to join and no tiles of 128 rows to fill.  That against those: a prompt of 300 tokens, 32 heads on 8 (600
// workgroups), 11.4 us and 12.5, of 400 15.9 and 14.1; 64 tokens at the end of 964 13.3 and 23.9; one of 1000, 4 heads, 9.6 and
// 18.2; eight sequences of one token behind 900 entries 13.0 and 13.9.
constexpr int KV_SHORT = 1024;
constexpr int KV_SHORT_GROUPS = 640;
constexpr int KV_OWN = 512;
// Workgroups that the pass over the prefixes is cut into: two a CU.
constexpr int KV_SLOTS = 2 * kCus;

cc_status kv_plan(const cc_problem* p, const cc_prefix* x, int max_len, KvPlan& c) {
  const int g = p->n_heads_q / p->n_heads_kv, hkv = p->n_heads_kv;
  const int longest = int(std::min<int64_t>(INT32_MAX, int64_t(max_len) + (x ? x->max_len : 0)));
  int64_t blocks16 = 0;
  int64_t few = 0, many = 0;   // sequences of few rows, blocks of the others
  for (int b = 0; b < p->n_seqs; ++b) {
    const int64_t rows = int64_t(p->cu_seqlens_h[b + 1] - p->cu_seqlens_h[b]) * g;
    blocks16 += (rows + 15) / 16;
    if (rows > FEW_ROWS)
      many += (rows + KV_ROWS - 1) / KV_ROWS;
    else
      few += rows > 0;
  }
  c.rows = (many || x) && longest <= KV_SHORT && blocks16 * hkv <= KV_SHORT_GROUPS;
  // Sequences of few rows beside prompts no shorter than any cache go along as blocks of 128 rows, before the others, in
  // place of launches of their own ahead of them: a prompt of 4001, 28 heads on 4, with eight tokens behind 4000 entries each
  // 135 us and 152, with 40 181 and 204; of 1100, 32 heads on 8, with two behind 1099 30.4 and 43.9, with 200 206 and 214; but
  // with 500 short ones 84 and 77.
  c.along = !x && !c.rows && few <= 8 * many && max_len <= ::max_len(p);
  c.ends = int(few * hkv);
  c.inside = x && c.rows;
  c.few_per = (p->n_seqs + KV_LIST - 1) / KV_LIST;
  for (int b = 0; b < p->n_seqs; ++b) {
    if (b % c.few_per == 0) c.few_at[b / c.few_per] = c.few_rows;
    const int seq0 = p->cu_seqlens_h[b], m = p->cu_seqlens_h[b + 1] - seq0;
    const int64_t rows = int64_t(m) * g;
    if (rows == 0) continue;
    if ((rows <= FEW_ROWS && !c.along) || c.rows) {
      if (c.n_few < KV_LIST) c.list[c.n_few] = b;
      ++c.n_few;
      c.few_rows += int(rows);
      c.R = int(std::max<int64_t>(c.R, rows));
    } else {
      c.many.add(b, seq0, m, g);
    }
  }
  std::fill(c.few_at + (p->n_seqs + c.few_per - 1) / c.few_per, c.few_at + KV_LIST, c.few_rows);
  const int64_t walked = int64_t(n_tokens(p)) * g / 16 + p->n_seqs;
  c.direct = c.rows || max_len <= kv_direct(int64_t(c.n_few) * hkv);
  // (listed sequences have the blocks of the longest)
  c.listed = c.n_few <= KV_LIST && (!c.direct || int64_t(c.n_few) * ((c.R + 15) / 16) <= walked);
  c.n_list = c.listed ? c.n_few : p->n_seqs;
  c.parts = 2 * kCus;
  // Behind prefixes results are joined anyhow, and a CU takes some 60 GB/s: pieces of what it takes in a few us.
  if (x && !c.inside && c.n_few) {
    c.direct = true;
    c.rpiece = std::max(KV_OWN, int((int64_t(max_len) + 32 * 16 - 1) / (32 * 16) * 16));
    c.rsplits = std::max(1, int((int64_t(max_len) + c.rpiece - 1) / c.rpiece));
    const size_t rows = size_t(c.rsplits) * c.few_rows * hkv;
    c.fpart = align_up(rows * p->head_dim * sizeof(float));
    c.ftotal = c.fpart + align_up(rows * sizeof(float2));
  } else if (c.n_few && !c.direct) {
    const size_t rows = (size_t(c.parts) + size_t(c.n_list) * hkv) * c.R;
    c.fpart = align_up(rows * p->head_dim * sizeof(float));
    c.fat = c.fpart + align_up(rows * sizeof(float2));
    c.ftotal = c.fat + align_up(size_t(c.n_list) * hkv * sizeof(int2));
  }
  CC_TRY(c.many.cut(p, p->n_seqs, max_len));
  if (x && !c.inside) {
    for (int i = 0; i < x->n_prefixes; ++i) {
      const int64_t m = p->cu_seqlens_h[x->first_seq_h[i + 1]] - p->cu_seqlens_h[x->first_seq_h[i]];
      c.pre_blocks += (m * g + KV_ROWS - 1) / KV_ROWS;
    }
    const int64_t groups = std::max<int64_t>(KV_SLOTS, c.pre_blocks * hkv);
    if (groups > MOST_GROUPS / 2) return CC_ERR_UNSUPPORTED;
    c.pre_at = align_up(size_t(x->n_prefixes) * sizeof(int2));
    c.ppart = c.pre_at + align_up(size_t(groups) * KV_ROWS * p->head_dim * sizeof(float));
    c.ptotal = c.ppart + align_up(size_t(groups) * KV_ROWS * sizeof(float2));
  }
  // (a launch by 16 rows a workgroup of 512)
  const int64_t by16 = (c.listed ? int64_t(c.n_list) * ((c.R + 15) / 16) : walked) * hkv * c.rsplits;
  if (c.n_few && c.direct && by16 > MOST_GROUPS / 2) return CC_ERR_UNSUPPORTED;
  return CC_OK;
}

KvPair make_pair(const cc_kv* kv) { return KvPair{make_view(kv, kv->k, 2), kv->v, kv->layout == CC_KV_PAGED}; }

// Both attentions.
cc_status run_attention_kv(const cc_problem* p, const void* q, const cc_prefix* prefix, const cc_kv* kv, int32_t layer,
                           const int32_t* kv_lens, int32_t max_kv_len, void* o, float* lse, void* ws, size_t ws_bytes,
                           void* stream) {
  CC_TRY(check_view16(p, kv, layer, max_kv_len));
  if (prefix) CC_TRY(check_view16(p, &prefix->kv, layer, prefix->max_len));
  const int N = n_tokens(p);
  if (N > 0 && (!q || !o || !kv_lens || !aligned16(q) || !aligned16(o))) return CC_ERR_ARG;
  if (N > 0 && prefix && (!prefix->first_seq_d || !prefix->lens)) return CC_ERR_ARG;
  KvPlan c;
  CC_TRY(kv_plan(p, prefix, max_kv_len, c));
  CC_TRY(check_ws(ws, ws_bytes, c.total()));
  if (N == 0) return CC_OK;
  KvAttnArgs a{};
  a.q = static_cast<const u16*>(q);
  a.o = static_cast<u16*>(o);
  a.lse = lse;
  a.own = make_pair(kv);
  a.cu = p->cu_seqlens_d;
  a.lens = kv_lens;
  if (prefix) {
    a.pre = make_pair(&prefix->kv);
    a.pre_first = prefix->first_seq_d;
    a.pre_lens = prefix->lens;
    a.n_prefixes = prefix->n_prefixes;
    a.pre_max = prefix->max_len;
  }
  a.n_seqs = p->n_seqs;
  a.layer = layer;
  a.max_len = max_kv_len;
  a.hq = p->n_heads_q;
  a.hkv = p->n_heads_kv;
  a.g = p->n_heads_q / p->n_heads_kv;
  a.head_dim = p->head_dim;
  a.N = N;
  a.scale = softmax_scale(p);
  a.c2 = a.scale * kLog2e;
  a.room = std::min(8.f / a.c2, FLT_MAX);   // (finite: a first logit passes -inf by more)
  hipStream_t st = static_cast<hipStream_t>(stream);
  size_t off = 0;
  auto many = [&](const KvMany& m) {
    a.items = m.items;
    a.blocks = int(m.blocks);
    a.few = c.along ? 0 : FEW_ROWS;
    if (m.skip) std::copy_n(c.few_at, KV_LIST, a.few_at);
    a.row0 = m.row0;
    a.places = m.places;
    a.skip = m.skip;
    a.ends = c.along ? c.ends : 0;
    a.piece = m.piece;
    a.splits = m.splits;
    a.part = m.total ? reinterpret_cast<float*>(at(ws, off)) : nullptr;
    a.part_ml = m.total ? reinterpret_cast<float2*>(at(ws, off + m.part)) : nullptr;
    off += m.total;
    return launch_attn_kv_many(a, st);
  };
  if (c.pre_blocks) {
    a.pre_at = reinterpret_cast<int2*>(at(ws, 0));
    a.ppart = reinterpret_cast<float*>(at(ws, c.pre_at));
    a.ppart_ml = reinterpret_cast<float2*>(at(ws, c.ppart));
    off = c.ptotal;
  }
  if (c.n_few) {
    a.n_list = c.n_list;
    a.listed = c.listed;
    a.R = c.R;
    a.most = c.rows ? INT32_MAX : FEW_ROWS;
    a.parts = c.parts;
    std::copy_n(c.list, c.listed ? c.n_few : 0, a.list);
    a.few_rows = c.few_rows;
    a.few_per = c.few_per;
    a.mixed = c.few_rows != N * a.g;
    a.rpiece = c.rpiece;
    a.rsplits = c.rsplits;
    (c.rpiece ? a.rpart : a.fpart) = c.ftotal ? reinterpret_cast<float*>(at(ws, off)) : nullptr;
    (c.rpiece ? a.rpart_ml : a.fpart_ml) = c.ftotal ? reinterpret_cast<float2*>(at(ws, off + c.fpart)) : nullptr;
    a.fpart_at = c.fat ? reinterpret_cast<int2*>(at(ws, off + c.fat)) : nullptr;
    off += c.ftotal;
  }
  if (c.pre_blocks) {
    KvAttnArgs pass = a;
    pass.own = a.pre;
    pass.lens = a.pre_lens;
    pass.max_len = a.pre_max;
    pass.n_seqs = a.n_prefixes;
    pass.blocks = int(c.pre_blocks);
    pass.slots = KV_SLOTS;
    std::copy_n(c.few_at, KV_LIST, pass.few_at);
    CC_HIP(launch_attn_prefix(pass, a, c.n_few > 0, st));
  } else if (c.n_few) {
    CC_HIP(c.direct ? launch_attn_rows(a, st) : launch_attn_few(a, st));
  }
  if (c.many.n) CC_HIP(many(c.many));
  return CC_OK;
}

// How a call's sequences of many rows are cut.
struct WeightsPlan {
  bool few = false;            // there are sequences of few rows, or without any
  int R = 0;                   // most rows of one
  int n = 0, n_list = 0, listed = 0, chunk = W_ROWS, chunks = 1;
  int32_t list[KV_LIST];
  size_t total = 0;
};

cc_status weights_plan(const cc_problem* p, int max_len, WeightsPlan& c) {
  const int g = p->n_heads_q / p->n_heads_kv, hkv = p->n_heads_kv;
  int64_t most = 0;
  double tiles = 0;            // (tile, block of entries) pairs that meet, in all
  const int64_t blocks = (int64_t(max_len) + W_KEYS - 1) / W_KEYS;
  const bool prompts = ::max_len(p) == max_len;   // as far as the host can tell
  for (int b = 0; b < p->n_seqs; ++b) {
    const int m = p->cu_seqlens_h[b + 1] - p->cu_seqlens_h[b];
    const int64_t rows = int64_t(m) * g;
    if (rows <= W_FEW_ROWS) {
      c.few = true;
      c.R = std::max(c.R, int(rows));
      continue;
    }
    if (c.n < KV_LIST) c.list[c.n] = b;
    ++c.n;
    most = std::max(most, rows);
    const double n = prompts ? m : std::max(max_len, m);
    tiles += (double(rows) / W_ROWS + 1) * ((n - 0.5 * m) / W_KEYS + 1) * hkv;
  }
  // A sequence's workgroups are a launch's at most (sequences are shared out over launches).
  if ((int64_t(max_len) + W_KEYS - 1) / W_KEYS * 2 * hkv > MOST_GROUPS) return CC_ERR_UNSUPPORTED;
  if (c.n == 0 || max_len == 0) return CC_OK;
  c.listed = c.n <= KV_LIST;
  c.n_list = c.listed ? c.n : p->n_seqs;
  const int64_t planes = int64_t(c.n_list) * hkv;
  // (a tile's rows by 32-bit offsets)
  if (int64_t(W_ROWS / g + 2) * p->n_heads_q * p->head_dim * 2 >= int64_t(1) << 32) return CC_ERR_UNSUPPORTED;
  // Chunks that make r rounds of two workgroups a CU, an item of a block ending half a chunk early, where a round costs
  // its tiles and four more to begin: the r of the least.
  const double slots = 2 * kCus, ends = 0.5 * double(blocks) * planes;
  int64_t each = 8;
  double least = 0;
  for (int r = 1; r <= 16; ++r) {
    if (r * slots <= 2 * ends) continue;
    const double t = std::max(4.0, tiles / (r * slots - ends));
    if (least == 0 || r * (t + 4) < least) {
      least = r * (t + 4);
      each = int64_t(t) + 1;
    }
  }
  if (least == 0) each = (most + W_ROWS - 1) / W_ROWS;   // workgroups enough without a cut
  const int64_t room = std::max<int64_t>(1, std::min(MOST_GROUPS / (2 * blocks * hkv), (int64_t(1) << 26) / (planes * std::max(max_len, 1))));
  each = std::max(each, ((most + W_ROWS - 1) / W_ROWS + room - 1) / room);
  c.chunk = int(std::min<int64_t>(each * W_ROWS, INT32_MAX / W_ROWS * W_ROWS));
  c.chunks = int((most + c.chunk - 1) / c.chunk);
  if (c.chunks > 1) c.total = align_up(size_t(c.chunks) * planes * max_len * sizeof(float));
  return CC_OK;
}

// written: each (sequence, KV head) needs a place of its own.  longest: entries of each that are reached.
cc_status check_weights(const cc_problem* p, const cc_weights* w, bool written, int longest) {
  if (!w || !w->base) return CC_ERR_ARG;
  if (w->seq_stride < 0 || w->head_stride < 0) return CC_ERR_SHAPE;
  if (w->entries != 0 && w->entries < longest) return CC_ERR_SHAPE;
  if (written && ((w->seq_stride == 0 && p->n_seqs > 1) || (w->head_stride == 0 && p->n_heads_kv > 1))) return CC_ERR_SHAPE;
  return CC_OK;
}

}  // namespace

extern "C" {

cc_status cc_attention_kv_workspace(const cc_problem* p, int32_t max_kv_len, size_t* bytes) {
  if (!bytes) return CC_ERR_ARG;
  CC_TRY(check_attention_kv(p, max_kv_len));
  KvPlan c;
  CC_TRY(kv_plan(p, nullptr, max_kv_len, c));
  *bytes = c.total();
  return CC_OK;
}

cc_status cc_attention_kv(const cc_problem* p, const void* q, const cc_kv* kv, int32_t layer, const int32_t* kv_lens,
                          int32_t max_kv_len, void* o, float* lse, void* ws, size_t ws_bytes, void* stream) {
  CC_TRY(check_attention_kv(p, max_kv_len));
  return run_attention_kv(p, q, nullptr, kv, layer, kv_lens, max_kv_len, o, lse, ws, ws_bytes, stream);
}

cc_status cc_attention_prefix_workspace(const cc_problem* p, const cc_prefix* prefix, int32_t max_kv_len,
                                        size_t* bytes) {
  if (!bytes) return CC_ERR_ARG;
  CC_TRY(check_attention_kv(p, max_kv_len));
  CC_TRY(check_prefix(p, prefix));
  KvPlan c;
  CC_TRY(kv_plan(p, prefix, max_kv_len, c));
  *bytes = c.total();
  return CC_OK;
}

cc_status cc_attention_prefix(const cc_problem* p, const void* q, const cc_prefix* prefix, const cc_kv* kv, int32_t layer,
                              const int32_t* kv_lens, int32_t max_kv_len, void* o, float* lse, void* ws, size_t ws_bytes,
                              void* stream) {
  CC_TRY(check_attention_kv(p, max_kv_len));
  CC_TRY(check_prefix(p, prefix));
  return run_attention_kv(p, q, prefix, kv, layer, kv_lens, max_kv_len, o, lse, ws, ws_bytes, stream);
}

cc_status cc_attention_weights_workspace(const cc_problem* p, int32_t max_kv_len, size_t* bytes) {
  if (!bytes) return CC_ERR_ARG;
  CC_TRY(check_attention_kv(p, max_kv_len));
  WeightsPlan c;
  CC_TRY(weights_plan(p, max_kv_len, c));
  *bytes = c.total;
  return CC_OK;
}

cc_status cc_attention_weights(const cc_problem* p, const void* q, const cc_kv* kv, int32_t layer, const int32_t* kv_lens,
                               int32_t max_kv_len, const float* lse, const cc_weights* prev, const int32_t* prev_lens,
                               const cc_weights* out, void* ws, size_t ws_bytes, void* stream) {
  CC_TRY(check_attention_kv(p, max_kv_len));
  CC_TRY(check_view16(p, kv, layer, max_kv_len));
  CC_TRY(check_weights(p, out, true, max_kv_len));
  if (prev) CC_TRY(check_weights(p, prev, false, prev_lens ? 0 : max_kv_len));
  if (prev && prev->base == out->base && (prev->seq_stride != out->seq_stride || prev->head_stride != out->head_stride))
    return CC_ERR_ARG;
  if (!prev && prev_lens) return CC_ERR_ARG;
  const int N = n_tokens(p);
  if (!kv_lens || (N > 0 && (!q || !lse || !aligned16(q)))) return CC_ERR_ARG;
  WeightsPlan c;
  CC_TRY(weights_plan(p, max_kv_len, c));
  CC_TRY(check_ws(ws, ws_bytes, c.total));
  if (max_kv_len == 0) return CC_OK;
  KvWeightsArgs a{};
  a.q = static_cast<const u16*>(q);
  a.lse = lse;
  a.own = make_pair(kv);
  a.cu = p->cu_seqlens_d;
  a.lens = kv_lens;
  a.prev_lens = prev_lens;
  if (prev) {
    a.prev = prev->base;
    a.prev_n = prev->entries ? int(std::min<int64_t>(prev->entries, INT32_MAX)) : INT32_MAX;
    a.prev_seq = prev->seq_stride;
    a.prev_head = prev->head_stride;
  }
  a.w = out->base;
  a.w_seq = out->seq_stride;
  a.w_head = out->head_stride;
  a.n_seqs = p->n_seqs;
  a.layer = layer;
  a.max_len = max_kv_len;
  a.hq = p->n_heads_q;
  a.hkv = p->n_heads_kv;
  a.g = p->n_heads_q / p->n_heads_kv;
  a.head_dim = p->head_dim;
  a.c2 = softmax_scale(p) * kLog2e;
  a.n_list = c.n_list;
  a.listed = c.listed;
  std::copy_n(c.list, c.listed ? c.n : 0, a.list);
  a.R = c.R;
  a.chunk = c.chunk;
  a.chunks = c.chunks;
  a.part = c.total ? static_cast<float*>(ws) : nullptr;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (c.few) CC_HIP(launch_weights_few(a, st));
  if (c.n) CC_HIP(launch_weights_many(a, st));
  return CC_OK;
}

cc_status cc_weight_scores(const cc_problem* p, const cc_weights* w, int32_t n_recent, int32_t per_head, float* scores,
                           void* stream) {
  CC_TRY(check_problem(p));
  if (per_head != 0 && per_head != 1) return CC_ERR_ARG;
  if (n_recent < 0) return CC_ERR_ARG;
  const int longest = max_len(p);
  CC_TRY(check_weights(p, w, false, longest));
  if (n_tokens(p) == 0) return CC_OK;
  if (!scores) return CC_ERR_ARG;
  if ((int64_t(longest) + 255) / 256 * (per_head ? p->n_heads_kv : 1) > MOST_GROUPS) return CC_ERR_UNSUPPORTED;
  const WeightScoresArgs a{w->base, w->seq_stride, w->head_stride, scores, p->cu_seqlens_d, p->n_seqs, p->n_heads_kv,
                           per_head, n_recent, p->n_frozen, longest, 0};
  CC_HIP(launch_weight_scores(a, static_cast<hipStream_t>(stream)));
  return CC_OK;
}

cc_status cc_compact_weights(const cc_problem* p, const cc_weights* w, const int32_t* keep_idx, const int32_t* k_h,
                             int32_t per_head, const cc_weights* out, void* stream) {
  CC_TRY(check_problem(p));
  if (per_head != 0 && per_head != 1) return CC_ERR_ARG;
  if (!k_h) return CC_ERR_ARG;
  CC_TRY(check_weights(p, w, !out, max_len(p)));
  if (out) {
    CC_TRY(check_weights(p, out, true, 0));
    if (out->base == w->base) return CC_ERR_ARG;
  }
  const int per = per_head ? p->n_heads_kv : 1;
  if (int64_t(p->n_heads_kv) >= 1 << 20 || int64_t(p->n_seqs) * p->n_heads_kv > INT32_MAX) return CC_ERR_UNSUPPORTED;
  int64_t all = 0;
  for (int64_t i = 0; i < int64_t(p->n_seqs) * per; ++i) {
    const int b = int(i / per);
    if (k_h[i] < 0 || k_h[i] > p->cu_seqlens_h[b + 1] - p->cu_seqlens_h[b]) return CC_ERR_SHAPE;
    if (out && out->entries != 0 && k_h[i] > out->entries) return CC_ERR_SHAPE;
    all += k_h[i];
  }
  if (all == 0) return CC_OK;
  if (!keep_idx) return CC_ERR_ARG;
  const cc_weights* to = out ? out : w;
  const CompactWeightsArgs a{w->base, to->base, w->seq_stride, w->head_stride, to->seq_stride, to->head_stride,
                             keep_idx, k_h, p->n_seqs, p->n_heads_kv, per_head};
  CC_HIP(launch_compact_weights(a, static_cast<hipStream_t>(stream)));
  return CC_OK;
}

}  // extern "C"

// ------------------------------------------------------------------ log-probabilities

namespace {
cc_status check_logprobs(int32_t dtype, int32_t n, int32_t vocab, int32_t hidden, int32_t top) {
  if (dtype != CC_F32 && dtype != CC_BF16) return CC_ERR_DTYPE;
  if (dtype != CC_BF16) return CC_ERR_UNSUPPORTED;
  if (n < 0 || vocab < 1 || hidden < 1) return CC_ERR_SHAPE;
  if (top < 0 || top > vocab || top > CC_LOGPROBS_MAX_TOP) return CC_ERR_ARG;
  if (hidden % 64 != 0) return CC_ERR_UNSUPPORTED;
  return CC_OK;
}
}  // namespace

extern "C" {

cc_status cc_lmhead_logprobs_workspace(int32_t dtype, int32_t n, int32_t vocab, int32_t hidden, int32_t top,
                                       size_t* bytes) {
  if (!bytes) return CC_ERR_ARG;
  CC_TRY(check_logprobs(dtype, n, vocab, hidden, top));
  *bytes = logprobs_ws_bytes(n, vocab, top);
  return CC_OK;
}

cc_status cc_lmhead_logprobs(int32_t dtype, const void* u, const void* w_lm, int32_t packed, int32_t n,
                             int32_t vocab, int32_t hidden, const int32_t* ids, int32_t top, float* logprob,
                             float* entropy, int32_t* top_ids, float* top_logprob, void* ws, size_t ws_bytes,
                             void* stream) {
  CC_TRY(check_logprobs(dtype, n, vocab, hidden, top));
  if (packed != 0 && packed != 1) return CC_ERR_ARG;
  if ((ids == nullptr) != (logprob == nullptr) && n > 0) return CC_ERR_ARG;
  if (n > 0 && (!u || !w_lm || !aligned16(u) || !aligned16(w_lm))) return CC_ERR_ARG;
  if (n > 0 && top > 0 && (!top_ids || !top_logprob)) return CC_ERR_ARG;
  CC_TRY(check_ws(ws, ws_bytes, logprobs_ws_bytes(n, vocab, top)));
  if (n == 0) return CC_OK;
  LogprobsLaunch a;
  a.u = static_cast<const u16*>(u);
  a.w = w_lm;
  a.packed = packed != 0;
  a.ids = ids;
  a.N = n;
  a.D = hidden;
  a.V = vocab;
  a.top = top;
  a.logprob = logprob;
  a.entropy = entropy;
  a.top_ids = top_ids;
  a.top_logprob = top_logprob;
  a.ws = ws;
  CC_HIP(launch_logprobs(a, static_cast<hipStream_t>(stream)));
  return CC_OK;
}

}  // extern "C"
