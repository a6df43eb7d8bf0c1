"""What the operators of the inference cycle refuse, on the host: every bad call ends with its status
before anything is enqueued (no GPU is needed), and the binding's own checks."""
import ctypes

import pytest
import torch

from paper_2607_27600_amd import cc

P = 0x100000   # an address that is checked, never read


def _problem(cu=(0, 3, 8), **kw):
    c = (ctypes.c_int32 * len(cu))(*cu)
    p = cc.c_problem()
    p.dtype, p.n_seqs = cc.CC_BF16, len(cu) - 1
    p.cu_seqlens_h = ctypes.cast(c, ctypes.POINTER(ctypes.c_int32))
    p.cu_seqlens_d = P
    p.n_heads_q, p.n_heads_kv, p.head_dim, p.hidden, p.vocab, p.rope_theta = 8, 2, 128, 64, 1, 1e4
    for k, v in kw.items():
        setattr(p, k, v)
    p._keep = c
    return p


def _kv(paged=True, es=1, **kw):
    s = cc.c_kv()
    s.layout, s.n_layers = (cc.CC_KV_PAGED if paged else cc.CC_KV_CONTIGUOUS), 2
    s.k, s.v = P, P
    s.layer_stride, s.head_stride, s.tok_stride, s.seq_stride = 1 << 20, 1 << 14, 128, 1 << 16
    s.page_stride, s.block_table, s.page_size, s.max_pages = 1 << 15, P, 16, 64
    for k, v in kw.items():
        setattr(s, k, v)
    return s


def _kv8(paged=True, **kw):
    s = cc.c_kv8()
    codes = {k: v for k, v in kw.items() if k in dict(cc.c_kv._fields_)}
    s.codes = _kv(paged, **codes)
    s.k_scale, s.v_scale, s.scale_block = P, P, 16
    s.scale_layer_stride, s.scale_head_stride, s.scale_page_stride, s.scale_seq_stride = 64, 8, 16, 128
    for k, v in kw.items():
        if k not in codes:
            setattr(s, k, v)
    return s


def _rows(**kw):
    r = cc.c_rows()
    r.base, r.layer_stride, r.tok_stride, r.head_stride = P, 8192, 1024, 128
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def _append(**kw):
    a = cc.c_append()
    a.k, a.v, a.q, a.q_out, a.cached = _rows(), _rows(), _rows(), P, P
    a.capacity, a.layer, a.n_layers, a.rotate = 0, 0, 1, 1
    for k, v in kw.items():
        setattr(a, k, v)
    return a


BAD_APPEND = [
    (dict(), dict(n_layers=0), {}, cc.CC_ERR_SHAPE),
    (dict(), dict(layer=-1), {}, cc.CC_ERR_SHAPE),
    (dict(), dict(layer=2), {}, cc.CC_ERR_SHAPE),
    (dict(), dict(layer=1, n_layers=2, q=cc.c_rows()), {}, cc.CC_ERR_SHAPE),
    (dict(), dict(n_layers=2), {}, cc.CC_ERR_UNSUPPORTED),            # queries belong to one layer
    (dict(), dict(rotate=2), {}, cc.CC_ERR_ARG),
    (dict(rope_theta=0.0), dict(), {}, cc.CC_ERR_ARG),
    (dict(rope_theta=float("inf")), dict(), {}, cc.CC_ERR_ARG),
    (dict(rope_theta=float("nan")), dict(), {}, cc.CC_ERR_ARG),
    (dict(), dict(capacity=-1), {}, cc.CC_ERR_SHAPE),
    (dict(), dict(cached=None), {}, cc.CC_ERR_ARG),
    (dict(), dict(k=_rows(base=None)), {}, cc.CC_ERR_ARG),
    (dict(), dict(v=_rows(base=P + 8)), {}, cc.CC_ERR_ARG),
    (dict(), dict(k=_rows(tok_stride=1020)), {}, cc.CC_ERR_UNSUPPORTED),
    (dict(), dict(k=_rows(head_stride=-128)), {}, cc.CC_ERR_SHAPE),
    (dict(), dict(q=_rows(tok_stride=4)), {}, cc.CC_ERR_UNSUPPORTED),
    (dict(), dict(q_out=None), {}, cc.CC_ERR_ARG),
    (dict(), dict(q_out=P + 4), {}, cc.CC_ERR_ARG),
    (dict(head_dim=96), dict(), {}, cc.CC_ERR_UNSUPPORTED),
    (dict(n_heads_kv=3), dict(), {}, cc.CC_ERR_SHAPE),
    (dict(dtype=9), dict(), {}, cc.CC_ERR_DTYPE),
    (dict(), dict(), dict(page_size=24), cc.CC_ERR_ARG),
    (dict(), dict(), dict(page_size=8), cc.CC_ERR_ARG),
    (dict(), dict(), dict(block_table=None), cc.CC_ERR_ARG),
    (dict(), dict(), dict(tok_stride=64), cc.CC_ERR_SHAPE),
    (dict(), dict(), dict(k=P + 1), cc.CC_ERR_ARG),
    (dict(), dict(), dict(max_pages=0), cc.CC_ERR_SHAPE),
]
BAD_KV8 = [
    (dict(k_scale=None), cc.CC_ERR_ARG),
    (dict(scale_block=8), cc.CC_ERR_UNSUPPORTED),
    (dict(scale_block=48), cc.CC_ERR_UNSUPPORTED),
    (dict(scale_block=256), cc.CC_ERR_UNSUPPORTED),
    (dict(scale_block=32), cc.CC_ERR_SHAPE),          # longer than a page of 16
    (dict(scale_page_stride=-1), cc.CC_ERR_SHAPE),
    (dict(scale_head_stride=-1), cc.CC_ERR_SHAPE),
    (dict(tok_stride=136), cc.CC_ERR_UNSUPPORTED),    # rows 16 bytes aligned
    (dict(page_stride=1 << 32), cc.CC_ERR_UNSUPPORTED),
]


def _ref(x):
    return ctypes.byref(x)


@pytest.mark.parametrize("n", range(len(BAD_APPEND)))
def test_append_refuses(n):
    pk, ak, kk, want = BAD_APPEND[n]
    a, p = _append(**ak), _problem(**pk)
    assert cc._lib.cc_append_kv8(_ref(p), _ref(a), _ref(_kv8(**kk)), None) == want
    if "tok_stride" not in kk:
        kv = _kv(**{**dict(tok_stride=128), **kk})
        assert cc._lib.cc_append_kv(_ref(p), _ref(a), _ref(kv), None) == want


def test_append_refuses_more():
    f8, f16 = cc._lib.cc_append_kv8, cc._lib.cc_append_kv
    p, a = _problem(), _append()
    assert f8(None, _ref(a), _ref(_kv8()), None) == cc.CC_ERR_ARG
    assert f8(_ref(p), None, _ref(_kv8()), None) == cc.CC_ERR_ARG
    assert f8(_ref(p), _ref(a), None, None) == cc.CC_ERR_ARG
    assert f16(_ref(p), _ref(a), None, None) == cc.CC_ERR_ARG
    # a contiguous cache needs its capacity said
    assert f8(_ref(p), _ref(a), _ref(_kv8(paged=False)), None) == cc.CC_ERR_ARG
    assert f16(_ref(p), _ref(a), _ref(_kv(paged=False)), None) == cc.CC_ERR_ARG
    # nothing to append: fine, whatever the rows
    empty = _problem((0, 0, 0))
    assert f8(_ref(empty), _ref(_append(k=cc.c_rows(), cached=None)), _ref(_kv8()), None) == cc.CC_OK


@pytest.mark.parametrize("n", range(len(BAD_KV8)))
def test_bad_8bit_caches(n):
    kw, want = BAD_KV8[n]
    kv, p, size = _kv8(**kw), _problem(), ctypes.c_size_t()
    assert cc._lib.cc_append_kv8(_ref(p), _ref(_append()), _ref(kv), None) == want
    k = (ctypes.c_int32 * 2)(1, 1)
    assert cc._lib.cc_compact_kv8(_ref(p), _ref(kv), P, k, 0, None, None, None, None) == want
    assert cc._lib.cc_compact_kv8(_ref(p), _ref(_kv8()), P, k, 0, None, None, _ref(kv), None) == want
    assert cc._lib.cc_attention_kv8(_ref(p), P, _ref(kv), 0, 0, P, 100, P, P, 1 << 30, None) == want


def test_compact_refuses():
    f, p = cc._lib.cc_compact_kv8, _problem()
    k = lambda *x: (ctypes.c_int32 * len(x))(*x)
    kv = _kv8()
    assert f(_ref(p), _ref(kv), P, None, 0, None, None, None, None) == cc.CC_ERR_ARG
    assert f(_ref(p), _ref(kv), P, k(1, 1), 2, None, None, None, None) == cc.CC_ERR_ARG
    assert f(_ref(p), _ref(kv), P, k(4, 1), 0, None, None, None, None) == cc.CC_ERR_SHAPE      # of 3
    assert f(_ref(p), _ref(kv), P, k(-1, 1), 0, None, None, None, None) == cc.CC_ERR_SHAPE
    assert f(_ref(p), _ref(kv), None, k(1, 1), 0, None, None, None, None) == cc.CC_ERR_ARG
    assert f(_ref(p), _ref(kv), P, k(1, 1), 0, None, None, _ref(_kv8(paged=False)), None) == cc.CC_ERR_ARG
    assert f(_ref(p), _ref(_kv8(page_size=32)), P, k(1, 1), 0, None, None, _ref(_kv8(page_size=32, scale_block=32)), None) == cc.CC_ERR_ARG
    assert f(_ref(p), _ref(kv), P, k(1, 1), 0, None, None, _ref(_kv8(n_layers=1)), None) == cc.CC_ERR_SHAPE
    assert f(_ref(p), _ref(_kv8(max_pages=0)), P, k(1, 1), 0, None, None, None, None) == cc.CC_ERR_SHAPE
    many = _problem(n_heads_q=130, n_heads_kv=65)
    assert f(_ref(many), _ref(kv), P, k(*[1] * 130), 1, None, None, None, None) == cc.CC_ERR_UNSUPPORTED
    assert f(_ref(p), _ref(kv), None, k(0, 0), 0, None, None, None, None) == cc.CC_OK


def test_attention_refuses():
    f, q = cc._lib.cc_attention_kv8, cc._lib.cc_attention_kv8_workspace
    p, kv, n = _problem(), _kv8(), ctypes.c_size_t()
    ok = [_ref(p), P, _ref(kv), 0, 0, P, 1000, P, P, 1 << 30, None]

    def call(i, x):
        return f(*[x if j == i else y for j, y in enumerate(ok)])

    assert call(1, None) == call(5, None) == call(7, None) == call(1, P + 8) == call(7, P + 2) == cc.CC_ERR_ARG
    assert call(3, -1) == call(3, 2) == call(4, 2) == call(4, -1) == cc.CC_ERR_ARG
    assert call(6, -1) == cc.CC_ERR_SHAPE
    assert call(6, 1025) == cc.CC_ERR_SHAPE            # 64 pages of 16
    assert call(6, 2 ** 31 - 1) == cc.CC_ERR_SHAPE
    assert call(0, _ref(_problem(dtype=cc.CC_F32))) == cc.CC_ERR_UNSUPPORTED
    assert call(0, _ref(_problem(head_dim=256))) == cc.CC_ERR_UNSUPPORTED
    wide = _kv8(max_pages=1 << 20)
    assert q(_ref(p), 0, 100000, _ref(n)) == cc.CC_OK and n.value > 0
    assert f(_ref(p), P, _ref(wide), 0, 0, P, 100000, P, P, n.value - 1, None) == cc.CC_ERR_WORKSPACE
    assert f(_ref(p), P, _ref(wide), 0, 0, P, 100000, P, None, n.value, None) == cc.CC_ERR_ARG
    assert f(_ref(p), P, _ref(wide), 0, 0, P, 100000, P, P + 16, n.value, None) == cc.CC_ERR_ARG
    assert q(_ref(p), 0, 100, None) == cc.CC_ERR_ARG
    assert q(_ref(p), 5, 100, _ref(n)) == cc.CC_ERR_ARG
    assert q(_ref(p), 0, -1, _ref(n)) == cc.CC_ERR_SHAPE
    empty = _problem((0, 0))
    assert f(_ref(empty), None, _ref(kv), 0, 0, None, 0, None, None, 0, None) == cc.CC_OK


def test_workspace_is_bounded():
    """Partial results do not grow with the product of lengths and sequences."""
    n = ctypes.c_size_t()
    big = _problem([0] + list(range(1, 4097)), n_heads_q=32, n_heads_kv=8)
    assert cc._lib.cc_attention_kv8_workspace(_ref(big), 0, 1 << 20, _ref(n)) == cc.CC_OK
    assert n.value < 1 << 28
    long = _problem([0, 1 << 20], n_heads_q=32, n_heads_kv=8)
    assert cc._lib.cc_attention_kv8_workspace(_ref(long), 0, 1 << 20, _ref(n)) == cc.CC_OK and n.value == 0


def test_logprobs_refuses():
    f, q, n = cc._lib.cc_lmhead_logprobs, cc._lib.cc_lmhead_logprobs_workspace, ctypes.c_size_t()
    ok = [cc.CC_BF16, P, P, 0, 4, 1000, 128, P, 5, P, P, P, P, P, 1 << 30, None]

    def call(i, x):
        return f(*[x if j == i else y for j, y in enumerate(ok)])

    assert call(0, cc.CC_F32) == cc.CC_ERR_UNSUPPORTED and call(0, 7) == cc.CC_ERR_DTYPE
    assert call(1, None) == call(2, None) == call(1, P + 2) == call(2, P + 8) == cc.CC_ERR_ARG
    assert call(3, 2) == cc.CC_ERR_ARG
    assert call(4, -1) == call(5, 0) == call(6, 0) == cc.CC_ERR_SHAPE
    assert call(6, 100) == cc.CC_ERR_UNSUPPORTED
    assert call(7, None) == call(9, None) == cc.CC_ERR_ARG     # ids and logprob go together
    assert call(8, -1) == call(8, 33) == cc.CC_ERR_ARG
    assert f(*[3 if j == 5 else y for j, y in enumerate(ok)]) == cc.CC_ERR_ARG   # 5 of 3 words
    assert call(11, None) == call(12, None) == cc.CC_ERR_ARG
    assert call(14, 16) == cc.CC_ERR_WORKSPACE
    assert call(13, None) == call(13, P + 64) == cc.CC_ERR_ARG
    assert f(*[0 if j == 4 else y for j, y in enumerate(ok)]) == cc.CC_OK
    assert q(cc.CC_BF16, 4, 1000, 128, 5, None) == cc.CC_ERR_ARG
    assert q(cc.CC_BF16, 100000, 128256, 4096, 32, _ref(n)) == cc.CC_OK
    assert n.value < 3 << 30          # rows are taken in slabs


def test_binding_refuses():
    p = cc.problem(dtype="bf16", cu_seqlens=[0, 2], n_heads_q=4, n_heads_kv=2, head_dim=64, hidden=64, vocab=1, rope_theta=1e4,
                   device="cpu")
    z = lambda *s, t=torch.bfloat16: torch.zeros(*s, dtype=t)
    codes, sc = z(1, 2, 32, 64, t=torch.uint8), z(1, 2, 2, t=torch.uint8)
    kw = dict(n_layers=1, layer_stride=4096, head_stride=2048, tok_stride=64, scale_block=16, scale_layer_stride=4,
              scale_head_stride=2)
    kv = cc.kv8_contiguous(codes, codes, sc, sc, **kw)
    with pytest.raises(ValueError, match="bytes"):
        cc.kv8_contiguous(z(1, 2, 32, 64), codes, sc, sc, **kw)
    k, lens = z(2, 2, 64), torch.zeros(1, dtype=torch.int32)
    ok = dict(capacity=32)
    with pytest.raises(ValueError, match="GPU"):
        cc.cc_append_kv8(p, kv, k, k, lens, **ok)
    with pytest.raises(ValueError, match="shape"):
        cc.cc_append_kv8(p, kv, z(3, 2, 64), k, lens, **ok)
    with pytest.raises(ValueError, match="float32"):
        cc.cc_append_kv8(p, kv, k, z(2, 2, 64, t=torch.float32), lens, **ok)
    with pytest.raises(ValueError, match="contiguous"):
        cc.cc_append_kv8(p, kv, z(2, 64, 2).transpose(1, 2), k, lens, **ok)
    with pytest.raises(ValueError, match="cached"):
        cc.cc_append_kv8(p, kv, k, k, lens.long(), **ok)
    with pytest.raises(ValueError, match="pos_ids"):
        cc.cc_append_kv8(p, kv, k, k, lens, pos_ids=torch.zeros(3, dtype=torch.int32), **ok)
    with pytest.raises(ValueError, match="q_out"):
        cc.cc_append_kv8(p, kv, k, k, lens, q=z(2, 4, 64), q_out=z(2, 4, 32), **ok)
    with pytest.raises(ValueError, match="kv_lens"):
        cc.cc_attention_kv8(p, z(2, 4, 64), kv, 0, torch.zeros(2, dtype=torch.int32), 10)
    with pytest.raises(ValueError, match="q must"):
        cc.cc_attention_kv8(p, z(3, 4, 64), kv, 0, lens, 10)
    with pytest.raises(ValueError, match="GPU"):
        cc.cc_attention_kv8(p, z(2, 4, 64), kv, 0, lens, 10)
    with pytest.raises(KeyError):
        cc.cc_attention_kv8_workspace(p, "both", 10)
    with pytest.raises(ValueError, match="budgets"):
        cc.cc_compact_kv8(p, kv, lens, [1, 1], 0)
    u, w = z(2, 64), z(10, 64)
    with pytest.raises(ValueError, match="w_lm"):
        cc.cc_lmhead_logprobs("bf16", u, w, 11, None, 1)
    with pytest.raises(ValueError, match="ids"):
        cc.cc_lmhead_logprobs("bf16", u, w, 10, torch.zeros(3, dtype=torch.int32), 1)
    with pytest.raises(ValueError, match="room"):
        cc.cc_lmhead_logprobs("bf16", u, w, 10, None, 3, cc.logprobs_out(2, 1, "cpu"))
    with pytest.raises(ValueError, match="packed"):
        cc.cc_lmhead_logprobs("bf16", u, w, 1000, None, 1, packed=True)


def test_struct_layouts_match_the_header(tmp_path):
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    classes = {"cc_kv8": cc.c_kv8, "cc_rows": cc.c_rows, "cc_append": cc.c_append}
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "cc.h"', "int main(void){"]
    for n, c in classes.items():
        lines.append(f'printf("%zu\\n", sizeof({n}));')
        lines += [f'printf("%zu\\n", offsetof({n}, {f[0]}));' for f in c._fields_]
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines + ["return 0;}"]))
    subprocess.run(["gcc", "-I", os.path.join(root, "include"), str(src), "-o", str(tmp_path / "layout")], check=True)
    got = subprocess.run([str(tmp_path / "layout")], capture_output=True, text=True, check=True).stdout.split()
    want = []
    for c in classes.values():
        want += [ctypes.sizeof(c)] + [getattr(c, f[0]).offset for f in c._fields_]
    assert [int(x) for x in got] == want


def test_attention_refuses_rows_whose_offsets_in_a_group_pass_32_bits():
    """Sixteen entries are addressed from one place by 32-bit offsets."""
    f = cc._lib.cc_attention_kv8
    lens = (P, 100, P, P, 1 << 30, None)
    assert f(_ref(_problem()), P, _ref(_kv8(paged=False, tok_stride=1 << 28)), 0, 0, *lens) == cc.CC_ERR_UNSUPPORTED
    assert f(_ref(_problem()), P, _ref(_kv8(paged=False, tok_stride=(1 << 40) + 128)), 0, 0, *lens) == cc.CC_ERR_UNSUPPORTED


def test_logprobs_out_of_wrong_sizes(monkeypatch):
    u, w = torch.zeros(3, 64, dtype=torch.bfloat16), torch.zeros(5, 64, dtype=torch.bfloat16)
    monkeypatch.setattr(cc, "_on_gpu", lambda *t: None)
    ids = torch.zeros(3, dtype=torch.int32)
    good = cc.logprobs_out(3, 2, "cpu")
    for name, bad in (("logprob", torch.zeros(2)), ("logprob", torch.zeros(3, dtype=torch.float64)), ("entropy", torch.zeros(2)),
                      ("entropy", torch.zeros(6)[::2]), ("top_ids", torch.zeros(3, 2)),
                      ("top_ids", torch.zeros(2, 2, dtype=torch.int32)), ("top_logprob", torch.zeros(3, 1))):
        out = cc.Logprobs(**{**good.__dict__, name: bad})
        with pytest.raises(ValueError, match=name):
            cc.cc_lmhead_logprobs("bf16", u, w, 5, ids, 2, out)


def test_strides_of_single_rows_do_not_matter():
    """A dimension of one element may have any stride."""
    r = cc.c_rows()
    t = torch.zeros(64, dtype=torch.bfloat16).as_strided((1, 1, 64), (3, 5, 1))
    cc._rows(r, t, torch.bfloat16, "k", (1, 1, 64))
    assert (r.layer_stride, r.tok_stride, r.head_stride) == (0, 0, 0)
    cc._rows(r, t[None], torch.bfloat16, "k", (1, 1, 1, 64))
    assert (r.layer_stride, r.tok_stride, r.head_stride) == (0, 0, 0)


def test_compaction_refuses_lists_of_another_type(monkeypatch):
    monkeypatch.setattr(cc, "_on_gpu", lambda *t: None)
    p, kv = cc.Problem(_problem(), None, None, []), cc.KV8(_kv8())
    for keep in (torch.zeros(3, dtype=torch.int64), torch.zeros(2, dtype=torch.int32), torch.zeros(6, dtype=torch.int32)[::2]):
        with pytest.raises(ValueError, match="keep_idx"):
            cc.cc_compact_kv8(p, kv, keep, [1, 2], 0)


def test_tensors_elsewhere(monkeypatch):
    """Tensors of one call lie on one GPU, the current one."""
    class T:
        def __init__(self, d):
            self.d, self.device = d, f"cuda:{d}"

        def get_device(self):
            return self.d
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    cc._on_gpu(T(0), None, T(0))
    for bad, what in (((T(0), T(1)), "different"), ((T(1), T(1)), "current device"), ((T(0), torch.zeros(1)), "must be on the GPU")):
        with pytest.raises(ValueError, match=what):
            cc._on_gpu(*bad)
    k = torch.zeros(16, dtype=torch.uint8)
    kv = cc.kv_contiguous(k, k, n_layers=1, layer_stride=0, head_stride=0, tok_stride=16)
    kv8 = cc.kv8_contiguous(k, k, k, k, n_layers=1, layer_stride=0, head_stride=0, tok_stride=16, scale_block=16,
                            scale_layer_stride=0, scale_head_stride=0)
    assert cc._codes(kv) is k and cc._codes(kv8) is k


def test_append_refuses_a_cache_of_another_type(monkeypatch):
    """Rows of four bytes into a cache of two would be written past its end."""
    monkeypatch.setattr(cc, "_on_gpu", lambda *t: None)
    monkeypatch.setattr(cc, "_stream", lambda s=None: None)
    lens = torch.zeros(1, dtype=torch.int32)
    for dtype, T, other in (("f32", torch.float32, torch.bfloat16), ("bf16", torch.bfloat16, torch.float32),
                            ("bf16", torch.bfloat16, torch.float16), ("bf16", torch.bfloat16, torch.uint8)):
        p = cc.problem(dtype=dtype, cu_seqlens=[0, 2], n_heads_q=4, n_heads_kv=2, head_dim=64, hidden=64, vocab=1, rope_theta=1e4,
                       device="cpu")
        k = torch.zeros(2, 2, 64, dtype=T)
        for pool in ((other, other), (T, other), (other, T)):
            pools = [torch.zeros(2, 32, 64, dtype=t) for t in pool]
            kw = dict(n_layers=1, layer_stride=4096, head_stride=2048, tok_stride=64)
            caches = [cc.kv_contiguous(*pools, **kw),
                      cc.kv_paged(*pools, torch.zeros(1, 2, dtype=torch.int32), page_stride=4096, page_size=32, **kw)]
            for kv in caches:
                # (layer 1 of one: the library refuses the call, so that nothing is launched where the binding does not)
                with pytest.raises(ValueError, match="the cache holds"):
                    cc.cc_append_kv(p, kv, k, k, lens, capacity=32, layer=1)


@pytest.mark.parametrize("which", ["token_ids", "pos_ids"])
def test_compaction_refuses_ids_of_another_type_or_too_few(monkeypatch, which):
    """int64 ids would be moved as pairs of words, a short tensor read and written past its end; a longer one
    (a buffer of the cache's capacity) is fine."""
    monkeypatch.setattr(cc, "_on_gpu", lambda *t: None)
    monkeypatch.setattr(cc, "_stream", lambda s=None: None)
    p, keep = cc.Problem(_problem(), None, None, []), torch.zeros(2, dtype=torch.int32)
    # (the library refuses the scale block, so that nothing is launched where the binding does not)
    kv = cc.KV8(_kv8(scale_block=8))
    for ids in (torch.zeros(8, dtype=torch.int64), torch.zeros(7, dtype=torch.int32), torch.zeros(16, dtype=torch.int32)[::2],
                torch.zeros(8)):
        with pytest.raises(ValueError, match=which):
            cc.cc_compact_kv8(p, kv, keep, [1, 1], 0, **{which: ids})
    for n in (8, 11):
        with pytest.raises(cc.CCError):
            cc.cc_compact_kv8(p, kv, keep, [1, 1], 0, **{which: torch.zeros(n, dtype=torch.int32)})


class _T:
    """A tensor somewhere, as far as the binding looks at one before the library does."""

    def __init__(self, device, dtype, shape=(1, 2)):
        self.d, self.dtype, self.shape, self.device = device, dtype, shape, f"cuda:{device}"

    def get_device(self):
        return self.d

    def element_size(self):
        return self.dtype.itemsize

    def data_ptr(self):
        return P

    def numel(self):
        return self.shape[0] * self.shape[1]

    def is_contiguous(self):
        return True

    def to(self, dtype):
        return self

    def contiguous(self):
        return self


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("odd", range(6))
def test_every_tensor_of_a_cache_and_a_problem_is_looked_at(monkeypatch, paged, odd):
    """Values, scales, the block table and the problem's lengths elsewhere count as much as the keys."""
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(cc, "_stream", lambda s=None: None)
    T = lambda i, dtype: _T(int(i == odd), dtype)
    kw = dict(n_layers=1, layer_stride=4096, head_stride=2048, tok_stride=64)
    kw8 = dict(scale_block=8, scale_layer_stride=4, scale_head_stride=2)   # (a scale block that the library refuses)

    def cache(eight):
        pools = [T(i, torch.uint8 if eight else torch.bfloat16) for i in (0, 1)]
        table = [T(2, torch.int32)] if paged else []
        scales = [T(i, torch.uint8) for i in (3, 4)]
        if not eight:
            return cc.kv_paged(*pools, *table, page_stride=4096, page_size=32, **kw) if paged else cc.kv_contiguous(*pools, **kw)
        if paged:
            return cc.kv8_paged(*pools, *scales, *table, page_stride=4096, page_size=32, scale_page_stride=4, **kw, **kw8)
        return cc.kv8_contiguous(*pools, *scales, **kw, **kw8)

    p = cc.Problem(_problem((0, 2), n_heads_q=4, head_dim=64), None, T(5, torch.int32), None)
    here = lambda dtype, *shape: _T(0, dtype, shape)
    lens = here(torch.int32, 1, 1)
    k = torch.zeros(2, 2, 64, dtype=torch.bfloat16)
    k.get_device = lambda: 0
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    q.get_device = lambda: 0
    away = odd in ({0, 1, 2, 5} if paged else {0, 1, 5})
    away8 = odd in ({0, 1, 2, 3, 4, 5} if paged else {0, 1, 3, 4, 5})
    for call, is_away in ((lambda: cc.cc_append_kv(p, cache(False), k, k, lens, capacity=32, layer=1), away),
                          (lambda: cc.cc_append_kv8(p, cache(True), k, k, lens, capacity=32), away8),
                          (lambda: cc.cc_compact_kv8(p, cache(True), lens, [1], 0, out=cache(True)), away8),
                          (lambda: cc.cc_attention_kv8(p, q, cache(True), 0, lens, 10, q, workspace=here(torch.uint8, 1, 1 << 16)), away8)):
        with pytest.raises(ValueError if is_away else cc.CCError, match="different devices" if is_away else None):
            call()


def test_logprobs_without_ids_have_no_logprob(monkeypatch):
    """No words given: none of the result is memory that nothing wrote."""
    calls = []
    monkeypatch.setattr(cc, "_on_gpu", lambda *t: None)
    monkeypatch.setattr(cc, "_stream", lambda s=None: None)
    monkeypatch.setattr(cc._lib, "cc_lmhead_logprobs", lambda *a: calls.append(a) or cc.CC_OK)
    u, w = torch.zeros(3, 64, dtype=torch.bfloat16), torch.zeros(5, 64, dtype=torch.bfloat16)
    r = cc.cc_lmhead_logprobs("bf16", u, w, 5, None, 2)
    assert r.logprob is None and r.entropy.shape == (3,) and r.top_ids.shape == (3, 2)
    out = cc.logprobs_out(3, 2, "cpu")
    out.logprob.fill_(7)
    r = cc.cc_lmhead_logprobs("bf16", u, w, 5, None, 2, out)
    assert r.logprob is None and r.entropy is out.entropy and torch.equal(out.logprob, torch.full((3,), 7.0))
    r = cc.cc_lmhead_logprobs("bf16", u, w, 5, None, 2, cc.logprobs_out(3, 2, "cpu", ids=False))
    assert r.logprob is None
    assert all(a[7] is None and a[9] is None for a in calls)   # ids and logprob
    with pytest.raises(ValueError, match="logprob"):
        cc.cc_lmhead_logprobs("bf16", u, w, 5, torch.zeros(3, dtype=torch.int32), 2, cc.logprobs_out(3, 2, "cpu", ids=False))
    r = cc.cc_lmhead_logprobs("bf16", u, w, 5, torch.zeros(3, dtype=torch.int32), 2, out)
    assert r is out and calls[-1][9].value == out.logprob.data_ptr()


def test_attention_refuses_more_sequences_than_a_launch_has_workgroups():
    """2^24 workgroups of 256 threads and more are not to be had: said before anything is queued."""
    f, q, n = cc._lib.cc_attention_kv8, cc._lib.cc_attention_kv8_workspace, ctypes.c_size_t()
    kv = _kv8(paged=False)
    for rows in (1, 33):    # both kernels
        for seqs, ok in ((1 << 18, False), ((1 << 18) - 1, True)):
            p = _problem(range(0, rows * seqs + 1, rows), n_heads_q=64, n_heads_kv=64, head_dim=64)
            for longest in (100, 100000):
                st = q(_ref(p), 0, longest, _ref(n))
                assert st == (cc.CC_OK if ok else cc.CC_ERR_UNSUPPORTED)
                if not ok:
                    assert f(_ref(p), P, _ref(kv), 0, 0, P, longest, P, P, 1 << 50, None) == cc.CC_ERR_UNSUPPORTED


def test_compaction_refuses_more_planes_than_a_launch_has_workgroups():
    f, p = cc._lib.cc_compact_kv8, _problem(n_heads_q=64, n_heads_kv=64)
    k = (ctypes.c_int32 * 2)(1, 1)
    for out in (None, _kv8(n_layers=1 << 14)):
        assert f(_ref(p), _ref(_kv8(n_layers=1 << 14)), P, k, 0, None, None, out and _ref(out), None) == cc.CC_ERR_UNSUPPORTED


def test_append_refuses_more_tokens_than_a_launch_has_workgroups():
    for cu in ((0, 1 << 26), range((1 << 22) + 1)):
        for paged in (False, True):
            p, kw = _problem(cu), dict(max_pages=1 << 23) if paged else {}
            assert cc._lib.cc_append_kv8(_ref(p), _ref(_append(capacity=100)), _ref(_kv8(paged, **kw)), None) == cc.CC_ERR_UNSUPPORTED
            assert cc._lib.cc_append_kv(_ref(p), _ref(_append(capacity=100)), _ref(_kv(paged, **kw)), None) == cc.CC_ERR_UNSUPPORTED


def test_workspace_of_ragged_chunks_goes_by_the_rows_there_are():
    """Pieces of a chunk beside many short ones: partial results of the rows that exist, not of as many for each
    sequence as the longest has."""
    import itertools
    n = ctypes.c_size_t()
    for new in ([5] * 99 + [1500], [1] * 5000 + [5] * 65 + [2000], [0] * 40 + [7, 3000, 9], [1] * 3000 + [900]):
        p = _problem([0, *itertools.accumulate(new)], n_heads_q=8, n_heads_kv=1, head_dim=128)
        assert cc._lib.cc_attention_kv8_workspace(_ref(p), 0, 5000, _ref(n)) == cc.CC_OK
        # a row of 128 floats, a maximum and a sum, in each of at most 20 pieces of 256; the shares of few rows
        # ((512 + sequences) * 32 rows) beside them
        rows = 8 * (sum(new) if sum(x > 4 for x in new) > 64 else sum(x for x in new if x > 4))
        few = (512 + len(new)) * 32
        assert 0 < n.value <= (20 * rows + few) * 520 + 1024
    p = _problem([0, *itertools.accumulate([5] * 99 + [1500])], n_heads_q=8, n_heads_kv=1, head_dim=128)
    assert cc._lib.cc_attention_kv8_workspace(_ref(p), 0, 5000, _ref(n)) == cc.CC_OK
    assert n.value <= 2 * 15960 * 520 + 1024      # two pieces


def test_attention_takes_a_few_chunks_among_millions_of_single_queries():
    """The pieces of the chunks are fewer, rather than the call refused."""
    import itertools
    n = ctypes.c_size_t()
    p = _problem([0, *itertools.accumulate([1] * 3_000_000 + [40] * 65)], n_heads_q=1, n_heads_kv=1, head_dim=64)
    for longest in (100, 100000):
        assert cc._lib.cc_attention_kv8_workspace(_ref(p), 0, longest, _ref(n)) == cc.CC_OK
