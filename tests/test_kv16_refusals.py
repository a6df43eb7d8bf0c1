"""What the attention over a bf16 cache, with shared prefixes, and eviction by attention weight refuse, on the host:
every bad call ends with its status before anything is enqueued (no GPU is needed), and the binding's own checks."""
import ctypes

import pytest
import torch

from paper_2607_27600_amd import cc

P = 0x100000   # an address that is checked, never read
I32 = ctypes.c_int32


def _problem(cu=(0, 3, 8), **kw):
    c = (I32 * len(cu))(*cu)
    p = cc.c_problem()
    p.dtype, p.n_seqs = cc.CC_BF16, len(cu) - 1
    p.cu_seqlens_h = ctypes.cast(c, ctypes.POINTER(I32))
    p.cu_seqlens_d = P
    p.n_heads_q, p.n_heads_kv, p.head_dim, p.hidden, p.vocab = 8, 2, 128, 64, 1
    for k, v in kw.items():
        setattr(p, k, v)
    p._keep = c
    return p


def _kv(paged=True, **kw):
    s = cc.c_kv()
    s.layout, s.n_layers = (cc.CC_KV_PAGED if paged else cc.CC_KV_CONTIGUOUS), 2
    s.k, s.v = P, P
    s.layer_stride, s.head_stride, s.tok_stride, s.seq_stride = 1 << 20, 1 << 14, 128, 1 << 16
    s.page_stride, s.block_table, s.page_size, s.max_pages = 1 << 15, P, 16, 64
    for k, v in kw.items():
        setattr(s, k, v)
    return s


def _prefix(first=(0, 1, 2), kv=None, **kw):
    f = (I32 * len(first))(*first)
    x = cc.c_prefix()
    x.kv, x.n_prefixes, x.max_len = _kv() if kv is None else kv, len(first) - 1, 100
    x.first_seq_h = ctypes.cast(f, ctypes.POINTER(I32))
    x.first_seq_d = x.lens = P
    for k, v in kw.items():
        setattr(x, k, v)
    x._keep = f
    return x


def _ref(x):
    return None if x is None else ctypes.byref(x)


def _attention(p=None, q=P, kv=None, layer=0, lens=P, longest=200, o=P, lse=P, ws=P, size=1 << 40, pre=None):
    p = _problem() if p is None else p
    kv = _kv() if kv is None else kv
    if pre is None:
        return cc._lib.cc_attention_kv(_ref(p), q, _ref(kv), layer, lens, longest, o, lse, ws, size, None)
    return cc._lib.cc_attention_prefix(_ref(p), q, _ref(pre), _ref(kv), layer, lens, longest, o, lse, ws, size, None)


BAD = [
    (dict(q=None), cc.CC_ERR_ARG),
    (dict(q=P + 8), cc.CC_ERR_ARG),
    (dict(o=None), cc.CC_ERR_ARG),
    (dict(o=P + 2), cc.CC_ERR_ARG),
    (dict(lens=None), cc.CC_ERR_ARG),
    (dict(layer=-1), cc.CC_ERR_ARG),
    (dict(layer=2), cc.CC_ERR_ARG),
    (dict(longest=-1), cc.CC_ERR_SHAPE),
    (dict(longest=2 ** 31 - 1), cc.CC_ERR_SHAPE),
    (dict(longest=16 * 64 + 1), cc.CC_ERR_SHAPE),                # the block table's rows end before
    (dict(p=_problem(dtype=cc.CC_F32)), cc.CC_ERR_UNSUPPORTED),
    (dict(p=_problem(dtype=5)), cc.CC_ERR_DTYPE),
    (dict(p=_problem(head_dim=96)), cc.CC_ERR_UNSUPPORTED),
    (dict(p=_problem(n_heads_kv=3)), cc.CC_ERR_SHAPE),
    (dict(p=_problem(softmax_scale=float("inf"))), cc.CC_ERR_ARG),
    (dict(p=_problem(cu=(0, 5, 4))), cc.CC_ERR_SHAPE),
    (dict(p=_problem(cu=(0, 1 << 29), n_heads_q=8, n_heads_kv=1)), cc.CC_ERR_UNSUPPORTED),      # 2^32 rows
    (dict(p=_problem(cu=(0, 1), n_heads_q=1 << 24, n_heads_kv=1 << 24)), cc.CC_ERR_UNSUPPORTED),
    (dict(kv=_kv(k=None)), cc.CC_ERR_ARG),
    (dict(kv=_kv(v=P + 4)), cc.CC_ERR_ARG),
    (dict(kv=_kv(tok_stride=64)), cc.CC_ERR_SHAPE),
    (dict(kv=_kv(tok_stride=132)), cc.CC_ERR_UNSUPPORTED),
    (dict(kv=_kv(page_size=24)), cc.CC_ERR_ARG),
    (dict(kv=_kv(block_table=None)), cc.CC_ERR_ARG),
    (dict(kv=_kv(page_stride=1 << 31)), cc.CC_ERR_UNSUPPORTED),
    (dict(kv=_kv(paged=False, tok_stride=1 << 27)), cc.CC_ERR_UNSUPPORTED),
    (dict(kv=_kv(paged=False, seq_stride=-8)), cc.CC_ERR_UNSUPPORTED),
]


@pytest.mark.parametrize("prefix", [False, True])
@pytest.mark.parametrize("i", range(len(BAD)))
def test_attention(i, prefix):
    kw, want = BAD[i]
    n = (kw["p"].n_seqs if "p" in kw else 2)
    assert _attention(pre=_prefix(first=(0, 1, n)) if prefix else None, **kw) == want, kw


BAD_PREFIX = [
    (dict(n_prefixes=0), cc.CC_ERR_ARG),
    (dict(first_seq_h=None), cc.CC_ERR_ARG),
    (dict(first_seq_d=None), cc.CC_ERR_ARG),
    (dict(lens=None), cc.CC_ERR_ARG),
    (dict(max_len=-1), cc.CC_ERR_SHAPE),
    (dict(first=(0, 1, 3)), cc.CC_ERR_SHAPE),        # sequences that are not there
    (dict(first=(0, 1)), cc.CC_ERR_SHAPE),           # one without a prefix
    (dict(first=(1, 2)), cc.CC_ERR_SHAPE),
    (dict(first=(0, 2, 1, 2)), cc.CC_ERR_SHAPE),
    (dict(max_len=16 * 64 + 1), cc.CC_ERR_SHAPE),    # the block table's rows end before
    (dict(kv=_kv(n_layers=0)), cc.CC_ERR_SHAPE),
    (dict(kv=_kv(k=None)), cc.CC_ERR_ARG),
    (dict(kv=_kv(paged=False, tok_stride=1 << 27)), cc.CC_ERR_UNSUPPORTED),
]


@pytest.mark.parametrize("i", range(len(BAD_PREFIX)))
def test_prefix(i):
    kw, want = BAD_PREFIX[i]
    assert _attention(pre=_prefix(**kw)) == want, kw


def test_layers_of_both_caches():
    assert _attention(layer=1, pre=_prefix(kv=_kv(n_layers=1))) == cc.CC_ERR_ARG


def test_workspaces():
    n = ctypes.c_size_t(0)
    p = _problem(cu=(0, 1, 2))
    assert cc._lib.cc_attention_kv_workspace(_ref(p), 1 << 20, None) == cc.CC_ERR_ARG
    assert cc._lib.cc_attention_kv_workspace(_ref(p), -1, ctypes.byref(n)) == cc.CC_ERR_SHAPE
    assert cc._lib.cc_attention_prefix_workspace(_ref(p), None, 1, ctypes.byref(n)) == cc.CC_ERR_ARG
    assert cc._lib.cc_attention_weights_workspace(_ref(p), 1, None) == cc.CC_ERR_ARG
    long = _kv(max_pages=1 << 16)
    for pre in (None, _prefix(kv=long, max_len=1 << 20)):
        args = (_ref(p),) if pre is None else (_ref(p), _ref(pre))
        query = cc._lib.cc_attention_kv_workspace if pre is None else cc._lib.cc_attention_prefix_workspace
        assert query(*args, 1 << 20, ctypes.byref(n)) == cc.CC_OK
        if n.value:
            assert _attention(p=p, kv=long, longest=1 << 20, size=n.value - 1, pre=pre) == cc.CC_ERR_WORKSPACE
            assert _attention(p=p, kv=long, longest=1 << 20, ws=None, size=n.value, pre=pre) == cc.CC_ERR_ARG
            assert _attention(p=p, kv=long, longest=1 << 20, ws=P + 16, size=n.value, pre=pre) == cc.CC_ERR_ARG


@pytest.mark.parametrize("cu", [(0, 0, 0), (0, 1, 2), (0, 40, 700), (0, 5000, 5001)])
@pytest.mark.parametrize("longest", [0, 1, 1 << 24, 2 ** 31 - 4097])
def test_workspaces_of_the_shortest_and_longest_plans(cu, longest):
    """(A division by the number of blocks would end the process.)"""
    n = ctypes.c_size_t(0)
    p, kv = _problem(cu=cu), _kv(paged=False)
    for call in (lambda: cc._lib.cc_attention_kv_workspace(_ref(p), longest, ctypes.byref(n)),
                 lambda: cc._lib.cc_attention_prefix_workspace(_ref(p), _ref(_prefix(kv=kv, max_len=longest)), longest, ctypes.byref(n)),
                 lambda: cc._lib.cc_attention_weights_workspace(_ref(p), longest, ctypes.byref(n))):
        n.value = 0
        st = call()
        assert st == cc.CC_OK or (longest > 1 << 24 and st == cc.CC_ERR_UNSUPPORTED)
        assert n.value < 1 << 36


def test_no_queries_need_nothing():
    assert _attention(p=_problem(cu=(0, 0, 0)), q=None, o=None, lens=None, lse=None, ws=None, size=0) == cc.CC_OK


def _w(**kw):
    w = cc.c_weights(P, 1000, 300)
    for k, v in kw.items():
        setattr(w, k, v)
    return w


def _weights(p=None, q=P, kv=None, layer=0, lens=P, longest=200, lse=P, prev=None, prev_lens=None, out=0, ws=P, size=1 << 40):
    p, kv = _problem() if p is None else p, _kv() if kv is None else kv
    out = _w() if out == 0 else out
    return cc._lib.cc_attention_weights(_ref(p), q, _ref(kv), layer, lens, longest, lse, _ref(prev), prev_lens, _ref(out), ws,
                                        size, None)


BAD_WEIGHTS = [
    (dict(q=None), cc.CC_ERR_ARG),
    (dict(q=P + 8), cc.CC_ERR_ARG),
    (dict(lse=None), cc.CC_ERR_ARG),
    (dict(lens=None), cc.CC_ERR_ARG),
    (dict(out=None), cc.CC_ERR_ARG),
    (dict(out=_w(base=None)), cc.CC_ERR_ARG),
    (dict(out=_w(seq_stride=-1)), cc.CC_ERR_SHAPE),
    (dict(out=_w(seq_stride=0)), cc.CC_ERR_SHAPE),         # sequences in one place
    (dict(out=_w(head_stride=0)), cc.CC_ERR_SHAPE),
    (dict(prev=_w(base=None)), cc.CC_ERR_ARG),
    (dict(prev=_w(head_stride=-3)), cc.CC_ERR_SHAPE),
    (dict(prev=_w(head_stride=400)), cc.CC_ERR_ARG),       # out's own place, laid out otherwise
    (dict(prev_lens=P), cc.CC_ERR_ARG),                    # without prev
    (dict(layer=2), cc.CC_ERR_ARG),
    (dict(longest=-1), cc.CC_ERR_SHAPE),
    (dict(longest=16 * 64 + 1), cc.CC_ERR_SHAPE),
    (dict(p=_problem(dtype=cc.CC_F32)), cc.CC_ERR_UNSUPPORTED),
    (dict(kv=_kv(tok_stride=64)), cc.CC_ERR_SHAPE),
    (dict(kv=_kv(paged=False, tok_stride=1 << 27)), cc.CC_ERR_UNSUPPORTED),
]


@pytest.mark.parametrize("i", range(len(BAD_WEIGHTS)))
def test_weights(i):
    kw, want = BAD_WEIGHTS[i]
    assert _weights(**kw) == want, kw


def _scores(p=None, w=0, recent=0, per_head=0, out=P):
    return cc._lib.cc_weight_scores(_ref(_problem() if p is None else p), _ref(_w() if w == 0 else w), recent, per_head, out, None)


def test_scores():
    assert _scores(w=None) == cc.CC_ERR_ARG
    assert _scores(recent=-1) == cc.CC_ERR_ARG
    assert _scores(per_head=2) == cc.CC_ERR_ARG
    assert _scores(out=None) == cc.CC_ERR_ARG
    assert _scores(w=_w(head_stride=-1)) == cc.CC_ERR_SHAPE
    assert _scores(p=_problem(n_frozen=-1)) == cc.CC_ERR_ARG
    assert _scores(p=_problem(cu=(0, 0, 0)), out=None) == cc.CC_OK


def _compact(p=None, w=0, keep=P, k=(1, 2), per_head=0, out=None):
    kk = (I32 * len(k))(*k) if k is not None else None
    return cc._lib.cc_compact_weights(_ref(_problem() if p is None else p), _ref(_w() if w == 0 else w), keep, kk, per_head,
                                      _ref(out), None)


def test_compaction():
    assert _compact(w=None) == cc.CC_ERR_ARG
    assert _compact(k=None) == cc.CC_ERR_ARG
    assert _compact(keep=None) == cc.CC_ERR_ARG
    assert _compact(per_head=2) == cc.CC_ERR_ARG
    assert _compact(k=(4, 2)) == cc.CC_ERR_SHAPE           # more than there are
    assert _compact(k=(1, -1)) == cc.CC_ERR_SHAPE
    assert _compact(k=(1, 3, 5, 6), per_head=1) == cc.CC_ERR_SHAPE
    assert _compact(w=_w(head_stride=0)) == cc.CC_ERR_SHAPE
    assert _compact(out=_w()) == cc.CC_ERR_ARG             # out's place is w's
    assert _compact(out=_w(base=2 * P, seq_stride=0)) == cc.CC_ERR_SHAPE
    assert _compact(k=(0, 0), keep=None) == cc.CC_OK


# ---- the binding's own checks, on tensors of the host

def _host(cu=(0, 2, 3), hq=4, hkv=2, d=64):
    p = cc.problem(dtype="bf16", cu_seqlens=cu, n_heads_q=hq, n_heads_kv=hkv, head_dim=d, hidden=64, vocab=1, device="cpu")
    n = cu[-1]
    k = torch.zeros(2, hkv, 8, d, dtype=torch.bfloat16)
    kv = cc.kv_contiguous(k, k.clone(), n_layers=1, seq_stride=hkv * 8 * d, layer_stride=0, head_stride=8 * d, tok_stride=d)
    return p, torch.zeros(n, hq, d, dtype=torch.bfloat16), kv, torch.tensor([2, 1], dtype=torch.int32)


def test_binding_attention():
    p, q, kv, lens = _host()
    call = lambda q=q, lens=lens, kv=kv, **kw: cc.cc_attention_kv(p, q, kv, 0, lens, 8, **kw)
    for bad in (dict(q=q.float()), dict(q=q[:2]), dict(q=q.transpose(0, 1)), dict(lens=lens.long()), dict(lens=lens[:1]),
                dict(o=torch.empty(3, 4, 64)), dict(o=torch.empty(3, 4, 32, dtype=torch.bfloat16)),
                dict(lse=torch.empty(3, 4, dtype=torch.bfloat16)), dict(lse=torch.empty(3, 3))):
        with pytest.raises(ValueError):
            call(**bad)
    k32 = torch.zeros(2, 2, 8, 64)
    kv32 = cc.kv_contiguous(k32, k32, n_layers=1, seq_stride=1024, layer_stride=0, head_stride=512, tok_stride=64)
    with pytest.raises(ValueError, match="bf16"):
        call(kv=kv32)
    with pytest.raises(ValueError, match="bf16"):
        cc.prefix(kv32, [0, 2], lens[:1], 8)
    with pytest.raises(ValueError, match="GPU"):
        call()


def test_binding_prefix():
    p, q, kv, lens = _host()
    for bad in (dict(first_seq=[0]), dict(first_seq=[0, 1, 2], lens=lens[:1]), dict(lens=lens[:1].long()),
                dict(lens=lens[:1], first_device=torch.tensor([0, 2]))):
        with pytest.raises(ValueError):
            cc.prefix(kv, **{"first_seq": [0, 2], "lens": lens, "max_len": 8, **bad})
    with pytest.raises(ValueError, match="GPU"):
        cc.cc_attention_prefix(p, q, cc.prefix(kv, [0, 2], lens[:1], 8), kv, 0, lens, 8)


def test_binding_weights():
    p, q, kv, lens = _host()
    lse, w = torch.zeros(3, 4), torch.zeros(2, 2, 8)
    call = lambda out=w, lse=lse, **kw: cc.cc_attention_weights(p, q, kv, 0, lens, 8, lse, out, **kw)
    for bad in (dict(out=w.double()), dict(out=w[:, :, :7]), dict(out=w[:1]), dict(out=w.flatten(1)), dict(lse=lse[:2]),
                dict(out=torch.zeros(2, 2, 16)[:, :, ::2]), dict(out=torch.zeros(1, 2, 8).expand(2, 2, 8)),
                dict(out=torch.zeros(30).as_strided((2, 2, 8), (16, 4, 1))),           # heads that overlap
                dict(prev=w.half()), dict(prev_lens=lens), dict(prev=w, prev_lens=lens.long())):
        with pytest.raises(ValueError):
            call(**bad)
    with pytest.raises(ValueError, match="GPU"):
        call()
    pe = cc.problem(dtype="bf16", cu_seqlens=[0, 8, 12], n_heads_q=2, n_heads_kv=2, head_dim=64, hidden=64, vocab=1, device="cpu")
    for bad in (dict(w=w[:, :, :7]), dict(scores=torch.zeros(11)), dict(scores=torch.zeros(12).half()), dict(per_head=1, scores=torch.zeros(12))):
        with pytest.raises(ValueError):
            cc.cc_weight_scores(pe, **{"w": w, "n_recent": 0, "per_head": 0, **bad})
    keep = torch.zeros(4, dtype=torch.int32)
    for bad in (dict(k=[2]), dict(k=[2, 3]), dict(keep_idx=keep.long()), dict(out=w.half()), dict(w=torch.zeros(1, 2, 8).expand(2, 2, 8)),
                dict(out=torch.zeros(2, 2, 1))):
        with pytest.raises(ValueError):
            cc.cc_compact_weights(pe, **{"w": w, "keep_idx": keep, "k": [2, 2], "per_head": 0, **bad})


def test_binding_block_tables():
    """A table with fewer rows than sequences, or prefixes, would be read past its end."""
    p, q, kv, lens = _host()
    pool, lse, w = torch.zeros(4, 16, 2, 64, dtype=torch.bfloat16), torch.zeros(3, 4), torch.zeros(2, 2, 8)
    paged = cc.kv_paged(pool, pool, torch.zeros(1, 1, dtype=torch.int32), n_layers=1, layer_stride=0, page_stride=2048, head_stride=64,
                        tok_stride=128, page_size=16)
    x = cc.prefix(paged, [0, 2], lens[:1], 8)
    for call in (lambda: cc.cc_attention_kv(p, q, paged, 0, lens, 8), lambda: cc.prefix(paged, [0, 1, 2], lens, 8),
                 lambda: cc.cc_attention_prefix(p, q, x, paged, 0, lens, 8),
                 lambda: cc.cc_attention_weights(p, q, paged, 0, lens, 8, lse, w)):
        with pytest.raises(ValueError, match="block table has 1 rows"):
            call()


def test_struct_layouts_match_header(tmp_path):
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    classes = {"cc_prefix": cc.c_prefix, "cc_weights": cc.c_weights}
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "cc.h"', "int main(void){"]
    for name, c in classes.items():
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        lines += [f'printf("%zu\\n", offsetof({name}, {f[0]}));' for f in c._fields_]
    (tmp_path / "x.c").write_text("\n".join([*lines, "return 0;}"]))
    subprocess.run(["gcc", "-I", os.path.join(root, "include"), str(tmp_path / "x.c"), "-o", str(tmp_path / "x")], check=True)
    got = [int(x) for x in subprocess.run([str(tmp_path / "x")], capture_output=True, text=True, check=True).stdout.split()]
    want = []
    for c in classes.values():
        want += [ctypes.sizeof(c), *(getattr(c, f[0]).offset for f in c._fields_)]
    assert got == want


def test_entries_of_weights():
    """Weights that say how many entries they hold are held against what a call reaches; earlier ones with lengths of
    their own are read as far as they go."""
    assert _weights(out=_w(entries=199)) == cc.CC_ERR_SHAPE
    assert _weights(out=_w(entries=-1)) == cc.CC_ERR_SHAPE
    assert _weights(prev=_w(base=2 * P, entries=199)) == cc.CC_ERR_SHAPE
    assert _weights(prev=_w(base=2 * P, entries=-1), prev_lens=P) == cc.CC_ERR_SHAPE
    assert _weights(out=_w(entries=200), prev=_w(base=2 * P, entries=3), prev_lens=P, lse=None) == cc.CC_ERR_ARG     # (as far as lse)
    assert _scores(w=_w(entries=4)) == cc.CC_ERR_SHAPE
    assert _compact(w=_w(entries=4)) == cc.CC_ERR_SHAPE
    assert _compact(out=_w(base=2 * P, entries=1)) == cc.CC_ERR_SHAPE
    assert _compact(w=_w(entries=5), out=_w(base=2 * P, entries=1), k=(0, 0)) == cc.CC_OK
    p, _, _, _ = _host()
    for w in (torch.zeros(2, 2, 8), torch.zeros(2, 2, 16)[:, :, :5], torch.zeros(2, 9, 2).transpose(1, 2)[:, :, :1]):
        assert cc._weights(p, w, "w", 1).entries == w.shape[2]


def _bytes_behind(new, prefix, longest, hq, hkv):
    n, p = ctypes.c_size_t(0), _problem(cu=[sum(new[:i]) for i in range(len(new) + 1)], n_heads_q=hq, n_heads_kv=hkv)
    x = _prefix(first=(0, len(new)), max_len=prefix)
    assert cc._lib.cc_attention_prefix_workspace(_ref(p), _ref(x), longest, ctypes.byref(n)) == cc.CC_OK
    return n.value


@pytest.mark.parametrize("few,many,longest,hq,hkv", [([1], [8000], 16384, 32, 8), ([1] * 40, [8192], 16384, 28, 4),
                                                     ([1] * 40, [16000], 32768, 32, 8), ([6] * 24, [40] * 3, 8000, 32, 8),
                                                     ([1] * 200, [3000, 100], 16384, 28, 4)])
def test_workspace_of_tokens_beside_prompts_behind_a_prefix(few, many, longest, hq, hkv):
    """What one call of both needs is no more than two calls need (results to be joined are those of the rows that have pieces)."""
    alone = _bytes_behind(few, 16000, longest, hq, hkv) + _bytes_behind(many, 16000, longest, hq, hkv)
    for new in (few + many, many + few, few[:1] + many + few[1:]):
        assert _bytes_behind(new, 16000, longest, hq, hkv) <= alone + 4096


def _bytes_of(new, longest, hq, hkv):
    n, p = ctypes.c_size_t(0), _problem(cu=[sum(new[:i]) for i in range(len(new) + 1)], n_heads_q=hq, n_heads_kv=hkv)
    assert cc._lib.cc_attention_kv_workspace(_ref(p), longest, ctypes.byref(n)) == cc.CC_OK
    return n.value


@pytest.mark.parametrize("few,many,longest,hq,hkv", [([1] * 1000, [16], 16384, 32, 8), ([1] * 128, [16], 16384, 28, 4),
                                                     ([2] * 300, [40, 33], 5000, 8, 2), ([1, 0] * 4000, [9] * 30, 60000, 4, 1)])
def test_workspace_of_tokens_beside_a_chunk(few, many, longest, hq, hkv):
    """What one call of both needs is no more than two calls need (results to be joined are those of the rows that are cut), but
    for what the few rows' shares need of every sequence: outputs, (maximum, sum) and a pair of whole numbers."""
    alone = _bytes_of(few, longest, hq, hkv) + _bytes_of(many, longest, hq, hkv)
    alone += len(many) * hkv * (max(few) * hq // hkv * (4 * 128 + 8) + 8)
    for new in (few + many, many + few, few[:7] + many + few[7:]):
        assert _bytes_of(new, longest, hq, hkv) <= alone + 4096
