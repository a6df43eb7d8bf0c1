"""Attention over a bf16 cache, alone and behind shared prefixes, against fp64: prompts, chunks, drafts and single
tokens, ragged batches, every layout, rows that see nothing, NaN and infinities where a row may not look."""
import numpy as np
import pytest
import torch

from oracle import kv16_oracle as O
from tests.gpu_util import assert_attention_close, f64
from tests.kv16_util import Cache16, cu_of, i32, logit_error, problem, queries

pytestmark = pytest.mark.gpu


def _oracle(cache, q, new, lens, hq, hkv, layer=0, scale=None, pre=None, first=None, pre_lens=None):
    """(o [N][Hq][d], lse [N][Hq], error bound of lse [N][Hq])"""
    g, qh, d = hq // hkv, f64(q), cache.d
    o, lse, tol = np.zeros(qh.shape), np.full(qh.shape[:2], -np.inf), np.zeros(qh.shape[:2])
    cu = cu_of(new)
    for b, m in enumerate(new):
        rows = slice(cu[b], cu[b + 1])
        for c in range(hkv if m else 0):
            k, v = (cache.values(layer, b, c, t, lens[b]) for t in "kv")
            kp = vp = None
            if pre is not None:
                i = sum(1 for x in first[1:] if x <= b)
                kp, vp = (pre.values(layer, i, c, t, pre_lens[i]) for t in "kv")
            ks = k if kp is None else np.concatenate([kp, k])
            for h in range(c * g, (c + 1) * g):
                o[rows, h], lse[rows, h] = O.attention(qh[rows, h], k, v, kp, vp, scale)
                tol[rows, h] = logit_error(qh[rows, h], np.nan_to_num(ks, posinf=0, neginf=0),
                                           d ** -0.5 if scale is None else scale)
    return o, lse, tol


def _same(o, lse, want, what=""):
    ro, rl, tol = want
    assert_attention_close(f64(o), ro, what)
    got = f64(lse)
    np.testing.assert_array_equal(np.isneginf(got), np.isneginf(rl), err_msg=what)
    fin = np.isfinite(rl)
    # (and the last rounding of a number of that size, the log's and the sum's)
    err = np.abs(got[fin] - rl[fin])
    bad = err > tol[fin] + 2.0 ** -22 * (1 + np.abs(rl[fin]))
    assert not bad.any(), f"{what}: lse off by {err[bad].max()}"


def _run(cc, cache, q, new, lens, hq, hkv, layer=0, longest=None, pre=None, first=None, pre_lens=None, pre_longest=None, **kw):
    p = problem(cc, new, hq, hkv, cache.d, **kw)
    o = torch.full_like(q, 7.0)
    lse = torch.full(q.shape[:2], 7.0, device="cuda")
    longest = max(lens) if longest is None else longest
    if pre is None:
        cc.cc_attention_kv(p, q, cache.view(cc), layer, i32(lens), longest, o, lse=lse)
    else:
        x = cc.prefix(pre.view(cc), first, i32(pre_lens), max(pre_lens) if pre_longest is None else pre_longest)
        cc.cc_attention_prefix(p, q, x, cache.view(cc), layer, i32(lens), longest, o, lse=lse)
    torch.cuda.synchronize()
    return o, lse


CASES = [
    # new, lens, hq, hkv, d, page
    ([1], [1], 4, 2, 128, 0),
    ([1], [17], 8, 1, 128, 0),
    ([1, 1, 1, 1], [1, 64, 65, 333], 28, 4, 128, 16),
    ([1, 1], [1500, 40], 32, 8, 128, 64),
    ([1, 3, 0, 8], [100, 3, 9, 257], 16, 4, 64, 16),
    ([5], [700], 20, 2, 128, 32),
    ([7], [130], 12, 4, 64, 128),
    ([20, 2], [20, 300], 8, 2, 128, 16),
    ([64], [1000], 4, 4, 128, 64),
    ([130, 33], [130, 500], 14, 2, 128, 16),
    ([200], [321], 8, 8, 64, 0),
    ([257], [257], 4, 2, 64, 32),
    ([300, 1, 0, 77, 640], [300, 1, 5, 77, 640], 4, 1, 128, 16),   # whole prompts, packed
    ([1000], [1000], 2, 1, 128, 0),
    ([63, 64, 65, 127, 128, 129], [63, 64, 65, 127, 128, 129], 2, 2, 64, 64),
    ([1], [50], 64, 1, 128, 16),
]


@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
def test_attention(case):
    from paper_2607_27600_amd import cc
    new, lens, hq, hkv, d, page = case
    print(f"[attn16] {case}", flush=True)
    cache = Cache16(lens, hkv, d, layers=2, page=page, seed=21)
    q = queries(new, hq, d, 22)
    _same(*_run(cc, cache, q, new, lens, hq, hkv, layer=1), _oracle(cache, q, new, lens, hq, hkv, layer=1), str(case))


PREFIXES = [
    # prefix lens, first, new, lens, hq, hkv, d, page
    ([1], [0, 1], [1], [1], 4, 2, 128, 0),
    ([100], [0, 3], [1, 1, 1], [1, 5, 30], 8, 2, 128, 16),
    ([333, 17], [0, 2, 5], [1, 4, 0, 2, 1], [70, 4, 3, 9, 1], 4, 1, 64, 16),
    ([0, 65, 4], [0, 1, 1, 3], [2, 1, 3], [2, 0, 200], 4, 2, 128, 32),      # an empty prefix, one without sequences, no own entries
    ([700], [0, 4], [40, 33, 1, 60], [40, 300, 1, 60], 14, 2, 128, 64),
    ([150, 90], [0, 1, 2], [200, 130], [200, 130], 2, 2, 64, 0),
    ([1300], [0, 20], [1] * 20, [i * 7 % 90 + 1 for i in range(20)], 28, 4, 128, 16),
]


@pytest.mark.parametrize("case", PREFIXES, ids=[str(i) for i in range(len(PREFIXES))])
def test_shared_prefix(case):
    from paper_2607_27600_amd import cc
    pl, first, new, lens, hq, hkv, d, page = case
    print(f"[prefix] {case}", flush=True)
    cache = Cache16(lens, hkv, d, layers=2, page=page, seed=31)
    pre = Cache16(pl, hkv, d, layers=2, page=16 if page else 0, seed=32)
    q = queries(new, hq, d, 33)
    kw = dict(layer=1, pre=pre, first=first, pre_lens=pl)
    _same(*_run(cc, cache, q, new, lens, hq, hkv, **kw), _oracle(cache, q, new, lens, hq, hkv, **kw), str(case))


def test_prefix_equals_one_cache():
    """What a sequence sees behind a prefix is what it sees of one cache that holds both."""
    from paper_2607_27600_amd import cc
    hq, hkv, d, new, lens, n = 8, 2, 128, [3, 1], [50, 9], 100
    one = Cache16([n + x for x in lens], hkv, d, page=16, seed=41)
    pre, own = Cache16([n], hkv, d, page=16, seed=42), Cache16(lens, hkv, d, page=16, seed=43)
    for b, m in enumerate(lens):
        for w in "kv":
            for t in range(n + m):
                src = (pre, 0, t) if t < n else (own, b, t - n)
                pg, sl = src[0]._where(src[1], np.asarray([src[2]]))
                to, at = one._where(b, np.asarray([t]))
                one.t[w][0, int(to[0]), :, int(at[0]), :d] = src[0].t[w][0, int(pg[0]), :, int(sl[0]), :d]
    q = queries(new, hq, d, 44)
    want = _oracle(one, q, new, [n + x for x in lens], hq, hkv)
    _same(*_run(cc, own, q, new, lens, hq, hkv, pre=pre, first=[0, 2], pre_lens=[n]), want)
    _same(*_run(cc, one, q, new, [n + x for x in lens], hq, hkv), want)


@pytest.mark.parametrize("new,d", [([3, 5, 2], 128), ([100, 5, 70], 128), ([100, 90, 2], 64)])
def test_rows_that_see_nothing(new, d):
    """More queries than entries: those that stand before the first see nothing, or their prefix alone."""
    from paper_2607_27600_amd import cc
    hq, hkv, lens = 4, 2, [2, 0, 1]
    cache = Cache16(lens, hkv, d, page=16, seed=25)
    q = queries(new, hq, d, 26)
    o, lse = _run(cc, cache, q, new, lens, hq, hkv, longest=16)
    want = _oracle(cache, q, new, lens, hq, hkv)
    _same(o, lse, want)
    empty = np.isneginf(want[1])
    assert empty.any() and np.all(f64(o)[empty] == 0)
    pre = Cache16([0, 40], hkv, d, page=16, seed=27)
    kw = dict(pre=pre, first=[0, 1, 3], pre_lens=[0, 40])
    _same(*_run(cc, cache, q, new, lens, hq, hkv, longest=16, **kw), _oracle(cache, q, new, lens, hq, hkv, **kw))


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("new,n", [([4], 100), ([40], 200), ([150], 150), ([33], 33)])
@pytest.mark.parametrize("d", [128, 64])
def test_what_is_not_finite_reaches_only_rows_that_see_it(new, n, d, value):
    from paper_2607_27600_amd import cc
    hq, hkv, m = 4, 2, new[0]
    print(f"[attn16 nan] {new} {n} {d} {value}", flush=True)
    cache = Cache16([n], hkv, d, page=16, seed=27)
    # a value in one dim, and a NaN key, in entries that only some of the queries see; a value in the last entry
    tv, tk = n - 2, n - 1 - m // 2
    q = queries(new, hq, d, 28)
    clean = _oracle(cache, q, new, [n], hq, hkv)
    cache.put(0, 0, 0, "v", tv, 5, value)
    cache.put(0, 0, 0, "v", n - 1, d - 1, -value)
    cache.put(0, 0, 1, "k", tk, 9, float("nan"))
    o, lse = _run(cc, cache, q, new, [n], hq, hkv)
    o, lse = f64(o), f64(lse)
    at = np.arange(m) + n - m
    hit = np.zeros(o.shape, bool)
    hit[np.ix_(at >= tv, [0, 1], [5])] = True
    hit[np.ix_(at >= n - 1, [0, 1], [d - 1])] = True
    if not np.isnan(value):
        assert np.all(o[np.ix_(at >= tv, [0, 1], [5])] == value) and np.all(o[np.ix_(at >= n - 1, [0, 1], [d - 1])] == -value)
    hit[np.ix_(at >= tk, [2, 3])] = True
    np.testing.assert_array_equal(~np.isfinite(o), hit)
    np.testing.assert_array_equal(np.isnan(lse), np.broadcast_to((at >= tk)[:, None] & (np.arange(hq) >= 2), lse.shape))
    assert_attention_close(np.where(hit, 0, o), np.where(hit, 0, clean[0]))


def test_lengths_on_the_device_in_a_graph():
    """A captured call follows its lengths, the prefix's too; lengths beyond the plan are cut to it, negative ones empty."""
    from paper_2607_27600_amd import cc
    hq, hkv, d, new = 8, 2, 128, [1, 1, 40]
    cache = Cache16([600, 300, 77], hkv, d, page=16, seed=32, room=600)
    pre = Cache16([500], hkv, d, page=16, seed=33, room=16)
    q = queries(new, hq, d, 34)
    p = problem(cc, new, hq, hkv, d)
    kv, lens, plens = cache.view(cc), i32([1, 1, 40]), i32([1])
    x = cc.prefix(pre.view(cc), [0, 3], plens, 500)
    need = max(cc.cc_attention_kv_workspace(p, 600), cc.cc_attention_prefix_workspace(p, x, 600))
    ws = torch.empty(max(1, need), dtype=torch.uint8, device="cuda")
    o, o2 = torch.empty_like(q), torch.empty_like(q)
    lse, lse2 = torch.empty(42, hq, device="cuda"), torch.empty(42, hq, device="cuda")

    def calls():
        cc.cc_attention_kv(p, q, kv, 0, lens, 600, o, lse=lse, workspace=ws)
        cc.cc_attention_prefix(p, q, x, kv, 0, lens, 600, o2, lse=lse2, workspace=ws)
    calls()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        calls()
    for now, pn in (([600, 300, 77], 500), ([1, 17, 40], 0), ([599, 0, 3], 10**6), ([10**6, -5, 77], -3)):
        lens.copy_(i32(now))
        plens.fill_(pn)
        for t in (o, o2, lse, lse2):
            t.fill_(3.0)
        ws.fill_(0x7f)
        g.replay()
        torch.cuda.synchronize()
        real, pr = [min(max(x, 0), 600) for x in now], [min(max(pn, 0), 500)]
        _same(o, lse, _oracle(cache, q, new, real, hq, hkv), str(now))
        _same(o2, lse2, _oracle(cache, q, new, real, hq, hkv, pre=pre, first=[0, 3], pre_lens=pr), f"{now} {pn}")


def test_many_sequences():
    """More sequences, and more prefixes, than any list by value holds."""
    from paper_2607_27600_amd import cc
    hq, hkv, d = 4, 2, 64
    r = np.random.default_rng(34)
    new = [int(x) for x in r.choice([0, 1, 1, 2, 40], 150)]
    lens = [m + int(x) for m, x in zip(new, r.integers(0, 60, 150))]
    cache = Cache16(lens, hkv, d, page=16, seed=35)
    q = queries(new, hq, d, 36)
    _same(*_run(cc, cache, q, new, lens, hq, hkv), _oracle(cache, q, new, lens, hq, hkv))
    pl = [int(x) for x in r.integers(0, 50, 70)]
    first = [0, *sorted(int(x) for x in r.integers(0, 151, 69)), 150]
    pre = Cache16(pl, hkv, d, page=16, seed=37)
    kw = dict(pre=pre, first=first, pre_lens=pl)
    _same(*_run(cc, cache, q, new, lens, hq, hkv, **kw), _oracle(cache, q, new, lens, hq, hkv, **kw))


@pytest.mark.parametrize("scale", [1.0, 0.01, 1e-20, 1e-38, 1e-40])
@pytest.mark.parametrize("new,lens,hq,hkv,d", [([1, 3], [200, 77], 8, 2, 128), ([70, 40], [300, 90], 4, 2, 64)])
def test_a_scale_of_the_callers(new, lens, hq, hkv, d, scale):
    from paper_2607_27600_amd import cc
    cache = Cache16(lens, hkv, d, page=16, seed=101)
    q = queries(new, hq, d, 102)
    _same(*_run(cc, cache, q, new, lens, hq, hkv, softmax_scale=scale), _oracle(cache, q, new, lens, hq, hkv, scale=scale))


@pytest.mark.parametrize("new,lens,hq,hkv,d,page", [([1], [9000], 4, 1, 128, 16), ([1, 1], [5001, 37], 4, 2, 64, 64),
                                                    ([70], [4100], 2, 1, 128, 16), ([300, 1], [3000, 2500], 2, 2, 64, 0),
                                                    ([40, 200, 0, 90], [40, 2000, 7, 90], 4, 1, 128, 32),
                                                    ([700], [700], 2, 1, 128, 128), ([33] * 20, [33 + 90 * i for i in range(20)], 2, 1, 64, 16)])
def test_pieces(new, lens, hq, hkv, d, page):
    """Long caches of few heads are cut into pieces and joined; the plan may reach beyond the longest.  The workspace holds
    no more than asked for, and the same call repeats bit for bit."""
    from paper_2607_27600_amd import cc
    print(f"[attn16 pieces] {new} {lens} {hq} {hkv} {d} {page}", flush=True)
    cache = Cache16(lens, hkv, d, page=page, seed=23, room=5000)
    q = queries(new, hq, d, 24)
    want = _oracle(cache, q, new, lens, hq, hkv)
    p, kv = problem(cc, new, hq, hkv, d), cache.view(cc)
    for longest in (max(lens), max(lens) + 4321):
        size = cc.cc_attention_kv_workspace(p, longest)
        ws = torch.full((size + 4096,), 0x7f, dtype=torch.uint8, device="cuda")
        got = []
        for _ in range(2):
            o, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
            cc.cc_attention_kv(p, q, kv, 0, i32(lens), longest, o, lse=lse, workspace=ws[:size])
            torch.cuda.synchronize()
            _same(o, lse, want, str(longest))
            got.append((o, lse))
        assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
        assert (ws[size:] == 0x7f).all()


LONG_PREFIXES = [
    # prefix lens, first, new, lens, hq, hkv, d, page: cut into pieces on the device, two and more row blocks, few and many rows behind
    ([5000], [0, 40], [1] * 40, [1 + 13 * i % 200 for i in range(40)], 8, 2, 128, 16),
    ([3000, 700, 0, 1500], [0, 9, 9, 12, 30], [6, 0, 1] * 10, [6 + 29 * i % 300 for i in range(30)], 16, 4, 64, 64),
    ([2500, 40], [0, 3, 6], [40, 200, 1, 90, 2, 64], [40, 900, 2500, 90, 3, 64], 4, 1, 128, 32),
    ([1200], [0, 2], [1, 1], [9000, 12], 4, 1, 128, 16),             # own entries that are cut too
    ([1100] * 70, list(range(71)), [1] * 70, [1 + i % 9 for i in range(70)], 2, 1, 64, 0),
    ([2000], [0, 1], [700], [700], 32, 8, 64, 16),
    ([1500], [0, 3], [700, 900, 1000], [700, 900, 1000], 16, 16, 64, 128),   # more (row block, head)s than workgroups at a time
]


@pytest.mark.parametrize("case", LONG_PREFIXES, ids=[str(i) for i in range(len(LONG_PREFIXES))])
def test_long_shared_prefix(case):
    from paper_2607_27600_amd import cc
    pl, first, new, lens, hq, hkv, d, page = case
    print(f"[prefix long] {case}", flush=True)
    cache = Cache16(lens, hkv, d, page=page, seed=61, room=400)
    pre = Cache16(pl, hkv, d, page=64 if page else 0, seed=62, room=700)
    q = queries(new, hq, d, 63)
    p, kv = problem(cc, new, hq, hkv, d), cache.view(cc)
    want = _oracle(cache, q, new, lens, hq, hkv, pre=pre, first=first, pre_lens=pl)
    for more in (0, 333):
        x = cc.prefix(pre.view(cc), first, i32(pl), max(pl) + more)
        size = cc.cc_attention_prefix_workspace(p, x, max(lens) + more)
        ws = torch.full((size + 4096,), 0x7f, dtype=torch.uint8, device="cuda")
        got = []
        for _ in range(2):
            o, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
            cc.cc_attention_prefix(p, q, x, kv, 0, i32(lens), max(lens) + more, o, lse=lse, workspace=ws[:size])
            torch.cuda.synchronize()
            _same(o, lse, want, str(more))
            got.append((o, lse))
        assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
        assert (ws[size:] == 0x7f).all()


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("n", [300, 3000])
def test_what_is_not_finite_in_a_prefix(n, value):
    """It reaches the rows of its run, and no others; what lies past a prefix reaches none."""
    from paper_2607_27600_amd import cc
    hq, hkv, d, new, lens = 4, 2, 128, [1, 40, 2, 3], [7, 40, 2, 30]
    cache, pre = Cache16(lens, hkv, d, page=16, seed=64), Cache16([n, n - 9], hkv, d, page=16, seed=65)
    q = queries(new, hq, d, 66)
    kw = dict(pre=pre, first=[0, 2, 4], pre_lens=[n, n - 9])
    clean = _oracle(cache, q, new, lens, hq, hkv, **kw)[0]
    pre.put(0, 1, 1, "v", n - 11, 17, value)
    o = f64(_run(cc, cache, q, new, lens, hq, hkv, **kw)[0])
    hit = np.zeros(o.shape, bool)
    hit[41:, 2:, 17] = True
    np.testing.assert_array_equal(~np.isfinite(o), hit)
    assert_attention_close(np.where(hit, 0, o), np.where(hit, 0, clean))


def test_a_plan_for_no_entries():
    """max_kv_len 0: every length is cut to it, every output is zero and no page is looked up; the prefix alone is seen."""
    from paper_2607_27600_amd import cc
    new, hq, hkv, d = [1, 40, 2, 300], 4, 2, 128
    cache = Cache16([9, 40, 2, 300], hkv, d, page=16, seed=61)
    cache.bt.fill_(-(1 << 30))
    q = queries(new, hq, d, 62)
    o, lse = _run(cc, cache, q, new, [9, 40, 2, 300], hq, hkv, longest=0)
    assert torch.count_nonzero(o) == 0 and torch.isneginf(lse).all()
    for n in (50, 3000):
        pre = Cache16([n], hkv, d, page=16, seed=63)
        kw = dict(pre=pre, first=[0, 4], pre_lens=[n])
        o, lse = _run(cc, cache, q, new, [9, 40, 2, 300], hq, hkv, longest=0, **kw)
        empty = Cache16([0] * 4, hkv, d, page=16, seed=64)
        _same(o, lse, _oracle(empty, q, new, [0] * 4, hq, hkv, **kw))
    pre.bt.fill_(-(1 << 30))
    o, lse = _run(cc, cache, q, new, [9, 40, 2, 300], hq, hkv, longest=0, pre_longest=0, **kw)
    assert torch.count_nonzero(o) == 0 and torch.isneginf(lse).all()


@pytest.mark.parametrize("new", [[1], [40], [150], [1, 3, 200]])
@pytest.mark.parametrize("prefix", [0, 60, 2000])
def test_a_query_that_is_not_finite(new, prefix):
    """It spoils its own outputs and no other row's."""
    from paper_2607_27600_amd import cc
    hq, hkv, d = 4, 2, 128
    lens = [m + 30 for m in new]
    cache = Cache16(lens, hkv, d, page=16, seed=67)
    q = queries(new, hq, d, 68)
    kw = dict(pre=Cache16([prefix], hkv, d, page=16, seed=69), first=[0, len(new)], pre_lens=[prefix]) if prefix else {}
    want, lse, tol = _oracle(cache, q, new, lens, hq, hkv, **kw)
    q[sum(new) // 2, 1, 7] = float("nan")
    o, got = _run(cc, cache, q, new, lens, hq, hkv, **kw)
    hit = np.zeros(lse.shape, bool)
    hit[sum(new) // 2, 1] = True
    np.testing.assert_array_equal(np.isnan(f64(got)), hit)
    np.testing.assert_array_equal(np.isnan(f64(o)), np.broadcast_to(hit[..., None], want.shape))
    assert_attention_close(np.where(hit[..., None], 0, f64(o)), np.where(hit[..., None], 0, want))


@pytest.mark.parametrize("new,hq,hkv,d", [([8] * 3, 16, 4, 128), ([8, 5], 16, 4, 64), ([1] * 40, 8, 8, 128)])
def test_few_rows_in_a_graph(new, hq, hkv, d):
    """Shares of the work of one and two row blocks, captured and replayed as the lengths change, from pieces to shares."""
    from paper_2607_27600_amd import cc
    cache = Cache16([3000] * len(new), hkv, d, page=16, seed=71)
    q, kv, lens = queries(new, hq, d, 72), cache.view(cc), i32([2000] * len(new))
    p = problem(cc, new, hq, hkv, d)
    o, lse = torch.empty_like(q), torch.empty(sum(new), hq, device="cuda")
    ws = torch.empty(max(1, cc.cc_attention_kv_workspace(p, 3000)), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        cc.cc_attention_kv(p, q, kv, 0, lens, 3000, o, lse=lse, workspace=ws)
    r = np.random.default_rng(73)
    for most in (3000, 45, 700, 2999):
        now = [int(x) for x in r.integers(min(most, 8), most + 1, len(new))]
        lens.copy_(i32(now))
        o.fill_(9.0)
        ws.fill_(0x7f)
        g.replay()
        torch.cuda.synchronize()
        _same(o, lse, _oracle(cache, q, new, now, hq, hkv), str(most))


@pytest.mark.parametrize("n,most,hkv", [(150, 5000, 2), (700, 3000, 1), (70, 4000, 3)])
def test_shares_of_many_sequences(n, most, hkv):
    """Work shared out over more sequences than a wave has lanes and than are listed; rows whose entries lie in one share,
    in a few and in many."""
    from paper_2607_27600_amd import cc
    d, hq = 64, 2 * hkv
    r = np.random.default_rng(n)
    new = [int(x) for x in r.choice([0, 1, 1, 3], n)]
    lens = [m + int(x) for m, x in zip(new, r.integers(0, 30, n))]
    lens[n // 3], lens[n - 1], new[n // 3], new[n - 1] = most, most - 1, 1, 2
    new[5], lens[5] = 40, 500            # one of many rows
    cache = Cache16(lens, hkv, d, page=16 if n == 150 else 0, seed=n + 1, fill=0.0)
    q = queries(new, hq, d, n + 2)
    want = _oracle(cache, q, new, lens, hq, hkv)
    _same(*_run(cc, cache, q, new, lens, hq, hkv), want)


def test_two_calls_at_once():
    """Two streams, each with its own workspace and outputs; nothing is shared."""
    from paper_2607_27600_amd import cc
    hq, hkv, d, new, lens = 8, 2, 128, [1, 40, 3], [3000, 900, 2500]
    cache, pre = Cache16(lens, hkv, d, page=16, seed=75), Cache16([2000], hkv, d, page=16, seed=76)
    qs = [queries(new, hq, d, s) for s in (77, 78)]
    p, kv, x, ld = problem(cc, new, hq, hkv, d), cache.view(cc), cc.prefix(pre.view(cc), [0, 3], i32([2000]), 2000), i32(lens)
    want = [(cc.cc_attention_kv(p, q, kv, 0, ld, 3000), cc.cc_attention_prefix(p, q, x, kv, 0, ld, 3000)) for q in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in qs]
    got = []
    for _ in range(5):
        for q, s in zip(qs, streams):
            got.append((cc.cc_attention_kv(p, q, kv, 0, ld, 3000, stream=s), cc.cc_attention_prefix(p, q, x, kv, 0, ld, 3000, stream=s)))
    torch.cuda.synchronize()
    for i, pair in enumerate(got):
        for a, b in zip(pair, want[i % 2]):
            assert torch.equal(a, b)


@pytest.mark.parametrize("new", [1, 40])
def test_offsets_past_32_bits(new, memory_given_back):
    """Entries 64 KiB apart, the ones that count beyond 4 GiB of their plane."""
    from paper_2607_27600_amd import cc
    n, d, hq, tok = 70000, 64, 4, 1 << 15
    free, _ = torch.cuda.mem_get_info()
    if free < (14 << 30):
        pytest.skip("needs 14 GiB of device memory")
    pools = {t: torch.zeros(n * tok, dtype=torch.bfloat16, device="cuda") for t in "kv"}
    rows = {t: x.view(n, tok)[:, :d] for t, x in pools.items()}
    g = torch.Generator().manual_seed(79)
    head, tail = 48, 500
    for t in "kv":
        rows[t][:head] = torch.randn(head, d, generator=g).to(torch.bfloat16).cuda()
        rows[t][n - tail:] = torch.randn(tail, d, generator=g).to(torch.bfloat16).cuda()
    rows["k"][head:n - tail] = -300.0            # (so far from the queries that they weigh nothing)
    q = torch.randn(new, hq, d, generator=g).abs().to(torch.bfloat16).cuda()
    kv = cc.kv_contiguous(pools["k"], pools["v"], n_layers=1, layer_stride=0, head_stride=0, tok_stride=tok)
    p, lens = problem(cc, [new], hq, 1, d), i32([n])
    lse = torch.empty(new, hq, device="cuda")
    o = cc.cc_attention_kv(p, q, kv, 0, lens, n, lse=lse)
    w = cc.cc_attention_weights(p, q, kv, 0, lens, n, lse, torch.full((1, 1, n), 7.0, device="cuda"))
    torch.cuda.synchronize()
    ends = np.r_[0:head, n - tail:n]
    k, v, qh = (f64(rows[t][torch.from_numpy(ends).cuda()]) for t in "kv"), None, f64(q)
    k, v = k
    ref, sums = np.zeros((new, hq, d)), np.zeros(len(ends))
    for h in range(hq):
        ref[:, h], r = O.attention(qh[:, h], k, v)
        sums += O.weights(qh[:, h], k, r)
    assert_attention_close(f64(o), ref)
    got = f64(w)[0, 0]
    np.testing.assert_allclose(got[ends], sums, rtol=2.0 ** -12, atol=1e-9)
    assert np.all(got[head:n - tail] == 0)
    # as a prefix
    x = cc.prefix(kv, [0, 1], lens, n)
    one = cc.kv_contiguous(pools["k"], pools["v"], n_layers=1, layer_stride=0, head_stride=0, tok_stride=tok)
    o = cc.cc_attention_prefix(p, q, x, one, 0, i32([0]), 0)
    torch.cuda.synchronize()
    full = np.stack([O.attention(qh[:, h], np.zeros((0, d)), np.zeros((0, d)), k, v)[0] for h in range(hq)], 1)
    assert_attention_close(f64(o), full)


@pytest.mark.parametrize("new,lens,hq,hkv,d,page", [
    ([1500, 1, 3, 700, 0], [1500, 1, 3, 700, 40], 28, 4, 128, 16),
    ([1, 1200, 2], [1199, 1200, 2], 4, 1, 64, 0),                       # a token behind as many entries as a prompt has
    ([300] + [40, 1] * 24 + [1100], [300] + [40, 1] * 24 + [1100], 8, 2, 64, 16),   # more than a launch lists
    ([1100] + [1] * 40, [1100] + list(range(1, 41)), 8, 2, 128, 32),    # more short ones than go along
])
@pytest.mark.parametrize("more", [0, 300])
def test_short_prompts_beside_long_ones(new, lens, hq, hkv, d, page, more):
    """Sequences of few rows in a call of prompts, which go along with them where no cache is longer than a prompt."""
    from paper_2607_27600_amd import cc
    cache = Cache16(lens, hkv, d, page=page, seed=91, room=more)
    q = queries(new, hq, d, 92)
    want = _oracle(cache, q, new, lens, hq, hkv)
    _same(*_run(cc, cache, q, new, lens, hq, hkv, longest=max(lens) + more), want)


MIXED_PREFIXES = [
    # prefix lens, first, new, lens, hq, hkv, d, page: few rows in pieces, among others, more sequences than a wave has lanes
    ([700, 1500], [0, 60, 150], [1, 40, 0, 2, 1] * 30, [1 + 41 * i % 1400 for i in range(150)], 4, 2, 64, 16),
    ([2000], [0, 90], [0] * 30 + [300] + [1, 3] * 29 + [0], [5] * 30 + [300] + [3 + 57 * i % 2100 for i in range(58)] + [9], 8, 2, 128, 64),
    ([1100], [0, 5], [1, 0, 500, 4, 1], [1900, 7, 500, 40, 1100], 28, 4, 128, 0),
    ([1200, 0], [0, 200, 300], [0] * 130 + [2] * 100 + [33] * 5 + [0] * 65, [1 + 11 * i % 900 for i in range(300)], 4, 1, 64, 16),
]


@pytest.mark.parametrize("case", MIXED_PREFIXES, ids=[str(i) for i in range(len(MIXED_PREFIXES))])
def test_few_rows_beside_many_behind_a_prefix(case):
    """The workspace holds no more than asked for, whose results to be joined are those of the few rows alone."""
    from paper_2607_27600_amd import cc
    pl, first, new, lens, hq, hkv, d, page = case
    print(f"[prefix mixed] {case[:2]} {hq} {hkv} {d} {page}", flush=True)
    cache = Cache16(lens, hkv, d, page=page, seed=103)
    pre = Cache16(pl, hkv, d, page=16 if page else 0, seed=104)
    q = queries(new, hq, d, 105)
    p, kv, x = problem(cc, new, hq, hkv, d), cache.view(cc), cc.prefix(pre.view(cc), first, i32(pl), max(pl))
    want = _oracle(cache, q, new, lens, hq, hkv, pre=pre, first=first, pre_lens=pl)
    size = cc.cc_attention_prefix_workspace(p, x, max(lens))
    ws = torch.full((size + 4096,), 0x7f, dtype=torch.uint8, device="cuda")
    o, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
    cc.cc_attention_prefix(p, q, x, kv, 0, i32(lens), max(lens), o, lse=lse, workspace=ws[:size])
    torch.cuda.synchronize()
    _same(o, lse, want)
    assert (ws[size:] == 0x7f).all()


@pytest.mark.parametrize("new,most,hq,hkv,d,page", [([1] * 20 + [40] + [1, 0, 2] * 10, 5000, 4, 1, 128, 16),
                                                    ([2] * 100 + [70] + [1, 0] * 30, 4000, 8, 2, 64, 64),        # more than a wave has lanes
                                                    ([0] * 70 + [1] * 90 + [33, 300] + [3] * 140, 6000, 4, 1, 64, 0),
                                                    ([1, 40] * 18 + [1] * 300, 3000, 2, 1, 128, 32)])            # more than a launch lists
def test_pieces_beside_few_rows(new, most, hq, hkv, d, page):
    """Chunks in pieces among single tokens and drafts: the workspace holds no more than asked for, whose results to be joined
    are those of the chunks alone."""
    from paper_2607_27600_amd import cc
    lens = [most - 3 * i if m * hq // hkv > 32 else m + 7 * i % 60 for i, m in enumerate(new)]
    print(f"[attn16 mixed] {len(new)} {most} {hq} {hkv} {d} {page}", flush=True)
    cache = Cache16(lens, hkv, d, page=page, seed=106, fill=0.0)
    q = queries(new, hq, d, 107)
    p = problem(cc, new, hq, hkv, d)
    most = max(lens)
    size = cc.cc_attention_kv_workspace(p, most)
    ws = torch.full((size + 4096,), 0x7f, dtype=torch.uint8, device="cuda")
    o, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
    cc.cc_attention_kv(p, q, cache.view(cc), 0, i32(lens), most, o, lse=lse, workspace=ws[:size])
    torch.cuda.synchronize()
    _same(o, lse, _oracle(cache, q, new, lens, hq, hkv))
    assert (ws[size:] == 0x7f).all()


@pytest.mark.parametrize("new,most,hq,hkv,d", [([16] + [1] * 50 + [16], 4000, 28, 4, 128), ([0, 40] + [1] * 200 + [40, 9, 2], 3000, 4, 1, 64),
                                               ([1] * 70 + [33, 2] * 2 + [3, 0, 1] * 60 + [50] + [1] * 5, 3000, 8, 2, 128)])
@pytest.mark.parametrize("prefix", [0, 1500])
def test_chunks_in_pieces_on_either_side_of_tokens(new, most, hq, hkv, d, prefix):
    """More rows of single tokens between the first and the last chunk than the chunks have: places for the chunks' alone."""
    from paper_2607_27600_amd import cc
    g = hq // hkv
    lens = [most - 5 * (i % 40) if m * g > 32 else m + 7 * i % 60 for i, m in enumerate(new)]
    print(f"[attn16 scattered] {len(new)} {most} {hq} {hkv} {d} {prefix}", flush=True)
    cache, q, p = Cache16(lens, hkv, d, page=16, seed=108, fill=0.0), queries(new, hq, d, 109), problem(cc, new, hq, hkv, d)
    most, kw = max(lens), {}
    o, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
    if prefix:
        pre = Cache16([prefix], hkv, d, page=16, seed=110)
        kw = dict(pre=pre, first=[0, len(new)], pre_lens=[prefix])
        x = cc.prefix(pre.view(cc), [0, len(new)], i32([prefix]), prefix)
        size = cc.cc_attention_prefix_workspace(p, x, most)
    else:
        size = cc.cc_attention_kv_workspace(p, most)
    ws = torch.full((size + 4096,), 0x7f, dtype=torch.uint8, device="cuda")
    if prefix:
        cc.cc_attention_prefix(p, q, x, cache.view(cc), 0, i32(lens), most, o, lse=lse, workspace=ws[:size])
    else:
        cc.cc_attention_kv(p, q, cache.view(cc), 0, i32(lens), most, o, lse=lse, workspace=ws[:size])
    torch.cuda.synchronize()
    _same(o, lse, _oracle(cache, q, new, lens, hq, hkv, **kw))
    assert (ws[size:] == 0x7f).all()


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("new,n,prefix", [([4], 900, 0), ([150], 700, 0), ([40], 5000, 0), ([1, 200, 3], 300, 1500), ([2, 70], 90, 2000)])
@pytest.mark.parametrize("d", [128, 64])
def test_a_key_that_is_not_finite_and_seen_by_all(new, n, prefix, d, value):
    """NaN logits spoil their rows, infinite ones those that they draw; what they repel sees the other entries."""
    from paper_2607_27600_amd import cc
    hq, hkv, lens = 4, 2, [n] * len(new)
    cache, q = Cache16(lens, hkv, d, page=16, seed=111), queries(new, hq, d, 112)
    kw = dict(pre=Cache16([prefix], hkv, d, page=16, seed=113), first=[0, len(new)], pre_lens=[prefix]) if prefix else {}
    clean, clean_lse, tol = _oracle(cache, q, new, lens, hq, hkv, **kw)
    where = kw["pre"] if prefix else cache
    for b in range(len(where.lens)):
        where.put(0, b, 1, "k", 37, 5, value)
    o, lse = (f64(x) for x in _run(cc, cache, q, new, lens, hq, hkv, **kw))
    # the entry's logit, of the second KV head's rows: NaN, drawn (+inf) or repelled (-inf)
    z = f64(q)[:, 2:, 5] * value
    spoilt = np.zeros(lse.shape, bool)
    spoilt[:, 2:] = ~np.isneginf(z)
    np.testing.assert_array_equal(np.isnan(lse), spoilt)
    np.testing.assert_array_equal(np.isnan(o), np.broadcast_to(spoilt[..., None], o.shape))
    want, rl, _ = _oracle(cache, q, new, lens, hq, hkv, **kw)
    assert_attention_close(np.where(spoilt[..., None], 0, o), np.where(spoilt[..., None], 0, want))
    assert np.all(np.abs(lse - rl)[~spoilt] <= (tol + 2.0 ** -22 * (1 + np.abs(clean_lse)))[~spoilt])


@pytest.mark.parametrize("prefix", [0, 1100])
def test_thousands_of_sequences(prefix):
    """More sequences than 64 groups of 64: tokens and drafts among sequences without queries, between chunks that are planned
    in pieces."""
    from paper_2607_27600_amd import cc
    hq, hkv, d, n = 4, 1, 64, 5000
    r = np.random.default_rng(114)
    new = [int(x) for x in r.choice([0, 0, 0, 1, 2], n)]
    for b in (3, 64, 4097, 4990):
        new[b] = 33 + b % 7
    lens = [m + int(x) for m, x in zip(new, r.integers(0, 25, n))]
    cache, q, p = Cache16(lens, hkv, d, seed=115, fill=0.0), queries(new, hq, d, 116), problem(cc, new, hq, hkv, d)
    kw = dict(pre=Cache16([prefix], hkv, d, page=16, seed=117), first=[0, n], pre_lens=[prefix]) if prefix else {}
    longest = 5000                       # (a contiguous cache may be planned for more than its sequences have)
    size = cc.cc_attention_kv_workspace(p, longest)
    if prefix:
        x = cc.prefix(kw["pre"].view(cc), [0, n], i32([prefix]), prefix)
        size = cc.cc_attention_prefix_workspace(p, x, longest)
    ws = torch.full((size + 4096,), 0x7f, dtype=torch.uint8, device="cuda")
    o, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
    if prefix:
        cc.cc_attention_prefix(p, q, x, cache.view(cc), 0, i32(lens), longest, o, lse=lse, workspace=ws[:size])
    else:
        cc.cc_attention_kv(p, q, cache.view(cc), 0, i32(lens), longest, o, lse=lse, workspace=ws[:size])
    torch.cuda.synchronize()
    _same(o, lse, _oracle(cache, q, new, lens, hq, hkv, **kw))
    assert (ws[size:] == 0x7f).all()
