"""Log-probabilities, entropies and alternatives of the LM head against fp64."""
import numpy as np
import pytest
import torch

from oracle import cc_oracle as O
from tests.gpu_util import f64

pytestmark = pytest.mark.gpu

# The inputs lie on a grid (u in steps of 1/16, w of 2^-11), so that every logit is exact in fp32 in
# any order and the order of the alternatives, ties included, belongs to the inputs.  What remains:
# a term's exponent z log2(e) - m is rounded at 2^-24 of up to 64 (4e-6 of the term), its
# exponential and the fp32 sums at some 2^-23, the logarithm and the last difference at 2^-23 of up to 64:
# under 2e-5; an entropy weighs its terms with up to 20 nats: five times that.
TOL, TOL_H = 2e-5, 1e-4


def _grid(n, D, V, seed, wide=1.0):
    g = torch.Generator().manual_seed(seed)
    u = (torch.randn(n, D, generator=g) * 16 * wide).round().clamp(-255, 255) / 16
    w = (torch.randn(V, D, generator=g) * 41).round().clamp(-255, 255) / 2048
    ids = torch.randint(0, V, (n,), generator=g, dtype=torch.int32)
    return u.to(torch.bfloat16), w.to(torch.bfloat16), ids


def _call(cc, u, w, ids, top, packed=False, out=None):
    V = w.shape[0]
    wd = w.cuda()
    if packed:
        wd = cc.cc_pack_lmhead(wd)
    r = cc.cc_lmhead_logprobs("bf16", u.cuda(), wd, V, None if ids is None else ids.cuda(), top, out, packed=packed)
    torch.cuda.synchronize()
    return r


def _check(r, u, w, ids, top):
    want = O.logprobs(f64(u), f64(w), None if ids is None else ids.numpy(), top)
    if ids is not None:
        np.testing.assert_allclose(f64(r.logprob), want["logprob"], rtol=0, atol=TOL)
        assert np.all(f64(r.logprob) <= 0)
    np.testing.assert_allclose(f64(r.entropy), want["entropy"], rtol=0, atol=TOL_H)
    assert np.all(f64(r.entropy) >= 0)
    if top:
        np.testing.assert_array_equal(r.top_ids.cpu().numpy()[:, :top], want["top_ids"])
        np.testing.assert_allclose(f64(r.top_logprob), want["top_logprob"], rtol=0, atol=TOL)


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("n,D,V,top", [(1, 64, 1, 1), (1, 64, 5, 5), (3, 128, 1000, 0), (17, 256, 1000, 1), (64, 192, 4099, 8),
                                       (65, 512, 257, 32), (200, 128, 20000, 5), (257, 64, 300, 20), (1000, 64, 2500, 3)])
def test_logprobs(n, D, V, top, packed):
    from paper_2607_27600_amd import cc
    print(f"[logprobs] {n} {D} {V} {top} packed={packed}", flush=True)
    u, w, ids = _grid(n, D, V, n + V)
    _check(_call(cc, u, w, ids, top, packed), u, w, ids, top)


def test_rows_beyond_a_slab():
    from paper_2607_27600_amd import cc
    u, w, ids = _grid(4500, 64, 700, 3)
    _check(_call(cc, u, w, ids, 4), u, w, ids, 4)


def test_no_ids_and_peaked_rows():
    from paper_2607_27600_amd import cc
    u, w, _ = _grid(70, 256, 3001, 4, wide=8.0)
    r = _call(cc, u, w, None, 6)
    _check(r, u, w, None, 6)


@pytest.mark.parametrize("order", ["equal", "falling", "rising", "few"])
def test_ties_and_orders(order):
    """All logits equal (the lowest ids first), rising or falling with the id, a handful of values."""
    from paper_2607_27600_amd import cc
    V, D, n, top = 3000, 64, 33, 32
    w = torch.zeros(V, D)
    v = torch.arange(V)
    if order == "falling":
        w[:, 0], w[:, 1] = -(v // 64).float(), -(v % 64).float() / 64
    elif order == "rising":
        w[:, 0], w[:, 1] = (v // 64).float(), (v % 64).float() / 64
    elif order == "few":
        w[:, 0] = (v % 7 == 3).float() - (v % 5 == 0).float()
    u = torch.zeros(n, D)
    u[:, 0] = u[:, 1] = 1
    u[1::2] *= -1
    u, w = u.to(torch.bfloat16), w.to(torch.bfloat16)
    ids = torch.arange(n, dtype=torch.int32) * 90
    _check(_call(cc, u, w, ids, top), u, w, ids, top)


def test_random_inputs_and_the_score():
    """Inputs off the grid; logprob is minus the score of cc_lmhead_score on the same rows."""
    from paper_2607_27600_amd import cc
    n, D, V, top = 128, 1024, 9000, 10
    g = torch.Generator().manual_seed(9)
    u, w = torch.randn(n, D, generator=g).to(torch.bfloat16), (torch.randn(V, D, generator=g) * 0.02).to(torch.bfloat16)
    ids = torch.randint(0, V, (n,), generator=g, dtype=torch.int32)
    r = _call(cc, u, w, ids, top)
    want = O.logprobs(f64(u), f64(w), ids.numpy(), top)
    # 1024 products of size up to 0.1 in fp32: under 1e-5 beside the bounds above
    np.testing.assert_allclose(f64(r.logprob), want["logprob"], rtol=0, atol=TOL + 1e-5)
    np.testing.assert_allclose(f64(r.top_logprob), want["top_logprob"], rtol=0, atol=TOL + 1e-5)
    got = np.take_along_axis(want["logits"], r.top_ids.cpu().numpy().astype(np.int64), 1)
    np.testing.assert_allclose(got, np.take_along_axis(want["logits"], want["top_ids"], 1), rtol=0, atol=1e-5)
    p = cc.problem(dtype="bf16", cu_seqlens=[0, n], n_heads_q=1, n_heads_kv=1, head_dim=64, hidden=D, vocab=V)
    s = torch.empty(n, device="cuda")
    cc.cc_lmhead_score(p, u.cuda(), w.cuda(), ids.cuda(), s)
    np.testing.assert_allclose(f64(s)[:-1], -f64(r.logprob)[:-1], rtol=0, atol=1e-5)


def test_nan_and_infinite_logits():
    """A NaN logit makes its row's numbers NaN and ranks last; other rows are untouched; a word of logit
    -inf has probability 0."""
    from paper_2607_27600_amd import cc
    u, w, ids = _grid(40, 64, 900, 11)
    clean = _call(cc, u, w, ids, 5)
    u2 = u.clone()
    u2[7, 3] = float("nan")
    r = _call(cc, u2, w, ids, 5)
    rows = np.arange(40) != 7
    for a, b in zip((r.logprob, r.entropy, r.top_logprob), (clean.logprob, clean.entropy, clean.top_logprob)):
        assert torch.equal(a[rows], b[rows]) and torch.isnan(a[7]).all()
    assert torch.equal(r.top_ids[rows], clean.top_ids[rows])
    assert sorted(r.top_ids[7].tolist()) == [0, 1, 2, 3, 4]
    u3, w3 = torch.ones(2, 64), torch.zeros(300, 64)
    w3[5:, 0] = -float("inf")
    u3[:, 1:] = 0
    r = _call(cc, u3.to(torch.bfloat16), w3.to(torch.bfloat16), torch.tensor([2, 7], dtype=torch.int32), 7)
    np.testing.assert_allclose(f64(r.entropy), np.log(5), atol=TOL_H)
    assert r.top_ids.cpu().tolist() == [[0, 1, 2, 3, 4, 5, 6]] * 2
    np.testing.assert_allclose(f64(r.logprob), [-np.log(5), -np.inf], atol=TOL)


def test_repeats_bit_for_bit_and_in_a_graph():
    from paper_2607_27600_amd import cc
    u, w, ids = _grid(300, 256, 30000, 12)
    ud, wd, idd = u.cuda(), w.cuda(), ids.cuda()
    ws = torch.empty(cc.cc_lmhead_logprobs_workspace("bf16", 300, 30000, 256, 8), dtype=torch.uint8, device="cuda")
    a, b = (cc.logprobs_out(300, 8) for _ in range(2))
    cc.cc_lmhead_logprobs("bf16", ud, wd, 30000, idd, 8, a, workspace=ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        cc.cc_lmhead_logprobs("bf16", ud, wd, 30000, idd, 8, b, workspace=ws)
    for i in range(4):
        for t in (b.logprob, b.entropy, b.top_logprob):
            t.zero_()
        ws.fill_(i * 85)      # whatever a workspace holds
        g.replay()
        torch.cuda.synchronize()
        for x, y in zip((a.logprob, a.entropy, a.top_ids, a.top_logprob), (b.logprob, b.entropy, b.top_ids, b.top_logprob)):
            assert torch.equal(x, y)


def test_ids_outside_the_vocabulary():
    """Rows of a padded batch (ids below 0 or at and past the vocabulary): NaN, whatever the workspace
    holds; their entropy and alternatives and the other rows stand."""
    from paper_2607_27600_amd import cc
    n, D, V = 70, 64, 1001
    u, w, ids = _grid(n, D, V, 14)
    bad = {0: -1, 5: -100, 17: V, 30: V + 1, 44: 1023, 51: 1024, 63: 2**31 - 1, 69: -2**31}
    for i, x in bad.items():
        ids[i] = x
    ws = torch.zeros(cc.cc_lmhead_logprobs_workspace("bf16", n, V, D, 3), dtype=torch.uint8, device="cuda")
    r = cc.cc_lmhead_logprobs("bf16", u.cuda(), w.cuda(), V, ids.cuda(), 3, workspace=ws)
    torch.cuda.synchronize()
    inside = [i for i in range(n) if i not in bad]
    clean = ids.clone()
    clean[list(bad)] = 0
    want = O.logprobs(f64(u), f64(w), clean.numpy(), 3)
    assert torch.isnan(r.logprob[list(bad)]).all()
    np.testing.assert_allclose(f64(r.logprob)[inside], want["logprob"][inside], rtol=0, atol=TOL)
    np.testing.assert_allclose(f64(r.entropy), want["entropy"], rtol=0, atol=TOL_H)
    np.testing.assert_array_equal(r.top_ids.cpu().numpy(), want["top_ids"])


def test_two_graphs_share_a_workspace():
    """Calls captured in two graphs that use one workspace in turn, with an eager call between them."""
    from paper_2607_27600_amd import cc
    n, D, V, top = 150, 128, 70000, 6
    sets = [tuple(x.cuda() for x in _grid(n, D, V, s)) for s in (15, 16)]
    want = [cc.cc_lmhead_logprobs("bf16", u, w, V, ids, top) for u, w, ids in sets]
    ws = torch.empty(cc.cc_lmhead_logprobs_workspace("bf16", n, V, D, top), dtype=torch.uint8, device="cuda")
    outs = [cc.logprobs_out(n, top) for _ in range(3)]
    torch.cuda.synchronize()
    graphs = []
    for (u, w, ids), out in zip(sets, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            cc.cc_lmhead_logprobs("bf16", u, w, V, ids, top, out, workspace=ws)
        graphs.append(g)
    for _ in range(3):
        for o in outs:
            for t in (o.logprob, o.entropy, o.top_ids, o.top_logprob):
                t.zero_()
        graphs[0].replay()
        cc.cc_lmhead_logprobs("bf16", *sets[1][:2], V, sets[1][2], top, outs[2], workspace=ws)
        graphs[1].replay()
        torch.cuda.synchronize()
        for o, x in zip(outs, (want[0], want[1], want[1])):
            for t in ("logprob", "entropy", "top_ids", "top_logprob"):
                assert torch.equal(getattr(o, t), getattr(x, t)), t


# ---- batches whose candidates go by a running bound: more than 64 rows and at least two rounds of tiles.  Which
# words are candidates there depends on the order of workgroups; the results may not.

def _bounded(cc, n, V, D, top):
    """Whether a call keeps a bound: its workspace has 32 slots and a bound a row behind the rest."""
    up = lambda x: -(-x // 256) * 256
    rows, tiles = min(n, 2048), -(-V // 256)
    rest = up(tiles * rows * 16) + up(2 * tiles * rows) + up(2 * tiles * rows * top * 8) + up(rows * 4)
    size = cc.cc_lmhead_logprobs_workspace("bf16", n, V, D, top)
    assert size in (rest, rest + up(rows * 128) + up(rows * 4))
    return size > rest


@pytest.mark.parametrize("n,D,V,top,packed", [(300, 64, 70000, 1, False), (300, 64, 70001, 5, True), (257, 128, 70000, 32, False),
                                              (600, 192, 50001, 20, True), (100, 64, 131073, 3, False)])
def test_rows_with_a_running_bound(n, D, V, top, packed):
    from paper_2607_27600_amd import cc
    assert _bounded(cc, n, V, D, top)
    print(f"[logprobs bounded] {n} {D} {V} {top} packed={packed}", flush=True)
    u, w, ids = _grid(n, D, V, n + V)
    _check(_call(cc, u, w, ids, top, packed), u, w, ids, top)


def test_a_running_bound_starts_anew_with_every_slab():
    """Rows of a second, shorter slab with logits far below the first's: a bound left over would drop them all."""
    from paper_2607_27600_amd import cc
    n, D, V, top = 2100, 64, 16385, 5
    assert _bounded(cc, n, V, D, top)
    u, w, ids = _grid(n, D, V, 17)
    w[:, 0] = 1
    u[:, 0] = 15
    u[2048:, 0] = -15
    _check(_call(cc, u, w, ids, top), u, w, ids, top)


@pytest.mark.parametrize("order", ["equal", "falling", "rising", "few"])
def test_ties_and_orders_with_a_running_bound(order):
    """All logits equal, rising or falling with the id (every tile passes the bound, or none), a handful of values."""
    from paper_2607_27600_amd import cc
    V, D, n, top = 70000, 64, 300, 32
    assert _bounded(cc, n, V, D, top)
    w = torch.zeros(V, D)
    v = torch.arange(V)
    if order in ("falling", "rising"):      # z = +-v / 1024, in three exact terms; |z| under 69
        s = -1.0 if order == "falling" else 1.0
        w[:, 0], w[:, 1], w[:, 2] = s * (v // 4096).float() * 4, s * (v // 64 % 64).float() / 16, s * (v % 64).float() / 1024
    elif order == "few":
        w[:, 0] = (v % 7 == 3).float() - (v % 5 == 0).float()
    u = torch.zeros(n, D)
    u[:, :3] = 1
    u[1::2] *= -1
    u, w = u.to(torch.bfloat16), w.to(torch.bfloat16)
    ids = torch.arange(n, dtype=torch.int32) * 200
    ids[2:] = ids[:2].repeat(n // 2)[:n - 2]
    r = _call(cc, u, w, ids, top)
    want = O.logprobs(f64(u[:2]), f64(w), ids[:2].numpy(), top)     # all rows are one of two
    for i in (0, 1):
        np.testing.assert_array_equal(r.top_ids[i::2].cpu().numpy(), np.tile(want["top_ids"][i], (n // 2, 1)))
        for t, tol in (("logprob", TOL), ("entropy", TOL_H), ("top_logprob", TOL)):
            got = f64(getattr(r, t)[i::2])
            np.testing.assert_allclose(got, np.broadcast_to(want[t][i], got.shape), rtol=0, atol=tol)


def test_nan_infinities_and_padding_with_a_running_bound():
    """Rows of NaN, rows of which five words are numbers and the others NaN or -inf, and ids of no word, among
    plain rows of a bounded call."""
    from paper_2607_27600_amd import cc
    n, D, V, top = 300, 64, 70000, 7
    assert _bounded(cc, n, V, D, top)
    u, w, ids = _grid(n, D, V, 18)
    w[:, 0] = 0
    w[:, 1] = 0
    u[:, 0] = u[:, 1] = 0
    clean = _call(cc, u, w, ids, top)
    _check(clean, u, w, ids, top)
    u2, ids2 = u.clone(), ids.clone()
    u2[9, 5] = u2[299, 1] = float("nan")
    ids2[[3, 150]] = torch.tensor([-1, V], dtype=torch.int32)
    r = _call(cc, u2, w, ids2, top)
    rows = np.setdiff1d(np.arange(n), [9, 299])
    for t in ("logprob", "entropy", "top_ids", "top_logprob"):
        x, y = getattr(r, t), getattr(clean, t)
        keep = np.setdiff1d(rows, [3, 150]) if t == "logprob" else rows
        assert torch.equal(x[keep], y[keep]), t
        if t != "top_ids":
            assert torch.isnan(x[[9, 299]]).all()
    assert torch.isnan(r.logprob[[3, 150]]).all()
    assert r.top_ids[[9, 299]].cpu().tolist() == [list(range(top))] * 2
    # -inf in w: rows of u0 = 1 have -inf in all words but five, rows of u0 = 0 NaN (0 times infinity)
    u3, w3 = torch.zeros(n, D), torch.zeros(V, D)
    w3[:, 1] = (torch.arange(V) % 64).float() / 16
    five = [3, 1000, 33333, 69998, 69999]
    w3[:, 0] = -float("inf")
    w3[five, 0] = 0
    u3[:, 1] = 1
    u3[::2, 0] = 1
    ids3 = torch.full((n,), 1000, dtype=torch.int32)
    r = _call(cc, u3.to(torch.bfloat16), w3.to(torch.bfloat16), ids3, top)
    z = np.array([x % 64 / 16 for x in five])
    lse = np.log(np.exp(z).sum())
    order = np.argsort(-z, kind="stable")
    want_ids = [five[i] for i in order] + [0, 1]
    assert (r.top_ids.cpu() == torch.tensor(want_ids, dtype=torch.int32)).all()
    np.testing.assert_allclose(f64(r.top_logprob[::2, :5]), np.tile(z[order] - lse, (n // 2, 1)), rtol=0, atol=TOL)
    assert torch.isneginf(r.top_logprob[::2, 5:]).all() and torch.isnan(r.top_logprob[1::2]).all()
    np.testing.assert_allclose(f64(r.logprob[::2]), z[1] - lse, rtol=0, atol=TOL)
    np.testing.assert_allclose(f64(r.entropy[::2]), -(np.exp(z - lse) * (z - lse)).sum(), rtol=0, atol=TOL_H)


def test_bounded_calls_repeat_bit_for_bit_in_graphs_that_share_a_workspace():
    """Two captured calls of one workspace, replayed in turn with an eager call between, whatever it holds."""
    from paper_2607_27600_amd import cc
    n, D, V, top = 300, 256, 70000, 8
    assert _bounded(cc, n, V, D, top)
    sets = [tuple(x.cuda() for x in _grid(n, D, V, s)) for s in (19, 20)]
    want = [cc.cc_lmhead_logprobs("bf16", u, w, V, ids, top) for u, w, ids in sets]
    for (u, w, ids), r in zip(sets, want):
        _check(r, u, w, ids.cpu(), top)
    ws = torch.empty(cc.cc_lmhead_logprobs_workspace("bf16", n, V, D, top), dtype=torch.uint8, device="cuda")
    outs = [cc.logprobs_out(n, top) for _ in range(3)]
    torch.cuda.synchronize()
    graphs = []
    for (u, w, ids), out in zip(sets, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            cc.cc_lmhead_logprobs("bf16", u, w, V, ids, top, out, workspace=ws)
        graphs.append(g)
    for i in range(5):
        for o in outs:
            for t in (o.logprob, o.entropy, o.top_ids, o.top_logprob):
                t.zero_()
        ws.fill_(i * 51)
        graphs[0].replay()
        cc.cc_lmhead_logprobs("bf16", *sets[1][:2], V, sets[1][2], top, outs[2], workspace=ws)
        graphs[1].replay()
        torch.cuda.synchronize()
        for o, x in zip(outs, (want[0], want[1], want[1])):
            for t in ("logprob", "entropy", "top_ids", "top_logprob"):
                assert torch.equal(getattr(o, t), getattr(x, t)), t
