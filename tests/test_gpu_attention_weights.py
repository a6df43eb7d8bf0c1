"""Accumulated attention weight, the scores made of it and its compaction, against fp64; the cycle of eviction by it."""
import numpy as np
import pytest
import torch

from oracle import cc_oracle
from oracle import kv16_oracle as O
from tests.gpu_util import f64
from tests.kv16_util import Cache16, cu_of, i32, logit_error, problem, queries

pytestmark = pytest.mark.gpu

CASES = [
    # new, lens, hq, hkv, d, page
    ([1], [1], 4, 2, 128, 0),
    ([1, 1, 1, 1], [1, 64, 65, 333], 28, 4, 128, 16),
    ([1, 3, 0, 8], [100, 3, 9, 257], 16, 4, 64, 16),
    ([5], [700], 20, 2, 128, 32),
    ([64], [1000], 4, 4, 128, 64),
    ([130, 33], [130, 500], 14, 2, 128, 16),
    ([300, 1, 0, 77, 640], [300, 1, 5, 77, 640], 4, 1, 128, 16),
    ([257], [257], 24, 1, 64, 0),
    ([9, 4], [3, 0], 4, 2, 128, 16),                # more queries than entries
    ([1500], [1500], 8, 2, 64, 128),
]


def _oracle(cache, q, new, lens, hq, hkv, layer=0, scale=None):
    """lse [N][Hq] (rounded to fp32), weights and the bound of their error [seq][Hkv][longest]."""
    g, qh, cu = hq // hkv, f64(q), cu_of(new)
    tau = cache.d ** -0.5 if scale is None else scale
    lse = np.full(qh.shape[:2], -np.inf, np.float32)
    w, tol = np.zeros((2, len(new), hkv, max(max(lens), 1)))
    for b, m in enumerate(new):
        rows, n = slice(cu[b], cu[b + 1]), lens[b]
        for c in range(hkv):
            k, v = (cache.values(layer, b, c, t, n) for t in "kv")
            for h in range(c * g, (c + 1) * g):
                lse[rows, h] = O.attention(qh[rows, h], k, v, scale=tau)[1]
                fin = np.isfinite(lse[rows, h])
                part = O.weights(qh[rows, h][fin], k, lse[rows, h][fin].astype(np.float64), tau) if fin.all() else sum(
                    np.where(np.arange(n) <= i + n - m, np.exp(tau * (k @ qh[cu[b] + i, h]) - lse[cu[b] + i, h]), 0.0)
                    for i in np.flatnonzero(fin)) if fin.any() else np.zeros(n)
                w[b, c, :n] += part
                # of a weight: its logit's error, that of lse's product with log2(e), and the power's own
                rel = logit_error(qh[rows, h], k, tau).max(initial=0) + 2.0 ** -22 * (
                    2 + np.abs(lse[rows, h][fin]).max(initial=0))
                tol[b, c, :n] += part * rel
        tol[b] += np.abs(w[b]) * (m * g / 16 + 8) * 2.0 ** -24      # the fp32 sums, the longest 16 rows at a time
    return lse, w, tol


@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
def test_weights(case):
    from paper_2607_27600_amd import cc
    new, lens, hq, hkv, d, page = case
    print(f"[weights] {case}", flush=True)
    cache = Cache16(lens, hkv, d, layers=2, page=page, seed=51)
    q = queries(new, hq, d, 52)
    lse, want, tol = _oracle(cache, q, new, lens, hq, hkv, layer=1)
    p, n = problem(cc, new, hq, hkv, d), max(max(lens), 1)
    had = [max(0, a - m) for a, m in zip(lens, new)]
    # prev is NaN where an entry has had nothing
    prev = torch.rand(len(new), hkv, n + 5, generator=torch.Generator().manual_seed(53)).cuda() * 4
    for b, x in enumerate(had):
        prev[b, :, x:] = float("nan")
    for start in ("none", "added", "in place"):
        out = prev if start == "in place" else torch.full((len(new), hkv, n + 5), 7.0, device="cuda")
        before = f64(out) if start == "in place" else np.full(out.shape, 7.0)
        base = np.zeros(out.shape)
        if start != "none":
            for b, x in enumerate(had):
                base[b, :, :x] = f64(prev)[b, :, :x]
        kw = {} if start == "none" else dict(prev=prev, prev_lens=i32(had))
        cc.cc_attention_weights(p, q, cache.view(cc), 1, i32(lens), n, torch.from_numpy(lse).cuda(), out, **kw)
        torch.cuda.synchronize()
        got = f64(out)
        for b, m in enumerate(lens):
            ref = base[b, :, :m] + want[b, :, :m]
            assert np.all(np.abs(got[b, :, :m] - ref) <= tol[b, :, :m] + 2.0 ** -24 * np.abs(ref)), f"{case} {start} {b}"
            np.testing.assert_array_equal(got[b, :, m:], before[b, :, m:])


def test_weights_sum_to_the_rows():
    """The weights that a row gives sum to one: over all entries, a head's sum is its number of rows."""
    from paper_2607_27600_amd import cc
    hq, hkv, d, new, lens = 28, 4, 128, [400, 1, 37], [400, 900, 1000]
    cache = Cache16(lens, hkv, d, page=64, seed=54)
    q = queries(new, hq, d, 55)
    p, lse = problem(cc, new, hq, hkv, d), torch.empty(sum(new), hq, device="cuda")
    cc.cc_attention_kv(p, q, cache.view(cc), 0, i32(lens), 1000, lse=lse)
    w = torch.zeros(3, hkv, 1000, device="cuda")
    cc.cc_attention_weights(p, q, cache.view(cc), 0, i32(lens), 1000, lse, w)
    torch.cuda.synchronize()
    # every weight is off by some 2^-16 of itself at most: (d + 16) 2^-24 of magnitudes around 16, and the lse's
    np.testing.assert_allclose(f64(w).sum(-1), np.repeat(np.array(new)[:, None] * (hq // hkv), hkv, 1), rtol=2.0 ** -12)


@pytest.mark.parametrize("d", [128, 64])
def test_entries_that_are_not_seen_do_not_count(d):
    """A NaN key gives NaN to the entries of the rows that see it, and leaves those that do not alone."""
    from paper_2607_27600_amd import cc
    hq, hkv, m, n = 4, 2, 40, 90
    cache = Cache16([n], hkv, d, page=16, seed=56)
    q = queries([m], hq, d, 57)
    lse, want, tol = _oracle(cache, q, [m], [n], hq, hkv)
    cache.put(0, 0, 0, "k", 70, 3, float("nan"))
    w = torch.zeros(1, hkv, n, device="cuda")
    cc.cc_attention_weights(problem(cc, [m], hq, hkv, d), q, cache.view(cc), 0, i32([n]), n, torch.from_numpy(lse).cuda(), w)
    torch.cuda.synchronize()
    got = f64(w)[0]
    nan = np.zeros((hkv, n), bool)
    nan[0, 70] = True
    np.testing.assert_array_equal(np.isnan(got), nan)
    assert np.all(np.abs(got - want[0])[~nan] <= tol[0][~nan])


@pytest.mark.parametrize("per_head", [0, 1])
@pytest.mark.parametrize("lens,hkv,first,recent", [([1], 1, 0, 0), ([700, 0, 33, 1], 4, 2, 30), ([300] * 70, 2, 0, 16),
                                                   ([40], 2, 100, 0), ([40, 3], 2, 0, 1000)])
def test_weight_scores(lens, hkv, first, recent, per_head):
    from paper_2607_27600_amd import cc
    w = torch.rand(len(lens), hkv, max(lens) + 3, generator=torch.Generator().manual_seed(58)).cuda()
    p = problem(cc, lens, hkv, hkv, 64, n_frozen=first)
    s = torch.full((sum(lens) * (hkv if per_head else 1) + 4,), 7.0, device="cuda")
    cc.cc_weight_scores(p, w, recent, per_head, s)
    torch.cuda.synchronize()
    want = []
    for b, n in enumerate(lens):
        x = w[b, :, :n].cpu().numpy()
        if per_head:
            want += [O.scores(x[h], first, recent) for h in range(hkv)]
        else:
            total = x[0].copy()
            for h in range(1, hkv):
                total = total + x[h]          # fp32, in order
            want.append(O.scores(total, first, recent))
    np.testing.assert_array_equal(s.cpu().numpy(), np.concatenate([*want, np.full(4, 7.0)]).astype(np.float32))


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("per_head", [0, 1])
@pytest.mark.parametrize("lens,keep,hkv", [([1], [1], 1), ([700, 0, 33, 1], [512, 0, 33, 0], 4), ([9000, 5000], [8500, 4097], 2),
                                           ([300] * 70, [100] * 70, 2)])
def test_compact_weights(lens, keep, hkv, per_head, in_place):
    from paper_2607_27600_amd import cc
    r = np.random.default_rng(59)
    n = max(lens) + 3
    w = torch.from_numpy(r.random((len(lens), hkv, n), np.float32)).cuda()
    lists = [np.sort(r.permutation(m)[:k]) for m, k in zip(lens, keep) for _ in range(hkv if per_head else 1)]
    want = w.cpu().numpy().copy() if in_place else np.full((len(lens), hkv, n), 7.0, np.float32)
    src = w.cpu().numpy().copy()
    for b in range(len(lens)):
        for h in range(hkv):
            x = lists[b * hkv + h] if per_head else lists[b]
            want[b, h, : len(x)] = src[b, h, x]
    out = None if in_place else torch.full_like(w, 7.0)
    budgets = [len(x) for x in lists]
    cc.cc_compact_weights(problem(cc, lens, hkv, hkv, 64), w, i32(np.concatenate(lists)), budgets, per_head, out=out)
    torch.cuda.synchronize()
    np.testing.assert_array_equal((w if in_place else out).cpu().numpy(), want)


@pytest.mark.parametrize("per_head", [0, 1])
def test_the_cycle_of_eviction(per_head):
    """Append, attend, accumulate, evict and attend again, as a managed cache runs them together, against the same cycle
    in 64 bits."""
    from paper_2607_27600_amd import cc
    hq, hkv, d, n_seqs, cap, J, m = 8, 2, 64, 2, 96, 48, 16
    g = torch.Generator().manual_seed(60)
    kc, vc = (torch.full((n_seqs, hkv, cap, d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in "kv")
    kv = cc.kv_contiguous(kc, vc, n_layers=1, seq_stride=hkv * cap * d, layer_stride=0, head_stride=cap * d, tok_stride=d)
    w = torch.full((n_seqs, hkv, cap), float("nan"), device="cuda")
    host = [[dict(k=np.zeros((0, d)), v=np.zeros((0, d)), w=np.zeros(0)) for _ in range(hkv)] for _ in range(n_seqs)]
    n = 0
    p = problem(cc, [m] * n_seqs, hq, hkv, d)
    for step in range(9):
        k, v = (torch.randn(n_seqs * m, hkv, d, generator=g).to(torch.bfloat16).cuda() for _ in "kv")
        q = torch.randn(n_seqs * m, hq, d, generator=g).to(torch.bfloat16).cuda()
        cached = i32([n] * n_seqs)
        cc.cc_append_kv(p, kv, k, v, cached, capacity=cap, rotate=False)
        n += m
        lens, lse = i32([n] * n_seqs), torch.empty(n_seqs * m, hq, device="cuda")
        o = cc.cc_attention_kv(p, q, kv, 0, lens, cap, lse=lse)
        cc.cc_attention_weights(p, q, kv, 0, lens, cap, lse, w, prev=w, prev_lens=cached)
        torch.cuda.synchronize()
        qh = f64(q)
        for b in range(n_seqs):
            rows = slice(b * m, b * m + m)
            for c in range(hkv):
                x = host[b][c]
                x["k"], x["v"] = np.concatenate([x["k"], f64(k)[rows, c]]), np.concatenate([x["v"], f64(v)[rows, c]])
                x["w"] = np.concatenate([x["w"], np.zeros(m)])
                for h in range(c * hq // hkv, (c + 1) * hq // hkv):
                    ro, rl = O.attention(qh[rows, h], x["k"], x["v"])
                    got = f64(o)[rows, h]
                    assert np.all(np.abs(got - ro) <= 2.0 ** -8 * np.abs(ro) + 2.0 ** -6 * np.sqrt((ro ** 2).mean(-1, keepdims=True)) + 1e-6)
                    x["w"] = x["w"] + O.weights(qh[rows, h], x["k"], rl)
                np.testing.assert_allclose(f64(w)[b, c, :n], x["w"], rtol=2.0 ** -12)
        if n <= J:
            continue
        pe = problem(cc, [n] * n_seqs, hq, hkv, d, n_frozen=2)
        lists = n_seqs * (hkv if per_head else 1)
        s = cc.cc_weight_scores(pe, w, 8, per_head)
        keep = torch.empty(lists * J, dtype=torch.int32, device="cuda")
        cc.cc_select_keep(s, [i * n for i in range(lists)], [n] * lists, [J] * lists, keep)
        cc.cc_compact_kv(pe, kv, keep, [J] * lists, per_head)
        cc.cc_compact_weights(pe, w, keep, [J] * lists, per_head)
        torch.cuda.synchronize()
        kept = keep.cpu().numpy().reshape(lists, J)
        for i in range(lists):
            np.testing.assert_array_equal(kept[i], cc_oracle.select_keep(s.cpu().numpy()[i * n:(i + 1) * n], J))
            assert set(kept[i]) >= {0, 1, *range(n - 8, n)}
        for b in range(n_seqs):
            for c in range(hkv):
                at = kept[b * hkv + c] if per_head else kept[b]
                host[b][c] = {name: x[at] for name, x in host[b][c].items()}
        n = J


@pytest.mark.parametrize("new,lens,hq,hkv,d,page", [([3000], [3000], 28, 4, 128, 16), ([1, 2100, 64, 700], [5, 2500, 9000, 700], 4, 1, 64, 32),
                                                    ([500] * 3, [500, 6000, 501], 8, 1, 128, 0), ([100] * 70, [100 + i for i in range(70)], 4, 2, 64, 16),
                                                    ([17], [30], 8, 2, 128, 16), ([300], [100], 8, 2, 64, 16), ([40, 65, 1], [900, 900, 900], 256, 2, 64, 64)])
def test_weights_in_chunks(new, lens, hq, hkv, d, page):
    """Many rows: tiles that a workgroup shares, chunks that are added up, beside sequences of few; the workspace holds no
    more than asked for, and the same call repeats bit for bit."""
    from paper_2607_27600_amd import cc
    print(f"[weights chunks] {new} {lens} {hq} {hkv} {d}", flush=True)
    cache = Cache16(lens, hkv, d, page=page, seed=71, room=300)
    q = queries(new, hq, d, 72)
    lse, want, tol = _oracle(cache, q, new, lens, hq, hkv)
    p, n = problem(cc, new, hq, hkv, d), max(lens)
    prev = torch.rand(len(new), hkv, n, generator=torch.Generator().manual_seed(73)).cuda() * 4
    for longest in (n, n + 300):
        size = cc.cc_attention_weights_workspace(p, longest)
        ws = torch.full((size + 4096,), 0x7f, dtype=torch.uint8, device="cuda")
        got = []
        for _ in range(2):
            out = torch.full((len(new), hkv, longest), 7.0, device="cuda")
            cc.cc_attention_weights(p, q, cache.view(cc), 0, i32(lens), longest, torch.from_numpy(lse).cuda(), out, prev=prev,
                                    prev_lens=i32(lens), workspace=ws[:size])
            torch.cuda.synchronize()
            got.append(out)
        assert torch.equal(*got) and (ws[size:] == 0x7f).all()
        for b, m in enumerate(lens):
            ref = f64(prev)[b, :, :m] + want[b, :, :m]
            err = np.abs(f64(got[0])[b, :, :m] - ref)
            assert np.all(err <= tol[b, :, :m] + 2.0 ** -24 * np.abs(ref)), (longest, b, err.max())
            assert (got[0][b, :, m:] == 7).all()


@pytest.mark.parametrize("new,most", [([1, 4], 300), ([70, 1], 900), ([400], 1500)])
def test_a_cycle_in_two_graphs(new, most):
    """Attention and its weights in place, captured twice with one workspace and replayed in turn as the lengths advance."""
    from paper_2607_27600_amd import cc
    hq, hkv, d = 8, 2, 64
    cache = Cache16([most] * len(new), hkv, d, page=16, seed=81)
    q, kv, p = queries(new, hq, d, 82), cache.view(cc), problem(cc, new, hq, hkv, d)
    ws = torch.empty(max(1, cc.cc_attention_kv_workspace(p, most), cc.cc_attention_weights_workspace(p, most)),
                     dtype=torch.uint8, device="cuda")
    lens, had = i32(new), i32([0] * len(new))
    lse, w = torch.empty(sum(new), hq, device="cuda"), torch.full((len(new), hkv, most), float("nan"), device="cuda")
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            cc.cc_attention_kv(p, q, kv, 0, lens, most, lse=lse, workspace=ws)
            cc.cc_attention_weights(p, q, kv, 0, lens, most, lse, w, prev=w, prev_lens=had, workspace=ws)
        graphs.append(g)
    want, tol, had_h = np.zeros(w.shape), np.zeros(w.shape), [0] * len(new)
    for step in range(4):
        now = [min(most, m * (step + 1) + 37 * step) for m in new]
        lens.copy_(i32(now))
        had.copy_(i32(had_h))
        ws.fill_(0x7f)
        graphs[step % 2].replay()
        torch.cuda.synchronize()
        _, x, t = _oracle(cache, q, new, now, hq, hkv)
        longest = x.shape[2]
        want[:, :, :longest] += x
        # (the kernel's own lse is off by the logits' error and its sum's, what the bound counts once already)
        tol[:, :, :longest] += 2 * t + 2.0 ** -22 * want[:, :, :longest]
        got = f64(w)
        for b, n in enumerate(now):
            assert np.all(np.abs(got[b, :, :n] - want[b, :, :n]) <= tol[b, :, :n]), (step, b)
            assert np.isnan(got[b, :, n:]).all()
        had_h = now


def test_a_query_that_is_not_finite_reaches_the_entries_it_sees():
    from paper_2607_27600_amd import cc
    hq, hkv, d = 4, 2, 64
    for new, n, bad in (([3], 50, 1), ([200], 700, 100)):
        cache, q = Cache16([n], hkv, d, page=16, seed=83), queries(new, hq, d, 84)
        lse, want, tol = _oracle(cache, q, new, [n], hq, hkv)
        q[bad, 3, 5] = float("nan")          # of the second KV head's group
        w = torch.full((1, hkv, n), 7.0, device="cuda")
        cc.cc_attention_weights(problem(cc, new, hq, hkv, d), q, cache.view(cc), 0, i32([n]), n, torch.from_numpy(lse).cuda(), w)
        torch.cuda.synchronize()
        hit = np.zeros((hkv, n), bool)
        hit[1, :n - new[0] + bad + 1] = True
        np.testing.assert_array_equal(np.isnan(f64(w)[0]), hit)
        assert np.all(np.abs(f64(w)[0] - want[0])[~hit] <= tol[0][~hit])


def test_weights_in_other_layouts():
    """Heads outermost, sequences spread, one earlier weight for all heads; the gaps stay as they are."""
    from paper_2607_27600_amd import cc
    new, lens, hq, hkv, d = [2, 90], [40, 300], 4, 2, 128
    cache, q = Cache16(lens, hkv, d, page=16, seed=85), queries(new, hq, d, 86)
    lse, want, tol = _oracle(cache, q, new, lens, hq, hkv)
    room = torch.full((hkv, 3, 333), 7.0, device="cuda")
    w = room[:, :2, :300].permute(1, 0, 2)
    prev = torch.rand(2, 1, 300, generator=torch.Generator().manual_seed(87)).cuda().expand(2, hkv, 300)
    cc.cc_attention_weights(problem(cc, new, hq, hkv, d), q, cache.view(cc), 0, i32(lens), 300, torch.from_numpy(lse).cuda(), w,
                            prev=prev)
    torch.cuda.synchronize()
    got = f64(room)
    for b, n in enumerate(lens):
        ref = want[b, :, :n] + f64(prev)[b, :, :n]
        assert np.all(np.abs(got[:, b, :n] - ref) <= tol[b, :, :n] + 2.0 ** -24 * np.abs(ref))
        assert (got[:, b, n:] == 7).all()
    assert (got[:, 2] == 7).all()
    # and compacted out of them
    keep = [0, 7, 39, 5, 299]
    out = torch.full((2, hkv, 8), 3.0, device="cuda")
    cc.cc_compact_weights(problem(cc, lens, hkv, hkv, d), w, i32(keep), [3, 2], 0, out=out)
    torch.cuda.synchronize()
    assert torch.equal(out[0, :, :3], w[0][:, keep[:3]]) and torch.equal(out[1, :, :2], w[1][:, keep[3:]])
    assert (out[0, :, 3:] == 3).all() and (out[1, :, 2:] == 3).all()


@pytest.mark.parametrize("new,lens,hq,hkv,d,page", [
    ([300, 1, 7, 900, 0], [300, 1, 7, 900, 40], 8, 2, 128, 16),
    ([1200, 2, 70], [1200, 1199, 2], 4, 1, 64, 0),                  # two tokens behind as many entries as a prompt has
    ([600] + [40, 1] * 40, [600] + [40, 1] * 40, 8, 4, 64, 16),     # more than a launch lists
    ([600] + [1] * 3, [600, 5, 1, 600], 8, 2, 128, 32),             # more short ones than go along
])
def test_weights_of_short_prompts_beside_long_ones(new, lens, hq, hkv, d, page):
    from paper_2607_27600_amd import cc
    cache, q = Cache16(lens, hkv, d, page=page, seed=93), queries(new, hq, d, 94)
    lse, want, tol = _oracle(cache, q, new, lens, hq, hkv)
    n = max(lens)
    had = [max(0, a - m) for a, m in zip(lens, new)]
    prev = torch.rand(len(new), hkv, n, generator=torch.Generator().manual_seed(95)).cuda()
    out = torch.full((len(new), hkv, n), 7.0, device="cuda")
    cc.cc_attention_weights(problem(cc, new, hq, hkv, d), q, cache.view(cc), 0, i32(lens), n, torch.from_numpy(lse).cuda(), out,
                            prev=prev, prev_lens=i32(had))
    torch.cuda.synchronize()
    for b, m in enumerate(lens):
        ref = want[b, :, :m].copy()
        ref[:, :had[b]] += f64(prev)[b, :, :had[b]]
        assert np.all(np.abs(f64(out)[b, :, :m] - ref) <= tol[b, :, :m] + 2.0 ** -24 * np.abs(ref)), b
        assert (out[b, :, m:] == 7).all()


@pytest.mark.parametrize("new,lens,hq,hkv,d,page", [
    ([8] * 8, [3000, 17, 64, 65, 1, 2999, 500, 8], 32, 8, 128, 16),       # 64 entries a wave
    ([32, 1, 0, 5] * 4, [2000, 63, 1999, 4] * 4, 16, 8, 64, 0),
    ([32], [1000], 2, 1, 64, 16),                                        # 32
])
def test_weights_of_drafts(new, lens, hq, hkv, d, page):
    from paper_2607_27600_amd import cc
    cache, q = Cache16(lens, hkv, d, page=page, seed=96), queries(new, hq, d, 97)
    lse, want, tol = _oracle(cache, q, new, lens, hq, hkv)
    n = max(lens)
    prev = torch.rand(len(new), hkv, n, generator=torch.Generator().manual_seed(98)).cuda()
    out = torch.full((len(new), hkv, n), 7.0, device="cuda")
    cc.cc_attention_weights(problem(cc, new, hq, hkv, d), q, cache.view(cc), 0, i32(lens), n, torch.from_numpy(lse).cuda(), out,
                            prev=prev)
    torch.cuda.synchronize()
    for b, m in enumerate(lens):
        ref = want[b, :, :m] + f64(prev)[b, :, :m]
        assert np.all(np.abs(f64(out)[b, :, :m] - ref) <= tol[b, :, :m] + 2.0 ** -24 * np.abs(ref)), b
        assert (out[b, :, m:] == 7).all()


@pytest.mark.parametrize("new,lens,hq,hkv,d,wide", [([1, 3], [900, 40], 8, 2, 128, 500), ([8] * 8, [3000, 17, 64, 65, 1, 2999, 500, 8], 32, 8, 128, 65),
                                                    ([90, 200], [900, 300], 8, 2, 64, 301), ([700], [700], 4, 1, 128, 1)])
def test_earlier_weights_end_where_their_tensor_does(new, lens, hq, hkv, d, wide):
    """Lengths on the device past the tensor of the earlier weights: entries beyond have had nothing."""
    from paper_2607_27600_amd import cc
    cache, q = Cache16(lens, hkv, d, page=16, seed=99), queries(new, hq, d, 100)
    lse, want, tol = _oracle(cache, q, new, lens, hq, hkv)
    n = max(lens)
    room = torch.full((len(new), hkv, n + 8), float("nan"), device="cuda")      # (what lies past the earlier weights)
    room[:, :, :wide] = torch.rand(len(new), hkv, wide, generator=torch.Generator().manual_seed(101)).cuda()
    prev = room[:, :, :wide]
    out = torch.full((len(new), hkv, n), 7.0, device="cuda")
    cc.cc_attention_weights(problem(cc, new, hq, hkv, d), q, cache.view(cc), 0, i32(lens), n, torch.from_numpy(lse).cuda(), out,
                            prev=prev, prev_lens=i32([10 ** 6] * len(new)))
    torch.cuda.synchronize()
    for b, m in enumerate(lens):
        ref = want[b, :, :m].copy()
        k = min(m, wide)
        ref[:, :k] += f64(prev)[b, :, :k]
        assert np.all(np.abs(f64(out)[b, :, :m] - ref) <= tol[b, :, :m] + 2.0 ** -24 * np.abs(ref)), b
        assert (out[b, :, m:] == 7).all()
