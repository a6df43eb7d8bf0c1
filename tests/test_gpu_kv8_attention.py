"""Attention over a cache in 8 bits against fp64: few and many rows, both masks, ragged batches, every
layout and scale block, pieces that are joined, rows that see nothing, NaN where a row may not look."""
import numpy as np
import pytest
import torch

from oracle import kv8_oracle as O8
from tests.gpu_util import assert_attention_close, f64
from tests.kv8_util import Cache8, cu_of, i32, quantize

pytestmark = pytest.mark.gpu


def _problem(cc, new, hq, hkv, d, **kw):
    return cc.problem(dtype="bf16", cu_seqlens=cu_of(new), n_heads_q=hq, n_heads_kv=hkv, head_dim=d, hidden=64, vocab=1, **kw)


def _oracle(cache, q, new, lens, hq, hkv, mask, inclusive=False, layer=0, scale=None):
    g, out, at = hq // hkv, [], 0
    qh = f64(q)
    for b, m in enumerate(new):
        o = np.zeros((m, hq, cache.d))
        for c in range(hkv):
            k, v = (cache.values(layer, b, c, t, lens[b]) for t in ("k", "v"))
            for h in range(c * g, (c + 1) * g):
                o[:, h] = O8.attention(qh[at:at + m, h], k, v, mask, inclusive, scale)
        out.append(o)
        at += m
    return np.concatenate(out)


def _run(cc, cache, q, new, lens, hq, hkv, mask, layer=0, longest=None, **kw):
    p = _problem(cc, new, hq, hkv, cache.d, **kw)
    o = torch.full_like(q, 7.0)
    cc.cc_attention_kv8(p, q, cache.view(cc), layer, i32(lens), max(lens) if longest is None else longest, o, mask=mask)
    torch.cuda.synchronize()
    return o


def _q(new, hq, d, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(sum(new), hq, d, generator=g).to(torch.bfloat16).cuda()


CASES = [
    # new, lens, hq, hkv, d, page, block
    ([1], [1], 4, 2, 128, 0, 16),
    ([1], [17], 8, 1, 128, 0, 16),
    ([1, 1, 1, 1], [1, 64, 65, 333], 28, 4, 128, 16, 16),
    ([1, 1], [1500, 40], 32, 8, 128, 64, 64),
    ([1, 3, 0, 8], [100, 3, 9, 257], 16, 4, 64, 16, 16),
    ([5], [700], 20, 2, 128, 32, 16),          # 50 rows of a KV head: four row blocks
    ([7], [130], 12, 4, 64, 128, 128),         # 21: two
    ([20, 2], [20, 300], 8, 2, 128, 16, 16),   # many beside few
    ([64], [1000], 4, 4, 128, 64, 32),
    ([130, 33], [130, 500], 14, 2, 128, 16, 16),
    ([200], [321], 8, 8, 64, 0, 64),
    ([257], [257], 4, 2, 64, 32, 32),
]


@pytest.mark.parametrize("mask", ["causal", "counter", "counter_inclusive"])
@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
def test_attention(case, mask):
    from paper_2607_27600_amd import cc
    new, lens, hq, hkv, d, page, block = case
    print(f"[attn8] {case} {mask}", flush=True)
    cache = Cache8(lens, hkv, d, layers=2, page=page, block=block, seed=21, fill=0x7f)
    q = _q(new, hq, d, 22)
    kw = dict(diag="inclusive") if mask == "counter_inclusive" else {}
    name = mask.split("_")[0]
    o = _run(cc, cache, q, new, lens, hq, hkv, name, layer=1, **kw)
    assert_attention_close(f64(o), _oracle(cache, q, new, lens, hq, hkv, name, bool(kw), layer=1), f"{case} {mask}")


@pytest.mark.parametrize("new,lens,hq,hkv,d", [([1], [9000], 4, 1, 128), ([1, 1], [5001, 37], 4, 2, 64),
                                               ([70], [4100], 2, 1, 128), ([300, 1], [3000, 2500], 2, 2, 64)])
def test_attention_in_pieces(new, lens, hq, hkv, d):
    """Long caches of few heads are cut into pieces and joined; the plan may reach beyond the longest."""
    from paper_2607_27600_amd import cc
    print(f"[attn8 pieces] {new} {lens} {hq} {hkv} {d}", flush=True)
    cache = Cache8(lens, hkv, d, page=16, block=16, seed=23, fill=0x7f, room=5000)
    q = _q(new, hq, d, 24)
    want = _oracle(cache, q, new, lens, hq, hkv, "causal")
    for longest in (max(lens), max(lens) + 4321):
        o = _run(cc, cache, q, new, lens, hq, hkv, "causal", longest=longest)
        assert_attention_close(f64(o), want, f"{longest}")
    again = _run(cc, cache, q, new, lens, hq, hkv, "causal", longest=max(lens))
    assert torch.equal(again, _run(cc, cache, q, new, lens, hq, hkv, "causal", longest=max(lens)))


@pytest.mark.parametrize("new,d", [([3, 5, 2], 128), ([100, 5, 70], 128), ([100, 90, 2], 64)])
def test_rows_that_see_nothing(new, d):
    """More queries than entries: those that stand before the first see nothing (causal); an empty sequence."""
    from paper_2607_27600_amd import cc
    hq, hkv = 4, 2
    lens = [2, 0, 1]
    cache = Cache8([max(x, 1) for x in lens], hkv, d, page=16, block=16, seed=25, fill=0x7f, room=64)
    q = _q(new, hq, d, 26)
    for mask in ("causal", "counter"):
        o = _run(cc, cache, q, new, lens, hq, hkv, mask, longest=90)
        want = _oracle(cache, q, new, lens, hq, hkv, mask)
        assert_attention_close(f64(o), want, mask)
        assert np.all(f64(o)[(want == 0).all(-1)] == 0)


@pytest.mark.parametrize("new,n", [([4], 100), ([40], 200), ([150], 150)])
@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("mask", ["causal", "counter"])
def test_nan_reaches_only_rows_that_see_it(new, n, d, mask):
    from paper_2607_27600_amd import cc
    hq, hkv, m = 4, 2, new[0]
    print(f"[attn8 nan] {new} {n} {d} {mask}", flush=True)
    cache = Cache8([n], hkv, d, page=16, block=16, seed=27, fill=0x7f, room=64)
    # a NaN value in one dim, and a NaN key, in entries that only some of the queries see
    tv, tk = n - 2, n - 1 - m // 2
    for c, t, e, which in ((0, tv, 5, "v"), (1, tk, 9, "k")):
        codes, sc = cache.plane(0, 0, c, which, n=n)
        codes[t, e] = 0xff
        cache.put(0, 0, c, which, codes, sc)
        cache.t[which].copy_(torch.from_numpy(cache.host[which]))
    q = _q(new, hq, d, 28)
    o = f64(_run(cc, cache, q, new, [n], hq, hkv, mask))
    want = _oracle(cache, q, new, [n], hq, hkv, mask)
    at = np.arange(m) + n - m
    sees = (lambda t: at >= t) if mask == "causal" else (lambda t: at < t)
    nan = np.zeros_like(want, dtype=bool)
    nan[np.ix_(sees(tv), [0, 1], [5])] = True
    nan[np.ix_(sees(tk), [2, 3])] = True
    np.testing.assert_array_equal(np.isnan(want), nan)
    np.testing.assert_array_equal(np.isnan(o), nan)
    assert_attention_close(np.where(nan, 0, o), np.where(nan, 0, want))


@pytest.mark.parametrize("new,n", [([1], 300), ([90], 300)])
def test_scales_far_apart_and_peaked_rows(new, n):
    """Blocks whose scales differ by 2^60, and logits so large that one entry takes all."""
    from paper_2607_27600_amd import cc
    hq, hkv, d = 4, 1, 128
    cache = Cache8([n], hkv, d, block=16, seed=29)
    codes, sc = cache.plane(0, 0, 0, "v", n=n)
    sc[:] = np.random.default_rng(30).integers(97, 157, len(sc))
    cache.put(0, 0, 0, "v", codes, sc)
    codes, sc = cache.plane(0, 0, 0, "k", n=n)
    sc[::3] += 4
    cache.put(0, 0, 0, "k", codes, sc)
    for t in ("k", "v", "ks", "vs"):
        cache.t[t].copy_(torch.from_numpy(cache.host[t]))
    q = _q(new, hq, d, 31)
    want = _oracle(cache, q, new, [n], hq, hkv, "causal")
    o = f64(_run(cc, cache, q, new, [n], hq, hkv, "causal"))
    # Relative to the row's probability-weighted magnitudes: the probabilities and the output are
    # rounded to bf16 (2^-8 each); logits reach some hundreds here, and fp32 sums of 128 products leave
    # up to 2^-17 of that, 1e-3 of a probability.
    k, v = cache.values(0, 0, 0, "k", n), np.abs(cache.values(0, 0, 0, "v", n))
    size = np.stack([O8.attention(f64(q)[:, h], k, v, "causal") for h in range(hq)], 1)
    assert np.all(np.abs(o - want) <= (2.0 ** -8 + 1e-3) * size + 2.0 ** -8 * np.abs(want))


def test_lengths_on_the_device_in_a_graph():
    """A captured call follows kv_lens; lengths beyond the plan are cut to it, negative ones are empty."""
    from paper_2607_27600_amd import cc
    hq, hkv, d, new = 8, 2, 128, [1, 1, 2]
    cache = Cache8([600, 300, 77], hkv, d, page=16, block=16, seed=32, room=200)
    q = _q(new, hq, d, 33)
    p = _problem(cc, new, hq, hkv, d)
    kv, lens = cache.view(cc), i32([1, 1, 2])
    o = torch.empty_like(q)
    ws = torch.empty(max(1, cc.cc_attention_kv8_workspace(p, "causal", 600)), dtype=torch.uint8, device="cuda")
    g = torch.cuda.CUDAGraph()
    cc.cc_attention_kv8(p, q, kv, 0, lens, 600, o, workspace=ws)
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        cc.cc_attention_kv8(p, q, kv, 0, lens, 600, o, workspace=ws)
    for now in ([600, 300, 77], [1, 17, 2], [599, 0, 40], [10**6, -5, 77]):
        lens.copy_(i32(now))
        o.fill_(3.0)
        g.replay()
        torch.cuda.synchronize()
        real = [min(max(x, 0), 600) for x in now]
        assert_attention_close(f64(o), _oracle(cache, q, new, real, hq, hkv, "causal"), str(now))


def test_sequences_beyond_the_listed_ones():
    """More sequences of both classes than a launch lists."""
    from paper_2607_27600_amd import cc
    hq, hkv, d = 4, 2, 64
    r = np.random.default_rng(34)
    new = [int(x) for x in r.choice([0, 1, 1, 2, 40], 150)]
    lens = [m + int(x) for m, x in zip(new, r.integers(1, 60, 150))]
    cache = Cache8(lens, hkv, d, page=16, block=16, seed=35, fill=0x7f)
    q = _q(new, hq, d, 36)
    o = _run(cc, cache, q, new, lens, hq, hkv, "causal")
    assert_attention_close(f64(o), _oracle(cache, q, new, lens, hq, hkv, "causal"))


def test_two_graphs_share_a_workspace():
    """Calls of both kernels captured in two graphs that use one workspace in turn, an eager call between."""
    from paper_2607_27600_amd import cc
    hq, hkv, d, lens = 8, 2, 128, [3000, 1500]
    cache = Cache8(lens, hkv, d, page=64, block=32, seed=41)
    kv, ld = cache.view(cc), i32(lens)
    calls = []
    for new in ([1, 2], [3, 40]):
        calls.append((_problem(cc, new, hq, hkv, d), _q(new, hq, d, 42 + new[0])))
    size = max(cc.cc_attention_kv8_workspace(p, "causal", 3000) for p, _ in calls)
    assert size > 0
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    want = [cc.cc_attention_kv8(p, q, kv, 0, ld, 3000) for p, q in calls]
    outs = [torch.empty_like(q) for _, q in (*calls, calls[1])]
    torch.cuda.synchronize()
    graphs = []
    for (p, q), o in zip(calls, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            cc.cc_attention_kv8(p, q, kv, 0, ld, 3000, o, workspace=ws)
        graphs.append(g)
    for i in range(3):
        for o in outs:
            o.fill_(5.0)
        ws.fill_(0x7f + i)
        graphs[0].replay()
        cc.cc_attention_kv8(*calls[1], kv, 0, ld, 3000, outs[2], workspace=ws)
        graphs[1].replay()
        torch.cuda.synchronize()
        for o, x in zip(outs, (want[0], want[1], want[1])):
            assert torch.equal(o, x)


@pytest.mark.parametrize("new", [1, 40])
def test_offsets_past_32_bits(new):
    """Entries 64 KiB apart: appended, attended to and compacted beyond 4 GiB of their plane."""
    from paper_2607_27600_amd import cc
    from tests.kv8_util import quantize
    n, d, hq, block, tok = 70000, 64, 4, 16, 1 << 16
    free, _ = torch.cuda.mem_get_info()
    if free < (12 << 30):
        pytest.skip("needs 12 GiB of device memory")
    r = np.random.default_rng(44)
    pools = {t: torch.zeros(n * tok, dtype=torch.uint8, device="cuda") for t in ("k", "v")}
    scales = {t: torch.full((-(-n // block),), 27, dtype=torch.uint8, device="cuda") for t in ("k", "v")}
    rows = {t: x.view(n, tok)[:, :d] for t, x in pools.items()}
    kv = cc.kv8_contiguous(pools["k"], pools["v"], scales["k"], scales["v"], n_layers=1, layer_stride=0, head_stride=0,
                           tok_stride=tok, scale_block=block, scale_layer_stride=0, scale_head_stride=0)
    # entries that count lie at both ends; keys of the rest are so far from the queries that they weigh nothing
    head, tail = 48, 500
    q = torch.randn(new, hq, d, generator=torch.Generator().manual_seed(45)).abs().to(torch.bfloat16).cuda()
    far = np.full((n - head - tail, d), -300.0)
    vals = {"k": np.concatenate([r.normal(0, 1, (head, d)), far]), "v": r.normal(0, 1, (n - tail, d))}
    want = {}
    for t, x in vals.items():
        codes, sc = quantize(x[:head], block)
        c2, s2 = quantize(x[head:1024], block)
        if t == "k":
            codes, sc = np.concatenate([codes, np.broadcast_to(c2[-1], (n - tail - head, d))]), np.concatenate(
                [sc, np.full(-(-(n - tail) // block) - head // block, s2[-1])])
        else:
            codes, sc = quantize(x, block)
        rows[t][: n - tail].copy_(torch.from_numpy(np.ascontiguousarray(codes)))
        scales[t][: len(sc)].copy_(torch.from_numpy(sc.astype(np.uint8)))
    p = cc.problem(dtype="bf16", cu_seqlens=[0, tail], n_heads_q=hq, n_heads_kv=1, head_dim=d, hidden=64, vocab=1)
    g = torch.Generator().manual_seed(46)
    add = {t: torch.randn(tail, 1, d, generator=g).to(torch.bfloat16).cuda() for t in ("k", "v")}
    cc.cc_append_kv8(p, kv, add["k"], add["v"], i32([n - tail]), capacity=n, rotate=False)
    torch.cuda.synchronize()

    def values(t, e):   # what the cache holds
        sv = O8.scale_value(scales[t].cpu().numpy())
        e = np.asarray(e)
        return O8.e4m3_decode(rows[t][torch.from_numpy(e).cuda()].cpu().numpy()) * sv[e // block][:, None]

    ends = np.concatenate([np.arange(head), np.arange(n - tail, n)])
    assert np.all(np.abs(values("k", ends[head:]) - f64(add["k"])[:, 0]) <= 2.0 ** -4 * np.abs(f64(add["k"])[:, 0]) + 2.0 ** -9)
    pq = _problem(cc, [new], hq, 1, d)
    o = cc.cc_attention_kv8(pq, q, kv, 0, i32([n]), n)
    torch.cuda.synchronize()
    k, v, qh = values("k", ends), values("v", ends), f64(q)
    # (the last `new` entries of `ends` are the queries' own, as in the whole cache)
    ref = np.stack([O8.attention(qh[:, h], k, v, "causal") for h in range(hq)], 1)
    assert_attention_close(f64(o), ref)
    keep = torch.arange(n - 64, n, dtype=torch.int32, device="cuda")
    moved = values("v", np.arange(n - 64, n))
    pc = cc.problem(dtype="bf16", cu_seqlens=[0, n], n_heads_q=1, n_heads_kv=1, head_dim=d, hidden=64, vocab=1)
    cc.cc_compact_kv8(pc, kv, keep, [64], 0)
    torch.cuda.synchronize()
    np.testing.assert_allclose(values("v", np.arange(64)), moved, rtol=2.0 ** -4, atol=2.0 ** -9)


@pytest.mark.parametrize("n,most,longest,hkv", [(150, 5000, 5000, 2), (4200, 40, 3000, 1), (700, 60, 3000, 3)])
def test_shares_of_many_sequences(n, most, longest, hkv):
    """Work shared out over more sequences than a wave has lanes, up to more than 64 for each lane; rows
    whose entries lie in one share, in a few and in many."""
    from paper_2607_27600_amd import cc
    d, hq = 64, 2 * hkv
    r = np.random.default_rng(n)
    new = [int(x) for x in r.choice([0, 1, 1, 3], n)]
    lens = [m + int(x) for m, x in zip(new, r.integers(0, 30, n))]
    lens[n // 3], lens[n - 1], new[n // 3], new[n - 1] = most, most - 1, 1, 2
    cache = Cache8(lens, hkv, d, page=16 if n == 150 else 0, block=16, seed=n + 1, fill=0x7f)
    q = _q(new, hq, d, n + 2)
    o = _run(cc, cache, q, new, lens, hq, hkv, "causal", longest=longest)
    assert_attention_close(f64(o), _oracle(cache, q, new, lens, hq, hkv, "causal"))


@pytest.mark.parametrize("new,n,hq,hkv,d", [([64], 9100, 12, 3, 64), ([300], 9100, 4, 4, 128), ([90, 70], 9000, 4, 2, 128),
                                            ([40], 300, 4, 2, 128)])
@pytest.mark.parametrize("mask", ["causal", "counter"])
def test_many_rows_in_pieces(new, n, hq, hkv, d, mask):
    """Rows in few and in more pieces than one group of lanes joins alone, and sequences shorter than the
    plan's, which have fewer."""
    from paper_2607_27600_amd import cc
    lens = [max(m, n // (b + 1) - 17 * b) for b, m in enumerate(new)]
    cache = Cache8(lens, hkv, d, page=64, block=32, seed=n + d, fill=0x7f)
    q = _q(new, hq, d, n + 1)
    o = _run(cc, cache, q, new, lens, hq, hkv, mask)
    assert_attention_close(f64(o), _oracle(cache, q, new, lens, hq, hkv, mask))


@pytest.mark.parametrize("new,lens,hq,hkv,d", [([1], [50], 64, 1, 128), ([2, 1], [300, 1], 96, 2, 64), ([1, 1], [2500, 3], 40, 1, 128)])
def test_many_heads_of_a_group(new, lens, hq, hkv, d):
    """A single query of a group of more heads than count as few rows."""
    from paper_2607_27600_amd import cc
    cache = Cache8(lens, hkv, d, page=16, block=16, seed=hq, fill=0x7f)
    q = _q(new, hq, d, hq + 1)
    for mask in ("causal", "counter"):
        o = _run(cc, cache, q, new, lens, hq, hkv, mask)
        assert_attention_close(f64(o), _oracle(cache, q, new, lens, hq, hkv, mask))


def test_a_plan_for_no_entries():
    """max_kv_len 0: every length is cut to it, every output is zero and no page is looked up."""
    from paper_2607_27600_amd import cc
    new, hq, hkv, d = [1, 40, 2], 4, 2, 128
    cache = Cache8([9, 40, 2], hkv, d, page=16, block=16, seed=61)
    cache.bt.fill_(-1)
    o = _run(cc, cache, _q(new, hq, d, 62), new, [9, 40, 2], hq, hkv, "causal", longest=0)
    assert torch.count_nonzero(o) == 0


@pytest.mark.parametrize("new,hq,hkv,d", [([8], 16, 4, 128), ([8, 5], 16, 4, 64), ([40], 8, 2, 128)])
def test_drafts_in_a_graph(new, hq, hkv, d):
    """Two row blocks, and the kernel for many, captured and replayed as the lengths grow."""
    from paper_2607_27600_amd import cc
    cache = Cache8([3000] * len(new), hkv, d, page=16, block=16, seed=71)
    q, kv, lens = _q(new, hq, d, 72), cache.view(cc), i32([2000] * len(new))
    p = _problem(cc, new, hq, hkv, d)
    o = torch.empty_like(q)
    ws = torch.empty(max(1, cc.cc_attention_kv8_workspace(p, "causal", 3000)), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        cc.cc_attention_kv8(p, q, kv, 0, lens, 3000, o, workspace=ws)
    for n in (2000, 2999, 45):
        lens.fill_(n)
        o.fill_(9.0)
        g.replay()
        torch.cuda.synchronize()
        assert_attention_close(f64(o), _oracle(cache, q, new, [n] * len(new), hq, hkv, "causal"), str(n))


@pytest.mark.parametrize("byte,code", [(247, 0x78), (250, 0x7e), (254, 0xc0), (255, 0x40)])
@pytest.mark.parametrize("new,n", [([4], 100), ([40], 200), ([150], 150)])
@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("mask", ["causal", "counter"])
def test_values_past_bf16_reach_only_rows_that_see_them(new, n, d, mask, byte, code):
    """Elements of 2^128 and more, which are infinite in bf16 (the first is what appending 3.4e38 writes): a row
    that may not see one is as if it held zero, a row that sees it is not finite there."""
    from paper_2607_27600_amd import cc
    hq, hkv, m = 4, 2, new[0]
    print(f"[attn8 wide] {new} {n} {d} {mask} {byte}", flush=True)
    cache = Cache8([n], hkv, d, page=16, block=16, seed=81, fill=0x7f, room=64)
    tv, tk, dims = n - 2, n - 1 - m // 2, [5, d - 1]
    want = None
    for held in (False, True):   # (the 64-bit result of rows that do not see them: they hold zeros)
        for c, t, which in ((0, tv, "v"), (1, tk, "k")):
            codes, sc = cache.plane(0, 0, c, which, n=n)
            sc[t // 16] = byte
            codes[t // 16 * 16:t // 16 * 16 + 16] = 0    # (others of the block: zeros)
            if held:
                codes[t, dims] = code
            cache.put(0, 0, c, which, codes, sc)
        if not held:
            q = _q(new, hq, d, 82)
            want = _oracle(cache, q, new, [n], hq, hkv, mask)
    for t in ("k", "v", "ks", "vs"):
        cache.t[t].copy_(torch.from_numpy(cache.host[t]))
    o = f64(_run(cc, cache, q, new, [n], hq, hkv, mask))
    at = np.arange(m) + n - m
    sees = (lambda t: at >= t) if mask == "causal" else (lambda t: at < t)
    assert sees(tv).any() and not sees(tv).all()
    hit = np.zeros(want.shape, bool)
    hit[np.ix_(sees(tv), [0, 1], dims)] = True
    assert not np.isfinite(o[hit]).any()
    hit[np.ix_(sees(tk), [2, 3])] = True       # (a logit past fp32 on one side or the other: nothing is asked)
    assert_attention_close(np.where(hit, 0, o), np.where(hit, 0, want))


def test_more_row_blocks_than_one_launch_has(memory_given_back):
    """A long chunk beside hundreds of short ones, 64 heads: (blocks of the longest) * sequences * heads passes
    2^24 workgroups; the long one's last block comes with a second launch."""
    from paper_2607_27600_amd import cc
    n_seqs, h, d, n, short = 600, 64, 64, 64, 33
    long = 436 * 128 + 77
    assert 437 * n_seqs * h >= 1 << 24 > 436 * n_seqs * h
    new = [short] * n_seqs
    new[7] = long
    r = np.random.default_rng(91)
    # one plane a head, which all sequences share
    codes, scales = zip(*(quantize(r.normal(0, 1, (n, d)), 16) for _ in range(2 * h)))
    t = lambda x: torch.from_numpy(np.stack(x)).cuda()
    k, v, ks, vs = t(codes[:h]), t(codes[h:]), t(scales[:h]), t(scales[h:])
    kv = cc.kv8_contiguous(k, v, ks, vs, n_layers=1, layer_stride=0, head_stride=n * d, tok_stride=d, scale_block=16,
                           scale_layer_stride=0, scale_head_stride=n // 16)
    q = torch.randn(sum(new), h, d, generator=torch.Generator("cuda").manual_seed(92), device="cuda").to(torch.bfloat16)
    o = torch.full_like(q, 7.0)
    cc.cc_attention_kv8(_problem(cc, new, h, h, d), q, kv, 0, i32([n] * n_seqs), n, o, mask="counter")
    torch.cuda.synchronize()
    cu = cu_of(new)
    val = lambda c, s, i: O8.values(c[i], s[i], 16)
    for b, i0, i1 in ((0, 0, short), (7, 0, 130), (7, 200 * 128, 200 * 128 + 8), (7, 436 * 128 - 3, long), (8, 0, short),
                      (n_seqs - 1, 0, short)):
        for c in (0, 31, 63):
            qq = f64(q[cu[b]:cu[b + 1], c])
            kk, vv = val(codes[:h], scales[:h], c), val(codes[h:], scales[h:], c)
            # (rows of a sequence stand at its cache's end: those asked for, as the last of a shorter one)
            want = O8.attention(qq[i0:], kk, vv, "counter")[: i1 - i0]
            assert_attention_close(f64(o[cu[b] + i0:cu[b] + i1, c])[:, None], want[:, None], f"{b} {i0} {c}")
    assert not (o == 7.0).all(-1).any()     # every row has been written


def test_more_rows_to_join_than_one_launch_has(memory_given_back):
    """Few rows of 130 sequences and 2^16 heads, 32 at the most: past 2^24 workgroups of the join, whose second
    launch has the last sequences; of the last one, heads 877 and 3364 are cut between two workgroups' shares."""
    from paper_2607_27600_amd import cc
    n_seqs, h, d, n = 130, 1 << 16, 64, 2400
    assert n_seqs * h * 32 // 16 >= 1 << 24 > (n_seqs - 3) * h * 32 // 16
    new, lens = [1] * n_seqs, [3] * n_seqs
    new[11], lens[11], lens[-1] = 32, 60, n
    p = _problem(cc, new, h, h, d)
    size = cc.cc_attention_kv8_workspace(p, "causal", n)
    free, _ = torch.cuda.mem_get_info()
    if free < size + (8 << 30):
        pytest.skip(f"needs {(size >> 30) + 8} GiB of device memory")
    r = np.random.default_rng(93)
    # one plane, which all sequences and heads share
    codes, scales = zip(*(quantize(r.normal(0, 1, (n, d)), 16) for _ in range(2)))
    t = lambda x: torch.from_numpy(x).cuda()
    kv = cc.kv8_contiguous(t(codes[0]), t(codes[1]), t(scales[0]), t(scales[1]), n_layers=1, layer_stride=0, head_stride=0,
                           tok_stride=d, scale_block=16, scale_layer_stride=0, scale_head_stride=0)
    q = torch.randn(sum(new), h, d, generator=torch.Generator("cuda").manual_seed(94), device="cuda").to(torch.bfloat16)
    o = torch.full_like(q, 7.0)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    cc.cc_attention_kv8(p, q, kv, 0, i32(lens), n, o, workspace=ws)
    torch.cuda.synchronize()
    del ws
    cu = cu_of(new)
    for b in (0, 11, n_seqs - 3, n_seqs - 2, n_seqs - 1):
        kk, vv = (O8.values(codes[i][:lens[b]], scales[i], 16) for i in (0, 1))
        for c in (0, 877, 3364, h - 1):
            want = O8.attention(f64(q[cu[b]:cu[b + 1], c]), kk, vv, "causal")
            assert_attention_close(f64(o[cu[b]:cu[b + 1], c])[:, None], want[:, None], f"{b} {c}")
    assert not (o == 7.0).all(-1).any()


@pytest.mark.parametrize("mask", ["causal", "counter"])
@pytest.mark.parametrize("new,hq,hkv,d", [([20, 0, 700, 1, 33, 17, 300], 4, 2, 128), ([40] * 20 + [1] * 40 + [3000] + [0, 17] * 50, 2, 1, 64)],
                         ids=["listed", "all"])
def test_ragged_chunks_in_pieces(new, hq, hkv, d, mask):
    """Pieces of sequences of different numbers of rows, beside sequences of few rows and none, listed and
    walked as a whole; the workspace holds no more than asked for."""
    from paper_2607_27600_amd import cc
    r = np.random.default_rng(95)
    lens = [m + int(x) for m, x in zip(new, r.integers(0, 2500, len(new)))]
    lens[2] = max(lens[2], 2900)
    cache = Cache8(lens, hkv, d, page=64, block=32, seed=96, fill=0x7f)
    q = _q(new, hq, d, 97)
    p = _problem(cc, new, hq, hkv, d)
    size = cc.cc_attention_kv8_workspace(p, mask, max(lens))
    assert size > sum(new) * hq * d * 4       # pieces
    ws = torch.full((size + 4096,), 0x7f, dtype=torch.uint8, device="cuda")
    o = torch.full_like(q, 7.0)
    cc.cc_attention_kv8(p, q, cache.view(cc), 0, i32(lens), max(lens), o, mask=mask, workspace=ws[:size])
    torch.cuda.synchronize()
    assert (ws[size:] == 0x7f).all()
    assert_attention_close(f64(o), _oracle(cache, q, new, lens, hq, hkv, mask))


# ---- equal shares: the kernel for few rows where there is much work.  A copy of its rule, to see that a case
# gets there and what its shares cut.

def _shares(new, lens, g, hkv, longest):
    """(mode, what the shares cut) of the few-row sequences of a call."""
    few = [0 < m * g <= 32 for m in new]
    n = sum(few)
    n_list = n if n <= 64 else len(new)
    if longest <= (2048 if n * hkv >= 128 else 1024):
        return "direct", set()
    units = [max(1, -(-min(max(x, 0), longest) // 128)) if f else 0 for x, f in zip(lens, few)]
    total, items, parts = sum(units) * hkv, n_list * hkv, 512
    if items < parts and -(-total // (parts - items)) <= 8:
        return "pieces", set()
    starts, at = [], 0                       # of every (sequence, head) along the line, two units ahead of its entries
    for u in units:
        for _ in range(hkv if u else 0):
            starts.append((at, u))
            at += u + 2
    parts = min(parts, at)
    cuts = [at * w // parts for w in range(parts + 1)]
    seen, i = set(), 0
    for w in range(1, parts):
        while starts[i][0] + starts[i][1] + 2 <= cuts[w]:
            i += 1
        off = cuts[w] - starts[i][0]
        seen.add("between" if off == 0 else "ahead of the entries" if off <= 2 else "entries")
    whole = np.searchsorted([s for s, _ in starts], cuts, side="right")
    if max(np.diff(whole)) >= 3:
        seen.add("several items in a share")
    if max(u for _, u in starts) >= 3 * at / parts:
        seen.add("an item in several shares")
    return "shares", seen


class _Windows:
    """One plane of n entries; sequence b's head h has the entries from 16 (b * step + h) on, in a contiguous cache or in
    pages of 16."""

    def __init__(self, cc, n, d, n_seqs, hkv, step, paged, seed):
        r = np.random.default_rng(seed)
        self.step = step
        n = -(-n // 16) * 16
        self.c, self.s, t = {}, {}, {}
        for w in "kv":
            self.c[w], self.s[w] = quantize(r.normal(0, 1, (n, d)) * np.exp2(r.integers(-2, 3, (n, 1))), 16)
            t[w], t[w + "s"] = torch.from_numpy(self.c[w]).cuda(), torch.from_numpy(self.s[w]).cuda()
        self.values = {w: O8.values(self.c[w], self.s[w], 16) for w in "kv"}
        if paged:
            pages = n // 16
            table = torch.arange(n_seqs)[:, None] * step + torch.arange(pages)[None]
            self.kv = cc.kv8_paged(t["k"], t["v"], t["ks"], t["vs"], table.clamp(max=pages - 1).to(torch.int32).cuda(), n_layers=1,
                                   layer_stride=0, page_stride=16 * d, head_stride=16 * d, tok_stride=d, page_size=16,
                                   scale_block=16, scale_layer_stride=0, scale_page_stride=1, scale_head_stride=1)
        else:
            self.kv = cc.kv8_contiguous(t["k"], t["v"], t["ks"], t["vs"], n_layers=1, layer_stride=0, seq_stride=16 * step * d,
                                        head_stride=16 * d, tok_stride=d, scale_block=16, scale_layer_stride=0,
                                        scale_seq_stride=step, scale_head_stride=1)

    def oracle(self, q, new, lens, hq, hkv, mask):
        g, out, at, qh = hq // hkv, [], 0, f64(q)
        for b, m in enumerate(new):
            o = np.zeros((m, hq, q.shape[2]))
            for h in range(hq if m else 0):
                i = 16 * (b * self.step + h // g)
                o[:, h] = O8.attention(qh[at:at + m, h], self.values["k"][i:i + lens[b]], self.values["v"][i:i + lens[b]], mask)
            out.append(o)
            at += m
        return np.concatenate(out)


ALL_CUTS = {"ahead of the entries", "entries", "several items in a share"}
SHARED = [
    # sequences, heads of a group, KV heads, head_dim, most new tokens, longest, paged, what is cut at least
    (300, 4, 2, 128, 4, 6000, True, ALL_CUTS),                            # walked as a whole, five sequences a lane; one row block
    (300, 4, 2, 64, 8, 6000, False, ALL_CUTS),                            # two row blocks
    (60, 2, 16, 128, 16, 3000, False, ALL_CUTS),                          # listed
    (40, 1, 20, 64, 3, 2500, True, ALL_CUTS),
    (1, 2, 16, 128, 2, 37000, False, {"entries", "an item in several shares"}),
    (3, 8, 8, 64, 4, 40000, True, {"entries", "an item in several shares"}),
    (700, 2, 1, 64, 1, 9000, False, ALL_CUTS),                            # most of them short, a few in several shares
]


@pytest.mark.parametrize("mask", ["causal", "counter"])
@pytest.mark.parametrize("case", SHARED, ids=[str(i) for i in range(len(SHARED))])
def test_equal_shares(case, mask):
    """Shares that begin and end inside an item, ahead of its entries or between items, and hold several."""
    from paper_2607_27600_amd import cc
    n, g, hkv, d, most, longest, paged, cut = case
    r = np.random.default_rng(n + d)
    new = [int(x) for x in r.integers(0 if n > 3 else 1, most + 1, n)]
    lens = [m + int(x) for m, x in zip(new, r.integers(0, 300 if n > 3 else longest, n))]
    for b in r.permutation(n)[:max(1, n // 8)]:
        new[b] = max(new[b], 1)
        lens[b] = int(r.integers(longest // 3, longest))
    if n > 100:
        new[5], lens[5], lens[6] = 40, 500, 0             # one of many rows, and one without entries
    lens[-1], new[-1] = longest, most
    mode, seen = _shares(new, lens, g, hkv, longest)
    assert mode == "shares" and cut <= seen, (mode, seen)
    print(f"[attn8 shares] {case} {mask} {seen}", flush=True)
    win = _Windows(cc, longest + 16 * (n + hkv) + 16, d, n, hkv, 1, paged, n)
    q = _q(new, g * hkv, d, n + 1)
    p = _problem(cc, new, g * hkv, hkv, d)
    for plan in (longest, longest + 900):
        if paged and plan > longest:
            continue                   # (a plan past the block table's rows is refused)
        o = torch.full_like(q, 7.0)
        cc.cc_attention_kv8(p, q, win.kv, 0, i32(lens), plan, o, mask=mask)
        torch.cuda.synchronize()
        assert_attention_close(f64(o), win.oracle(q, new, lens, g * hkv, hkv, mask), f"{plan}")


def test_pieces_and_shares_under_one_plan_in_a_graph():
    """Device lengths that take a captured call from pieces to equal shares and back."""
    from paper_2607_27600_amd import cc
    n, g, hkv, d, longest = 50, 2, 8, 64, 9000
    new = [1 + b % 3 for b in range(n)]
    r = np.random.default_rng(98)
    win = _Windows(cc, longest + 16 * (n + hkv) + 16, d, n, hkv, 1, True, 99)
    q, lens = _q(new, g * hkv, d, 100), i32([3] * n)
    p = _problem(cc, new, g * hkv, hkv, d)
    o = torch.empty_like(q)
    ws = torch.empty(max(1, cc.cc_attention_kv8_workspace(p, "causal", longest)), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cc.cc_attention_kv8(p, q, win.kv, 0, lens, longest, o, workspace=ws)
    modes = []
    for most in (20, longest, 600, 0, 4000, 150):
        now = [int(x) for x in r.integers(0, most + 1, n)]
        now[17] = most
        modes.append(_shares(new, now, g, hkv, longest)[0])
        lens.copy_(i32(now))
        o.fill_(9.0)
        ws.fill_(0x7f)
        graph.replay()
        torch.cuda.synchronize()
        assert_attention_close(f64(o), win.oracle(q, new, now, g * hkv, hkv, "causal"), str(most))
    assert {"pieces", "shares"} <= set(modes), modes


@pytest.mark.parametrize("scale", [1.0, 0.2, 0.01, 1e-20, 1e-38, 1e-40])
@pytest.mark.parametrize("new,lens,hq,hkv,d", [([1, 3], [200, 77], 8, 2, 128), ([2], [3000], 4, 1, 64), ([70, 40], [300, 90], 4, 2, 128),
                                               ([90], [2500], 2, 1, 64)])
def test_a_scale_of_the_callers(new, lens, hq, hkv, d, scale):
    """softmax_scale, few and many rows, whole and in pieces: from peaked rows to ones whose logits vanish."""
    from paper_2607_27600_amd import cc
    cache = Cache8(lens, hkv, d, page=16, block=16, seed=101, fill=0x7f, std=0.5)
    q = _q(new, hq, d, 102)
    for mask in ("causal", "counter"):
        o = _run(cc, cache, q, new, lens, hq, hkv, mask, softmax_scale=scale)
        assert_attention_close(f64(o), _oracle(cache, q, new, lens, hq, hkv, mask, scale=scale), f"{scale} {mask}")
