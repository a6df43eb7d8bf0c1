"""RefreshLoop on a bf16 cache with the inference cycle's attention, and eviction by accumulated attention weight: the cycle
against the same one in 64 bits, and a decode step of a batch behind a shared prefix captured in one graph."""
import numpy as np
import pytest
import torch

from oracle import cc_oracle, kv16_oracle as O
from synth import gen
from tests.gpu_util import assert_attention_close, bf16_host, dev, f64
from tests.kv16_util import Cache16, cu_of, i32, problem, queries

pytestmark = pytest.mark.gpu

L, HQ, HKV, DH, D, V = 2, 4, 2, 128, 512, 1000


def _model():
    from paper_2607_27600_amd.refresh import Model
    return Model(mode="last_layer", n_layers=L, n_heads_q=HQ, n_heads_kv=HKV, head_dim=DH, hidden=D, vocab=V,
                 w_lm=dev(gen.normal_bf16(7, 1, (V, D), 0.05)), w_o=dev(gen.normal_bf16(7, 2, (D, HQ * DH), 0.05)))


@pytest.mark.parametrize("recent", [0, 6])
def test_weight_cycle(recent):
    """The prompt in chunks, then single tokens; each chunk attends in every layer, a refresh keeps the heaviest."""
    from paper_2607_27600_amd.refresh import RefreshLoop
    J, h, T_prompt, T = 40, 24, 96, 160
    loop = RefreshLoop(_model(), J, h, policy="weight", n_recent=recent)
    g = torch.Generator().manual_seed(5)
    k, v = (torch.randn(L, HKV, T, DH, generator=g).to(torch.bfloat16).cuda() for _ in "kv")
    q = torch.randn(L, T, HQ, DH, generator=g).to(torch.bfloat16).cuda()
    ids, pos = torch.randint(0, V, (T,), generator=g, dtype=torch.int32).cuda(), torch.arange(T, dtype=torch.int32).cuda()
    rows = torch.randn(T, HQ * DH, generator=g).to(torch.bfloat16).cuda()
    at, w, t = np.zeros(0, int), np.zeros(0), 0      # the entries that are cached, by position, and their sums
    while t < T:
        m = min(h, T_prompt - t) if t < T_prompt else 1
        sl = slice(t, t + m)
        loop.append(k[:, :, sl], v[:, :, sl], ids[sl], pos[sl], rows[sl])
        at, w = np.concatenate([at, np.arange(t, t + m)]), np.concatenate([w, np.zeros(m)])
        for layer in range(L):
            o = loop.attend(layer, q[layer, sl].contiguous())
            torch.cuda.synchronize()
            want = np.zeros((m, HQ, DH))
            for x in range(HQ):
                kk, vv = f64(k)[layer, x // 2, at], f64(v)[layer, x // 2, at]
                want[:, x], lse = O.attention(f64(q)[layer, sl, x], kk, vv)
                w = w + O.weights(f64(q)[layer, sl, x], kk, lse)
            assert_attention_close(f64(o), want)
        n = len(at)
        assert loop.n == n
        # sums of up to 2 layers * 4 heads * 160 rows, each weight off by some 2^-16 of itself (fp32 logits)
        np.testing.assert_allclose(f64(loop.w)[0, :, :n].sum(0), w, rtol=2.0 ** -12)
        t += m
        if t % h or n <= J:
            continue
        seen = {}
        keep = loop.refresh(lambda s, kept: seen.update(s=s.cpu().numpy(), k=kept.cpu().numpy()))
        torch.cuda.synchronize()
        kept = keep.cpu().numpy()
        np.testing.assert_array_equal(kept, cc_oracle.select_keep(seen["s"], J))
        np.testing.assert_array_equal(np.isinf(seen["s"]), np.arange(n) >= n - recent)
        np.testing.assert_allclose(seen["s"][: n - recent], w[: n - recent], rtol=2.0 ** -12)
        at, w = at[kept], w[kept]
        np.testing.assert_array_equal(loop.pos.cpu().numpy()[:J], at)
        np.testing.assert_array_equal(loop.ids.cpu().numpy()[:J], ids.cpu().numpy()[at])
        np.testing.assert_array_equal(bf16_host(loop.rows)[:J], bf16_host(rows)[at])
        np.testing.assert_array_equal(bf16_host(loop.k)[:, :, :J], bf16_host(k)[:, :, at])
        np.testing.assert_allclose(f64(loop.w)[0, :, :J].sum(0), w, rtol=2.0 ** -12)
    assert loop.refreshes >= 4


def test_surprise_cycle_attends():
    """The counter-causal loop on a bf16 cache has the same attention."""
    from paper_2607_27600_amd.refresh import RefreshLoop
    loop = RefreshLoop(_model(), 20, 12)
    g = torch.Generator().manual_seed(6)
    k, v = (torch.randn(L, HKV, 30, DH, generator=g).to(torch.bfloat16).cuda() for _ in "kv")
    i = torch.arange(30, dtype=torch.int32).cuda()
    loop.append(k, v, i, i, torch.randn(30, HQ * DH, generator=g).to(torch.bfloat16).cuda())
    kept = loop.refresh().cpu().numpy()
    q = queries([3], HQ, DH, 7)
    for layer in range(L):
        want = np.stack([O.attention(f64(q)[:, x], f64(k)[layer, x // 2, kept], f64(v)[layer, x // 2, kept])[0] for x in range(HQ)], 1)
        assert_attention_close(f64(loop.attend(layer, q)), want)


def test_loop_refuses():
    from paper_2607_27600_amd.refresh import RefreshLoop
    for kw in (dict(policy="age"), dict(policy="weight", cache="e4m3"), dict(n_recent=4), dict(policy="weight", n_recent=-1)):
        with pytest.raises(ValueError):
            RefreshLoop(_model(), 4, 4, **kw)
    with pytest.raises(ValueError):
        RefreshLoop(_model(), 4, 4, policy="weight").attend(0, torch.zeros(1, HQ, DH, dtype=torch.bfloat16, device="cuda"))


def test_a_served_step_in_a_graph():
    """A batch behind a shared prefix: append, attend, accumulate, in one captured step that is replayed as lengths advance."""
    from paper_2607_27600_amd import cc
    hq, hkv, d, n_seqs, n, steps = 8, 2, 128, 5, 700, 6
    lens0 = [3, 100, 0, 41, 7]
    own = Cache16(lens0, hkv, d, page=16, seed=8, room=steps + 16, fill=0.0)
    pre = Cache16([n], hkv, d, page=16, seed=9)
    p, kv = problem(cc, [1] * n_seqs, hq, hkv, d, rope_theta=1e4), own.view(cc)
    x = cc.prefix(pre.view(cc), [0, n_seqs], i32([n]), n)
    cached, lens, pos = i32(lens0), i32(lens0), i32([n + m for m in lens0])
    most = max(lens0) + steps + 1
    new = {t: torch.empty(n_seqs, hkv, d, dtype=torch.bfloat16, device="cuda") for t in "kv"}
    qn, qr = (torch.empty(n_seqs, hq, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    o, lse = torch.empty_like(qr), torch.empty(n_seqs, hq, device="cuda")
    w = torch.zeros(n_seqs, hkv, most, device="cuda")
    ws = torch.empty(cc.cc_attention_prefix_workspace(p, x, most) + 256, dtype=torch.uint8, device="cuda")
    ww = torch.empty(max(1, cc.cc_attention_weights_workspace(p, most)), dtype=torch.uint8, device="cuda")

    def step():
        cc.cc_append_kv(p, kv, new["k"], new["v"], cached, pos_ids=pos, q=qn, q_out=qr)
        lens.copy_(cached + 1)
        cc.cc_attention_prefix(p, qr, x, kv, 0, lens, most, o, lse=lse, workspace=ws)
        cc.cc_attention_weights(p, qr, kv, 0, lens, most, lse, w, prev=w, prev_lens=cached, workspace=ww)
        cached.add_(1)
        pos.add_(1)
    for t in (*new.values(), qn):
        t.zero_()
    step()          # (a warm-up, taken back)
    torch.cuda.synchronize()
    cached.copy_(i32(lens0))
    pos.copy_(i32([n + m for m in lens0]))
    w.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    torch.cuda.synchronize()
    g = torch.Generator().manual_seed(10)
    sums = np.zeros((n_seqs, hkv, most))
    for i in range(steps):
        for t in (*new.values(), qn):
            t.copy_(torch.randn(t.shape, generator=g).to(torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        now = [m + i + 1 for m in lens0]
        assert cached.tolist() == now
        ro, rl = np.zeros((n_seqs, hq, d)), np.zeros((n_seqs, hq))
        for b in range(n_seqs):
            for c in range(hkv):
                kk, vv = (own.values(0, b, c, t, now[b]) for t in "kv")
                kp, vp = (pre.values(0, 0, c, t) for t in "kv")
                for hh in range(c * 4, c * 4 + 4):
                    qh = f64(qr)[b:b + 1, hh]
                    ro[b, hh], rl[b, hh] = (y[0] for y in O.attention(qh, kk, vv, kp, vp))
                    sums[b, c, : now[b]] += O.weights(qh, kk, rl[b:b + 1, hh])
        assert_attention_close(f64(o), ro)
        np.testing.assert_allclose(f64(lse), rl, atol=1e-4)     # (128 products of some 10 in all, 2^-24 each)
        np.testing.assert_allclose(f64(w), sums, rtol=2.0 ** -12, atol=1e-9)
        assert float(w.sum()) < hq * n_seqs * (i + 1)           # the rest is the prefix's
