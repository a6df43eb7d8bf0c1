"""The operators together, as a program runs them: the refresh cycle on a cache in 8 bits against the
oracle at every step, and a decode step of a served batch (append, attention, output projection, LM
head) in one captured graph."""
import numpy as np
import pytest
import torch

from oracle import cc_oracle as O
from oracle import kv8_oracle as O8
from synth import gen
from tests.gpu_util import assert_attention_close, assert_scores_close, bf16_host, dev, f64
from tests.kv8_util import Cache8, cu_of, i32

pytestmark = pytest.mark.gpu

L, HQ, HKV, DH, D, V = 2, 4, 2, 128, 512, 1000


def _model(mode, packed):
    from paper_2607_27600_amd import cc
    from paper_2607_27600_amd.refresh import Model
    host = dict(w_lm=gen.normal_bf16(7, 1, (V, D), 0.05), w_o=gen.normal_bf16(7, 2, (D, HQ * DH), 0.05))
    w_lm = dev(host["w_lm"])
    if mode == "last_layer_fused":
        w_lm = cc.cc_fuse_wo_lmhead("bf16", w_lm, dev(host["w_o"]))
    m = Model(mode=mode, n_layers=L, n_heads_q=HQ, n_heads_kv=HKV, head_dim=DH, hidden=D, vocab=V, w_lm=w_lm,
              w_o=dev(host["w_o"]))
    if packed:
        m.w_lm_packed = cc.cc_pack_lmhead(w_lm)
    return m, host


def _planes(loop, block):
    """Codes and scales of the loop's cache on the host."""
    return {k: getattr(loop, n).cpu().numpy().copy() for k, n in
            (("k", "k"), ("v", "v"), ("ks", "k_scale"), ("vs", "v_scale"))}


@pytest.mark.parametrize("mode,chunked,packed,block", [("last_layer", True, False, 16), ("last_layer", False, True, 32),
                                                       ("last_layer_fused", True, False, 16),
                                                       ("last_layer_fused", True, True, 64)])
def test_refresh_cycle(mode, chunked, packed, block):
    from paper_2607_27600_amd.refresh import RefreshLoop, run_stream
    print(f"[loop8] {mode} {chunked} {packed} {block}", flush=True)
    J, h, T_prompt, T = 40, 24, 100, 130
    model, host = _model(mode, packed)
    loop = RefreshLoop(model, J, h, capacity=None if chunked else T, cache="e4m3", scale_block=block)
    r = np.random.default_rng(3)
    k, v = gen.normal_bf16(3, 100, (L, HKV, T, DH)), gen.normal_bf16(3, 101, (L, HKV, T, DH))
    rows, ids = gen.normal_bf16(3, 102, (T, model.row_width)), r.integers(0, V, T).astype(np.int32)
    kd, vd, rd, idd = dev(k), dev(v), dev(rows), torch.from_numpy(ids).cuda()
    k64, v64 = gen.bf16_to_f64(k), gen.bf16_to_f64(v)
    # the oracle's cache, appended and compacted beside the loop's
    cap = loop.cap
    state = {"n": 0, "ids": np.zeros(cap, np.int32), "rows": np.zeros((cap, model.row_width), np.uint16),
             "pos": np.zeros(cap, np.int32)}
    for t in ("k", "v"):
        state[t] = np.zeros((L, HKV, cap, DH), np.uint8)
        state[t + "s"] = np.zeros((L, HKV, -(-cap // block)), np.uint8)

    def entry(t0, t1):
        n = state["n"]
        for l in range(L):
            for c in range(HKV):
                for t, x in (("k", k64), ("v", v64)):
                    O8.append(state[t][l, c], state[t + "s"][l, c], n, x[l, c, t0:t1], block, cap)
        sl = slice(n, n + t1 - t0)
        state["ids"][sl], state["rows"][sl], state["pos"][sl] = ids[t0:t1], rows[t0:t1], np.arange(t0, t1)
        state["n"] = n + t1 - t0
        return (kd[:, :, t0:t1], vd[:, :, t0:t1], idd[t0:t1], torch.arange(t0, t1, dtype=torch.int32, device="cuda"),
                rd[t0:t1])

    checked = []

    def compare():
        n = state["n"]
        got = _planes(loop, block)
        for t in ("k", "v"):
            np.testing.assert_array_equal(got[t][:, :, :n], state[t][:, :, :n])
            np.testing.assert_array_equal(got[t + "s"][:, :, : -(-n // block)], state[t + "s"][:, :, : -(-n // block)])

    def hook(scores, keep):
        n = state["n"]
        compare()
        dense = [np.stack([O8.values(state[t][-1, c][:n], state[t + "s"][-1, c], block) for c in range(HKV)])
                 for t in ("k", "v")]
        q = gen.bf16_to_f64(state["rows"][:n]).reshape(n, HQ, DH)
        want = O.last_layer_scores(q, *dense, host["w_o"], host["w_lm"], state["ids"][:n], [0, n])
        assert_scores_close(f64(scores), want, "bf16", f"refresh at {n}")
        kl = O.select_keep(scores.cpu().numpy(), J)
        np.testing.assert_array_equal(keep.cpu().numpy(), kl)
        for l in range(L):
            for c in range(HKV):
                for t in ("k", "v"):
                    codes, sc = O8.compact(state[t][l, c][:n], state[t + "s"][l, c], kl, block)
                    state[t][l, c][:J] = codes
                    state[t + "s"][l, c][: len(sc)] = sc
        for a in ("ids", "rows", "pos"):
            state[a][:J] = state[a][kl]
        state["n"] = J
        checked.append(n)

    run_stream(loop, entry, T_prompt, T, chunked=chunked, hook=hook)
    torch.cuda.synchronize()
    assert len(checked) == (T // h if chunked else 1) or len(checked) == loop.refreshes
    assert loop.refreshes == len(checked) > 0
    compare()
    n = state["n"]
    np.testing.assert_array_equal(loop.ids.cpu().numpy()[:n], state["ids"][:n])
    np.testing.assert_array_equal(loop.pos.cpu().numpy()[:n], state["pos"][:n])
    np.testing.assert_array_equal(bf16_host(loop.rows)[:n], state["rows"][:n])
    # the inference cycle's attention over what is left
    q = torch.randn(3, HQ, DH, generator=torch.Generator().manual_seed(4)).to(torch.bfloat16).cuda()
    for layer in range(L):
        o = loop.attend(layer, q)
        want = np.zeros((3, HQ, DH))
        for c in range(HKV):
            kk, vv = (O8.values(state[t][layer, c][:n], state[t + "s"][layer, c], block) for t in ("k", "v"))
            for hq in range(c * 2, c * 2 + 2):
                want[:, hq] = O8.attention(f64(q)[:, hq], kk, vv, "causal")
        assert_attention_close(f64(o), want)


def test_loop_refuses():
    from paper_2607_27600_amd.refresh import RefreshLoop
    model, _ = _model("last_layer", False)
    with pytest.raises(ValueError):
        RefreshLoop(model, 4, 4, cache="int4")
    with pytest.raises(ValueError):
        RefreshLoop(model, 4, 4, cache="e4m3", scale_block=24)
    with pytest.raises(ValueError):
        RefreshLoop(model, 4, 4).attend(0, torch.zeros(1, HQ, DH, dtype=torch.bfloat16, device="cuda"))
    loop = RefreshLoop(model, 4, 4, cache="e4m3")
    with pytest.raises(ValueError):
        loop.attend(0, torch.zeros(1, HQ, DH, dtype=torch.bfloat16, device="cuda"))
    model.mode = "last_layer_h"
    with pytest.raises(ValueError):
        RefreshLoop(model, 4, 4, cache="e4m3")


def test_decode_step_of_a_batch_in_a_graph():
    """Append, attention, W_o and log-probabilities of one layer, captured once and replayed while the
    lengths advance; every step against the oracle's own cache."""
    from paper_2607_27600_amd import cc
    theta, hq, hkv, d, block, steps = 1e4, 4, 2, 64, 16, 6
    lens = [14, 0, 31, 200]
    B = len(lens)
    cache = Cache8(lens, hkv, d, page=16, block=block, seed=41, room=steps)
    ref = {(b, c, t): cache.plane(0, b, c, t) for b in range(B) for c in range(hkv) for t in ("k", "v")}
    g = torch.Generator().manual_seed(42)
    qkv = torch.randn(steps, B, hq + 2 * hkv, d, generator=g).to(torch.bfloat16)
    w_o = (torch.randn(64, hq * d, generator=g) * 0.1).to(torch.bfloat16).cuda()
    w_lm = (torch.randn(501, 64, generator=g) * 0.3).to(torch.bfloat16).cuda()
    p = cc.problem(dtype="bf16", cu_seqlens=cu_of([1] * B), n_heads_q=hq, n_heads_kv=hkv, head_dim=d, hidden=64, vocab=501,
                   rope_theta=theta)
    kv, most = cache.view(cc), max(lens) + steps
    cached, row = i32(lens), torch.empty_like(qkv[0], device="cuda")
    after = cached + 1
    ids = torch.arange(B, dtype=torch.int32, device="cuda")
    q2, o = torch.empty(B, hq, d, dtype=torch.bfloat16, device="cuda"), torch.empty(B, hq, d, dtype=torch.bfloat16, device="cuda")
    u, out = torch.empty(B, 64, dtype=torch.bfloat16, device="cuda"), cc.logprobs_out(B, 5)
    ws = torch.empty(max(1, cc.cc_attention_kv8_workspace(p, "causal", most)), dtype=torch.uint8, device="cuda")
    ws2 = torch.empty(cc.cc_lmhead_logprobs_workspace("bf16", B, 501, 64, 5), dtype=torch.uint8, device="cuda")

    def step():
        q, k, v = row.split([hq, hkv, hkv], 1)
        cc.cc_append_kv8(p, kv, k, v, cached, q=q, q_out=q2)
        cc.cc_attention_kv8(p, q2, kv, 0, after, most, o, workspace=ws)
        cc.cc_linear("bf16", o.view(B, hq * d), w_o, u)
        cc.cc_lmhead_logprobs("bf16", u, w_lm, 501, ids, 5, out, workspace=ws2)
        cached.add_(1)
        after.add_(1)

    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        step()
    cached.copy_(i32(lens))
    after.copy_(i32([x + 1 for x in lens]))
    for t in range(steps):
        row.copy_(qkv[t])
        graph.replay()
        torch.cuda.synchronize()
        h = f64(qkv[t])
        pos = np.array(lens) + t
        kr = O8.rotate(h[:, hq:hq + hkv], pos, theta)
        for b in range(B):
            want = np.zeros((hq, d))
            for c in range(hkv):
                # (the device's own codes: a rotated key may round either way)
                got = {x: cache.plane(0, b, c, x, src=cache.read(), n=int(pos[b]) + 1) for x in ("k", "v")}
                O8.append(*ref[b, c, "v"], int(pos[b]), h[b:b + 1, hq + hkv + c], block, cache.cap)
                np.testing.assert_array_equal(got["v"][0], ref[b, c, "v"][0][: pos[b] + 1])
                kk, vv = (O8.values(*got[x], block) for x in ("k", "v"))
                assert np.all(np.abs(kk[-1] - kr[b, c]) <= 2.0 ** -4 * np.abs(kr[b, c]) + 2.0 ** -10 * O8.scale_value(got["k"][1][-1]) + 1e-5)
                for x in range(c * 2, c * 2 + 2):
                    want[x] = O8.attention(f64(q2)[b:b + 1, x], kk, vv, "causal")[0]
            assert_attention_close(f64(o)[b][None], want[None])
        lp = O.logprobs(f64(u), f64(w_lm), np.arange(B), 5)
        np.testing.assert_allclose(f64(out.logprob), lp["logprob"], rtol=0, atol=3e-5)
        np.testing.assert_allclose(f64(out.top_logprob), lp["top_logprob"], rtol=0, atol=3e-5)


def test_calls_on_another_stream():
    """Every operator on a stream that is not the current one, with memory that the call allocates."""
    from paper_2607_27600_amd import cc
    hq, hkv, d, new, cached = 4, 2, 128, [3, 40], [20, 9]
    caches = [Cache8(cached, hkv, d, page=16, block=16, seed=51, room=50) for _ in range(2)]
    g = torch.Generator().manual_seed(52)
    qkv = torch.randn(43, hq + 2 * hkv, d, generator=g).to(torch.bfloat16).cuda()
    u, w = torch.randn(70, 128, generator=g).to(torch.bfloat16).cuda(), torch.randn(20000, 128, generator=g).to(torch.bfloat16).cuda()
    ids = torch.arange(70, dtype=torch.int32, device="cuda")
    p = cc.problem(dtype="bf16", cu_seqlens=cu_of(new), n_heads_q=hq, n_heads_kv=hkv, head_dim=d, hidden=64, vocab=1,
                   rope_theta=1e4)
    whole = cc.problem(dtype="bf16", cu_seqlens=cu_of([23, 49]), n_heads_q=hq, n_heads_kv=hkv, head_dim=d, hidden=64, vocab=1)
    lens, after = i32(cached), i32([23, 49])
    keep = i32([0, 5, 22, 1, 2, 48])
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = []
    for cache, stream in zip(caches, (None, side)):
        kv = cache.view(cc)
        q, k, v = qkv.split([hq, hkv, hkv], 1)
        q2 = cc.cc_append_kv8(p, kv, k, v, lens, q=q, stream=stream)
        o = cc.cc_attention_kv8(p, q2, kv, 0, after, 60, stream=stream)
        lp = cc.cc_lmhead_logprobs("bf16", u, w, 20000, ids, 7, stream=stream)
        cc.cc_compact_kv8(whole, kv, keep, [3, 3], 0, stream=stream)
        torch.cuda.synchronize()
        got.append((q2, o, lp.logprob, lp.entropy, lp.top_ids, lp.top_logprob, *cache.t.values()))
    for a, b in zip(*got):
        assert torch.equal(a.view(torch.uint8) if a.dtype == torch.bfloat16 else a, b.view(torch.uint8) if b.dtype == torch.bfloat16 else b)
