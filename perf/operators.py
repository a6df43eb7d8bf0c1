"""The operators of the inference cycle between refreshes, through the library's public entry
points, beside their plain forms.

  append    cc_append_kv, cc_append_kv8: new keys (rotated to their positions on the way) and values
            into a paged or contiguous cache, in bf16 or in 8 bits (E4M3 codes, a power-of-two scale
            for each block of tokens and head); the queries of the same tokens are rotated with them
  attn      cc_attention_kv8: attention over a cache in 8 bits; causal (single tokens and chunks of a
            prompt) or counter-causal (the scoring pass)
  compact   cc_compact_kv8: the kept entries of a cache in 8 bits, moved to the front of their planes
  logprobs  cc_lmhead_logprobs: log-probabilities of given tokens from the hidden rows and the LM
            head, with the entropy and the most probable alternatives of each row

Shapes are those of the two model families of the repository's workloads (32 query heads on 8, 4096
wide, vocabulary 128256; 28 on 4, 3584 wide, vocabulary 152064), and generic ones.  Keys, values and
queries are N(0, 1), LM-head weights N(0, 0.02^2).
"""
import math
import random

import torch

own = False

DEV = "cuda"
BF, F32, F64 = torch.bfloat16, torch.float32, torch.float64
E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
THETA = 5e5
LOW = 27            # the smallest scale that a block is given: 2^(27 - 127)

LLAMA = dict(hq=32, hkv=8, d=128)
QWEN = dict(hq=28, hkv=4, d=128)
SMALL = dict(hq=16, hkv=4, d=64)


def listed():
    return [
        # a decode step of a served batch of eight: one token each into a paged cache in 8 bits
        dict(name="append_decode_8", kind="append", bits=8, new="1", times=8, cached="2048,777,15,4000,3001,64,1200,0",
             page=16, block=16, **QWEN),
        # prompts of mixed length entering a paged bf16 cache, a decoding sequence among them
        dict(name="append_ragged_bf16", kind="append", bits=16, new="1711,333,1,97,1024", times=1,
             cached="0,100,4001,33,2047", page=16, block=16, **LLAMA),
        # one chunk of a long prompt into a cache in 8 bits with a scale for 64 tokens
        dict(name="append_chunk_8192", kind="append", bits=8, new="8192", times=1, cached="8200", page=64, block=64,
             **LLAMA),
        # one sequence decoding on a short cache, where latency counts
        dict(name="attn_decode_1", kind="attn", mask="causal", new="1", times=1, cached="1023", page=0, block=16, **LLAMA),
        # a served batch decoding: 64 ragged sequences in a paged cache
        dict(name="attn_decode_64", kind="attn", mask="causal", new="1", times=64,
             cached="4395,14550,15987,6282,655,8070,1201,7860,2048,31,512,9000,333,2777,4096,1500", page=16, block=16, **QWEN),
        # four sequences decoding at long context
        dict(name="attn_decode_long", kind="attn", mask="causal", new="1", times=4, cached="131071", page=64, block=64,
             **LLAMA),
        # a chunk of a long prompt against what is cached of it
        dict(name="attn_chunk_32k", kind="attn", mask="causal", new="512", times=1, cached="32257", page=64, block=64,
             **LLAMA),
        # the scoring pass's attention over a managed cache
        dict(name="attn_score_4096", kind="attn", mask="counter", new="4096", times=1, cached="0", page=0, block=16,
             **LLAMA),
        # eviction in the refresh loop: 512 of 768 kept, 28-layer cache, ids and positions with it
        dict(name="compact_768", kind="compact", lens="768", keep="512", layers=28, page=0, block=16, **QWEN),
        # eviction in a served batch: a quarter of each sequence kept, paged
        dict(name="compact_paged", kind="compact", lens="4395,1455,15987,6282", keep="1099,364,3997,1571", layers=8,
             page=16, block=16, **QWEN),
        # the next token's distribution of a decoding batch, with eight alternatives
        dict(name="logprobs_64", kind="logprobs", n=64, D=4096, V=128256, k=8, packed=False),
        # a prompt's tokens scored with their five best alternatives
        dict(name="logprobs_2000", kind="logprobs", n=2000, D=3584, V=152064, k=5, packed=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _ints(text):
    return [int(x) for x in str(text).split(",")]


def draw(rng):
    kind = rng.choice(["append", "append", "attn", "attn", "attn", "compact", "logprobs"])
    heads = dict(rng.choice([LLAMA, QWEN, SMALL, dict(hq=8, hkv=1, d=128), dict(hq=4, hkv=4, d=64)]))
    page, block = rng.choice([(0, 16), (0, 64), (16, 16), (32, 16), (64, 64), (128, 32), (128, 128)])
    if kind == "append":
        n = _log(rng, 1, 24)
        most = 1 if rng.random() < 0.4 else _log(rng, 2, 4096)
        new = [max(0, min(most, _log(rng, 1, most))) for _ in range(n)]
        new[rng.randrange(n)] = most
        cached = [rng.choice([0, _log(rng, 1, 3000)]) for _ in range(n)]
        return dict(kind="append", bits=rng.choice([8, 8, 16]), new=",".join(map(str, new)), times=1,
                    cached=",".join(map(str, cached)), page=page, block=block, **heads)
    if kind == "attn":
        mask = rng.choice(["causal", "causal", "causal", "counter"])
        if mask == "counter":
            n = _log(rng, 1, 4)
            new = [_log(rng, 1, 3000) for _ in range(n)]
            cached = [0] * n
        else:
            form = rng.choice(["one", "few", "chunk"])
            n = _log(rng, 1, 3 if form == "chunk" else 48)
            new = [1 if form == "one" else rng.randint(0, 12) if form == "few" else _log(rng, 16, 700) for _ in range(n)]
            new[0] = max(1, new[0])
            top = _log(rng, 64, 16000 if n > 4 else 60000 if form != "chunk" else 20000)
            cached = [_log(rng, 1, top) for _ in range(n)]
            cached[-1] = top
        return dict(kind="attn", mask=mask, new=",".join(map(str, new)), times=1, cached=",".join(map(str, cached)),
                    page=page, block=block, **heads)
    if kind == "compact":
        n = _log(rng, 1, 6)
        lens = [_log(rng, 1, 9000) for _ in range(n)]
        keep = [max(0, min(x, int(x * rng.uniform(0.05, 1.0)))) for x in lens]
        keep[0] = max(1, keep[0])
        return dict(kind="compact", lens=",".join(map(str, lens)), keep=",".join(map(str, keep)), layers=_log(rng, 1, 16),
                    page=page, block=block, **heads)
    return dict(kind="logprobs", n=_log(rng, 1, 1500), D=64 * _log(rng, 2, 64), V=_log(rng, 500, 152064),
                k=rng.randint(0, 20), packed=rng.random() < 0.5)


# ------------------------------------------------------------------ inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 7919 + 17)
    return g


def _normal(g, *shape, dtype=BF):
    return torch.randn(*shape, generator=g, device=DEV).to(dtype)


def _step(amax):
    """The exponent code (127 + e) of the smallest power of two 2^e with amax <= 448 * 2^e."""
    m, x = torch.frexp(amax / 448)               # amax / 448 = m 2^x, 0.5 <= m < 1
    e = torch.where(m == 0.5, x - 1, x) + 127
    return torch.where(amax > 0, e.clamp(LOW, 254), torch.full_like(e, LOW))


def _factor(code):
    return torch.exp2(code.to(F32) - 127)


def _layout(c, lens):
    """Pages of a pool that holds `lens` entries a sequence, and the table of them; a contiguous cache
    is a pool of one page a sequence."""
    rng = random.Random(len(lens) * 1000003 + sum(lens))
    if c["page"] == 0:
        P = max(c["block"], -(-max(lens) // c["block"]) * c["block"])
        return P, len(lens), [[b] for b in range(len(lens))]
    P = c["page"]
    per = [max(1, -(-x // P)) for x in lens]
    order = list(range(sum(per)))
    rng.shuffle(order)
    table, at = [], 0
    for m in per:
        table.append(order[at:at + m] + [-1] * (max(per) - m))
        at += m
    return P, sum(per), table


def _pool(g, c, pages, P, layers):
    """Codes [layers][pages][Hkv][P][d] and scale codes [layers][pages][Hkv][P / block] of N(0, 1) entries."""
    hkv, d, B = c["hkv"], c["d"], c["block"]
    codes = torch.empty(layers, pages, hkv, P, d, dtype=torch.uint8, device=DEV)
    scale = torch.empty(layers, pages, hkv, P // B, dtype=torch.uint8, device=DEV)
    piece = max(1, (1 << 27) // (hkv * P * d))
    for l in range(layers):
        for lo in range(0, pages, piece):
            x = torch.randn(min(piece, pages - lo), hkv, P // B, B, d, generator=g, device=DEV)
            e = _step(x.abs().amax((-1, -2)))
            codes[l, lo:lo + piece] = (x / _factor(e)[..., None, None]).to(E4M3).view(torch.uint8).view(-1, hkv, P, d)
            scale[l, lo:lo + piece] = e.to(torch.uint8)
    return codes, scale


def _cu(lens):
    cu = [0]
    for x in lens:
        cu.append(cu[-1] + x)
    return cu


def _view8(cc, c, k, v, ks, vs, table, P):
    layers, pages, hkv, _, d = k.shape
    s = P // c["block"]
    if c["page"] == 0:
        return cc.kv8_contiguous(k, v, ks, vs, n_layers=layers, seq_stride=hkv * P * d, layer_stride=pages * hkv * P * d,
                                 head_stride=P * d, tok_stride=d, scale_block=c["block"], scale_seq_stride=hkv * s,
                                 scale_layer_stride=pages * hkv * s, scale_head_stride=s)
    return cc.kv8_paged(k, v, ks, vs, table, n_layers=layers, layer_stride=pages * hkv * P * d, page_stride=hkv * P * d,
                        head_stride=P * d, tok_stride=d, page_size=P, scale_block=c["block"],
                        scale_layer_stride=pages * hkv * s, scale_page_stride=hkv * s, scale_head_stride=s)


def _view16(cc, c, k, v, table, P):
    layers, pages, hkv, _, d = k.shape
    if c["page"] == 0:
        return cc.kv_contiguous(k, v, n_layers=layers, seq_stride=hkv * P * d, layer_stride=pages * hkv * P * d,
                                head_stride=P * d, tok_stride=d)
    return cc.kv_paged(k, v, table, n_layers=layers, layer_stride=pages * hkv * P * d, page_stride=hkv * P * d,
                       head_stride=P * d, tok_stride=d, page_size=P)


def _problem(cc, c, cu, cu_d, **kw):
    return cc.problem(dtype="bf16", cu_seqlens=cu, n_heads_q=c["hq"], n_heads_kv=c["hkv"], head_dim=c["d"], hidden=64,
                      vocab=1, device=DEV, cu_device=cu_d, **kw)


def prepare(case, seed):
    c, g = dict(case), _gen(seed)
    s = {"c": c, "kind": c["kind"]}
    if c["kind"] == "logprobs":
        # On a grid (activations of step 1/16, weights of step 2^-11, as coarse as bf16 has them at the
        # ends of their ranges) every logit is exact in 32 bits in any order of summation, so that
        # the order of the alternatives belongs to the inputs.
        n, D, V = c["n"], c["D"], c["V"]
        s["u"] = (torch.randn(n, D, generator=g, device=DEV) * 16).round().clamp(-128, 128).div(16).to(BF)
        w = torch.empty(V, D, dtype=BF, device=DEV)
        for lo in range(0, V, 1 << 15):
            rows = min(1 << 15, V - lo)
            w[lo:lo + rows] = (torch.randn(rows, D, generator=g, device=DEV) * 41).round().clamp(-256, 256).div(2048).to(BF)
        s["w"] = w
        s["ids"] = torch.randint(0, V, (n,), generator=g, device=DEV, dtype=torch.int32)
        if own:
            from paper_2607_27600_amd import cc
            s["weight"] = cc.cc_pack_lmhead(w) if c["packed"] else w
            s["out"] = cc.logprobs_out(n, c["k"], DEV)
            s["ws"] = torch.empty(max(1, cc.cc_lmhead_logprobs_workspace("bf16", n, V, D, c["k"])), dtype=torch.uint8,
                                  device=DEV)
        return s
    if c["kind"] == "compact":
        lens, keep = _ints(c["lens"]), _ints(c["keep"])
        P, pages, table = _layout(c, lens)
        s.update(P=P, lens=lens, keep=keep, cu=_cu(lens), table=torch.tensor(table, dtype=torch.int32, device=DEV))
        s["k"], s["ks"] = _pool(g, c, pages, P, c["layers"])
        s["v"], s["vs"] = _pool(g, c, pages, P, c["layers"])
        s["k2"], s["v2"], s["ks2"], s["vs2"] = (torch.zeros_like(x) for x in (s["k"], s["v"], s["ks"], s["vs"]))
        s["list"] = torch.cat([torch.randperm(n, generator=g, device=DEV)[:m].sort().values.to(torch.int32)
                               for n, m in zip(lens, keep)])
        at = torch.tensor([b for b, m in enumerate(keep) for _ in range(m)], dtype=torch.int64, device=DEV)
        s["of"], s["to"] = at, torch.cat([torch.arange(m, device=DEV) for m in keep])
        s["ids"] = torch.randint(0, 128256, (sum(lens),), generator=g, device=DEV, dtype=torch.int32)
        s["cu_d"] = torch.tensor(s["cu"], dtype=torch.int32, device=DEV)
        if own:
            from paper_2607_27600_amd import cc
            s["p"] = _problem(cc, c, s["cu"], s["cu_d"])
            s["kv"] = _view8(cc, c, s["k"], s["v"], s["ks"], s["vs"], s["table"], P)
            s["kv2"] = _view8(cc, c, s["k2"], s["v2"], s["ks2"], s["vs2"], s["table"], P)
        return s
    new, cached = _ints(c["new"]) * c["times"], _ints(c["cached"])
    cached = (cached * len(new))[:len(new)]
    lens = [a + b for a, b in zip(new, cached)]
    P, pages, table = _layout(c, lens)
    M, hq, hkv, d = sum(new), c["hq"], c["hkv"], c["d"]
    s.update(P=P, new=new, cu=_cu(new), most=max(lens), table=torch.tensor(table, dtype=torch.int32, device=DEV))
    s["cu_d"] = torch.tensor(s["cu"], dtype=torch.int32, device=DEV)
    s["seq"] = torch.tensor([b for b, m in enumerate(new) for _ in range(m)], dtype=torch.int64, device=DEV)
    s["nth"] = torch.tensor([i for m in new for i in range(m)], dtype=torch.int64, device=DEV)
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    s["cached"] = torch.tensor(cached, dtype=torch.int32, device=DEV)
    if c["kind"] == "attn":
        s["q"] = _normal(g, M, hq, d)
        s["k"], s["ks"] = _pool(g, c, pages, P, 1)
        s["v"], s["vs"] = _pool(g, c, pages, P, 1)
        if own:
            from paper_2607_27600_amd import cc
            s["p"] = _problem(cc, c, s["cu"], s["cu_d"])
            s["kv"] = _view8(cc, c, s["k"], s["v"], s["ks"], s["vs"], s["table"], P)
            s["o"] = torch.empty_like(s["q"])
            s["ws"] = torch.empty(max(1, cc.cc_attention_kv8_workspace(s["p"], c["mask"], s["most"])), dtype=torch.uint8,
                                  device=DEV)
        return s
    # the projections of a layer leave queries, keys and values side by side in one row a token
    s["qkv"] = _normal(g, M, hq + 2 * hkv, d)
    # positions of a managed cache: those that the entries had before evictions, far beyond its length
    s["pos"] = (s["cached"][s["seq"]] + s["nth"] + 100000 * (s["seq"] % 3)).to(torch.int32)
    s["q2"] = torch.empty(M, hq, d, dtype=BF, device=DEV)
    if c["bits"] == 8:
        s["k"], s["ks"] = _pool(g, c, pages, P, 1)
        s["v"], s["vs"] = _pool(g, c, pages, P, 1)
    else:
        s["k"], s["v"] = _normal(g, 1, pages, hkv, P, d), _normal(g, 1, pages, hkv, P, d)
    if own:
        from paper_2607_27600_amd import cc
        s["p"] = _problem(cc, c, s["cu"], s["cu_d"], rope_theta=THETA)
        s["kv"] = (_view8(cc, c, s["k"], s["v"], s["ks"], s["vs"], s["table"], P) if c["bits"] == 8
                   else _view16(cc, c, s["k"], s["v"], s["table"], P))
    return s


# ------------------------------------------------------------------ plain forms

def _rotate(x, pos, d):
    """Elements e and e + d/2 turned by pos * theta^(-2e/d); angles in 64 bits, for far positions."""
    f = torch.pow(torch.tensor(THETA, dtype=F64, device=DEV), -torch.arange(d // 2, device=DEV, dtype=F64) * 2 / d)
    a = pos.to(F64)[:, None] * f
    cos, sin = a.cos().to(F32)[:, None], a.sin().to(F32)[:, None]
    lo, hi = x[..., :d // 2].to(F32), x[..., d // 2:].to(F32)
    return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], -1)


def _store8(s, x, codes, scale):
    """x [M][Hkv][d] (32 bits) appended to the codes and scales of layer 0."""
    c, P = s["c"], s["P"]
    B, hkv, d = c["block"], c["hkv"], c["d"]
    n = len(s["new"])
    pos = s["cached"].long()[s["seq"]] + s["nth"]
    first = s["cached"].long() // B                                # each sequence's first block touched
    most = max(s["new"]) // B + 2
    at = pos // B - first[s["seq"]]
    top = torch.zeros(n, most, hkv, device=DEV).view(-1, hkv)
    top = top.scatter_reduce(0, (s["seq"] * most + at)[:, None].expand(-1, hkv), x.abs().amax(-1), "amax").view(n, most, hkv)
    e = _step(top)
    blocks = first[:, None] + torch.arange(most, device=DEV)
    past = blocks * B < s["cached"][:, None]                        # a block that holds entries already
    here = blocks * B < (s["cached"] + (s["cu_d"][1:] - s["cu_d"][:-1]))[:, None]
    here &= (s["cu_d"][1:] > s["cu_d"][:-1])[:, None]
    page = s["table"].long().gather(1, (blocks * B // P).clamp(max=s["table"].shape[1] - 1)).clamp(min=0)
    slot = blocks % (P // B)
    view = codes[0].view(-1, hkv, P // B, B, d)
    old = scale[0][page, :, slot].to(e.dtype)                       # [n][most][Hkv]
    e = torch.where(past[..., None], torch.maximum(old, e), e)
    kept = view[page, :, slot]                                      # [n][most][Hkv][B][d]
    again = (kept.view(E4M3).to(F32) * _factor(old - e + 127)[..., None, None]).to(E4M3).view(torch.uint8)
    held = (blocks * B)[..., None] + torch.arange(B, device=DEV) < s["cached"][:, None, None]
    again = torch.where(held[:, :, None, :, None], again, kept)
    grown = past & here
    view[page[grown], :, slot[grown]] = again[grown]
    scale[0][page[here], :, slot[here]] = e[here].to(torch.uint8)
    codes[0][s["table"].long()[s["seq"], pos // P], :, pos % P] = (
        x / _factor(e[s["seq"], at])[..., None]).to(E4M3).view(torch.uint8)


def _append(s):
    c = s["c"]
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    q, k, v = s["qkv"].split([hq, hkv, hkv], 1)
    s["q2"].copy_(_rotate(q, s["pos"], d))
    k, v = _rotate(k, s["pos"], d), v.to(F32)
    if c["bits"] == 8:
        _store8(s, k, s["k"], s["ks"])
        _store8(s, v, s["v"], s["vs"])
    else:
        pos = s["cached"].long()[s["seq"]] + s["nth"]
        page = s["table"].long()[s["seq"], pos // s["P"]]
        s["k"][0][page, :, pos % s["P"]] = k.to(BF)
        s["v"][0][page, :, pos % s["P"]] = v.to(BF)
    return _append_out(s)


def _append_out(s):
    if s["c"]["bits"] == 16:
        return {"q": s["q2"], "k": s["k"], "v": s["v"]}
    return {"q": s["q2"], "k": s["k"].view(E4M3), "v": s["v"].view(E4M3), "ks": s["ks"].view(E8M0), "vs": s["vs"].view(E8M0)}


def _dense(s, codes, scale, dtype):
    """Entries [sequences][Hkv][longest][d] of layer 0 as the numbers that they stand for."""
    P, B = s["P"], s["c"]["block"]
    t = torch.arange(s["most"], device=DEV)
    page = s["table"].long()[:, t // P].clamp(min=0)                # [n][T]
    f = torch.exp2(scale[0][page, :, t % P // B].to(dtype) - 127)   # [n][T][Hkv]
    x = codes[0][page, :, t % P].view(E4M3).to(dtype)               # [n][T][Hkv][d]
    return (x * f[..., None]).transpose(1, 2)


def _attend(s):
    c = s["c"]
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    n, m = len(s["new"]), max(s["new"])
    grp = hq // hkv
    q = torch.zeros(n, m, hq, d, device=DEV)
    q[s["seq"], s["nth"]] = s["q"].to(F32)
    q = q.view(n, m, hkv, grp, d).permute(0, 2, 1, 3, 4).reshape(n, hkv, m * grp, d)
    t = torch.arange(s["most"], device=DEV)
    k, v = _dense(s, s["k"], s["ks"], F32), _dense(s, s["v"], s["vs"], F32)
    z = (q @ k.transpose(2, 3)) / math.sqrt(d)
    row = torch.arange(m, device=DEV) + (s["lens"] - (s["cu_d"][1:] - s["cu_d"][:-1]))[:, None]   # [n][m]
    ok = t <= row[..., None] if c["mask"] == "causal" else t > row[..., None]
    ok &= t < s["lens"][:, None, None]
    ok = ok[:, None, :, None].expand(n, 1, m, grp, s["most"]).reshape(n, 1, m * grp, s["most"])
    z.masked_fill_(~ok, -math.inf)
    top = z.amax(-1, keepdim=True).clamp(min=-1e30)
    z = z.sub_(top).exp_()
    total = z.sum(-1, keepdim=True)
    o = (z @ v) / torch.where(total > 0, total, torch.ones_like(total))
    o = o.view(n, hkv, m, grp, d).permute(0, 2, 1, 3, 4).reshape(n, m, hq, d)
    return o[s["seq"], s["nth"]].to(BF)


def _compact8(s, codes, scale, codes2, scale2):
    c, P = s["c"], s["P"]
    B, hkv, d, L = c["block"], c["hkv"], c["d"], codes.shape[0]
    src = s["list"].long()
    page = s["table"].long()[s["of"], src // P]
    f = _factor(scale[:, page, :, src % P // B])                                     # [kept][L][Hkv]
    x = codes[:, page, :, src % P].view(E4M3).to(F32) * f[..., None]                 # [kept][L][Hkv][d]
    most = max(s["keep"]) // B + 1
    at = s["of"] * most + s["to"] // B
    top = torch.zeros(len(s["keep"]) * most, L, hkv, device=DEV)
    top = top.scatter_reduce(0, at[:, None, None].expand(-1, L, hkv), x.abs().amax(-1), "amax")
    e = _step(top)[at]                                                               # [kept][L][Hkv]
    x = (x / _factor(e)[..., None]).to(E4M3).view(torch.uint8)
    page2 = s["table"].long()[s["of"], s["to"] // P]
    codes2[:, page2, :, s["to"] % P] = x
    scale2[:, page2, :, s["to"] % P // B] = e.to(torch.uint8)


def _compact_out(s):
    return {"k": s["k2"].view(E4M3), "v": s["v2"].view(E4M3), "ks": s["ks2"].view(E8M0), "vs": s["vs2"].view(E8M0)}


def _logprobs(s):
    c = s["c"]
    z = s["u"].to(F32) @ s["w"].to(F32).T
    top = z.amax(-1, keepdim=True)
    e = (z - top).exp()
    total = e.sum(-1, keepdim=True)
    lse = top + total.log()
    out = {"logprob": (z.gather(1, s["ids"].long()[:, None]) - lse)[:, 0],
           "entropy": (total.log() - (e * (z - top)).sum(-1, keepdim=True) / total)[:, 0]}
    if c["k"]:
        order = z.sort(dim=-1, descending=True, stable=True)
        out["top_ids"] = order.indices[:, :c["k"]].to(torch.int32)
        out["top_logprob"] = order.values[:, :c["k"]] - lse
    return out


def run(state):
    s, kind = state, state["kind"]
    if not own:
        if kind == "append":
            return _append(s)
        if kind == "attn":
            return _attend(s)
        if kind == "logprobs":
            return _logprobs(s)
        _compact8(s, s["k"], s["ks"], s["k2"], s["ks2"])
        _compact8(s, s["v"], s["vs"], s["v2"], s["vs2"])
        return _compact_out(s)
    from paper_2607_27600_amd import cc
    c = s["c"]
    if kind == "append":
        q, k, v = s["qkv"].split([c["hq"], c["hkv"], c["hkv"]], 1)
        call = cc.cc_append_kv8 if c["bits"] == 8 else cc.cc_append_kv
        call(s["p"], s["kv"], k, v, s["cached"], capacity=s["P"] * s["table"].shape[1], pos_ids=s["pos"], q=q, q_out=s["q2"])
        return _append_out(s)
    if kind == "attn":
        return cc.cc_attention_kv8(s["p"], s["q"], s["kv"], 0, s["lens"], s["most"], s["o"], mask=c["mask"],
                                   workspace=s["ws"])
    if kind == "logprobs":
        out = s["out"]
        cc.cc_lmhead_logprobs("bf16", s["u"], s["weight"], c["V"], s["ids"], c["k"], out, packed=c["packed"],
                              workspace=s["ws"])
        got = {"logprob": out.logprob, "entropy": out.entropy}
        return {**got, "top_ids": out.top_ids, "top_logprob": out.top_logprob} if c["k"] else got
    cc.cc_compact_kv8(s["p"], s["kv"], s["list"], s["keep"], 0, out=s["kv2"])
    return _compact_out(s)


# ------------------------------------------------------------------ work

def work(case):
    c = dict(case)
    if c["kind"] == "logprobs":
        n, D, V, k = c["n"], c["D"], c["V"], c["k"]
        return {"bytes": 2.0 * (n * D + V * D) + 4 * n * (3 + 2 * k), "flops": 2.0 * n * D * V}
    hq, hkv, d, B = c["hq"], c["hkv"], c["d"], c["block"]
    if c["kind"] == "compact":
        K = sum(_ints(c["keep"]))
        return {"bytes": 2.0 * 2 * c["layers"] * hkv * K * (d + 1 / B) + 4 * K, "flops": 0}
    new = _ints(c["new"]) * c["times"]
    cached = (_ints(c["cached"]) * len(new))[:len(new)]
    M = sum(new)
    if c["kind"] == "append":
        row = d + 1 / B if c["bits"] == 8 else 2 * d
        return {"bytes": M * (2.0 * d * (hq + 2 * hkv) + 2 * d * hq + 2 * hkv * row + 4), "flops": 3.0 * M * d * (hq + hkv)}
    if c["mask"] == "causal":
        pairs = sum(m * n + m * (m + 1) // 2 for m, n in zip(new, cached))
    else:
        pairs = sum(m * (m - 1) // 2 for m in new)
    T = sum(m + n for m, n in zip(new, cached) if m)
    return {"bytes": 2.0 * T * hkv * (d + 1 / B) + 2.0 * 2 * M * hq * d, "flops": 4.0 * d * hq * pairs}


# ------------------------------------------------------------------ 64 bits

def _turned(x, pos, d):
    """The rotation as a product of complex numbers."""
    e = torch.arange(d // 2, device=DEV, dtype=F64)
    angle = pos.double()[:, None] * torch.exp(e * (-2.0 / d * math.log(THETA)))
    z = torch.complex(x[..., :d // 2].double(), x[..., d // 2:].double()) * torch.polar(torch.ones_like(angle), angle)[:, None]
    return torch.cat([z.real, z.imag], -1)


def _ceil_scale(amax):
    """log2 of the scale of a block, from its largest magnitude."""
    x = torch.ceil(torch.log2(amax.clamp(min=2.0 ** -90) / 448))
    x = torch.where(amax > 448 * torch.exp2(x), x + 1, x)
    return torch.where(amax <= 224 * torch.exp2(x), x - 1, x).clamp(min=float(LOW - 127))


def exact(case, seed):
    s = prepare(case, seed)
    c = s["c"]
    if c["kind"] == "logprobs":
        if c["n"] * c["V"] > 1 << 30:
            return None
        z = torch.cat([s["u"].double() @ s["w"][lo:lo + 16384].double().t() for lo in range(0, c["V"], 16384)], 1)
        lp = torch.log_softmax(z, -1)
        out = {"logprob": lp.gather(1, s["ids"].long()[:, None]).squeeze(1), "entropy": -(lp.exp() * lp).sum(-1)}
        if c["k"]:
            # one number for (logit, position): the logits are whole multiples of 2^-15
            key = (z * 32768).round().long() * (1 << 18) + ((1 << 18) - 1 - torch.arange(c["V"], device=DEV))
            ids = key.topk(c["k"], -1).indices
            out["top_ids"], out["top_logprob"] = ids.to(torch.int32), lp.gather(1, ids)
        return out
    hkv, d, B, P = c["hkv"], c["d"], c["block"], s["P"]
    tab = s["table"].long()
    if c["kind"] == "compact":
        out = {}
        for name in ("k", "v"):
            codes, e = s[name].view(E4M3).double(), s[name + "s"].double() - 127
            to, toe = torch.zeros_like(codes), torch.zeros_like(e)
            toe -= 127                      # an untouched scale code of zero stands for 2^-127
            at = 0
            for b, m in enumerate(s["keep"]):
                src = s["list"][at:at + m].long()
                at += m
                if m == 0:
                    continue
                x = codes[:, tab[b, src // P], :, src % P] * torch.exp2(e[:, tab[b, src // P], :, src % P // B])[..., None]
                for lo in range(0, m, B):
                    y = x[lo:lo + B]
                    z = _ceil_scale(y.abs().amax((0, 3)))
                    page, slot = int(tab[b, lo // P]), lo % P
                    to[:, page, :, slot:slot + y.shape[0]] = (y / torch.exp2(z)[..., None]).permute(1, 2, 0, 3)
                    toe[:, page, :, slot // B] = z
            out[name], out[name + "s"] = to, torch.exp2(toe)
        return out
    if c["kind"] == "attn":
        if len(s["new"]) * max(s["new"]) * c["hq"] * s["most"] > 1 << 31:
            return None
        grp, out = c["hq"] // hkv, []
        for b, m in enumerate(s["new"]):
            T = int(s["lens"][b])
            t = torch.arange(T, device=DEV)
            kv = [s[x][0][tab[b, t // P], :, t % P].view(E4M3).double()
                  * torch.exp2(s[x + "s"][0][tab[b, t // P], :, t % P // B].double() - 127)[..., None] for x in ("k", "v")]
            q = s["q"][s["cu"][b]:s["cu"][b + 1]].double()
            o = torch.zeros_like(q)
            i = torch.arange(m, device=DEV)[:, None] + T - m
            ok = (t <= i) if c["mask"] == "causal" else (t > i)
            live = ok.any(1)
            for h in range(c["hq"]):
                z = (q[:, h] @ kv[0][:, h // grp].t()) * d ** -0.5
                o[live, h] = torch.softmax(z.masked_fill(~ok, -math.inf)[live], -1) @ kv[1][:, h // grp]
            out.append(o)
        return torch.cat(out)
    hq = c["hq"]
    q, k, v = s["qkv"][:, :hq], s["qkv"][:, hq:hq + hkv], s["qkv"][:, hq + hkv:]
    out = {"q": _turned(q, s["pos"], d)}
    for name, x in (("k", _turned(k, s["pos"], d)), ("v", v.double())):
        pool = s[name].view(E4M3).double() if c["bits"] == 8 else s[name].double()
        if c["bits"] == 8:
            e = s[name + "s"].double() - 127
        for b, m in enumerate(s["new"]):
            lo = int(s["cached"][b])
            t = torch.arange(lo, lo + m, device=DEV)
            y = x[s["cu"][b]:s["cu"][b + 1]]
            if c["bits"] == 16:
                pool[0][tab[b, t // P], :, t % P] = y
                continue
            for blk in range(lo // B, (lo + m + B - 1) // B if m else lo // B):
                a, z = max(lo, blk * B), min(lo + m, (blk + 1) * B)
                page, slot = int(tab[b, blk * B // P]), blk * B % P
                part = y[a - lo:z - lo]
                step = _ceil_scale(part.abs().amax((0, 2)))
                if a > blk * B:
                    was = e[0, page, :, slot // B]
                    step = torch.maximum(step, was)
                    old = pool[0, page, :, slot:slot + a - blk * B]
                    old *= torch.exp2(was - step)[:, None, None]
                e[0, page, :, slot // B] = step
                here = slice(slot + a - blk * B, slot + z - blk * B)
                pool[0, page, :, here] = (part / torch.exp2(step)[:, None]).transpose(0, 1)
        out[name] = pool
        if c["bits"] == 8:
            out[name + "s"] = torch.exp2(e)
    return out
