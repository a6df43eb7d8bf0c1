"""Attention over a cache in bf16, attention of a batch that shares a prefix, and eviction by accumulated
attention weight, through the library's public entry points, beside their plain forms.

  attn      cc_attention_kv: causal attention of packed queries over a bf16 cache: whole prompts of
            different lengths, chunks, single tokens; with each row's log-sum-exp
  prefix    cc_attention_prefix: the same where runs of sequences share the entries before their own,
            which are read once for all
  weights   cc_attention_weights: what each cached entry receives of the queries' attention, added to
            what it has received so far
  evict     cc_weight_scores, cc_select_keep, cc_compact_kv, cc_compact_weights: the entries of the
            least accumulated weight leave the cache, but for the first and the most recent ones

Shapes are those of the two model families of the repository's workloads (32 query heads on 8; 28 on 4),
and generic ones.  Keys, values and queries are N(0, 1).
"""
import math
import random

import torch

own = False

DEV = "cuda"
BF, F32, F64 = torch.bfloat16, torch.float32, torch.float64

LLAMA = dict(hq=32, hkv=8, d=128)
QWEN = dict(hq=28, hkv=4, d=128)
SMALL = dict(hq=16, hkv=4, d=64)


def listed():
    return [
        # one short prompt, where latency counts
        dict(name="attn_prompt_200", kind="attn", new="200", times=1, cached="0", page=0, **LLAMA),
        # prompts of mixed length entering a paged cache together
        dict(name="attn_prompt_packed", kind="attn", new="1711,333,1,97,4001,1024,2500,640", times=1, cached="0", page=16,
             **QWEN),
        # one long prompt as a whole
        dict(name="attn_prompt_16384", kind="attn", new="16384", times=1, cached="0", page=0, **LLAMA),
        # one sequence decoding on a short cache
        dict(name="attn_decode_1", kind="attn", new="1", times=1, cached="2047", page=0, **LLAMA),
        # a served batch decoding: 48 ragged sequences in a paged cache
        dict(name="attn_decode_48", kind="attn", new="1", times=48,
             cached="4395,14550,15987,6282,655,8070,1201,7860,2048,31,512,9000,333,2777,4096,1500", page=16, **QWEN),
        # four samples of one short prompt, their first tokens
        dict(name="prefix_4", kind="prefix", prefix="900", runs="4", new="1", times=4, cached="0,3,1,7", page=0, **LLAMA),
        # a served batch behind one long system prompt, each sequence with a conversation of its own
        dict(name="prefix_decode_40", kind="prefix", prefix="16000", runs="40", new="1", times=40,
             cached="5,1800,640,0,97,1201,333,64", page=16, **QWEN),
        # drafts of six tokens behind two shared documents, one far longer than the other
        dict(name="prefix_drafts_24", kind="prefix", prefix="30001,6000", runs="16,8", new="6", times=24,
             cached="17,500,128,1023", page=64, **LLAMA),
        # one decode step of a served batch: what its queries attend to
        dict(name="weights_decode_8", kind="weights", new="1", times=8, cached="2048,777,15,4000,9001,64,1200,12000", page=16,
             **QWEN),
        # a whole prompt: what its entries received
        dict(name="weights_prompt_4096", kind="weights", new="4096", times=1, cached="0", page=0, **LLAMA),
        # eviction in a managed cache: 512 of 768 kept, 28 layers, the last 64 entries among them
        dict(name="evict_768", kind="evict", lens="768", keep="512", recent=64, first=0, heads=False, layers=28, page=0, **QWEN),
        # eviction in a served batch, each KV head by its own weights: a quarter of each sequence kept, paged
        dict(name="evict_heads_paged", kind="evict", lens="4395,1455,15987,6282", keep="1099,364,3997,1571", recent=128,
             first=4, heads=True, layers=8, page=16, **QWEN),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _ints(text):
    return [int(x) for x in str(text).split(",")]


def _text(xs):
    return ",".join(map(str, xs))


def draw(rng):
    kind = rng.choice(["attn", "attn", "attn", "prefix", "prefix", "weights", "weights", "evict"])
    heads = dict(rng.choice([LLAMA, QWEN, SMALL, dict(hq=8, hkv=1, d=128), dict(hq=4, hkv=4, d=64)]))
    page = rng.choice([0, 16, 32, 64, 128])
    if kind in ("attn", "weights"):
        form = rng.choice(["prompt", "prompt", "one", "few", "chunk"])
        if form == "prompt":
            n = _log(rng, 1, 12)
            new = [_log(rng, 1, 12000 if n == 1 else 4000) for _ in range(n)]
            cached = [0] * n
        else:
            n = _log(rng, 1, 3 if form == "chunk" else 48)
            new = [1 if form == "one" else rng.randint(0, 12) if form == "few" else _log(rng, 16, 700) for _ in range(n)]
            new[0] = max(1, new[0])
            top = _log(rng, 64, 16000 if n > 4 else 60000 if form != "chunk" else 20000)
            cached = [_log(rng, 1, top) for _ in range(n)]
            cached[-1] = top
        return dict(kind=kind, new=_text(new), times=1, cached=_text(cached), page=page, **heads)
    if kind == "prefix":
        runs = [_log(rng, 1, 24) for _ in range(rng.choice([1, 1, 2, 3]))]
        n = sum(runs)
        most = rng.choice([1, 1, 4, _log(rng, 8, 200)])
        new = [rng.randint(0, most) for _ in range(n)]
        new[rng.randrange(n)] = most
        return dict(kind="prefix", prefix=_text(_log(rng, 30, 40000 // len(runs)) for _ in runs), runs=_text(runs),
                    new=_text(new), times=1, cached=_text(rng.choice([0, _log(rng, 1, 3000)]) for _ in new), page=page, **heads)
    n = _log(rng, 1, 6)
    lens = [_log(rng, 2, 9000) for _ in range(n)]
    keep = [max(1, int(x * rng.uniform(0.05, 1.0))) for x in lens]
    first = rng.choice([0, 0, 1, 4])
    recent = rng.choice([0, 16, _log(rng, 1, 300)])
    return dict(kind="evict", lens=_text(lens), keep=_text(keep), recent=recent, first=first, heads=rng.random() < 0.5,
                layers=_log(rng, 1, 16), page=page, **heads)


# ------------------------------------------------------------------ inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 7919 + 29)
    return g


def _normal(g, *shape):
    out = torch.empty(*shape, dtype=BF, device=DEV)
    flat = out.view(-1)
    for lo in range(0, flat.numel(), 1 << 27):
        flat[lo:lo + (1 << 27)] = torch.randn(min(1 << 27, flat.numel() - lo), generator=g, device=DEV)
    return out


def _i32(xs):
    return torch.tensor(xs, dtype=torch.int32, device=DEV)


def _layout(c, lens):
    """Pages of a pool that holds `lens` entries a sequence, and the table of them; a contiguous cache
    is a pool of one page a sequence."""
    rng = random.Random(len(lens) * 1000003 + sum(lens))
    if c["page"] == 0:
        return max(1, max(lens)), len(lens), [[b] for b in range(len(lens))]
    P = c["page"]
    per = [max(1, -(-x // P)) for x in lens]
    order = list(range(sum(per)))
    rng.shuffle(order)
    table, at = [], 0
    for m in per:
        table.append(order[at:at + m] + [-1] * (max(per) - m))
        at += m
    return P, sum(per), table


def _cu(lens):
    cu = [0]
    for x in lens:
        cu.append(cu[-1] + x)
    return cu


def _pool(g, c, lens, layers=1):
    """Keys and values [layers][pages][Hkv][P][d] of sequences of `lens` entries, their table, P."""
    P, pages, table = _layout(c, lens)
    shape = (layers, pages, c["hkv"], P, c["d"])
    return dict(k=_normal(g, *shape), v=_normal(g, *shape), table=_i32(table), P=P, lens=lens)


def _view(cc, c, pool, k=None, v=None):
    k, v = pool["k"] if k is None else k, pool["v"] if v is None else v
    layers, pages, hkv, P, d = k.shape
    if c["page"] == 0:
        return cc.kv_contiguous(k, v, n_layers=layers, seq_stride=hkv * P * d, layer_stride=pages * hkv * P * d,
                                head_stride=P * d, tok_stride=d)
    return cc.kv_paged(k, v, pool["table"], n_layers=layers, layer_stride=pages * hkv * P * d, page_stride=hkv * P * d,
                       head_stride=P * d, tok_stride=d, page_size=P)


def _problem(cc, c, cu, cu_d, **kw):
    return cc.problem(dtype="bf16", cu_seqlens=cu, n_heads_q=c["hq"], n_heads_kv=c["hkv"], head_dim=c["d"], hidden=64,
                      vocab=1, device=DEV, cu_device=cu_d, **kw)


def prepare(case, seed):
    c, g = dict(case), _gen(seed)
    s = {"c": c, "kind": c["kind"]}
    if c["kind"] == "evict":
        lens, keep = _ints(c["lens"]), _ints(c["keep"])
        n, hkv = len(lens), c["hkv"]
        s.update(lens=lens, keep=keep, cu=_cu(lens), kv=_pool(g, c, lens, c["layers"]))
        s["cu_d"] = _i32(s["cu"])
        # Whole multiples of 2^-8, so that sums over the heads are exact in any order and the order of the entries
        # belongs to the inputs; a few entries have nearly all, as attention has it.
        w = torch.rand(n, hkv, max(lens), generator=g, device=DEV).clamp(min=1e-4).pow(-0.7)
        s["w"] = (w.mul(256).round() / 256).clamp(max=4096)
        s["k2"], s["v2"], s["w2"] = torch.zeros_like(s["kv"]["k"]), torch.zeros_like(s["kv"]["v"]), torch.zeros_like(s["w"])
        lists = [(b, h) for b in range(n) for h in range(hkv if c["heads"] else 1)]
        s["budgets"] = [keep[b] for b, _ in lists]
        s["seg_len"] = [lens[b] for b, _ in lists]
        s["seg_start"] = _cu(s["seg_len"])[:-1]
        s["list"] = torch.zeros(sum(s["budgets"]), dtype=torch.int32, device=DEV)
        s["scores"] = torch.empty(sum(s["seg_len"]), dtype=F32, device=DEV)
        if own:
            from paper_2607_27600_amd import cc
            s["p"] = _problem(cc, c, s["cu"], s["cu_d"], n_frozen=c["first"])
            s["view"] = _view(cc, c, s["kv"])
            s["view2"] = _view(cc, c, s["kv"], s["k2"], s["v2"])
        return s
    new = _ints(c["new"]) * c["times"]
    new = new[:c["times"]] if c["times"] > 1 else new
    cached = (_ints(c["cached"]) * len(new))[:len(new)]
    lens = [a + b for a, b in zip(new, cached)]
    s.update(new=new, cu=_cu(new), most=max(lens), kv=_pool(g, c, lens))
    s["cu_d"], s["lens"], s["cached"] = _i32(s["cu"]), _i32(lens), _i32(cached)
    M = sum(new)
    s["q"] = _normal(g, M, c["hq"], c["d"])
    s["o"] = torch.empty_like(s["q"])
    s["lse"] = torch.empty(M, c["hq"], dtype=F32, device=DEV)
    if c["kind"] == "prefix":
        pre, runs = _ints(c["prefix"]), _ints(c["runs"])
        s["first"], s["pre"], s["pre_lens"] = _cu(runs), _pool(g, c, pre), _i32(pre)
    if c["kind"] == "weights":
        # what the attention of the same queries has left
        for b, m in enumerate(new):
            k = _entries(s["kv"], "k", b).to(F32)
            for lo, hi in _pieces(m, c["hq"] * lens[b]):
                z = _logits(s, b, lo, hi, k, lens[b])
                s["lse"][s["cu"][b] + lo:s["cu"][b] + hi] = z.logsumexp(-1).permute(2, 0, 1).reshape(hi - lo, c["hq"])
        s["prev"] = torch.rand(len(new), c["hkv"], max(lens), generator=g, device=DEV) * 8
        s["w"] = torch.zeros_like(s["prev"])
    if own:
        from paper_2607_27600_amd import cc
        s["p"] = _problem(cc, c, s["cu"], s["cu_d"])
        s["view"] = _view(cc, c, s["kv"])
        if c["kind"] == "prefix":
            s["prefix"] = cc.prefix(_view(cc, c, s["pre"]), s["first"], s["pre_lens"], max(s["pre"]["lens"]))
            size = cc.cc_attention_prefix_workspace(s["p"], s["prefix"], s["most"])
        elif c["kind"] == "attn":
            size = cc.cc_attention_kv_workspace(s["p"], s["most"])
        else:
            size = cc.cc_attention_weights_workspace(s["p"], s["most"])
        s["ws"] = torch.empty(max(1, size), dtype=torch.uint8, device=DEV)
    return s


# ------------------------------------------------------------------ plain forms

def _entries(pool, which, b):
    """Entries [Hkv][n][d] of sequence b, layer 0."""
    t = torch.arange(pool["lens"][b], device=DEV)
    return pool[which][0][pool["table"][b].long()[t // pool["P"]], :, t % pool["P"]].transpose(0, 1)


def _pieces(m, each):
    """Queries lo..hi of m, so that `each` numbers a query stay within 4 GiB in 32 bits."""
    step = max(1, (1 << 30) // max(1, each))
    return [(lo, min(m, lo + step)) for lo in range(0, m, step)]


def _logits(s, b, lo, hi, k, n):
    """Logits [Hkv][g][queries][n] of queries lo..hi of sequence b, -inf where the entry comes after the query."""
    c = s["c"]
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    q = s["q"][s["cu"][b] + lo:s["cu"][b] + hi].to(F32).view(hi - lo, hkv, hq // hkv, d).permute(1, 2, 0, 3)
    z = (q.reshape(hkv, -1, d) @ k.transpose(1, 2).contiguous()).view(hkv, hq // hkv, hi - lo, n) / math.sqrt(d)
    at = torch.arange(lo, hi, device=DEV) + n - s["new"][b]
    return z.masked_fill_(torch.arange(n, device=DEV) > at[:, None], -math.inf)


def _attend(s):
    """Attention of every sequence's queries to its prefix (if any) and to its own entries up to their own."""
    c = s["c"]
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    for b, m in enumerate(s["new"]):
        if m == 0:
            continue
        n = s["kv"]["lens"][b]
        k, v = _entries(s["kv"], "k", b).to(F32), _entries(s["kv"], "v", b).to(F32)
        np = 0
        if s["kind"] == "prefix":
            i = next(i for i in range(len(s["first"])) if s["first"][i + 1] > b)
            kp, vp = _entries(s["pre"], "k", i).to(F32), _entries(s["pre"], "v", i).to(F32)
            np = s["pre"]["lens"][i]
            v = torch.cat([vp, v], 1)
        for lo, hi in _pieces(m, hq * (n + np)):
            z = _logits(s, b, lo, hi, k, n)
            if np:
                q = s["q"][s["cu"][b] + lo:s["cu"][b] + hi].to(F32).view(hi - lo, hkv, hq // hkv, d).permute(1, 2, 0, 3)
                far = (q.reshape(hkv, -1, d) @ kp.transpose(1, 2).contiguous()).view(*z.shape[:3], np) / math.sqrt(d)
                z = torch.cat([far, z], -1)
            top = z.amax(-1, keepdim=True)
            z = z.sub_(top).exp_()
            total = z.sum(-1, keepdim=True)
            o = (z.view(hkv, -1, n + np) @ v).view(*z.shape[:3], d) / total
            rows = slice(s["cu"][b] + lo, s["cu"][b] + hi)
            s["o"][rows] = o.permute(2, 0, 1, 3).reshape(hi - lo, hq, d).to(BF)
            s["lse"][rows] = (top + total.log())[..., 0].permute(2, 0, 1).reshape(hi - lo, hq)
    return {"o": s["o"], "lse": s["lse"]}


def _weights(s):
    c = s["c"]
    hq, hkv = c["hq"], c["hkv"]
    for b, m in enumerate(s["new"]):
        n = s["kv"]["lens"][b]
        if m == 0:
            s["w"][b, :, :n] = s["prev"][b, :, :n]
            continue
        k = _entries(s["kv"], "k", b).to(F32)
        total = torch.zeros(hkv, n, device=DEV)
        for lo, hi in _pieces(m, hq * n):
            lse = s["lse"][s["cu"][b] + lo:s["cu"][b] + hi].view(hi - lo, hkv, hq // hkv).permute(1, 2, 0)
            total += _logits(s, b, lo, hi, k, n).sub_(lse[..., None]).exp_().sum((1, 2))
        total[:, :n - m] += s["prev"][b, :, :n - m]
        s["w"][b, :, :n] = total
    return s["w"]


def _evict(s):
    c, P = s["c"], s["kv"]["P"]
    at = 0
    for b, (n, m) in enumerate(zip(s["lens"], s["keep"])):
        w = s["w"][b, :, :n]
        score = w.clone() if c["heads"] else w.sum(0, keepdim=True)
        score[:, :c["first"]] = math.inf
        score[:, max(0, n - c["recent"]):] = math.inf
        kept = score.sort(dim=-1, descending=True, stable=True).indices[:, :m].sort(-1).values
        s["list"][at:at + kept.numel()] = kept.view(-1).to(torch.int32)
        at += kept.numel()
        kept = kept.expand(c["hkv"], m)
        t, h = torch.arange(m, device=DEV), torch.arange(c["hkv"], device=DEV)[:, None]
        page = s["kv"]["table"][b].long()
        for src, dst in ((s["kv"]["k"], s["k2"]), (s["kv"]["v"], s["v2"])):
            dst[:, page[t // P], h, t % P] = src[:, page[kept // P], h, kept % P]
        s["w2"][b, :, :m] = w.gather(1, kept)
    return _evict_out(s)


def _evict_out(s):
    return {"keep": s["list"], "k": s["k2"], "v": s["v2"], "w": s["w2"]}


def run(state):
    s, kind = state, state["kind"]
    if not own:
        return _evict(s) if kind == "evict" else _weights(s) if kind == "weights" else _attend(s)
    from paper_2607_27600_amd import cc
    c = s["c"]
    if kind == "attn":
        cc.cc_attention_kv(s["p"], s["q"], s["view"], 0, s["lens"], s["most"], s["o"], lse=s["lse"], workspace=s["ws"])
        return {"o": s["o"], "lse": s["lse"]}
    if kind == "prefix":
        cc.cc_attention_prefix(s["p"], s["q"], s["prefix"], s["view"], 0, s["lens"], s["most"], s["o"], lse=s["lse"],
                               workspace=s["ws"])
        return {"o": s["o"], "lse": s["lse"]}
    if kind == "weights":
        return cc.cc_attention_weights(s["p"], s["q"], s["view"], 0, s["lens"], s["most"], s["lse"], s["w"], prev=s["prev"],
                                       prev_lens=s["cached"], workspace=s["ws"])
    cc.cc_weight_scores(s["p"], s["w"], c["recent"], c["heads"], s["scores"])
    cc.cc_select_keep(s["scores"], s["seg_start"], s["seg_len"], s["budgets"], s["list"])
    cc.cc_compact_kv(s["p"], s["view"], s["list"], s["budgets"], int(c["heads"]), out=s["view2"])
    cc.cc_compact_weights(s["p"], s["w"], s["list"], s["budgets"], c["heads"], out=s["w2"])
    return _evict_out(s)


# ------------------------------------------------------------------ work

def work(case):
    c = dict(case)
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    if c["kind"] == "evict":
        lens, keep = _ints(c["lens"]), _ints(c["keep"])
        K = sum(keep)
        return {"bytes": 2.0 * 2 * c["layers"] * hkv * K * 2 * d + 4 * hkv * sum(lens) + 4 * hkv * K
                + 4 * K * (hkv if c["heads"] else 1), "flops": 0}
    new = _ints(c["new"]) * c["times"]
    new = new[:c["times"]] if c["times"] > 1 else new
    cached = (_ints(c["cached"]) * len(new))[:len(new)]
    M = sum(new)
    pairs = sum(m * n + m * (m + 1) // 2 for m, n in zip(new, cached))
    T = sum(m + n for m, n in zip(new, cached) if m)
    if c["kind"] == "weights":
        every = sum(m + n for m, n in zip(new, cached))
        return {"bytes": 2.0 * T * hkv * d + 2.0 * M * hq * d + 4 * M * hq + 4 * hkv * (every + sum(cached)),
                "flops": 2.0 * d * hq * pairs}
    if c["kind"] == "prefix":
        pre, runs, at = _ints(c["prefix"]), _ints(c["runs"]), 0
        for n, r in zip(pre, runs):
            m = sum(new[at:at + r])
            at += r
            pairs += n * m
            T += n if m else 0
    return {"bytes": 4.0 * T * hkv * d + 4.0 * M * hq * d + 4 * M * hq, "flops": 4.0 * d * hq * pairs}


# ------------------------------------------------------------------ 64 bits

def _plane(pool, which, b, h):
    """Entries [n][d] of one head of a sequence in 64 bits."""
    n, P = pool["lens"][b], pool["P"]
    rows = [pool[which][0, int(pg), h] for pg in pool["table"][b].tolist()[:-(-n // P)]]
    return torch.cat(rows)[:n].double() if rows else torch.zeros(0, pool[which].shape[-1], dtype=F64, device=DEV)


def exact(case, seed):
    s = prepare(case, seed)
    c = s["c"]
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    grp = hq // hkv
    if c["kind"] == "evict":
        lists, k2, v2, w2 = [], torch.zeros_like(s["k2"]), torch.zeros_like(s["v2"]), torch.zeros_like(s["w2"])
        P = s["kv"]["P"]
        for b, (n, m) in enumerate(zip(s["lens"], s["keep"])):
            tab = s["kv"]["table"][b].tolist()
            planes = torch.cat([s["kv"]["k"][:, pg] for pg in tab if pg >= 0], 2), torch.cat(
                [s["kv"]["v"][:, pg] for pg in tab if pg >= 0], 2)
            keep = None
            for h in range(hkv):
                if c["heads"] or h == 0:
                    x = s["w"][b, h, :n].double() if c["heads"] else s["w"][b, :, :n].double().sum(0)
                    # one whole number for (weight, position): weights are multiples of 2^-8, pinned ones above all
                    i = torch.arange(n, device=DEV)
                    key = (x * 256).round().long()
                    key[(i < c["first"]) | (i >= n - c["recent"])] = 1 << 40
                    keep = (key * (1 << 17) + (n - 1 - i)).topk(m).indices.sort().values
                    lists.append(keep.to(torch.int32))
                w2[b, h, :m] = s["w"][b, h, keep]
                for x, out in zip(planes, (k2, v2)):
                    kept = x[:, h, keep]
                    for lo in range(0, m, P):
                        out[:, tab[lo // P], h, :min(P, m - lo)] = kept[:, lo:lo + P]
        return {"keep": torch.cat(lists), "k": k2.double(), "v": v2.double(), "w": w2.double()}
    if hq * d * sum(m * n for m, n in zip(s["new"], s["kv"]["lens"])) > 1 << 42:
        return None
    q = s["q"].double() * d ** -0.5
    if c["kind"] == "weights":
        out = torch.zeros_like(s["w"], dtype=F64)
        for b, m in enumerate(s["new"]):
            n = s["kv"]["lens"][b]
            out[b, :, :n - m] = s["prev"][b, :, :n - m]
            for h in range(hq if m else 0):
                k = _plane(s["kv"], "k", b, h // grp)
                for i0 in range(0, m, 4096):
                    i = torch.arange(i0, min(m, i0 + 4096), device=DEV)
                    rows = s["cu"][b] + i
                    p = torch.exp(torch.mm(q[rows, h], k.t()) - s["lse"][rows, h, None].double())
                    out[b, h // grp, :n] += torch.where(torch.arange(n, device=DEV)[None] <= i[:, None] + n - m, p, 0.0).sum(0)
        return out
    o, lse = torch.zeros_like(q), torch.zeros(q.shape[:2], dtype=F64, device=DEV)
    for b, m in enumerate(s["new"]):
        n = s["kv"]["lens"][b]
        for c_ in range(hkv if m else 0):
            k, v = _plane(s["kv"], "k", b, c_), _plane(s["kv"], "v", b, c_)
            np = 0
            if c["kind"] == "prefix":
                i = sum(1 for x in s["first"][1:] if x <= b)
                np = s["pre"]["lens"][i]
                k = torch.cat([_plane(s["pre"], "k", i, c_), k])
                v = torch.cat([_plane(s["pre"], "v", i, c_), v])
            for h in range(c_ * grp, (c_ + 1) * grp):
                for i0 in range(0, m, 4096):
                    i = torch.arange(i0, min(m, i0 + 4096), device=DEV)
                    rows = s["cu"][b] + i
                    z = torch.mm(q[rows, h], k.t())
                    z = z.masked_fill(torch.arange(np + n, device=DEV)[None] > (i + np + n - m)[:, None], -math.inf)
                    lse[rows, h] = torch.logsumexp(z, -1)
                    o[rows, h] = torch.mm(torch.softmax(z, -1), v)
    return {"o": o, "lse": lse}
