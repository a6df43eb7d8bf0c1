"""Caches in bf16 for tests: pools with padding and a shuffled block table, or contiguous planes with gaps, NaN (or what
is asked for) wherever no entry lies, and numpy copies of single planes."""
import numpy as np
import torch

from tests.gpu_util import f64


class Cache16:
    def __init__(self, lens, hkv, d, layers=1, page=0, room=0, seed=0, fill=float("nan"), device="cuda"):
        r = np.random.default_rng(seed)
        self.lens, self.hkv, self.d, self.layers, self.page = list(lens), hkv, d, layers, page
        n, cap = len(lens), max(max(lens) + room, 1)
        if page:
            self.P = page
            self.max_pages = -(-cap // page) + 1
            order = r.permutation(n * self.max_pages + 3)
            self.table = order[: n * self.max_pages].reshape(n, self.max_pages).astype(np.int32)
            pages = len(order)
        else:
            self.P = cap
            self.table = np.arange(n, dtype=np.int32)[:, None]
            pages = n
        self.tok = d + 8                     # a gap of 16 bytes behind each token row
        g = torch.Generator().manual_seed(seed)
        self.t = {}
        for w in "kv":
            x = torch.full((layers, pages, hkv, self.P, self.tok), fill, dtype=torch.bfloat16)
            for b, m in enumerate(self.lens):
                pg, sl = self._where(b, np.arange(m))
                x[:, pg, :, sl, :d] = torch.randn(m, layers, hkv, d, generator=g).to(torch.bfloat16)
            self.t[w] = x.to(device)
        # pages past a sequence's entries are no pages
        tab = self.table.copy()
        if page:
            for b, m in enumerate(self.lens):
                tab[b, -(-m // page):] = -(1 << 30) if room == 0 else tab[b, -(-m // page):]
        self.bt = torch.from_numpy(tab).to(device)

    def _where(self, b, t):
        if self.page:
            return self.table[b, t // self.P], t % self.P
        return np.full_like(t, b), t

    def put(self, l, b, h, which, t, e, x):
        pg, sl = self._where(b, np.asarray([t]))
        self.t[which][l, int(pg[0]), h, int(sl[0]), e] = x

    def values(self, l, b, h, which, n=None):
        pg, sl = self._where(b, np.arange(self.lens[b] if n is None else n))
        return f64(self.t[which][l, torch.from_numpy(pg).long(), h, torch.from_numpy(sl).long(), : self.d])

    def view(self, cc):
        pages, row = self.t["k"].shape[1], self.P * self.tok
        kw = dict(n_layers=self.layers, layer_stride=pages * self.hkv * row, head_stride=row, tok_stride=self.tok)
        if self.page:
            return cc.kv_paged(self.t["k"], self.t["v"], self.bt, page_stride=self.hkv * row, page_size=self.P, **kw)
        return cc.kv_contiguous(self.t["k"], self.t["v"], seq_stride=self.hkv * row, **kw)


def cu_of(lens):
    return [0] + np.cumsum(lens).tolist()


def i32(x, device="cuda"):
    return torch.tensor(list(x), dtype=torch.int32, device=device)


def queries(new, hq, d, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(sum(new), hq, d, generator=g).to(torch.bfloat16).cuda()


def problem(cc, new, hq, hkv, d, **kw):
    return cc.problem(dtype="bf16", cu_seqlens=cu_of(new), n_heads_q=hq, n_heads_kv=hkv, head_dim=d, hidden=64, vocab=1, **kw)


def logit_error(q, ks, scale):
    """Bound of the error of a row's logits (rows q [m][d], keys [n][d]): d products, their fp32 sums in any order,
    the scale's rounding, and what 2^x and log add, 16 roundings more, all relative to the sum of magnitudes."""
    d = q.shape[1]
    size = (np.abs(q) @ np.abs(ks).T).max(1, initial=0.0) if len(ks) else np.zeros(len(q))
    return (d + 16) * 2.0 ** -24 * size * scale
