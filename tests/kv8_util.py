"""Caches in 8 bits for tests: pools with padding and a shuffled block table, or contiguous planes
with gaps, random bytes where no entry lies, and numpy copies of single planes."""
import numpy as np
import torch

from oracle import kv8_oracle as O8


class Cache8:
    """fill: byte of every code and scale that no entry owns (0x7f: NaN codes)."""

    def __init__(self, lens, hkv, d, layers=1, page=0, block=16, room=0, seed=0, fill=None, std=1.0, device="cuda"):
        r = np.random.default_rng(seed)
        self.lens, self.hkv, self.d, self.layers, self.page, self.block = list(lens), hkv, d, layers, page, block
        n = len(lens)
        cap = max(max(self.lens) + room, 1)
        if page:
            P = page
            self.max_pages = -(-cap // P) + 1
            order = r.permutation(n * self.max_pages + 3)
            self.table = order[: n * self.max_pages].reshape(n, self.max_pages).astype(np.int32)
            pages = len(order)
            self.cap = (self.max_pages - 1) * P
        else:
            P = -(-cap // block) * block
            self.table = np.arange(n, dtype=np.int32)[:, None]
            pages = n
            self.cap = P
            self.max_pages = 1
        self.P = P
        # a gap of 16 bytes behind each token row, of two scales behind each head's scales
        self.tok = d + 16
        shape = (layers, pages, hkv, P, self.tok)
        sshape = (layers, pages, hkv, P // block + 2)
        draw = lambda s: r.integers(0, 0x7f, s).astype(np.uint8) if fill is None else np.full(s, fill, np.uint8)
        self.host = {"k": draw(shape), "v": draw(shape), "ks": r.integers(100, 150, sshape).astype(np.uint8),
                     "vs": r.integers(100, 150, sshape).astype(np.uint8)}
        for l in range(layers):
            for b, m in enumerate(self.lens):
                for h in range(hkv):
                    for t in ("k", "v"):
                        x = r.normal(0, std, (m, d)) * np.exp2(r.integers(-3, 4))
                        self.put(l, b, h, t, *quantize(x, block))
        self.t = {k: torch.from_numpy(v.copy()).to(device) for k, v in self.host.items()}
        self.bt = torch.from_numpy(self.table).to(device)

    def _where(self, b, t):
        if self.page:
            return self.table[b, t // self.P], t % self.P
        return np.full_like(t, b), t

    def put(self, l, b, h, which, codes, scales):
        t = np.arange(len(codes))
        pg, sl = self._where(b, t)
        self.host[which][l, pg, h, sl, : self.d] = codes
        t = np.arange(len(scales)) * self.block
        pg, sl = self._where(b, t)
        self.host[which + "s"][l, pg, h, sl // self.block] = scales

    def plane(self, l, b, h, which, src=None, n=None):
        """(codes [n][d], scales) of a plane, of all its room by default."""
        src = self.host if src is None else src
        n = self.cap if n is None else n
        t = np.arange(n)
        pg, sl = self._where(b, t)
        codes = src[which][l, pg, h, sl, : self.d].copy()
        t = np.arange(-(-n // self.block)) * self.block
        pg, sl = self._where(b, t)
        return codes, src[which + "s"][l, pg, h, sl // self.block].copy()

    def values(self, l, b, h, which, n):
        c, s = self.plane(l, b, h, which, n=n)
        return O8.values(c, s, self.block)

    def read(self):
        return {k: v.cpu().numpy() for k, v in self.t.items()}

    def view(self, cc):
        t, pages = self.t, self.host["k"].shape[1]
        row, sr = self.P * self.tok, self.P // self.block + 2
        if self.page:
            return cc.kv8_paged(t["k"], t["v"], t["ks"], t["vs"], self.bt, n_layers=self.layers,
                                layer_stride=pages * self.hkv * row, page_stride=self.hkv * row, head_stride=row,
                                tok_stride=self.tok, page_size=self.P, scale_block=self.block,
                                scale_layer_stride=pages * self.hkv * sr, scale_page_stride=self.hkv * sr,
                                scale_head_stride=sr)
        return cc.kv8_contiguous(t["k"], t["v"], t["ks"], t["vs"], n_layers=self.layers,
                                 layer_stride=pages * self.hkv * row, seq_stride=self.hkv * row, head_stride=row,
                                 tok_stride=self.tok, scale_block=self.block,
                                 scale_layer_stride=pages * self.hkv * sr, scale_seq_stride=self.hkv * sr,
                                 scale_head_stride=sr)


def quantize(x, block):
    codes = np.empty(x.shape, np.uint8)
    scales = np.empty(-(-len(x) // block), np.uint8)
    for b0 in range(0, len(x), block):
        scales[b0 // block] = O8.scale_byte(O8.top(x[b0:b0 + block]))
        codes[b0:b0 + block] = O8.encode(x[b0:b0 + block], int(scales[b0 // block]))
    return codes, scales


def cu_of(lens):
    return [0] + np.cumsum(lens).tolist()


def i32(x, device="cuda"):
    return torch.tensor(list(x), dtype=torch.int32, device=device)
