"""Compaction of a cache in 8 bits: codes, scales, ids and positions bit for bit as the oracle's, in place
and out of place, contiguous and paged, one list or one per head; other bytes untouched."""
import numpy as np
import pytest
import torch

from oracle import kv8_oracle as O8
from tests.kv8_util import Cache8, cu_of, i32

pytestmark = pytest.mark.gpu

CASES = [
    # lens, kept, hkv, d, layers, page, block, per_head
    ([1], [1], 1, 64, 1, 0, 16, 0),
    ([40], [0], 2, 128, 1, 0, 16, 0),
    ([768], [512], 4, 128, 2, 0, 16, 0),
    ([300, 5, 130], [77, 5, 1], 2, 128, 2, 16, 16, 0),
    ([1000, 257], [1000, 129], 2, 128, 1, 64, 64, 0),
    ([513], [400], 2, 64, 1, 128, 128, 0),
    ([700, 90], [513, 17], 2, 64, 1, 32, 32, 1),
    ([260], [131], 3, 128, 1, 128, 128, 1),
]


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
def test_compact(case, in_place):
    from paper_2607_27600_amd import cc
    lens, kept, hkv, d, layers, page, block, per_head = case
    print(f"[compact8] {case} in_place={in_place}", flush=True)
    r = np.random.default_rng(11)
    c = Cache8(lens, hkv, d, layers=layers, page=page, block=block, seed=12)
    dst = c if in_place else Cache8(lens, hkv, d, layers=layers, page=page, block=block, seed=13)
    per = hkv if per_head else 1
    budgets = [max(0, min(n, k + (h if k else 0))) for n, k in zip(lens, kept) for h in range(per)]
    lists = [np.sort(r.permutation(lens[i // per])[:k]).astype(np.int32) for i, k in enumerate(budgets)]
    N = sum(lens)
    ids = r.integers(0, 1000, N).astype(np.int32)
    pos = r.integers(0, 1 << 20, N).astype(np.int32)
    idd, posd = torch.from_numpy(ids.copy()).cuda(), torch.from_numpy(pos.copy()).cuda()
    keep = torch.from_numpy(np.concatenate(lists + [np.zeros(1, np.int32)])).cuda()
    p = cc.problem(dtype="bf16", cu_seqlens=cu_of(lens), n_heads_q=hkv, n_heads_kv=hkv, head_dim=d, hidden=64, vocab=1)
    cc.cc_compact_kv8(p, c.view(cc), keep, budgets, per_head, idd, posd, out=None if in_place else dst.view(cc))
    torch.cuda.synchronize()
    after = dst.read()
    want = {k: v.copy() for k, v in dst.host.items()}
    cu = cu_of(lens)
    for b in range(len(lens)):
        for h in range(hkv):
            kl = lists[b * per + (h if per_head else 0)]
            for l in range(layers):
                for t in ("k", "v"):
                    codes, sc = O8.compact(*c.plane(l, b, h, t, n=lens[b]), kl, block)
                    e = np.arange(len(kl))
                    pg, sl = dst._where(b, e)
                    want[t][l, pg, h, sl, :d] = codes
                    e = np.arange(0, len(kl), block)
                    pg, sl = dst._where(b, e)
                    want[t + "s"][l, pg, h, sl // block] = sc
        first = lists[b * per]
        ids[cu[b]:cu[b] + len(first)] = ids[cu[b] + first]
        pos[cu[b]:cu[b] + len(first)] = pos[cu[b] + first]
    for k in want:
        np.testing.assert_array_equal(after[k], want[k], err_msg=k)
    if not in_place:
        for k, v in c.read().items():
            np.testing.assert_array_equal(v, c.host[k])
    np.testing.assert_array_equal(idd.cpu().numpy(), ids)
    np.testing.assert_array_equal(posd.cpu().numpy(), pos)


def test_many_sequences_take_several_launches():
    from paper_2607_27600_amd import cc
    r = np.random.default_rng(15)
    lens = r.integers(0, 90, 150).tolist()
    lens[0] = 90
    kept = [int(x) for x in (np.array(lens) * r.uniform(0, 1, 150)).astype(int)]
    c = Cache8(lens, 1, 64, page=16, block=16, seed=16)
    lists = [np.sort(r.permutation(n)[:k]).astype(np.int32) for n, k in zip(lens, kept)]
    keep = torch.from_numpy(np.concatenate(lists)).cuda()
    p = cc.problem(dtype="bf16", cu_seqlens=cu_of(lens), n_heads_q=1, n_heads_kv=1, head_dim=64, hidden=64, vocab=1)
    cc.cc_compact_kv8(p, c.view(cc), keep, kept, 0)
    torch.cuda.synchronize()
    after = c.read()
    for b, kl in enumerate(lists):
        for t in ("k", "v"):
            codes, sc = O8.compact(*c.plane(0, b, 0, t, n=max(lens[b], 1)), kl, 16)
            gc, gs = c.plane(0, b, 0, t, src=after, n=max(len(kl), 1))
            np.testing.assert_array_equal(gc[: len(kl)], codes)
            np.testing.assert_array_equal(gs[: len(sc)], sc)


def test_nan_codes_and_extreme_scales():
    """NaN codes stay NaN and do not count; scales far apart in one block."""
    from paper_2607_27600_amd import cc
    c = Cache8([64], 1, 128, block=16, seed=17)
    codes, sc = c.plane(0, 0, 0, "k", n=64)
    sc[:] = [27, 120, 60, 200]
    codes[1, 3], codes[33, 4], codes[50] = 0x7f, 0xff, 0
    c.put(0, 0, 0, "k", codes, sc)
    c.t["k"].copy_(torch.from_numpy(c.host["k"]))
    c.t["ks"].copy_(torch.from_numpy(c.host["ks"]))
    kl = np.array([0, 1, 2, 17, 20, 33, 40, 47, 48, 49, 50, 63], np.int32)
    p = cc.problem(dtype="bf16", cu_seqlens=[0, 64], n_heads_q=1, n_heads_kv=1, head_dim=128, hidden=64, vocab=1)
    cc.cc_compact_kv8(p, c.view(cc), torch.from_numpy(kl).cuda(), [len(kl)], 0)
    torch.cuda.synchronize()
    want, ws = O8.compact(codes, sc, kl, 16)
    gc, gs = c.plane(0, 0, 0, "k", src=c.read(), n=len(kl))
    nan = (want & 0x7f) == 0x7f
    np.testing.assert_array_equal((gc & 0x7f) == 0x7f, nan)
    np.testing.assert_array_equal(gc[~nan], want[~nan])
    np.testing.assert_array_equal(gs, ws)


@pytest.mark.parametrize("d", [64, 128])
def test_zeros_kept_from_blocks_of_large_scales(d):
    """All that stays of blocks with scales up to 2^120 are zeros and NaN: the new scale is the smallest,
    2^220 below, and zeros stay zeros."""
    from paper_2607_27600_amd import cc
    c = Cache8([64], 1, d, block=16, seed=18)
    codes, sc = c.plane(0, 0, 0, "v", n=64)
    sc[:] = [247, 160, 230, 155]
    codes[0:64:2] = 0
    codes[6], codes[34, 5] = 0x80, 0x7f
    c.put(0, 0, 0, "v", codes, sc)
    c.t["v"].copy_(torch.from_numpy(c.host["v"]))
    c.t["vs"].copy_(torch.from_numpy(c.host["vs"]))
    kl = np.arange(0, 64, 2, dtype=np.int32)
    p = cc.problem(dtype="bf16", cu_seqlens=[0, 64], n_heads_q=1, n_heads_kv=1, head_dim=d, hidden=64, vocab=1)
    cc.cc_compact_kv8(p, c.view(cc), torch.from_numpy(kl).cuda(), [len(kl)], 0)
    torch.cuda.synchronize()
    gc, gs = c.plane(0, 0, 0, "v", src=c.read(), n=len(kl))
    np.testing.assert_array_equal(gs, [27, 27])
    nan = np.zeros(gc.shape, bool)
    nan[17, 5] = True
    np.testing.assert_array_equal((gc & 0x7f) == 0x7f, nan)
    assert np.all((gc[~nan] & 0x7f) == 0)


def test_two_graphs_and_an_eager_call_in_turn():
    """Calls captured in two graphs, replayed in turn with an eager call between them."""
    from paper_2607_27600_amd import cc
    r = np.random.default_rng(21)
    lens, kept, hkv, d = [300, 70], [120, 41], 2, 128
    c = Cache8(lens, hkv, d, layers=2, page=16, block=16, seed=22)
    outs = [Cache8(lens, hkv, d, layers=2, page=16, block=16, seed=23) for _ in range(3)]
    p = cc.problem(dtype="bf16", cu_seqlens=cu_of(lens), n_heads_q=hkv, n_heads_kv=hkv, head_dim=d, hidden=64, vocab=1)
    lists = [[np.sort(r.permutation(n)[:k]).astype(np.int32) for n, k in zip(lens, kept)] for _ in range(2)]
    keeps = [torch.from_numpy(np.concatenate(x)).cuda() for x in lists]
    src = c.view(cc)
    graphs = []
    for keep, out in zip(keeps, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            cc.cc_compact_kv8(p, src, keep, kept, 0, out=out.view(cc))
        graphs.append(g)
    for _ in range(3):
        for o in outs:
            for t in ("k", "v", "ks", "vs"):
                o.t[t].copy_(torch.from_numpy(o.host[t]))
        graphs[0].replay()
        cc.cc_compact_kv8(p, src, keeps[1], kept, 0, out=outs[2].view(cc))
        graphs[1].replay()
        torch.cuda.synchronize()
        for o, ll in zip(outs, (lists[0], lists[1], lists[1])):
            after = o.read()
            for b, kl in enumerate(ll):
                codes, sc = O8.compact(*c.plane(1, b, 1, "v", n=lens[b]), kl, 16)
                gc, gs = o.plane(1, b, 1, "v", src=after, n=len(kl))
                np.testing.assert_array_equal(gc, codes)
                np.testing.assert_array_equal(gs, sc)


@pytest.mark.parametrize("page,page2", [(16, 64), (128, 32)])
def test_pages_of_another_size(page, page2):
    """Out of place between pools whose pages differ."""
    from paper_2607_27600_amd import cc
    r = np.random.default_rng(31)
    lens, kept, hkv, d = [400, 130], [333, 100], 2, 128
    c = Cache8(lens, hkv, d, page=page, block=16, seed=32)
    dst = Cache8([333, 100], hkv, d, page=page2, block=16, room=70, seed=33)
    lists = [np.sort(r.permutation(n)[:k]).astype(np.int32) for n, k in zip(lens, kept)]
    p = cc.problem(dtype="bf16", cu_seqlens=cu_of(lens), n_heads_q=hkv, n_heads_kv=hkv, head_dim=d, hidden=64, vocab=1)
    cc.cc_compact_kv8(p, c.view(cc), torch.from_numpy(np.concatenate(lists)).cuda(), kept, 0, out=dst.view(cc))
    torch.cuda.synchronize()
    after = dst.read()
    for b, kl in enumerate(lists):
        for h in range(hkv):
            for t in ("k", "v"):
                codes, sc = O8.compact(*c.plane(0, b, h, t, n=lens[b]), kl, 16)
                gc, gs = dst.plane(0, b, h, t, src=after, n=len(kl))
                np.testing.assert_array_equal(gc, codes)
                np.testing.assert_array_equal(gs, sc)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_the_largest_scales(d, in_place):
    """Scales from 2^119 to 2^127 (byte 255 reads as 254), whose elements pass fp32: kept where they are the
    block's largest, rounded again where others are."""
    from paper_2607_27600_amd import cc
    r = np.random.default_rng(24)
    n = 176
    c = Cache8([n], 1, d, block=16, seed=25)
    codes, sc = c.plane(0, 0, 0, "k", n=n)
    codes = (r.integers(0, 127, codes.shape) | (r.integers(0, 2, codes.shape) << 7)).astype(np.uint8)
    codes[1, 3], codes[40, 4], codes[100] = 0x7f, 0xff, 0
    sc[:] = [246, 247, 248, 250, 252, 253, 254, 255, 253, 27, 249]
    c.put(0, 0, 0, "k", codes, sc)
    for t in ("k", "ks"):
        c.t[t].copy_(torch.from_numpy(c.host[t]))
    # a destination block of each kind: of one source scale, of several, with and without those past fp32
    kl = np.concatenate([np.arange(0, 30, 2), np.arange(31, 60, 3), np.arange(64, 176, 5)]).astype(np.int32)
    p = cc.problem(dtype="bf16", cu_seqlens=[0, n], n_heads_q=1, n_heads_kv=1, head_dim=d, hidden=64, vocab=1)
    dst = c if in_place else Cache8([n], 1, d, block=16, seed=26)
    cc.cc_compact_kv8(p, c.view(cc), torch.from_numpy(kl).cuda(), [len(kl)], 0, out=None if in_place else dst.view(cc))
    torch.cuda.synchronize()
    want, ws = O8.compact(codes, np.minimum(sc, 254), kl, 16)
    gc, gs = dst.plane(0, 0, 0, "k", src=dst.read(), n=len(kl))
    assert ws.max() == 254 and ws.min() < 250
    np.testing.assert_array_equal(gs, ws)
    nan = (want & 0x7f) == 0x7f
    np.testing.assert_array_equal((gc & 0x7f) == 0x7f, nan)
    np.testing.assert_array_equal(gc[~nan], want[~nan])


def test_more_chunks_than_one_launch_has(memory_given_back):
    """Out of place, 64 lists of 32 layers and 64 heads, one of them so long that the chunks of all pass 2^24
    workgroups: the longest list's last chunks come with a second launch.  Ids move once."""
    from paper_2607_27600_amd import cc
    layers, h, d, page, n = 32, 64, 64, 16, 16640
    assert 64 * layers * h * 2 * (n // 256) >= 1 << 24 > 64 * layers * h * 2 * (n // 256 - 2)
    free, _ = torch.cuda.mem_get_info()
    if free < (12 << 30):
        pytest.skip("needs 12 GiB of device memory")
    lens = [n] + [40] * 63
    per = n // page
    pages = per + 63 * 3
    table = torch.zeros(64, per, dtype=torch.int32)
    table[0] = torch.arange(per)
    table[1:, :3] = per + torch.arange(63 * 3).view(63, 3)
    g = torch.Generator("cuda").manual_seed(27)
    row = page * d
    # one layer of codes for all; 448 in every row, so that kept blocks of kept blocks' scales are bit copies
    src = torch.randint(0, 127, (pages, h, page, d), generator=g, device="cuda", dtype=torch.uint8)
    src[..., 0] = 0x7e
    ssc = torch.randint(100, 150, (pages, h), generator=g, device="cuda", dtype=torch.uint8)
    dst = torch.zeros(layers, pages, h, page, d, dtype=torch.uint8, device="cuda")
    dst_v, dsc = torch.zeros_like(dst), torch.zeros(layers, pages, h, dtype=torch.uint8, device="cuda")
    dsc_v = torch.zeros_like(dsc)
    kw = dict(n_layers=layers, page_stride=h * row, head_stride=row, tok_stride=d, page_size=page, scale_block=16,
              scale_page_stride=h, scale_head_stride=1)
    bt = table.cuda()
    kv = cc.kv8_paged(src, src, ssc, ssc, bt, layer_stride=0, scale_layer_stride=0, **kw)
    out = cc.kv8_paged(dst, dst_v, dsc, dsc_v, bt, layer_stride=pages * h * row, scale_layer_stride=pages * h, **kw)
    p = cc.problem(dtype="bf16", cu_seqlens=cu_of(lens), n_heads_q=h, n_heads_kv=h, head_dim=d, hidden=64, vocab=1)
    keep = [n] + [9] * 63
    lists = torch.cat([torch.arange(n)] + [31 + torch.arange(9)] * 63).to(torch.int32).cuda()
    ids = torch.arange(sum(lens), dtype=torch.int32, device="cuda")
    cc.cc_compact_kv8(p, kv, lists, keep, 0, token_ids=ids, out=out)
    torch.cuda.synchronize()
    for got, gs in ((dst, dsc), (dst_v, dsc_v)):
        for l in range(layers):
            assert torch.equal(got[l, :per], src[:per]) and torch.equal(gs[l, :per], ssc[:per]), l
    # the short lists: entries 31 to 39 of each, from its second and third pages
    p1, p2 = per + 1, per + 2
    x = torch.cat([src[p1::3, :, 15:], src[p2::3, :, :8]], 2)
    top = torch.maximum(ssc[p1::3], ssc[p2::3])
    got = dst_v[layers - 1, per::3]
    assert torch.equal(dsc_v[layers - 1, per::3], top)
    same = torch.cat([ssc[p1::3, :, None] == top[:, :, None], (ssc[p2::3] == top)[:, :, None].expand(-1, -1, 8)], 2)
    assert torch.equal(got[:, :, :9][same], x[same])
    assert torch.count_nonzero(got[:, :, 9:]) == 0
    cu = cu_of(lens)
    assert torch.equal(ids[cu[5]:cu[5] + 9].cpu(), cu[5] + 31 + torch.arange(9, dtype=torch.int32))
    assert torch.equal(ids[:n].cpu(), torch.arange(n, dtype=torch.int32))
