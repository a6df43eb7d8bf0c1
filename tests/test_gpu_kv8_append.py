"""Appending to a cache: rotated keys, values and queries against fp64, in 8 bits and in the cache's own
type, every layout, lengths and block fills where a block is new, partly held or overfull; bytes
that belong to no new entry stay as they were."""
import numpy as np
import pytest
import torch

from oracle import kv8_oracle as O8
from tests.gpu_util import f64
from tests.kv8_util import Cache8, cu_of, i32

pytestmark = pytest.mark.gpu
THETA = 5e5

# Rotation in fp32: the angle is off by up to 2^-25 of a revolution (2e-7), its sine and cosine by an
# ulp or two, the two products and their sum by 2^-24 each: under 1e-6 of the pair's length.
ROT = 1e-6


def _problem(cc, new, hq, hkv, d, dtype="bf16", **kw):
    return cc.problem(dtype=dtype, cu_seqlens=cu_of(new), n_heads_q=hq, n_heads_kv=hkv, head_dim=d, hidden=64,
                      vocab=1, rope_theta=THETA, **kw)


def _inputs(M, hq, hkv, d, dtype, seed, layers=1):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(layers, M, hq + 2 * hkv, d, generator=g) * torch.exp2(torch.randint(-4, 5, (layers, M, 1, 1), generator=g).float())
    return x.to(torch.bfloat16 if dtype == "bf16" else torch.float32)


def _length(x):
    """Length of each element's rotation pair."""
    d = x.shape[-1]
    h = np.hypot(x[..., : d // 2], x[..., d // 2:])
    return np.concatenate([h, h], -1)


def _check8(cache, before, after, new, cached, rows, rot, cap):
    """rows: which -> fp64 values [layers][M][Hkv][d] appended; rot: which -> pair lengths (0: not rotated)."""
    cu = cu_of(new)
    want = {k: v.copy() for k, v in before.items()}
    B = cache.block
    for l in range(cache.layers):
        for b, m in enumerate(new):
            for h in range(cache.hkv):
                for t in ("k", "v"):
                    c, s = cache.plane(l, b, h, t, src=before)
                    x = rows[t][l, cu[b]:cu[b + 1], h]
                    O8.append(c, s, cached[b], x, B, cap)
                    gc, gs = cache.plane(l, b, h, t, src=after)
                    n0, n1 = cached[b], min(cached[b] + m, cap)
                    if n1 > n0:
                        if rot[t] is None:
                            np.testing.assert_array_equal(gs, s)
                            np.testing.assert_array_equal(gc, c)
                        else:
                            np.testing.assert_array_equal(gs, s)
                            sv = np.repeat(O8.scale_value(gs), B)[n0:n1, None]
                            got = O8.e4m3_decode(gc[n0:n1]) * sv
                            x = x[: n1 - n0]
                            lim = 2.0 ** -4 * np.abs(x) + 2.0 ** -10 * sv + ROT * rot[t][l, cu[b]:cu[b] + n1 - n0, h]
                            assert np.all(np.abs(got - x) <= lim)
                            # entries before: as the oracle has them
                            np.testing.assert_array_equal(gc[n0 // B * B:n0], c[n0 // B * B:n0])
                        cache_put(cache, want, l, b, h, t, gc, gs, n0, n1)
    for k in want:
        np.testing.assert_array_equal(after[k], want[k], err_msg=f"{k}: bytes outside the new entries changed")


def cache_put(cache, dst, l, b, h, t, codes, scales, n0, n1):
    lo = n0 // cache.block * cache.block
    e = np.arange(lo, n1)
    pg, sl = cache._where(b, e)
    dst[t][l, pg, h, sl, : cache.d] = codes[lo:n1]
    e = np.arange(lo, n1, cache.block)
    pg, sl = cache._where(b, e)
    dst[t + "s"][l, pg, h, sl // cache.block] = scales[e // cache.block]


CASES = [
    # new, cached, hq, hkv, d, page, block, dtype, layers
    ([1], [0], 4, 2, 128, 0, 16, "bf16", 1),
    ([1, 1, 1, 1, 1], [0, 15, 16, 17, 100], 28, 4, 128, 16, 16, "bf16", 1),
    ([5, 0, 33, 1], [3, 9, 0, 63], 8, 8, 128, 64, 64, "bf16", 1),
    ([130, 1, 17], [127, 128, 200], 7, 1, 128, 128, 128, "bf16", 1),
    ([300], [70], 32, 8, 128, 32, 16, "bf16", 1),
    ([3, 40], [250, 7], 4, 4, 64, 16, 16, "bf16", 1),
    ([129], [1], 16, 4, 64, 0, 128, "bf16", 1),
    ([20, 2], [5, 30], 6, 3, 64, 32, 32, "f32", 1),
    ([31], [33], 4, 2, 128, 0, 32, "f32", 1),
    ([9, 16], [16, 2], 4, 2, 128, 16, 16, "bf16", 3),
]


MORE_HEADS = [([3, 1], [14, 0], 66, 66, 64, 16, 16, "bf16", 1), ([40], [7], 130, 65, 64, 0, 32, "bf16", 2)]


@pytest.mark.parametrize("case", MORE_HEADS, ids=["66", "65"])
def test_more_heads_than_a_workgroup_takes(case):
    test_append_8bit(case, False)


@pytest.mark.parametrize("pos_given", [True, False])
@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
def test_append_8bit(case, pos_given):
    from paper_2607_27600_amd import cc
    new, cached, hq, hkv, d, page, block, dtype, layers = case
    print(f"[append8] {case} pos={pos_given}", flush=True)
    cache = Cache8(cached, hkv, d, layers=layers, page=page, block=block, room=max(new), seed=1)
    M = sum(new)
    x = _inputs(M, hq, hkv, d, dtype, 2, layers)
    xd = x.cuda()
    pos = np.concatenate([np.arange(c, c + m) for c, m in zip(cached, new)])
    if pos_given:
        pos = pos + np.random.default_rng(3).integers(0, 900000, M)
    p = _problem(cc, new, hq, hkv, d, dtype)
    q, k, v = xd.split([hq, hkv, hkv], 2)
    with_q = layers == 1
    out = cc.cc_append_kv8(p, cache.view(cc), k if layers > 1 else k[0], v if layers > 1 else v[0], i32(cached),
                           capacity=0 if page else cache.cap, n_layers=layers,
                           pos_ids=i32(pos) if pos_given else None, q=q[0] if with_q else None)
    torch.cuda.synchronize()
    h = f64(x)
    kr = np.stack([O8.rotate(h[l, :, hq:hq + hkv], pos, THETA) for l in range(layers)])
    _check8(cache, cache.host, cache.read(), new, cached, {"k": kr, "v": h[:, :, hq + hkv:]},
            {"k": _length(h[:, :, hq:hq + hkv]), "v": None}, cache.cap if not page else cache.max_pages * page)
    if with_q:
        want = O8.rotate(h[0, :, :hq], pos, THETA)
        half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
        assert np.all(np.abs(f64(out) - want) <= half * np.abs(want) + ROT * _length(h[0, :, :hq]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,page", [(128, 0), (128, 16), (64, 32)])
def test_append_own_type(dtype, d, page):
    from paper_2607_27600_amd import cc
    new, cached, hq, hkv = [17, 0, 1, 40], [0, 3, 31, 16], 6, 2
    print(f"[append] {dtype} {d} {page}", flush=True)
    T = torch.bfloat16 if dtype == "bf16" else torch.float32
    M, n = sum(new), len(new)
    P = page or 64
    per = -(-64 // P) if page else 1
    g = torch.Generator().manual_seed(5)
    pool = [torch.randn(n * per, hkv, P, d + 8, generator=g).to(T) for _ in range(2)]
    table = torch.randperm(n * per, generator=g).to(torch.int32).view(n, per)
    k, v = (t.clone().cuda() for t in pool)
    kw = dict(n_layers=1, layer_stride=k.numel(), head_stride=P * (d + 8), tok_stride=d + 8)
    if page:
        kv = cc.kv_paged(k, v, table.cuda(), page_stride=hkv * P * (d + 8), page_size=P, **kw)
    else:
        table = torch.arange(n, dtype=torch.int32).view(n, 1)
        kv = cc.kv_contiguous(k, v, seq_stride=hkv * P * (d + 8), **kw)
    x = _inputs(M, hq, hkv, d, dtype, 6)[0]
    q, kn, vn = x.cuda().split([hq, hkv, hkv], 1)
    pos = np.concatenate([np.arange(c, c + m) for c, m in zip(cached, new)])
    out = cc.cc_append_kv(_problem(cc, new, hq, hkv, d, dtype), kv, kn, vn, i32(cached), capacity=64, q=q)
    torch.cuda.synchronize()
    h = f64(x)
    want = [t.clone() for t in pool]
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    kr = O8.rotate(h[:, hq:hq + hkv], pos, THETA)
    ln = _length(h[:, hq:hq + hkv])
    got = [k.cpu(), v.cpu()]
    at = 0
    for b, m in enumerate(new):
        for i in range(m):
            t = cached[b] + i
            pg, sl = int(table[b, t // P]), t % P
            assert torch.equal(got[1][pg, :, sl, :d], x[at, hq + hkv:])
            err = np.abs(f64(got[0][pg, :, sl, :d]) - kr[at])
            assert np.all(err <= half * np.abs(kr[at]) + ROT * ln[at])
            for w, o in zip(want, got):
                w[pg, :, sl, :d] = o[pg, :, sl, :d]
            at += 1
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    qr = O8.rotate(h[:, :hq], pos, THETA)
    assert np.all(np.abs(f64(out) - qr) <= half * np.abs(qr) + ROT * _length(h[:, :hq]))


def test_append_stops_at_capacity_and_missing_pages():
    from paper_2607_27600_amd import cc
    cache = Cache8([30, 20], 2, 128, page=16, block=16, room=40, seed=4)
    cache.table[1, 2] = -1            # tokens 32..47 of sequence 1 have no page
    cache.bt = torch.from_numpy(cache.table).cuda()
    new, cached, cap = [20, 30], [30, 20], 45
    x = _inputs(50, 2, 2, 128, "bf16", 8)
    q, k, v = x.cuda().split([2, 2, 2], 2)
    cc.cc_append_kv8(_problem(cc, new, 2, 2, 128), cache.view(cc), k[0], v[0], i32(cached), capacity=cap, rotate=False)
    torch.cuda.synchronize()
    after = cache.read()
    h = f64(x)[0]
    want = {t: w.copy() for t, w in cache.host.items()}
    for b, at in ((0, 0), (1, 20)):
        for hh in range(2):
            for t, off in (("k", 2), ("v", 4)):
                stop = cap if b == 0 else 32
                c, s = cache.plane(0, b, hh, t, n=48)
                O8.append(c, s, cached[b], h[at:at + new[b], off + hh], 16, stop)
                cache_put(cache, want, 0, b, hh, t, c, s, cached[b], stop)
    for t in want:
        np.testing.assert_array_equal(after[t], want[t])


def test_append_non_finite():
    """NaN and infinities become NaN codes and leave the scale to the others; an all-zero block has the least."""
    from paper_2607_27600_amd import cc
    cache = Cache8([0], 2, 64, block=16, room=32, seed=6)
    x = _inputs(20, 2, 2, 64, "bf16", 9)
    x[0, 3, 2, 5] = float("inf")
    x[0, 4, 4, 7] = float("nan")
    x[0, 5, 5, 9] = -float("inf")
    x[0, 16:, 3] = 0
    q, k, v = x.cuda().split([2, 2, 2], 2)
    cc.cc_append_kv8(_problem(cc, [20], 2, 2, 64), cache.view(cc), k[0], v[0], i32([0]), capacity=cache.cap, rotate=False)
    torch.cuda.synchronize()
    after, h = cache.read(), f64(x)[0]
    for hh in range(2):
        for t, off in (("k", 2), ("v", 4)):
            c, s = cache.plane(0, 0, hh, t)
            O8.append(c, s, 0, h[:, off + hh], 16, 32)
            gc, gs = cache.plane(0, 0, hh, t, src=after)
            np.testing.assert_array_equal(gs, s)
            nan = (c & 0x7f) == 0x7f
            np.testing.assert_array_equal((gc & 0x7f) == 0x7f, nan)
            np.testing.assert_array_equal(gc[~nan], c[~nan])


def test_append_token_by_token_follows_device_lengths_in_a_graph():
    """One captured call, replayed with lengths that a kernel advances between replays: the same cache as
    eager single appends."""
    from paper_2607_27600_amd import cc
    new = [1, 1, 1]
    caches = [Cache8([0, 14, 31], 2, 128, page=16, block=16, room=40, seed=7) for _ in range(2)]
    x = _inputs(3 * 35, 4, 2, 128, "bf16", 10)[0].view(35, 3, 8, 128).cuda()
    p = _problem(cc, new, 4, 2, 128)
    lens = i32([0, 14, 31])
    for t in range(35):
        q, k, v = x[t].split([4, 2, 2], 1)
        cc.cc_append_kv8(p, caches[0].view(cc), k, v, lens, q=q)
        lens += 1
    row = x[0].clone()
    lens2, one = i32([0, 14, 31]), torch.ones(3, dtype=torch.int32, device="cuda")
    view = caches[1].view(cc)
    q, k, v = row.split([4, 2, 2], 1)
    qo = torch.empty(3, 4, 128, dtype=torch.bfloat16, device="cuda")
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        cc.cc_append_kv8(p, view, k, v, lens2, q=q, q_out=qo)
        lens2.add_(one)
    for t in range(35):
        row.copy_(x[t])
        g.replay()
    torch.cuda.synchronize()
    a, b = caches[0].read(), caches[1].read()
    for t in a:
        np.testing.assert_array_equal(a[t], b[t])
    assert lens2.tolist() == [35, 49, 66]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_append_to_a_block_of_the_largest_scale(d, dtype):
    """A held block of scale byte 254, 2^127: new elements of up to 2^128 are rounded in it, not lost; byte 255
    reads as 254."""
    from paper_2607_27600_amd import cc
    cache = Cache8([5, 3], 2, d, block=16, room=32, seed=61)
    T = torch.bfloat16 if dtype == "bf16" else torch.float32
    for t in ("k", "v"):
        for b, n in ((0, 5), (1, 3)):
            for hh in range(2):
                codes, sc = cache.plane(0, b, hh, t, n=n)
                sc[:] = 254 + (b == 1)
                cache.put(0, b, hh, t, codes, sc)
        cache.t[t + "s"].copy_(torch.from_numpy(cache.host[t + "s"]))
    # magnitudes 2^119 to 2^128, in steps that the type holds: in units of the scale from 2^-8 to 2
    g = torch.Generator().manual_seed(62)
    x = (torch.randint(128, 256, (6, 6, d), generator=g).float() * torch.exp2(torch.randint(112, 121, (6, 6, 1), generator=g).float())
         * torch.where(torch.rand(6, 6, d, generator=g) < 0.5, -1.0, 1.0)).to(T)
    assert torch.isfinite(x).all()
    q, k, v = x.cuda().split([2, 2, 2], 1)
    p = _problem(cc, [4, 2], 2, 2, d, dtype)
    cc.cc_append_kv8(p, cache.view(cc), k, v, i32([5, 3]), capacity=cache.cap, rotate=False)
    torch.cuda.synchronize()
    after, h = cache.read(), f64(x)
    for b, n, at, m in ((0, 5, 0, 4), (1, 3, 4, 2)):
        for hh in range(2):
            for t, off in (("k", 2), ("v", 4)):
                c, s = cache.plane(0, b, hh, t)
                s[0] = 254
                O8.append(c, s, n, h[at:at + m, off + hh], 16, cache.cap)
                gc, gs = cache.plane(0, b, hh, t, src=after)
                assert gs[0] == s[0] == 254
                assert np.all(c[n:n + m] & 0x7f)     # all of them above 2^-9 of the scale
                np.testing.assert_array_equal(gc, c)


def test_more_layers_than_one_launch_has_workgroups_for(memory_given_back):
    """One token each of 4096 sequences into 2100 layers: past 2^24 workgroups, the last layers come with a
    second launch."""
    from paper_2607_27600_amd import cc
    n, layers, d = 4096, 2100, 64
    assert 2 * n * layers >= 1 << 24
    free, _ = torch.cuda.mem_get_info()
    if free < (12 << 30):
        pytest.skip("needs 12 GiB of device memory")
    g = torch.Generator("cuda").manual_seed(63)
    x = torch.randint(0, 30000, (2, layers, n, 1, d), generator=g, device="cuda", dtype=torch.int16).view(torch.bfloat16)
    # a cache of two entries a sequence: the second is written
    pools = [torch.zeros(layers, n, 2, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    kv = cc.kv_contiguous(*pools, n_layers=layers, layer_stride=n * 2 * d, seq_stride=2 * d, head_stride=0, tok_stride=d)
    p = _problem(cc, [1] * n, 1, 1, d)
    cc.cc_append_kv(p, kv, x[0], x[1], i32([1] * n), capacity=2, n_layers=layers, rotate=False)
    torch.cuda.synchronize()
    for pool, y in zip(pools, x):
        assert torch.equal(pool[:, :, 1].view(torch.int16), y[:, :, 0].view(torch.int16))
        assert torch.count_nonzero(pool[:, :, 0].view(torch.int16)) == 0


@pytest.mark.parametrize("new", [[2, 2], [3, 1]])
@pytest.mark.parametrize("d", [64, 128])
def test_negative_lengths_are_zero(new, d):
    """Keys and queries of a sequence stand at the same positions."""
    from paper_2607_27600_amd import cc
    x = _inputs(sum(new), 4, 2, d, "bf16", 64)[0].cuda()
    q, k, v = x.split([4, 2, 2], 1)
    p, out = _problem(cc, new, 4, 2, d), []
    for cached in ([0, 5], [-7, 5]):
        cache = Cache8([0, 5], 2, d, block=16, room=32, seed=65)
        qo = cc.cc_append_kv8(p, cache.view(cc), k, v, i32(cached), capacity=cache.cap, q=q)
        torch.cuda.synchronize()
        out.append((f64(qo), cache.read()))
    np.testing.assert_array_equal(out[0][0], out[1][0])
    for t in out[0][1]:
        np.testing.assert_array_equal(out[0][1][t], out[1][1][t])
