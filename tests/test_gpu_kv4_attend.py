"""scap_kv4_attend against attention in 64 bits over the values that the cache stands for."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from kv4_testlib import Cache, quantise64, starts, tokens
from test_gpu_kv4 import SHAPES, fake_cache

BF, HF = torch.bfloat16, torch.float16


def filled(lens, heads, D, group, dt=BF, page=64, seed=0, fill=None, **kw):
    """A cache with random tokens, and scale, zero, codes of its keys and values in 64 bits."""
    c = Cache(lens, page=page, heads=heads, D=D, group=group, dt=dt, seed=seed, **kw)
    if fill is not None:
        c.raw[1:-1] = fill
    n = sum(lens)
    k = tokens(n, heads, D, BF, seed + 1) * 0.5 if n else torch.zeros(0, heads, D, device="cuda")
    v = tokens(n, heads, D, BF, seed + 2) if n else k
    k, v = k.clamp(-300, 300).to(dt), v.clamp(-300, 300).to(dt)
    if n:
        c.scap.scap_kv4_append(c.cache, k, v, starts(lens))
    c.kv = (k, v)
    return c


def side64(x, group):
    s, z, q = quantise64(x.double().cpu().numpy(), group)
    s, z, q = (torch.tensor(a, device="cuda") for a in (s, z, q))
    return (s[..., None] * (q - z[..., None])).flatten(-2), 15 * s.repeat_interleave(group, -1)  # values, and the size of a code's part


def check(c, q, out, lse, lens, nq, scale, window, missing=()):
    B, _, Hq, D = q.shape
    g = Hq // c.heads
    k64, kmag = side64(c.kv[0], c.group)
    v64, vmag = side64(c.kv[1], c.group)
    at = 0
    worst = 0.0
    for b, n in enumerate(lens):
        rows = slice(at, at + n)
        at += n
        pos = torch.arange(n, device="cuda")
        there = torch.ones(n, dtype=torch.bool, device="cuda")
        for lo, hi in missing:
            there &= (pos < lo) | (pos >= hi)
        for i in range(nq):
            last = n - nq + i
            seen = there & (pos <= last) & ((pos > last - window) if window else True)
            for h in range(c.heads):
                o, ls = out[b, i, h * g:(h + 1) * g].double(), lse[b, i, h * g:(h + 1) * g].double()
                if not bool(seen.any()):
                    assert bool((o == 0).all()) and bool((ls == -math.inf).all())
                    continue
                idx = rows.start + seen.nonzero().flatten()
                qq = q[b, i, h * g:(h + 1) * g].double()
                s = scale * qq @ k64[idx, h].T
                want_l = torch.logsumexp(s, -1)
                p = torch.exp(s - want_l[:, None])
                want = p @ v64[idx, h]
                # A score is a sum of D exact products of q and codes (up to 15 scales) and as many of q and zero points: D / 8 + 16
                # additions and multiplications in fp32, the tensor core's with truncation.  2^x is good to 2^-22.
                es = scale * 2 * (qq.abs() @ kmag[idx, h].T) * (D / 8 + 16) * 2.0 ** -23 + 2.0 ** -21
                # p v: the rounding of p s to 11 bits acts on v; p itself is off by its score, and the sum it is divided by likewise
                err = (p * (2.0 ** -11 + 2 * es)) @ v64[idx, h].abs() + (p * 2 * es).sum(-1, keepdim=True) * want.abs()
                # code and zero-point parts are added up apart, two additions per tile and as many rescalings
                err = err + 2 * (p @ vmag[idx, h]) * (len(idx) / 16 + 32) * 2.0 ** -23 + want.abs() * torch.finfo(out.dtype).eps / 2 * 1.001
                err = err + vmag[idx, h].amax() * len(idx) * 2.0 ** -38 + 2.0 ** -25
                r = ((o - want).abs() / err).max()
                el = es.amax(-1) + 2.0 ** -22 * (want_l.abs() + math.log(n) + 4)
                rl = ((ls - want_l).abs() / el).max()
                worst = max(worst, float(r), float(rl))
                assert float(r) <= 1 and float(rl) <= 1, (b, i, h, float(r), float(rl))
    return worst


def attend(c, q, scale, window=0, nan=True):
    B, nq, Hq, D = q.shape
    out = torch.full_like(q, float("nan") if nan else 0.0)
    lse = torch.full((B, nq, Hq), float("nan"), device="cuda")
    ws = torch.full((c.scap.scap_kv4_attend_workspace(B, nq, Hq, c.heads, D),), 255, dtype=torch.uint8, device="cuda")
    c.scap.scap_kv4_attend(c.cache, q, out, scale, ws, window=window, lse=lse)
    torch.cuda.synchronize()
    assert c.guards_intact()
    c.scap.scap_device_status()
    return out, lse


def queries(B, nq, Hq, D, dt, seed=9):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(B, nq, Hq, D, generator=g, device="cuda").to(dt)


@pytest.mark.gpu
@pytest.mark.parametrize("D,group", SHAPES)
@pytest.mark.parametrize("dt", [BF, HF])
def test_shapes(D, group, dt):
    lens = [1, 32, 33, 100, 0, 517]
    c = filled(lens, 2, D, group, dt, page=32, fill=255)  # what lies behind the last token is NaN
    q = queries(len(lens), 1, 6, D, dt)
    out, lse = attend(c, q, D ** -0.5)
    check(c, q, out, lse, lens, 1, D ** -0.5, 0)


@pytest.mark.gpu
@pytest.mark.parametrize("nq,g,heads", [(2, 1, 3), (3, 5, 1), (4, 4, 2), (5, 7, 1), (16, 1, 1), (16, 16, 1), (7, 16, 2), (1, 16, 2), (1, 33, 1), (9, 2, 1)])
@pytest.mark.parametrize("window", [0, 20])
def test_rows(nq, g, heads, window):
    lens = [3, 64, 130, 0, 16, 300]
    c = filled(lens, heads, 64, 32, page=64, fill=255, seed=nq)
    q = queries(len(lens), nq, g * heads, 64, BF)
    out, lse = attend(c, q, 0.125, window)
    check(c, q, out, lse, lens, nq, 0.125, window)


@pytest.mark.gpu
@pytest.mark.parametrize("window", [0, 1, 31, 32, 33, 1000, 1 << 30])
def test_windows_and_cuts(window):
    lens = [2000, 1, 5000, 129]
    c = filled(lens, 1, 128, 64, page=128, seed=4, fill=255)
    q = queries(4, 3, 4, 128, BF)
    out, lse = attend(c, q, 128 ** -0.5, window)
    check(c, q, out, lse, lens, 3, 128 ** -0.5, window)


@pytest.mark.gpu
@pytest.mark.parametrize("B,most", [(1, 40000), (300, 70), (130, 700), (2, 9000)])
def test_many_and_long(B, most):
    rng = np.random.default_rng(B)
    lens = rng.integers(0, most, B).tolist()
    lens[0] = most
    c = filled(lens, 2, 64, 64, HF, page=64, seed=B)
    q = queries(B, 1, 4, 64, HF)
    out, lse = attend(c, q, 0.125)
    check(c, q, out, lse, lens, 1, 0.125, 0)
    again, lse2 = attend(c, q, 0.125)
    assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.gpu
@pytest.mark.parametrize("D,group,heads,B,most,nq,g,window", [(64, 32, 8, 200, 90, 1, 3, 0), (128, 128, 16, 90, 300, 2, 4, 0), (128, 32, 6, 260, 60, 1, 8, 25),
                                                              (256, 128, 4, 240, 50, 1, 2, 0), (64, 64, 40, 41, 2500, 1, 1, 700)])
def test_a_warp_for_every_item(D, group, heads, B, most, nq, g, window):
    """So many sequences and heads that each warp works on its own, lengths from none to a few that are cut."""
    rng = np.random.default_rng(B)
    lens = (most * rng.random(B) ** 3).astype(int).tolist()
    lens[B // 2] = 4 * most
    c = filled(lens, heads, D, group, page=32, seed=B, fill=255)
    q = queries(B, nq, g * heads, D, BF)
    out, lse = attend(c, q, D ** -0.5, window)
    check(c, q, out, lse, lens, nq, D ** -0.5, window)
    again, lse2 = attend(c, q, D ** -0.5, window)
    assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.gpu
def test_peaked_and_large_scores():
    lens = [700, 64]
    for scale in (3.0, -0.5, 0.0, 50.0):
        c = filled(lens, 1, 64, 32, seed=7)
        q = queries(2, 2, 2, 64, BF) * 4
        out, lse = attend(c, q, scale)
        check(c, q, out, lse, lens, 2, abs(scale), 0) if scale >= 0 else check(c, -q, out, lse, lens, 2, -scale, 0)


@pytest.mark.gpu
def test_sizes_of_queries_and_values():
    """Queries far from one in size, values of very different size per token, values that are all zero."""
    lens, D = [200], 128
    for kind in range(4):
        c = Cache(lens, heads=1, D=D, group=64)
        k = tokens(200, 1, D, BF, 1) * 0.1
        v = tokens(200, 1, D, BF, 2).clamp(-300, 300)
        if kind == 1:
            v = v * torch.logspace(-4, 4, 200, base=2, device="cuda")[:, None, None]
        if kind == 2:
            v = v * 2.0 ** 90
        if kind == 3:
            v = torch.zeros_like(v)
        k, v = k.to(BF), v.to(BF)
        c.kv = (k, v)
        c.scap.scap_kv4_append(c.cache, k, v, starts(lens))
        up = 2.0 ** (60 if kind == 1 else (-60 if kind == 2 else 0))
        q = (queries(1, 1, 2, D, BF) * up).to(BF)
        out, lse = attend(c, q, D ** -0.5 / up)
        check(c, q, out, lse, lens, 1, D ** -0.5 / up, 0)


@pytest.mark.gpu
def test_rows_of_different_size():
    """Eight rows share a power of two: those 2^-14 as large as the largest keep all of their bits."""
    lens = [150, 33]
    c = filled(lens, 2, 128, 64, seed=17)
    q = queries(2, 2, 8, 128, HF)
    q = (q * torch.tensor([1.0, 2.0 ** -14, 4.0, 2.0 ** -7, 2.0 ** -3, 0.0, 1.0, 2.0 ** -14], device="cuda")[:, None].half()).to(HF)
    out, lse = attend(c, q, 128 ** -0.5)
    check(c, q, out, lse, lens, 2, 128 ** -0.5, 0)


@pytest.mark.gpu
def test_non_finite_values_stay_with_the_rows_that_see_them():
    lens, D, nq = [100, 100], 64, 4
    c = Cache(lens, heads=2, D=D, group=64)
    k, v = tokens(200, 2, D, BF, 1).clamp(-50, 50), tokens(200, 2, D, BF, 2).clamp(-50, 50)
    c.scap.scap_kv4_append(c.cache, k, v, starts(lens))
    q = queries(2, nq, 4, D, BF)
    clean, _ = attend(c, q, 0.125)
    v[98, 0, 3] = float("nan")    # the value of the second token from the end of sequence 0, head 0
    k[199, 1, 5] = float("inf")   # the key of the last token of sequence 1, head 1
    c.scap.scap_kv4_append(c.cache, k, v, starts(lens))
    q[0, 0, 3, 2] = float("nan")  # a query of head 1
    out, _ = attend(c, q, 0.125)
    bad = ~torch.isfinite(out).all(-1)
    want = torch.zeros_like(bad)
    want[0, 2:, 0:2] = True       # tokens 98 and 99 see token 98
    want[1, 3, 2:4] = True
    want[0, 0, 3] = True
    assert torch.equal(bad, want)
    assert torch.equal(out[~want], clean[~want])


@pytest.mark.gpu
def test_missing_pages_are_not_seen():
    lens = [200]
    c = filled(lens, 1, 128, 128, page=32, seed=3)
    c.table[0, 2] = -1
    c.table[0, 4] = 1 << 20
    q = queries(1, 2, 2, 128, BF)
    out, lse = attend(c, q, 128 ** -0.5)
    check(c, q, out, lse, lens, 2, 128 ** -0.5, 0, missing=[(64, 96), (128, 160)])
    c.table.fill_(-1)
    out, lse = attend(c, q, 128 ** -0.5)
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())


@pytest.mark.gpu
def test_slices_graph_and_stream():
    lens, heads, D = [50, 130], 2, 128
    c = filled(lens, heads, D, 64, room=200)
    qkv = torch.randn(2, 12, D, device="cuda").to(BF)   # a fused row: 8 query, 2 key, 2 value heads
    q = qkv[:, None, :8]
    wide = torch.zeros(2, 1, 12, D, dtype=BF, device="cuda")
    out, lse = wide[:, :, 2:10], torch.empty(2, 1, 8, device="cuda")
    ws = torch.empty(c.scap.scap_kv4_attend_workspace(2, 1, 8, heads, D), dtype=torch.uint8, device="cuda")
    kn, vn = qkv[:, 8:10], qkv[:, 10:12]

    def step():
        c.lens += 1
        c.scap.scap_kv4_append(c.cache, kn, vn)
        c.scap.scap_kv4_attend(c.cache, q, out, D ** -0.5, ws, lse=lse)
    k, v = ([t[:50], t[50:]] for t in c.kv)

    def expect():
        for b in range(2):
            k[b], v[b] = torch.cat((k[b], kn[b:b + 1])), torch.cat((v[b], vn[b:b + 1]))
        c.kv = (torch.cat(k), torch.cat(v))
        check(c, q, out, lse, [len(x) for x in k], 1, D ** -0.5, 0)
        assert bool((wide[:, :, :2] == 0).all()) and bool((wide[:, :, 10:] == 0).all())
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    s.synchronize()
    expect()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(3):
        qkv.copy_(torch.randn_like(qkv))
        graph.replay()
        torch.cuda.synchronize()
        expect()


@pytest.mark.gpu
@pytest.mark.parametrize("B,heads,tokens,nq,g,window", [(1, 32, 215000, 1, 2, 0), (2, 16, 180000, 2, 8, 0), (110, 8, 4200, 1, 2, 0), (100, 8, 6000, 2, 1, 4000)])
def test_more_than_32_tiles_per_warp(B, heads, tokens, nq, g, window):
    """The addresses of a warp's tiles come 32 at a time.  Some heads of some sequences against 64 bits."""
    import paper_2412_07174_b200 as scap
    D, page, dev = 64, 128, "cuda"
    rng = np.random.default_rng(tokens)
    lens = [tokens - int(rng.integers(0, 200)) for _ in range(B)]
    width = -(-tokens // page)
    table = torch.tensor(rng.permutation(B * width).reshape(B, width), dtype=torch.int32, device=dev)
    n = torch.tensor(lens, dtype=torch.int32, device=dev)
    pool = torch.zeros(B * width, scap.scap_kv4_page_bytes(page, heads, D, 64), dtype=torch.uint8, device=dev)
    cache = scap.ScapKv4(pool, page, heads, D, 64, table, n)
    gen = torch.Generator(device=dev).manual_seed(3)
    k = torch.empty(sum(lens), heads, D, dtype=BF, device=dev).normal_(generator=gen)
    v = torch.empty(sum(lens), heads, D, dtype=BF, device=dev).normal_(generator=gen)
    at = starts(lens)
    scap.scap_kv4_append(cache, k, v, at)
    q = queries(B, nq, g * heads, D, BF)
    out, lse = torch.empty_like(q), torch.empty(B, nq, g * heads, device=dev)
    ws = torch.empty(scap.scap_kv4_attend_workspace(B, nq, g * heads, heads, D), dtype=torch.uint8, device=dev)
    scap.scap_kv4_attend(cache, q, out, 0.125, ws, window=window, lse=lse)
    torch.cuda.synchronize()
    scap.scap_device_status()

    class One:  # one head of one sequence, as a cache of its own
        pass
    for b, h in {(0, 0), (B - 1, heads - 1), (B // 2, 3)}:
        c = One()
        c.heads, c.group = 1, 64
        rows = slice(int(at[b]), int(at[b + 1]))
        c.kv = (k[rows, h:h + 1], v[rows, h:h + 1])
        check(c, q[b:b + 1, :, h * g:(h + 1) * g], out[b:b + 1, :, h * g:(h + 1) * g], lse[b:b + 1, :, h * g:(h + 1) * g], lens[b:b + 1], nq, 0.125, window)


@pytest.mark.gpu
def test_offsets_beyond_32_bits():
    import paper_2412_07174_b200 as scap
    n, stride = 40, 1 << 27   # 5.4 GB
    pool = torch.empty(n, stride, dtype=torch.uint8, device="cuda")
    table = torch.tensor([[39, 0, 33], [38, 17, 36]], dtype=torch.int32, device="cuda")
    lens = [90, 70]
    c = Cache(lens, page=32, heads=2, D=128, group=128)
    c.table, c.lens, c.view = table, torch.tensor(lens, dtype=torch.int32, device="cuda"), pool[:, (stride - c.bytes) // 16 * 16:]
    c.cache = scap.ScapKv4(c.view, 32, 2, 128, 128, c.table, c.lens)
    c.kv = (tokens(160, 2, 128, BF, 1).clamp(-99, 99), tokens(160, 2, 128, BF, 2).clamp(-99, 99))
    scap.scap_kv4_append(c.cache, *c.kv, starts(lens))
    q = queries(2, 1, 4, 128, BF)
    out, lse = attend(c, q, 128 ** -0.5)
    check(c, q, out, lse, lens, 1, 128 ** -0.5, 0)


@pytest.mark.gpu
def test_a_wait_that_runs_out_is_reported():
    import paper_2412_07174_b200 as scap
    c = filled([3000], 2, 128, 128)
    q = queries(1, 1, 2, 128, BF)
    ws = torch.empty(scap.scap_kv4_attend_workspace(1, 1, 2, 2, 128), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(q)
    scap.scap_tune("tc_spin", 1)
    try:
        scap.scap_kv4_attend(c.cache, q, out, 0.1, ws)
        try:
            scap.scap_device_status()
        except scap.ScapError as e:
            assert e.code == 7
    finally:
        scap.scap_tune("tc_spin", 0)
    out, lse = attend(c, q, 128 ** -0.5)
    check(c, q, out, lse, [3000], 1, 128 ** -0.5, 0)


def test_refusals():
    from paper_2412_07174_b200 import binding, build
    build.build()
    L = binding.lib()
    P = 0x10000

    def call(q=P, ldq=1024, out=P, ldo=1024, lse=P, nq=2, hq=8, scale=0.1, window=0, dt=1, ws=P, wsb=1 << 30, **kw):
        c = fake_cache(binding, **kw)
        return L.scap_kv4_attend(C.addressof(c), q, ldq, out, ldo, lse, nq, hq, scale, window, dt, ws, wsb, None)
    assert L.scap_kv4_attend(None, P, 1024, P, 1024, P, 2, 8, 0.1, 0, 1, P, 1 << 30, None) == 1
    assert call(q=None) == 1 and call(out=None) == 1 and call(ws=None) == 1
    assert call(scale=float("nan")) == 1 and call(scale=float("inf")) == 1
    assert call(nq=0) == 2 and call(nq=17) == 2 and call(hq=7) == 2 and call(hq=1) == 2 and call(hq=1026, ldq=1 << 20, ldo=1 << 20) == 2
    assert call(window=-1) == 2 and call(ldq=1016) == 2 and call(ldo=1023) == 2 and call(page_tokens=16) == 2
    assert call(dt=2) == 3
    assert call(ldq=1028) == 4 and call(q=P + 2) == 4 and call(out=P + 2) == 4 and call(lse=P + 4) == 4 and call(ws=P + 4) == 4
    n = L.scap_kv4_attend_workspace(2, 2, 8, 2, 128)
    assert n > 0 and call(wsb=n - 1) == 5
    assert L.scap_kv4_attend_workspace(0, 2, 8, 2, 128) == 0 and L.scap_kv4_attend_workspace(2, 2, 8, 3, 128) == 0 and L.scap_kv4_attend_workspace(2, 2, 8, 2, 100) == 0
