"""scap_kv4_attend where rows and tokens differ much in size, and where a sum is long: bounds that follow the products of a row, not its largest value."""
import functools
import math

import pytest
import torch

from kv4_testlib import Cache, starts
from test_gpu_kv4_attend import attend, check, filled, queries, side64

BF, HF = torch.bfloat16, torch.float16


@pytest.mark.gpu
@pytest.mark.parametrize("nq,g,heads,B", [(1, 8, 2, 3), (4, 2, 1, 2), (5, 4, 1, 2), (1, 4, 8, 100)])  # eight rows, eight of several tokens, sixteen, a warp for an item
@pytest.mark.parametrize("size", [2.0 ** 40, 2.0 ** 100, 2.0 ** 127, 2.0 ** -110])
def test_a_row_does_not_depend_on_the_rows_beside_it(nq, g, heads, B, size):
    """One query head of a very different size (finite, as a padded or an outlier one): the others keep their bits, and are right."""
    lens = [150 + b % 40 for b in range(B)]
    c = filled(lens, heads, 64, 64, seed=21)
    q = queries(B, nq, g * heads, 64, BF)
    clean, lse = attend(c, q, 0.125)
    if B < 10:
        check(c, q, clean, lse, lens, nq, 0.125, 0)
    odd = q.clone()
    odd[:, nq // 2, 1] = torch.sign(odd[:, nq // 2, 1]) * size
    out, lse2 = attend(c, odd, 0.125)
    same = torch.ones(B, nq, g * heads, dtype=torch.bool, device="cuda")
    same[:, nq // 2, 1] = False
    assert torch.equal(out[same], clean[same]) and torch.equal(lse2[same], lse[same])


@pytest.mark.gpu
@pytest.mark.parametrize("up", [-95, -20, 60, 120])
def test_queries_of_any_size(up):
    """Queries times 2^up with the scale divided by it: the same bits."""
    lens, D = [200, 31], 64
    c = filled(lens, 1, D, 64, seed=22)
    q = queries(2, 2, 2, D, BF).clamp(-3, 3)
    want, lse = attend(c, q, 0.125)
    check(c, q, want, lse, lens, 2, 0.125, 0)
    big = (q.double() * 2.0 ** up).to(BF)
    assert torch.equal(big.double() * 2.0 ** -up, q.double())
    out, lse2 = attend(c, big, 0.125 * 2.0 ** -up)
    assert torch.equal(out, want) and torch.equal(lse2, lse)


def tight(c, q, out, lse, lens, nq, scale, run=512):
    """Against attention in 64 bits, with a bound made of the products of a weight and a value that a row has.  run: additions into one accumulator."""
    B, _, Hq, D = q.shape
    g = Hq // c.heads
    k64, kmag = side64(c.kv[0], c.group)
    v64, vmag = side64(c.kv[1], c.group)
    at = 0
    for b, n in enumerate(lens):
        for i in range(nq):
            idx = slice(at, at + n - nq + i + 1)
            for h in range(c.heads):
                o, ls = out[b, i, h * g:(h + 1) * g].double(), lse[b, i, h * g:(h + 1) * g].double()
                qq = q[b, i, h * g:(h + 1) * g].double()
                s = scale * qq @ k64[idx, h].T
                want_l = torch.logsumexp(s, -1)
                p = torch.exp(s - want_l[:, None])
                want = p @ v64[idx, h]
                # A score: as in `check`, D / 8 + 16 additions and multiplications in fp32.  s - m is rounded once and below 2^8: 2^-17 of the weight.
                es = scale * 2 * (qq.abs() @ kmag[idx, h].T) * (D / 8 + 16) * 2.0 ** -23 + 2.0 ** -17
                # Of 16 products that it adds at a time the tensor core drops from each what lies below 2^-24 of the largest one's exponent (the largest itself has no
                # such bits).  A code is held as a subnormal number, 2^-8 of what its exponent stands for, so that is 2^-16 of the largest product of a weight and a
                # scale, from codes or from zero points, which are subtracted.
                block = (p[..., None] * vmag[idx, h] / 15).amax(-1)
                block = torch.nn.functional.pad(block, (0, -block.shape[-1] % 16)).unflatten(-1, (-1, 16)).amax(-1)
                others = (len(s[0]) - 16 * torch.arange(block.shape[-1], device="cuda")).clamp(max=16) - 1
                drop = (block * others).sum(-1, keepdim=True) * 2.0 ** -16
                # A weight times the scale of its value is rounded to fp16: 2^-11 of it, or half a step of the subnormal numbers, 2^-25, where the largest
                # product of the row is 2^10 or more, 16 times more in half of the blocks: 2^-31 of the largest (a value is up to 15 scales).
                err = (p * (2.0 ** -11 + 2 * es)) @ v64[idx, h].abs() + (p * 2 * es).sum(-1, keepdim=True) * want.abs()
                err = err + (p[..., None] * vmag[idx, h]).amax((-2, -1))[:, None] * len(s[0]) * 2.0 ** -31
                # code and zero-point parts are added up apart, two additions per tile
                err = err + 2 * (p @ vmag[idx, h]) * min(len(s[0]) / 16 + 2, run) * 2.0 ** -23 + drop
                err = err + want.abs() * torch.finfo(out.dtype).eps / 2 * 1.001 + (2.0 ** -25 if out.dtype is HF else 2.0 ** -134)
                assert bool(((o - want).abs() <= err).all()), (b, i, h, float(((o - want).abs() / err).max()))
                el = es.amax(-1) + 2.0 ** -22 * (want_l.abs() + math.log(n) + 4)
                assert bool(((ls - want_l).abs() <= el).all()), (b, i, h, float(((ls - want_l).abs() / el).max()))
        at += n


def spiked(lens, D, group, where, key, value, dt=BF, seed=31):
    """Tokens of ordinary size, and in every sequence one at `where` (of its length): its key is `key` times the direction of the queries, its values `value`
    times larger."""
    c = Cache(lens, heads=1, D=D, group=group, dt=dt)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda", dtype=torch.float64)  # noqa: E731
    base = rand(D)
    k, v = 0.3 * rand(sum(lens), 1, D), rand(sum(lens), 1, D) + 0.5
    at = 0
    for n in lens:
        t = at + int(where * (n - 1))
        k[t, 0] = key * base
        v[t, 0] *= value
        at += n
    c.kv = (k.to(dt), v.to(dt))
    c.scap.scap_kv4_append(c.cache, *c.kv, starts(lens))
    return c, (base + 0.05 * rand(len(lens), 1, 4, D)).to(dt)


@pytest.mark.gpu
@pytest.mark.parametrize("D,group", [(64, 64), (128, 64), (128, 32), (256, 128)])
@pytest.mark.parametrize("where", [0.0, 0.4, 1.0])
def test_a_large_value_of_next_to_no_weight(D, group, where):
    """A token with a weight of about 2^-60 and values 2^30 times as large as the others' takes no bits from them."""
    lens = [40, 300, 2500]
    c, q = spiked(lens, D, group, where, -42 / D ** 0.5, 2.0 ** 30)
    out, lse = attend(c, q, D ** -0.5)
    tight(c, q, out, lse, lens, 1, D ** -0.5)


@pytest.mark.gpu
@pytest.mark.parametrize("where", [0.0, 0.5])
@pytest.mark.parametrize("value", [0.0, 2.0 ** -20, 2.0 ** -40])
def test_a_token_of_all_the_weight_and_small_values(where, value):
    """An attention sink: nearly all of the weight, values of zero or nearly so.  What the other tokens add is still right."""
    lens = [40, 300, 2500]
    c, q = spiked(lens, 128, 128, where, 25 / 128 ** 0.5, value)
    out, lse = attend(c, q, 128 ** -0.5)
    tight(c, q, out, lse, lens, 1, 128 ** -0.5)


@pytest.mark.gpu
@pytest.mark.parametrize("up", [-70, -40, 40, 100, 123])
def test_values_of_any_size(up):
    lens, D = [200, 1000], 64
    c, q = spiked(lens, D, 32, 0.5, 0.1, 2.0 ** -6)
    c.kv = (c.kv[0], (c.kv[1].double().clamp(-7, 7) * 2.0 ** up).to(BF))
    c.scap.scap_kv4_append(c.cache, *c.kv, starts(lens))
    out, lse = attend(c, q, D ** -0.5)
    tight(c, q, out, lse, lens, 1, D ** -0.5)


@functools.lru_cache(2)
def long_values(n, heads, D, group):
    """Keys and values of one sequence, and what a cache holds of them in 64 bits."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    k, v = (torch.empty(n, heads, D, dtype=HF, device="cuda").normal_(generator=gen) for _ in range(2))
    return k, v, side64(k, group)[0], side64(v, group)[0]


@pytest.mark.gpu
@pytest.mark.parametrize("B,heads,g,nq", [(120, 8, 1, 1), (1, 8, 1, 1), (40, 1, 4, 4), (60, 8, 1, 2)])  # a warp for an item; one item over the device; sixteen rows; a CTA for an item
@pytest.mark.parametrize("scale,hole", [(0.0, 0), (0.125, 0), (0.125, 1800)])
def test_a_long_mean(B, heads, g, nq, scale, hole):
    """Means of up to 400000 values, 1 / 630 of their size, as many as 4000 tiles of them in one warp; where there is a hole the first pages are missing.  The
    sequences share their pages."""
    long_mean(B, heads, g, nq, scale, hole, 64, 64, 400000)


@pytest.mark.gpu
@pytest.mark.parametrize("D,group,B,g,nq,n", [(128, 32, 120, 2, 1, 60000), (256, 64, 80, 1, 2, 40000), (128, 128, 30, 4, 4, 100000), (256, 128, 20, 16, 1, 70000)])
def test_a_long_mean_of_other_shapes(D, group, B, g, nq, n):
    long_mean(B, 8, g, nq, 0.05, 0, D, group, n)


def long_mean(B, heads, g, nq, scale, hole, D, group, n):
    import paper_2412_07174_b200 as scap
    page, dev = 128, "cuda"
    width = -(-n // page)
    gen = torch.Generator(device=dev).manual_seed(6)
    k, v, k64, v64 = long_values(n, heads, D, group)
    pool = torch.zeros(width, scap.scap_kv4_page_bytes(page, heads, D, group), dtype=torch.uint8, device=dev)
    row = torch.randperm(width, generator=gen, device=dev).to(torch.int32)
    lens = torch.full((B,), n, dtype=torch.int32, device=dev)
    one = scap.ScapKv4(pool, page, heads, D, group, row[None].contiguous(), lens[:1])
    scap.scap_kv4_append(one, k, v, torch.tensor([0, n], dtype=torch.int32, device=dev))
    row[:hole] = -1
    cache = scap.ScapKv4(pool, page, heads, D, group, row.expand(B, width).contiguous(), lens)
    q = queries(B, nq, g * heads, D, HF)
    out = torch.empty_like(q)
    lse = torch.empty(B, nq, g * heads, device=dev)
    ws = torch.full((scap.scap_kv4_attend_workspace(B, nq, g * heads, heads, D),), 255, dtype=torch.uint8, device=dev)
    scap.scap_kv4_attend(cache, q, out, scale, ws, lse=lse)
    torch.cuda.synchronize()
    scap.scap_device_status()
    for b in {0, B - 1}:
        for i in range(nq):
            seen = slice(hole * page, n - nq + i + 1)
            s = scale * torch.einsum("hgd,nhd->hgn", q[b, i].view(heads, g, D).double(), k64[seen])
            want_l = torch.logsumexp(s, -1)
            want = torch.einsum("hgn,nhd->hgd", torch.exp(s - want_l[..., None]), v64[seen])
            # The product of a weight with the scale of its value is off by at most 2^-11 of it, differently from token to token: in the mean of independent
            # values 2^-11 of its size at most (as a root of mean squares); the rounding of the result likewise.
            off = (out[b, i].double().view(heads, g, D) - want).square().mean().sqrt() / want.square().mean().sqrt()
            assert float(off) <= 2.0 ** -10, (b, i, float(off))
            # a score is off by at most 2 scale sum |q| |k| (D / 8 + 16) 2^-23 (codes and zero points apart, 15 scales each), a weight by 2^-17
            es = scale * 2 * q[b, i].double().abs().sum(-1).max() * k64.abs().max() * 2 * (D / 8 + 16) * 2.0 ** -23 + 2.0 ** -17
            assert bool(((lse[b, i].double().view(heads, g) - want_l).abs() <= es).all())


@pytest.mark.gpu
@pytest.mark.parametrize("B,heads,n,nq,g", [(1, 32, 215000, 1, 2), (2, 16, 180000, 2, 8), (110, 8, 4200, 1, 2), (2, 2, 9000, 4, 4)])
def test_no_tile_is_lost(B, heads, n, nq, g):
    """The values of every page lie around a mean of its own, the keys too: a tile that is left out, read twice or taken for another shows in the root of mean
    squares of all outputs, whatever the bounds of one of them."""
    import paper_2412_07174_b200 as scap
    D, page, dev = 64, 128, "cuda"
    width = -(-n // page)
    gen = torch.Generator(device=dev).manual_seed(n)
    lens = torch.randint(n - 200, n + 1, (B,), generator=gen, device=dev).to(torch.int32)
    table = torch.randperm(B * width, generator=gen, device=dev).to(torch.int32).view(B, width)
    pool = torch.zeros(B * width, scap.scap_kv4_page_bytes(page, heads, D, 64), dtype=torch.uint8, device=dev)
    cache = scap.ScapKv4(pool, page, heads, D, 64, table, lens)
    at = starts(lens.tolist())
    total = int(at[-1])
    mean = torch.empty(2, total // 32 + 1, heads, D, dtype=BF, device=dev).normal_(generator=gen).repeat_interleave(32, 1)[:, :total]
    k, v = ((m + torch.empty_like(m).normal_(generator=gen)).contiguous() for m in mean)
    scap.scap_kv4_append(cache, k, v, at)
    q = queries(B, nq, g * heads, D, BF)
    out, lse = torch.empty_like(q), torch.empty(B, nq, g * heads, device=dev)
    ws = torch.empty(scap.scap_kv4_attend_workspace(B, nq, g * heads, heads, D), dtype=torch.uint8, device=dev)
    scap.scap_kv4_attend(cache, q, out, 0.125, ws, lse=lse)
    torch.cuda.synchronize()
    scap.scap_device_status()
    for b in {0, B // 2, B - 1}:
        rows, some = slice(int(at[b]), int(at[b + 1])), sorted({0, heads // 2, heads - 1})
        k64, v64 = side64(k[rows][:, some], 64)[0], side64(v[rows][:, some], 64)[0]
        for i in range(nq):
            m = len(k64) - nq + i + 1
            p = torch.softmax(0.125 * torch.einsum("hgd,nhd->hgn", q[b, i].view(heads, g, D)[some].double(), k64[:m]), -1)
            want = torch.einsum("hgn,nhd->hgd", p, v64[:m])
            off = (out[b, i].view(heads, g, D)[some].double() - want).square().mean().sqrt() / want.square().mean().sqrt()
            # The rounding of a weight times its scale (2^-11 of it) and of the result (2^-8): 2^-7 of the outputs together.  One tile of 6700, with a 6700th of the weight,
            # holds a value 1 / 82 of the outputs' size or more: of the tiles of a warp beyond the first 32 there are a tenth.
            assert float(off) <= 2.0 ** -7, (b, i, float(off))


@pytest.mark.gpu
@pytest.mark.parametrize("lens,heads,nq", [([200000], 8, 1), ([20000] * 20, 8, 1), ([2000] * 200, 8, 1)])
def test_waits_that_run_out_are_reported(lens, heads, nq):
    """One try of 4 us at most per wait, beside first copies that take longer (three tiles of 4352 bytes for each of 2368 warps, 31 MB: 4.7 us at the rate of the
    memory): scap_device_status says so."""
    import paper_2412_07174_b200 as scap
    c = filled(lens, heads, 128, 128, seed=1)
    q = queries(len(lens), nq, heads, 128, BF)
    out = torch.empty_like(q)
    ws = torch.empty(scap.scap_kv4_attend_workspace(len(lens), nq, heads, heads, 128), dtype=torch.uint8, device="cuda")
    scap.scap_kv4_attend(c.cache, q, out, 0.1, ws)
    want = out.clone()
    flush = torch.zeros(1 << 28, dtype=torch.uint8, device="cuda")  # nothing of the cache in L2
    torch.cuda.synchronize()
    scap.scap_device_status()
    scap.scap_tune("tc_spin", 1)
    try:
        scap.scap_kv4_attend(c.cache, q, out, 0.1, ws)
        with pytest.raises(scap.ScapError) as e:
            scap.scap_device_status()
        assert e.value.code == 7
    finally:
        scap.scap_tune("tc_spin", 0)
    scap.scap_kv4_attend(c.cache, q, out, 0.1, ws)
    scap.scap_device_status()  # and is done with it
    assert torch.equal(out, want) and flush is not None


@pytest.mark.gpu
@pytest.mark.parametrize("every", [700, 20])  # in one tile, in all of them
def test_a_group_that_is_not_finite_stays_in_its_channels(every):
    """Values of one group of channels that are NaN make those channels NaN; the other groups of the same tokens count, in size too."""
    lens, D, group = [40, 300, 2500], 128, 32
    c, q = spiked(lens, D, group, 0.5, 0.2, 2.0 ** 12)
    k, v = c.kv
    v[7::every, 0, 40] = float("nan")
    c.scap.scap_kv4_append(c.cache, k, v, starts(lens))
    out, lse = attend(c, q, D ** -0.5)
    assert bool(out[..., 32:64].isnan().all()) if every == 20 else bool(out[0, ..., 32:64].isnan().all())
    v[7::every, 0, 32:64] = 0.0
    c.scap.scap_kv4_append(c.cache, k, v, starts(lens))
    zero, lse0 = attend(c, q, D ** -0.5)
    tight(c, q, zero, lse0, lens, 1, D ** -0.5)
    assert bool(torch.isfinite(out[..., :32]).all()) and bool(torch.isfinite(out[..., 64:]).all())
    tight(c, q, torch.cat((out[..., :32], zero[..., 32:64], out[..., 64:]), -1), lse, lens, 1, D ** -0.5)


@pytest.mark.gpu
@pytest.mark.parametrize("D,group", [(64, 32), (64, 64), (128, 128), (256, 64)])
@pytest.mark.parametrize("where", [0, 5, 7])
def test_small_values_beside_a_large_one(D, group, where):
    """A token with nine tenths of the weight and a large scale, whose value is zero in most channels: what the tokens that are added with it have there."""
    lens = [8, 18, 33, 64]
    c = Cache(lens, heads=1, D=D, group=group, dt=HF)
    gen = torch.Generator(device="cuda").manual_seed(D + where)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda", dtype=torch.float64)  # noqa: E731
    base = rand(D)
    k = 0.1 * rand(sum(lens), 1, D)
    v = (1 + 0.3 * torch.rand(sum(lens), 1, 1, generator=gen, device="cuda", dtype=torch.float64)) * torch.where(torch.arange(D, device="cuda") % 2 == 0, -1.0, 1.0)
    at = 0
    for n in lens:
        k[at + where, 0] = base * (math.log(9 * n) / float(base @ base) * D ** 0.5)
        v[at + where] = 0.0
        v[at + where, 0, ::group], v[at + where, 0, 1::group] = 320.0, -280.0
        at += n
    c.kv = (k.to(HF), v.to(HF))
    c.scap.scap_kv4_append(c.cache, *c.kv, starts(lens))
    q = (base + 0.02 * rand(len(lens), 1, 4, D)).to(HF)
    out, lse = attend(c, q, D ** -0.5)
    tight(c, q, out, lse, lens, 1, D ** -0.5)
