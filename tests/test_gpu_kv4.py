"""scap_kv4_append and scap_kv4_read: what the cache holds is what its format says, exactly."""
import ctypes as C

import numpy as np
import pytest
import torch

from kv4_testlib import Cache, stored64, starts, tokens

BF, HF = torch.bfloat16, torch.float16
SHAPES = [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128), (256, 64), (256, 128)]


def read_back(c, rows, counts):
    ko = torch.full((rows, c.heads, c.D), 99.0, dtype=c.dt, device="cuda")
    vo = torch.full_like(ko, 99.0)
    c.scap.scap_kv4_read(c.cache, ko, vo, starts(counts))
    torch.cuda.synchronize()
    return ko, vo


def same(got, want64):
    """Bit for bit: the value is exact in binary32, its rounding to the type of the tensor is the only one."""
    want = torch.tensor(want64, device="cuda").float().to(got.dtype)
    return torch.equal(torch.nan_to_num(got.float(), nan=12345.0), torch.nan_to_num(want.float(), nan=12345.0))


@pytest.mark.gpu
@pytest.mark.parametrize("D,group", SHAPES)
@pytest.mark.parametrize("dt", [BF, HF])
def test_prompt_then_single_tokens(D, group, dt):
    lens = [1, 31, 32, 33, 97, 0, 64]
    c = Cache(lens, page=32, heads=3, D=D, group=group, dt=dt, room=130, seed=D + group)
    k, v = tokens(sum(lens), 3, D, dt, 1), tokens(sum(lens), 3, D, dt, 2)
    c.scap.scap_kv4_append(c.cache, k, v, starts(lens))
    ko, vo = read_back(c, sum(lens), lens)
    assert same(ko, stored64(k, group)) and same(vo, stored64(v, group)) and c.guards_intact()
    all_k, all_v = [k[a:b] for a, b in zip(starts(lens)[:-1].tolist(), starts(lens)[1:].tolist())], None
    all_v = [v[a:b] for a, b in zip(starts(lens)[:-1].tolist(), starts(lens)[1:].tolist())]
    for step in range(3):  # single tokens, one for each sequence
        c.lens += 1
        kn, vn = tokens(len(lens), 3, D, dt, 10 + step), tokens(len(lens), 3, D, dt, 20 + step)
        c.scap.scap_kv4_append(c.cache, kn, vn)
        all_k = [torch.cat((a, kn[b:b + 1])) for b, a in enumerate(all_k)]
        all_v = [torch.cat((a, vn[b:b + 1])) for b, a in enumerate(all_v)]
    n = [len(a) for a in all_k]
    ko, vo = read_back(c, sum(n), n)
    assert same(ko, stored64(torch.cat(all_k), group)) and same(vo, stored64(torch.cat(all_v), group)) and c.guards_intact()


@pytest.mark.gpu
def test_random_lengths_and_rows_left_alone():
    rng = np.random.default_rng(5)
    for trial in range(4):
        B = int(rng.integers(1, 70))
        past, new = rng.integers(0, 200, B), rng.integers(0, 120, B)
        new[rng.random(B) < 0.3] = 0
        lens = (past + new).tolist()
        c = Cache(lens, page=64, heads=2, D=128, group=64, seed=trial)
        first, tail = int(rng.integers(0, 5)), int(rng.integers(0, 5))  # rows before the first sequence and behind the last
        st = starts(new) + first
        rows = int(new.sum()) + first + tail
        if rows == 0:
            continue
        k, v = tokens(rows, 2, 128, BF, trial), tokens(rows, 2, 128, BF, trial + 50)
        c.scap.scap_kv4_append(c.cache, k, v, st)
        ko, vo = torch.full_like(k, 99.0), torch.full_like(v, 99.0)
        c.scap.scap_kv4_read(c.cache, ko, vo, st)
        torch.cuda.synchronize()
        n = rows - first - tail
        assert same(ko[first:first + n], stored64(k[first:first + n], 64)) and same(vo[first:first + n], stored64(v[first:first + n], 64))
        for t in (ko, vo):
            assert bool((t[:first] == 99.0).all()) and bool((t[first + n:] == 99.0).all())
        assert c.guards_intact()


@pytest.mark.gpu
@pytest.mark.parametrize("B,page", [(33, 4096), (1000, 32), (4096, 32)])
def test_many_sequences(B, page):
    rng = np.random.default_rng(B)
    new = rng.integers(0, 4, B)
    new[rng.random(B) < 0.5] = 0
    new[:3], new[-3:] = 0, 0     # empty ones at both ends
    past = rng.integers(0, 30, B)
    c = Cache((past + new).tolist(), page=page, heads=1, D=64, group=64, seed=B, room=40)
    n = int(new.sum())
    k, v = tokens(n, 1, 64, BF, 1), tokens(n, 1, 64, BF, 2)
    c.scap.scap_kv4_append(c.cache, k, v, starts(new))
    ko, vo = read_back(c, n, new)
    assert same(ko, stored64(k, 64)) and same(vo, stored64(v, 64)) and c.guards_intact()


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF, HF])
def test_values_at_the_borders(dt):
    D, group = 128, 64
    rows = [torch.zeros(D), torch.full((D,), 3.0), torch.full((D,), -3.0)]
    r = torch.arange(D).float()
    rows.append((r % 16) - 7.5)                       # ties of x / s: s = 1 exactly
    rows.append(((r % 31) - 15) * 0.5)                # many exact halves
    rows.append((r % 2) * 2.0 ** -24)                 # subnormal fp16; tiny bf16
    rows.append(torch.where(r == 5, float("nan"), r))
    rows.append(torch.where(r == 70, float("inf"), -r))
    rows.append(torch.where(r == 70, -float("inf"), -r))
    rows.append(torch.full((D,), 65504.0) * torch.where(r % 2 == 0, 1.0, -1.0))
    if dt is BF:
        rows.append((r - 64) * 2.0 ** 120)            # beyond half precision, difference beyond single
        rows.append((r - 64) * 2.0 ** -140)           # scales in the subnormal numbers
        rows.append((r % 3) * 2.0 ** -133)
        rows.append(torch.where(r % 2 == 0, 3.38e38, -3.38e38))
    x = torch.stack(rows).to(dt).cuda()[:, None, :]
    n = len(rows)
    c = Cache([n], page=32, heads=1, D=D, group=group, dt=dt)
    c.scap.scap_kv4_append(c.cache, x, x, starts([n]))
    ko, vo = read_back(c, n, [n])
    want = stored64(x, group)
    assert same(ko, want) and same(vo, want)


@pytest.mark.gpu
def test_error_is_at_most_half_a_step_and_a_bit():
    x = tokens(500, 2, 128, HF, 3)
    c = Cache([500], heads=2, dt=HF)
    c.scap.scap_kv4_append(c.cache, x, x, starts([500]))
    ko, _ = read_back(c, 500, [500])
    g = x.double().unflatten(-1, (-1, 64))
    step = (g.amax(-1).clamp(min=0) - g.amin(-1).clamp(max=0)) / 15
    err = (ko.double() - x.double()).abs().unflatten(-1, (-1, 64))
    # s is off by at most 2^-20 of the step.  Not clipped: |x - s (q - zero)| <= s / 2.  Clipped at 15: round(x / s) + zero = 16 while
    # (hi - lo) / s <= 15 (1 + 2^-20) and zero <= -lo / s + 1/2, so x / s - (15 - zero) <= 1/2 + 15 2^-20; at 0 likewise.
    # The value read is rounded to fp16: 2^-11 of it, and it is at most |x| + s (so not of |x| alone: half a step beside a small x is larger
    # than x), or half of the least subnormal.
    bound = step[..., None] * (0.5 + 16 * 2.0 ** -20) + (g.abs() + step[..., None]) * 2.0 ** -11 + 2.0 ** -25
    finite = torch.isfinite(g).all(-1, keepdim=True).expand_as(g)  # (the largest tokens overflow fp16: such groups read as NaN)
    assert bool((err <= bound)[finite].all()) and bool(torch.isnan(err[~finite]).all()) and bool(finite.any())


@pytest.mark.gpu
def test_slices_of_a_fused_projection_and_layers_of_a_page():
    lens, heads, D = [70, 5], 2, 64
    n = sum(lens)
    c0 = Cache(lens, heads=heads, D=D, group=64, layers=3, layer=1)
    qkv = torch.randn(n, 10, D, device="cuda").to(BF)
    k, v = qkv[:, 6:8], qkv[:, 8:10]
    c0.scap.scap_kv4_append(c0.cache, k, v, starts(lens))
    wide = torch.full((n, 10, D), 99.0, dtype=BF, device="cuda")
    c0.scap.scap_kv4_read(c0.cache, wide[:, 2:4], wide[:, 4:6], starts(lens))
    torch.cuda.synchronize()
    assert same(wide[:, 2:4], stored64(k, 64)) and same(wide[:, 4:6], stored64(v, 64))
    assert bool((wide[:, :2] == 99.0).all()) and bool((wide[:, 6:] == 99.0).all())
    other = c0.pool.view(len(c0.pool), 3, -1)
    assert bool((other[:, 0] == 0xA5).all()) and bool((other[:, 2] == 0xA5).all()) and c0.guards_intact()


@pytest.mark.gpu
def test_pages_that_are_not_there_are_skipped():
    lens = [100, 40]
    c = Cache(lens, page=32, heads=1, D=128, group=128)
    c.table[0, 1] = -1
    c.table[1, 0] = 10 ** 6
    before = c.pool.clone()
    k = tokens(140, 1, 128, BF, 1)
    c.scap.scap_kv4_append(c.cache, k, k, starts(lens))
    ko, vo = read_back(c, 140, lens)
    want = stored64(k, 128)
    for rows, there in ((slice(0, 32), True), (slice(32, 64), False), (slice(64, 100), True), (slice(100, 132), False), (slice(132, 140), True)):
        if there:
            assert same(ko[rows], want[rows]) and same(vo[rows], want[rows])
        else:
            assert bool((ko[rows] == 99.0).all()) and bool((vo[rows] == 99.0).all())
    used = set(c.table[0, [0, 2, 3]].tolist()) | set(c.table[1, 1:2].tolist())
    for p in range(len(c.pool)):
        if p not in used:
            assert torch.equal(c.pool[p], before[p])
    # more rows than a sequence has tokens, and more tokens than its table has room for
    c.lens.copy_(torch.tensor([3, 10 ** 5], dtype=torch.int32))
    c.scap.scap_kv4_append(c.cache, k, k, starts(lens))
    torch.cuda.synchronize()
    assert c.guards_intact()


@pytest.mark.gpu
def test_graph_stream_and_other_rows_of_a_word():
    lens = [40, 40]
    c = Cache(lens, heads=2)
    k = tokens(80, 2, 128, BF, 1)
    c.scap.scap_kv4_append(c.cache, k, k, starts(lens))
    kn = tokens(2, 2, 128, BF, 2)
    graph = torch.cuda.CUDAGraph()
    c.scap.scap_kv4_append(c.cache, kn, kn)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        c.lens += 1
        c.scap.scap_kv4_append(c.cache, kn, kn)
    seqs = [[k[:40]], [k[40:]]]
    seqs[0][0][39:40] = kn[0:1]
    seqs[1][0][39:40] = kn[1:2]
    for step in range(5):
        kn.copy_(tokens(2, 2, 128, BF, 30 + step))
        graph.replay()
        for b in range(2):
            seqs[b].append(kn[b:b + 1].clone())
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    ko, vo = torch.empty(90, 2, 128, dtype=BF, device="cuda"), torch.empty(90, 2, 128, dtype=BF, device="cuda")
    st = starts([45, 45])
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        c.scap.scap_kv4_read(c.cache, ko, vo, st)
    s.synchronize()
    want = stored64(torch.cat(seqs[0] + seqs[1]), 64)
    assert same(ko, want) and same(vo, want)


def fake_cache(binding, **kw):
    c = binding.ScapKv4.__new__(binding.ScapKv4)
    base = dict(pages=0x10000, page_stride=1 << 20, n_pages=8, page_tokens=64, heads=2, head_dim=128, group=64, table_stride=4, n_seqs=2, table=0x20000, lens=0x30000, refs=0x40000)
    base.update(kw)
    for n, v in base.items():
        setattr(c, n, v)
    return c


def test_refusals():
    from paper_2412_07174_b200 import binding, build
    build.build()
    L = binding.lib()
    P = 0x10000

    def call(f=L.scap_kv4_append, cache=None, k=P, ldk=256, v=P, ldv=256, start=P, rows=4, dt=1, **kw):
        c = cache or fake_cache(binding, **kw)
        return f(C.addressof(c), k, ldk, v, ldv, start, rows, dt, None)
    for f in (L.scap_kv4_append, L.scap_kv4_read):
        assert f(None, P, 256, P, 256, P, 4, 1, None) == 1
        assert call(f, pages=None) == 1 and call(f, table=None) == 1 and call(f, lens=None) == 1 and call(f, k=None) == 1 and call(f, v=None) == 1
        assert call(f, n_pages=0) == 2 and call(f, page_tokens=48) == 2 and call(f, page_tokens=0) == 2 and call(f, heads=0) == 2
        assert call(f, head_dim=96) == 2 and call(f, group=16) == 2 and call(f, group=256) == 2 and call(f, head_dim=256, group=32, ldk=512, ldv=512) == 2
        assert call(f, table_stride=0) == 2 and call(f, n_seqs=0) == 2 and call(f, n_seqs=4097) == 2 and call(f, page_stride=1024) == 2
        assert call(f, rows=-1) == 2 and call(f, rows=(1 << 20) + 1) == 2 and call(f, start=None, rows=3) == 2
        assert call(f, ldk=255) == 2 and call(f, ldv=248) == 2
        assert call(f, dt=2) == 3
        assert call(f, k=P + 2) == 4 and call(f, ldk=257) == 4 and call(f, pages=P + 8) == 4 and call(f, page_stride=(1 << 20) + 8) == 4
        assert call(f, table=P + 4) == 4 and call(f, lens=P + 4) == 4 and call(f, start=P + 2) == 4
        assert call(f, rows=0) == 0
    assert L.scap_kv4_page_bytes(64, 8, 128, 64) == 8 * 2 * (32 * 128 + 2 * 2 * 128)
    assert L.scap_kv4_page_bytes(63, 8, 128, 64) == 0 and L.scap_kv4_page_bytes(64, 8, 100, 64) == 0


# Many rows times heads take the form with eight channels of a lane, from 16 rows and heads per multiprocessor on (2368 on 148 of them).
@pytest.mark.gpu
@pytest.mark.parametrize("D,group", SHAPES)
@pytest.mark.parametrize("dt", [BF, HF])
def test_long_prompts_in_pieces(D, group, dt):
    pieces = [[45, 0, 3, 77, 31], [50, 33, 1, 90, 60], [7, 64, 32, 0, 29]]
    heads = 24
    total = np.sum(pieces, 0).tolist()
    c = Cache(total, page=64, heads=heads, D=D, group=group, dt=dt, seed=D + group)
    c.lens.zero_()
    k = [[] for _ in total]
    v = [[] for _ in total]
    for i, counts in enumerate(pieces):
        n = sum(counts)
        assert n * heads >= 2368
        kn, vn = tokens(n, heads, D, dt, 3 * i), tokens(n, heads, D, dt, 3 * i + 1)
        c.lens += torch.tensor(counts, dtype=torch.int32, device="cuda")
        c.scap.scap_kv4_append(c.cache, kn, vn, starts(counts))
        at = np.concatenate(([0], np.cumsum(counts)))
        for b in range(len(total)):
            k[b].append(kn[at[b]:at[b + 1]])
            v[b].append(vn[at[b]:at[b + 1]])
    ko, vo = read_back(c, sum(total), total)
    want = [torch.cat([torch.cat(x) for x in y]) for y in (k, v)]
    assert same(ko, stored64(want[0], group)) and same(vo, stored64(want[1], group)) and c.guards_intact()


@pytest.mark.gpu
@pytest.mark.parametrize("D,group", SHAPES)
@pytest.mark.parametrize("dt", [BF, HF])
def test_values_at_the_borders_of_many_heads(D, group, dt):
    heads, r = 300, torch.arange(D).float()
    rows = [torch.zeros(D), torch.full((D,), -3.0), (r % 16) - 7.5, ((r % 31) - 15) * 0.5, (r % 2) * 2.0 ** -24, torch.where(r == 5, float("nan"), r),
            torch.where(r == D - 2, float("inf"), -r), torch.where(r == D - 2, -float("inf"), r), torch.where(r % 2 == 0, 65504.0, -65504.0), (r % 16) * 0.1, -(r % 16) / 3]
    if dt is BF:
        rows += [(r - D / 2) * 2.0 ** 118, (r - 64) * 2.0 ** -140, (r % 3) * 2.0 ** -133, torch.where(r % 2 == 0, 3.38e38, -3.38e38), (r % 15) * 2.0 ** -101, (r % 15 - 7) * 2.0 ** -99]
    x = torch.stack(rows)[:, None, :].expand(-1, heads, -1).to(dt).to("cuda")
    k, v = x.contiguous(), x.flip(0).contiguous()
    n = x.shape[0]
    assert n * heads >= 2368
    c = Cache([n], page=32, heads=heads, D=D, group=group, dt=dt)
    c.scap.scap_kv4_append(c.cache, k, v, starts([n]))
    ko, vo = read_back(c, n, [n])
    assert same(ko, stored64(k, group)) and same(vo, stored64(v, group)) and c.guards_intact()
