"""The calls on pages of the 4-bit cache against a plain restatement of what they do, in Python integers."""
import ctypes as C

import numpy as np
import pytest
import torch

from test_gpu_kv4 import fake_cache


class Plain:
    """Table, lengths, counts and pages as lists and arrays."""

    def __init__(self, table, lens, refs, pool, page):
        self.table, self.lens, self.refs, self.pool, self.page = table.copy(), lens.copy(), refs.copy(), pool.copy(), page

    def free_list(self):
        return [p for p in range(len(self.refs)) if self.refs[p] == 0]

    def fork(self, src, dst):
        S, width = self.table.shape
        free, failed, named = self.free_list(), 0, set()
        dests = {int(d) for d in dst if 0 <= d < S}
        copies = []
        for a, b in zip(src, dst):
            first = b not in named
            named.add(b)
            if not (0 <= a < S and 0 <= b < S) or not first or a in dests or self.lens[b] > 0 or self.lens[a] > width * self.page:
                failed += 1
                continue
            full, part = divmod(int(self.lens[a]), self.page)
            if part and not free:
                failed += 1
                continue
            row = [-1] * width
            row[:full] = self.table[a, :full]
            for p in row[:full]:
                self.refs[p] += 1
            if part:
                p = free.pop(0)
                copies.append((self.table[a, full], p))
                self.refs[p] = 1
                row[full] = p
            self.table[b], self.lens[b] = row, self.lens[a]
        for a, p in copies:
            self.pool[p] = self.pool[a]
        return failed

    def free(self, rows):
        for b in rows:
            if 0 <= b < len(self.lens) and self.lens[b] > 0:
                for p in self.table[b, :-(-int(self.lens[b]) // self.page)]:
                    self.refs[p] -= 1
                self.table[b], self.lens[b] = -1, 0

    def reserve(self, add):
        free, taken, failed = self.free_list(), 0, 0
        start = len(free)
        for b, n in enumerate(add):
            n = max(0, int(n))
            have, need = -(-int(self.lens[b]) // self.page), -(-(int(self.lens[b]) + n) // self.page)
            if need > self.table.shape[1]:
                failed += 1
                continue
            more = need - have
            taken += more
            if more and taken > start:
                failed += 1
                continue
            for k in range(more):
                p = free[taken - more + k]
                self.table[b, have + k], self.refs[p] = p, 1
            self.lens[b] += n
        return failed

    def compact(self):
        used = int((self.refs > 0).sum())
        holes = [p for p in range(used) if self.refs[p] == 0]
        movers = [p for p in range(used, len(self.refs)) if self.refs[p] > 0]
        place = dict(zip(movers, holes))
        for a, b in place.items():
            self.pool[b] = self.pool[a]
            self.refs[b], self.refs[a] = self.refs[a], 0
        self.table = np.vectorize(lambda p: place.get(int(p), p))(self.table).astype(np.int32)
        return used


class Pool:
    def __init__(self, S, width, pages, page=32, stride=4112, seed=0, fill=0.6, shared=True):
        import paper_2412_07174_b200 as scap
        self.scap, self.page = scap, page
        rng = np.random.default_rng(seed)
        ids = rng.permutation(pages).tolist()
        table, lens, refs = np.full((S, width), -1, np.int32), np.zeros(S, np.int32), np.zeros(pages, np.int32)
        for b in range(S):
            if rng.random() > fill:
                continue
            n = int(rng.integers(1, width * page + 1))
            need = -(-n // page)
            share = 0
            if shared and b and rng.random() < 0.4 and lens[b - 1] > 0:
                share = min(n, int(lens[b - 1])) // page
            if len(ids) < need - share:
                continue
            table[b, :share] = table[b - 1, :share]
            table[b, share:need] = [ids.pop() for _ in range(need - share)]
            refs[table[b, :need]] += 1
            lens[b] = n
        pool = rng.integers(0, 256, (pages, stride), dtype=np.uint8)
        self.plain = Plain(table, lens, refs, pool, page)
        self.raw = torch.full((pages + 2, stride), 0x5A, dtype=torch.uint8, device="cuda")
        self.raw[1:-1] = torch.from_numpy(pool).cuda()
        self.table, self.lens, self.refs = (torch.from_numpy(x.copy()).cuda() for x in (table, lens, refs))
        self.cache = scap.ScapKv4(self.raw[1:-1], page, 0, 0, 0, self.table, self.lens, refs=self.refs)
        self.ws = torch.full((scap.scap_kv4_pages_workspace(pages, S),), 0xEE, dtype=torch.uint8, device="cuda")
        self.out = torch.full((1,), -7, dtype=torch.int32, device="cuda")

    def same(self):
        torch.cuda.synchronize()
        p = self.plain
        assert np.array_equal(self.table.cpu().numpy(), p.table)
        assert np.array_equal(self.lens.cpu().numpy(), p.lens)
        assert np.array_equal(self.refs.cpu().numpy(), p.refs)
        assert np.array_equal(self.raw[1:-1].cpu().numpy(), p.pool)
        assert bool((self.raw[0] == 0x5A).all()) and bool((self.raw[-1] == 0x5A).all())
        # the state is consistent
        count = np.zeros(len(p.refs), np.int64)
        for b in range(len(p.lens)):
            held = p.table[b, :-(-int(p.lens[b]) // self.page)]
            np.add.at(count, held, 1)
        assert np.array_equal(count, p.refs)


def i32(x):
    return torch.tensor(list(x), dtype=torch.int32, device="cuda")


def fork(p, src, dst):
    p.scap.scap_kv4_fork(p.cache, i32(src), i32(dst), p.out, p.ws)
    assert int(p.out.item()) == p.plain.fork(src, dst)
    p.same()


@pytest.mark.gpu
@pytest.mark.parametrize("S,width,pages,stride", [(1, 1, 2, 16), (5, 3, 16, 4112), (40, 6, 300, 4112), (200, 4, 900, 48), (2500, 3, 8000, 16), (12, 3, 60, 100000)])
def test_random_steps(S, width, pages, stride):
    rng = np.random.default_rng(S)
    p = Pool(S, width, pages, stride=stride, seed=S)
    p.same()
    for step in range(6):
        empty, held = np.flatnonzero(p.plain.lens == 0), np.flatnonzero(p.plain.lens > 0)
        if len(empty) and len(held):
            n = int(rng.integers(1, len(empty) + 1))
            fork(p, rng.choice(held, n).tolist(), rng.permutation(empty)[:n].tolist())
        rows = rng.integers(-2, S + 2, max(1, S // 4)).tolist()
        p.scap.scap_kv4_free(p.cache, i32(rows))
        p.plain.free(rows)
        p.same()
        add = rng.integers(0, 40, S) * (rng.random(S) < 0.7)
        p.scap.scap_kv4_reserve(p.cache, i32(add), p.out, p.ws)
        assert int(p.out.item()) == p.plain.reserve(add)
        p.same()
        if step % 2:
            p.scap.scap_kv4_compact(p.cache, p.out, p.ws)
            assert int(p.out.item()) == p.plain.compact()
            p.same()


@pytest.mark.gpu
def test_requests_that_are_left_out():
    p = Pool(8, 3, 40, fill=1.0, shared=False, seed=3)
    p.scap.scap_kv4_free(p.cache, i32([4, 5, 6, 7, 4, 4]))   # the same row three times
    p.plain.free([4, 5, 6, 7])
    p.same()
    # named twice; not empty; out of range; a source that is a destination; itself
    fork(p, [0, 1, 2, 9, 0, 5, 3, 6], [4, 4, 1, 5, -1, 6, 8, 6])
    fork(p, [0, 0, 0], [5, 6, 7])


@pytest.mark.gpu
def test_no_pages_left():
    p = Pool(20, 4, 24, fill=0.5, seed=11)
    held, empty = np.flatnonzero(p.plain.lens > 0), np.flatnonzero(p.plain.lens == 0)
    fork(p, [int(held[i % len(held)]) for i in range(len(empty))], empty.tolist())
    add = np.full(20, 50)
    p.scap.scap_kv4_reserve(p.cache, i32(add), p.out, p.ws)
    assert int(p.out.item()) == p.plain.reserve(add) > 0
    p.same()
    add[:] = 2 ** 31 - 1
    add[3] = -5
    add[4] = 0
    p.scap.scap_kv4_reserve(p.cache, i32(add), None, p.ws)
    p.plain.reserve(add)
    p.same()


@pytest.mark.gpu
def test_empty_full_and_compacted_pools():
    p = Pool(4, 2, 50, fill=0.0)
    for _ in range(2):
        p.scap.scap_kv4_compact(p.cache, p.out, p.ws)
        assert int(p.out.item()) == p.plain.compact() == 0
        p.same()
    p = Pool(4, 4, 16, fill=1.0, shared=False, seed=2)
    p.scap.scap_kv4_compact(p.cache, None, p.ws)
    p.plain.compact()
    p.same()
    p.scap.scap_kv4_compact(p.cache, p.out, p.ws)
    p.same()


@pytest.mark.gpu
def test_copy_and_large_pages():
    import paper_2412_07174_b200 as scap
    pool = torch.randint(0, 256, (40, 70000), device="cuda", dtype=torch.uint8)
    want = pool.clone()
    src, dst = [0, 5, 5, 39, -1, 3, 40], [20, 21, 22, 23, 24, 99, 25]
    cache = scap.ScapKv4(pool, 32, 0, 0, 0, i32([0])[None], i32([0]))
    scap.scap_kv4_copy(cache, i32(src), i32(dst))
    for a, b in zip(src, dst):
        if 0 <= a < 40 and 0 <= b < 40:
            want[b] = want[a]
    torch.cuda.synchronize()
    assert torch.equal(pool, want)
    # pages beyond 4 GB, of several layers
    big = torch.empty(34, 1 << 27, dtype=torch.uint8, device="cuda")
    big[33].random_(0, 256)
    big[1].zero_()
    cache = scap.ScapKv4(big, 32, 0, 0, 0, i32([0])[None], i32([0]))
    scap.scap_kv4_copy(cache, i32([33]), i32([1]))
    assert torch.equal(big[1], big[33])


@pytest.mark.gpu
def test_many_pages():
    """Counts over several rounds of the plan's CTA, the last round partly filled."""
    p = Pool(300, 5, 40011, stride=16, fill=0.9, seed=8)
    p.scap.scap_kv4_free(p.cache, i32(range(0, 300, 2)))
    p.plain.free(range(0, 300, 2))
    p.same()
    fork(p, [1 + 2 * (i % 140) for i in range(150)], list(range(0, 300, 2)))
    p.scap.scap_kv4_compact(p.cache, p.out, p.ws)
    assert int(p.out.item()) == p.plain.compact()
    p.same()


@pytest.mark.gpu
def test_a_step_in_a_graph_on_another_stream():
    p = Pool(12, 4, 80, fill=0.5, seed=5)
    held, empty = np.flatnonzero(p.plain.lens > 0).tolist(), np.flatnonzero(p.plain.lens == 0).tolist()
    src, dst, rows, add = i32([held[0]] * len(empty)), i32(empty), i32(held[:1]), i32([1] * 12)
    saved = [t.clone() for t in (p.table, p.lens, p.refs, p.raw)]

    def step():
        p.scap.scap_kv4_fork(p.cache, src, dst, p.out, p.ws)
        p.scap.scap_kv4_free(p.cache, rows)
        p.scap.scap_kv4_reserve(p.cache, add, None, p.ws)
        p.scap.scap_kv4_compact(p.cache, None, p.ws)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    s.synchronize()
    p.plain.fork([held[0]] * len(empty), empty)
    p.plain.free(held[:1])
    p.plain.reserve([1] * 12)
    p.plain.compact()
    p.same()
    for t, v in zip((p.table, p.lens, p.refs, p.raw), saved):
        t.copy_(v)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    graph.replay()
    p.same()


@pytest.mark.gpu
def test_a_decoding_run():
    """Prompts through the FC, into the cache, forked into beams, decoded by single tokens with the pages moved meanwhile."""
    import paper_2412_07174_b200 as scap
    from kv4_testlib import stored64
    torch.manual_seed(0)
    B, heads, g, D, K, page, S = 3, 2, 2, 64, 256, 32, 8
    width = (g + 2) * heads * D
    W = (0.06 * torch.randn(K, width, device="cuda")).bfloat16()
    Wo = (0.06 * torch.randn(g * heads * D, K, device="cuda")).bfloat16()
    n = scap.scap_kv4_page_bytes(page, heads, D, 32)
    pool = torch.zeros(60, n, dtype=torch.uint8, device="cuda")
    table, lens, refs = torch.full((S, 5), -1, dtype=torch.int32, device="cuda"), torch.zeros(S, dtype=torch.int32, device="cuda"), torch.zeros(60, dtype=torch.int32, device="cuda")
    cache = scap.ScapKv4(pool, page, heads, D, 32, table, lens, refs=refs)
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    fail = torch.zeros(1, dtype=torch.int32, device="cuda")
    prompt = [40, 7, 65]
    x = torch.randn(sum(prompt), K, device="cuda").bfloat16()
    qkv = torch.empty(sum(prompt), width, dtype=torch.bfloat16, device="cuda")
    scap.scap_fc_act(x, W, None, qkv, ws)
    assert torch.allclose(qkv.float(), x.float() @ W.float(), atol=0.05, rtol=0.02)
    heads_of = lambda t: t.view(len(t), -1, D)  # noqa: E731
    add = i32(prompt + [0] * (S - B))
    scap.scap_kv4_reserve(cache, add, fail, ws)
    st = i32([0] + np.cumsum(prompt).tolist() + [sum(prompt)] * (S - B))
    k, v = heads_of(qkv)[:, g * heads:(g + 1) * heads], heads_of(qkv)[:, (g + 1) * heads:]
    scap.scap_kv4_append(cache, k, v, st)
    past = {b: (k[sum(prompt[:b]):sum(prompt[:b + 1])], v[sum(prompt[:b]):sum(prompt[:b + 1])]) for b in range(B)}
    # sequence 2 becomes four beams, sequence 1 ends
    scap.scap_kv4_fork(cache, i32([2, 2, 2]), i32([3, 4, 5]), fail, ws)
    scap.scap_kv4_free(cache, i32([1]))
    for b in (3, 4, 5):
        past[b] = past[2]
    del past[1]
    assert int(fail.item()) == 0
    ones = i32([0 if b in (1, 6, 7) else 1 for b in range(S)])
    y = torch.empty(S, K, dtype=torch.bfloat16, device="cuda")
    for step in range(4):
        x1 = torch.randn(S, K, device="cuda").bfloat16()
        q1 = torch.empty(S, width, dtype=torch.bfloat16, device="cuda")
        scap.scap_fc_act(x1, W, None, q1, ws)
        scap.scap_kv4_reserve(cache, ones, fail, ws)
        k1, v1 = heads_of(q1)[:, g * heads:(g + 1) * heads], heads_of(q1)[:, (g + 1) * heads:]
        rows = [b for b in range(S) if b in past]
        scap.scap_kv4_append(cache, k1, v1)       # rows of the empty sequences have no place and are left out
        for b in rows:
            past[b] = (torch.cat((past[b][0], k1[b:b + 1])), torch.cat((past[b][1], v1[b:b + 1])))
        if step == 1:
            scap.scap_kv4_compact(cache, None, ws)
        o = torch.empty(S, 1, g * heads, D, dtype=torch.bfloat16, device="cuda")
        scap.scap_kv4_attend(cache, heads_of(q1)[:, None, :g * heads], o, D ** -0.5, ws)
        scap.scap_fc_act(o.view(S, -1), Wo, None, y, ws, res=x1)
        assert lens.tolist() == [len(past[b][0]) if b in past else 0 for b in range(S)]
        for b in range(S):
            want = torch.zeros(g * heads, D, dtype=torch.float64, device="cuda")
            if b in past:
                kk, vv = (torch.tensor(stored64(t, 32), device="cuda") for t in past[b])
                for h in range(heads):
                    p = torch.softmax(heads_of(q1)[b, h * g:(h + 1) * g].double() @ kk[:, h].T * D ** -0.5, -1)
                    want[h * g:(h + 1) * g] = p @ vv[:, h]
            assert torch.allclose(o[b, 0].double(), want, atol=0.01, rtol=0.01)
        assert torch.allclose(y.float(), o.view(S, -1).float() @ Wo.float() + x1.float(), atol=0.05, rtol=0.02)
    assert int(fail.item()) == 0
    scap.scap_device_status()


def test_refusals():
    from paper_2412_07174_b200 import binding, build
    build.build()
    L = binding.lib()
    P, big = 0x10000, 1 << 30
    addr = lambda c: C.addressof(c)  # noqa: E731

    def both(f, *args, **kw):
        c = fake_cache(binding, heads=0, head_dim=0, group=0, **kw)
        return f(addr(c), *args)
    calls = [(L.scap_kv4_fork, (P, P, 2, P, P, big, None)), (L.scap_kv4_free, (P, 2, None)), (L.scap_kv4_reserve, (P, P, P, big, None)), (L.scap_kv4_compact, (P, P, big, None))]
    for f, args in calls:
        assert f(None, *args) == 1
        for name in ("pages", "table", "lens", "refs"):
            assert both(f, *args, **{name: None}) == 1
        for kw in (dict(n_pages=0), dict(n_pages=(1 << 20) + 1), dict(page_tokens=33), dict(table_stride=0), dict(n_seqs=0), dict(n_seqs=4097), dict(page_stride=0)):
            assert both(f, *args, **kw) == 2
        for kw in (dict(pages=P + 8), dict(page_stride=24), dict(table=P + 4), dict(lens=P + 8), dict(refs=P + 4)):
            assert both(f, *args, **kw) == 4
    assert both(L.scap_kv4_fork, P, P, 3, P, P, big, None) == 2 and both(L.scap_kv4_fork, P, P, -1, P, P, big, None) == 2
    assert both(L.scap_kv4_fork, None, P, 2, P, P, big, None) == 1 and both(L.scap_kv4_fork, P, P, 2, P, None, big, None) == 1
    n = L.scap_kv4_pages_workspace(8, 2)
    assert n > 0 and both(L.scap_kv4_fork, P, P, 2, P, P, n - 1, None) == 5
    assert both(L.scap_kv4_reserve, P, P, P, 15, None) == 5 and both(L.scap_kv4_compact, P, P, 15, None) == 5
    assert both(L.scap_kv4_free, None, 2, None) == 1 and both(L.scap_kv4_free, P, 4097, None) == 2 and both(L.scap_kv4_free, P + 4, 2, None) == 4
    assert both(L.scap_kv4_copy, P, None, 2, None) == 1 and both(L.scap_kv4_copy, P, P, -1, None) == 2 and both(L.scap_kv4_copy, P, P + 8, 2, None) == 4
    for f, args in ((L.scap_kv4_fork, (P, P, 0, P, P, big, None)), (L.scap_kv4_free, (P, 0, None)), (L.scap_kv4_copy, (P, P, 0, None))):
        assert both(f, *args) == 0
    assert L.scap_kv4_pages_workspace(0, 1) == 0 and L.scap_kv4_pages_workspace(8, 4097) == 0


def test_counts_that_lie_between_two_ints_are_refused():
    from paper_2412_07174_b200 import binding, build
    build.build()
    L = binding.lib()
    P, big = 0x10000, 1 << 30
    c = fake_cache(binding, heads=0, head_dim=0, group=0)
    for off in (1, 2, 3):
        assert L.scap_kv4_fork(C.addressof(c), P, P, 2, P + off, P, big, None) == 4
        assert L.scap_kv4_reserve(C.addressof(c), P, P + off, P, big, None) == 4
        assert L.scap_kv4_compact(C.addressof(c), P + off, P, big, None) == 4
