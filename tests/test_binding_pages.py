"""The binding of the calls on pages: what they may be given.  CPU tensors and a stand-in for the entry points: nothing is launched."""
import pytest
import torch

from paper_2412_07174_b200 import binding
from test_binding_new_calls import built, seen  # noqa: F401 (fixtures)


def i32(*shape):
    return torch.zeros(*shape, dtype=torch.int32)


def cache(pages, n_seqs=3):
    return binding.ScapKv4(pages, 32, 2, 64, 32, i32(n_seqs, 4), i32(n_seqs), refs=i32(pages.shape[0]))


def calls(c):
    i, ws = i32(2), torch.zeros(64, dtype=torch.uint8)
    return [lambda: binding.scap_kv4_copy(c, i, i, stream=0), lambda: binding.scap_kv4_fork(c, i, i, None, ws, stream=0), lambda: binding.scap_kv4_compact(c, None, ws, stream=0)]


def test_pages_move_whole(seen):  # noqa: F811
    """A copy takes all bytes from one page to the next: from the middle of a page that is the end of one and the beginning of another, and beyond the pool at its
    end.  So a layer inside the pages is refused; the pool, a slice of its pages and its first layer are what they were."""
    one = binding.scap_kv4_page_bytes(32, 2, 64, 32)
    raw = torch.zeros(10, 3 * one, dtype=torch.uint8)
    for pool in (raw, raw[1:-1], raw[2:3], raw[:, :one], raw[1:, :2 * one], torch.zeros(16 + 8 * one, dtype=torch.uint8)[16:].view(8, one)):
        for f in calls(cache(pool)):
            f()
    assert len(seen) == 18
    seen.clear()
    for layer in (raw[:, one:2 * one], raw[1:-1, 2 * one:], raw[:1, one:], raw[:, 16:16 + one]):
        for f in calls(cache(layer)):
            with pytest.raises(ValueError):
                f()
    short = torch.as_strided(torch.zeros(7 * 3 * one + one, dtype=torch.uint8), (8, one), (3 * one, 1))  # the last page ends with its first layer
    for f in calls(cache(short)):
        with pytest.raises(ValueError):
            f()
    assert not seen
    c = cache(raw[:, one:2 * one])  # what moves no bytes takes it
    binding.scap_kv4_free(c, i32(2), stream=0)
    binding.scap_kv4_reserve(c, i32(3), None, torch.zeros(64, dtype=torch.uint8), stream=0)
    assert len(seen) == 2


def test_counts_are_int32(seen):  # noqa: F811
    c, i, ws = cache(torch.zeros(8, binding.scap_kv4_page_bytes(32, 2, 64, 32), dtype=torch.uint8)), i32(2), torch.zeros(64, dtype=torch.uint8)
    calls = (lambda t: binding.scap_kv4_fork(c, i, i, t, ws, stream=0), lambda t: binding.scap_kv4_reserve(c, i32(3), t, ws, stream=0), lambda t: binding.scap_kv4_compact(c, t, ws, stream=0))
    for f in calls:
        for bad in (torch.zeros(1), torch.zeros(1, dtype=torch.int64), torch.zeros(1, dtype=torch.int16), i32(0)):
            with pytest.raises(ValueError):
                f(bad)
    assert not seen
    for f in calls:
        for good in (None, i32(1), i32(()), i32(4), 0x10000):
            f(good)
    assert len(seen) == 15


def test_a_cache_lies_on_one_device():
    pages = torch.zeros(8, binding.scap_kv4_page_bytes(32, 2, 64, 32), dtype=torch.uint8)
    good = dict(pages=pages, table=i32(3, 4), lens=i32(3), refs=i32(8))
    make = lambda pages, table, lens, refs: binding.ScapKv4(pages, 32, 2, 64, 32, table, lens, refs=refs)  # noqa: E731
    make(**good)
    for name in good:
        with pytest.raises(ValueError):
            make(**{**good, name: other(good[name])})


class Elsewhere(torch.Tensor):
    def get_device(self):
        return 3


def other(t):
    return t.as_subclass(Elsewhere)


def test_tensors_lie_on_the_device_of_the_cache(seen):  # noqa: F811
    """Memory of another device, or of the host, would be read and written by a kernel that cannot reach it."""
    c, ws, i = cache(torch.zeros(8, binding.scap_kv4_page_bytes(32, 2, 64, 32), dtype=torch.uint8)), torch.zeros(64, dtype=torch.uint8), i32(2)
    k, q = torch.zeros(5, 2, 64, dtype=torch.float16), torch.zeros(3, 1, 4, 64, dtype=torch.float16)
    x, W, y, b = torch.zeros(5, 16, dtype=torch.float16), torch.zeros(16, 8, dtype=torch.float16), torch.zeros(5, 8), torch.zeros(8)
    calls = [
        (lambda k, v, st: binding.scap_kv4_append(c, k, v, st, stream=0), [k, k, i32(4)]),
        (lambda k, v, st: binding.scap_kv4_read(c, k, v, st, stream=0), [k, k, i32(4)]),
        (lambda q, o, lse, ws: binding.scap_kv4_attend(c, q, o, 0.5, ws, lse=lse, stream=0), [q, q, torch.zeros(3, 1, 4), ws]),
        (lambda x, W, b, y, ws, r: binding.scap_fc_act(x, W, b, y, ws, res=r, stream=0), [x, W, b, y, ws, y]),
        (lambda a, b: binding.scap_kv4_copy(c, a, b, stream=0), [i, i]),
        (lambda a, b, f, ws: binding.scap_kv4_fork(c, a, b, f, ws, stream=0), [i, i, i32(1), ws]),
        (lambda a: binding.scap_kv4_free(c, a, stream=0), [i]),
        (lambda a, f, ws: binding.scap_kv4_reserve(c, a, f, ws, stream=0), [i32(3), i32(1), ws]),
        (lambda f, ws: binding.scap_kv4_compact(c, f, ws, stream=0), [i32(1), ws]),
    ]
    for f, args in calls:
        f(*args)
        assert seen.pop() and not seen
        for n in range(len(args)):
            with pytest.raises(ValueError):
                f(*[other(a) if m == n else a for m, a in enumerate(args)])
    assert not seen


def test_the_device_is_the_current_one(monkeypatch):
    """A launch goes to the current device, so memory of another one is refused."""
    class On0:
        def get_device(self):
            return 0
    monkeypatch.setattr(binding, "_getDevice", lambda: 1)
    with pytest.raises(ValueError):
        binding._stream_on(0, 5, On0())
    monkeypatch.setattr(binding, "_getDevice", lambda: 0)
    monkeypatch.setattr(binding, "_getCurrentRawStream", lambda device: 70 + device)
    assert binding._stream_on(0, 5, On0(), None) == 5 and binding._stream_on(0, None, On0()) == 70
