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
            make(**{**good, name: good[name].to("meta")})  # a device that is not the others'
