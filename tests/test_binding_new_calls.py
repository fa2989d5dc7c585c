"""The binding of scap_fc_act and the scap_kv4 calls: what it refuses before the library is called, the strides and numbers that it passes on, and the two ways
it calls (the native helper and ctypes).  CPU tensors and a stand-in for the entry points: nothing is launched."""
import ctypes as C

import pytest
import torch

from paper_2412_07174_b200 import binding, build


@pytest.fixture(scope="module", autouse=True)
def built():
    build.build()
    binding.lib()


@pytest.fixture()
def seen(monkeypatch):
    """Arguments of the calls, as _invoke and _invoke_real get them."""
    calls = []
    monkeypatch.setattr(binding, "_invoke", lambda name, *args: calls.append((name, args)))
    monkeypatch.setattr(binding, "_invoke_real", lambda name, x, at, *args: calls.append((name, args[:at] + (x,) + args[at:])))
    return calls


def cache(S=3, n=8, heads=2, D=64, group=32, page=32, refs=True):
    pages = torch.zeros(n, binding.scap_kv4_page_bytes(page, heads, D, group), dtype=torch.uint8)
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    return binding.ScapKv4(pages, page, heads, D, group, i32(S, 4), i32(S), refs=i32(n) if refs else None)


def test_cache_description():
    c = cache()
    assert (c.n_pages, c.page_tokens, c.heads, c.head_dim, c.group, c.table_stride, c.n_seqs) == (8, 32, 2, 64, 32, 4, 3)
    assert c.page_stride == binding.scap_kv4_page_bytes(32, 2, 64, 32) and C.addressof(c) == c.address
    pages, t, n = torch.zeros(8, 1 << 16, dtype=torch.uint8), torch.zeros(3, 4, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    assert binding.ScapKv4(pages[:, 4096:20000], 32, 2, 64, 32, t, n).page_stride == 1 << 16   # a layer inside wider pages
    for bad in (dict(pages=pages.int()), dict(pages=pages.t()), dict(table=t.long()), dict(table=torch.zeros(4, 3, dtype=torch.int32).t()), dict(lens=n[:2]), dict(lens=n.long()),
                dict(refs=torch.zeros(7, dtype=torch.int32)), dict(pages=pages[:, :100])):
        args = dict(pages=pages, table=t, lens=n, refs=None, **{})
        args.update(bad)
        with pytest.raises(ValueError):
            binding.ScapKv4(args["pages"], 32, 2, 64, 32, args["table"], args["lens"], refs=args["refs"])


def test_rows_of_the_cache(seen):
    c = cache()
    qkv = torch.zeros(5, 8, 64, dtype=torch.bfloat16)
    k, v = qkv[:, 4:6], qkv[:, 6:8]
    st = torch.zeros(4, dtype=torch.int32)
    binding.scap_kv4_append(c, k, v, st, stream=0)
    name, a = seen.pop()
    assert name == "scap_kv4_append" and a[0] == c.address and a[2] == a[4] == 512 and a[6] == 5 and a[7] == binding.SCAP_BF16
    binding.scap_kv4_read(c, k[:1], v[:1], None, stream=0)
    assert seen.pop()[1][2] == 512
    for bad in ((k, v.half()), (k[:3], v), (k[:, :1], v[:, :1]), (k[..., :32], v[..., :32]), (k.transpose(0, 1).contiguous().transpose(0, 1), v)):
        with pytest.raises(ValueError):
            binding.scap_kv4_append(c, bad[0], bad[1], st, stream=0)
    with pytest.raises(ValueError):
        binding.scap_kv4_append(c, k, v, st[:3], stream=0)
    with pytest.raises(TypeError):
        binding.scap_kv4_append(c, k.float(), v.float(), st, stream=0)
    assert not seen


def test_attend(seen):
    c, ws = cache(), torch.zeros(64, dtype=torch.uint8)
    q = torch.zeros(3, 2, 4, 64, dtype=torch.float16)
    lse = torch.zeros(3, 2, 4)
    binding.scap_kv4_attend(c, q, torch.empty_like(q), 0.5, ws, window=7, lse=lse, stream=0)
    name, a = seen.pop()
    assert name == "scap_kv4_attend" and a[2] == a[4] == 256 and a[6:11] == (2, 4, 0.5, 7, binding.SCAP_F16)
    wide = torch.zeros(3, 8, 64, dtype=torch.float16)[:, None, :4]      # one token of a fused row
    binding.scap_kv4_attend(c, wide, torch.empty(3, 1, 4, 64, dtype=torch.float16), 0.5, ws, stream=0)
    assert seen.pop()[1][2] == 512
    for bad in (dict(q=q[:2]), dict(out=torch.empty(3, 2, 4, 64)), dict(out=torch.empty(3, 2, 4, 32, dtype=torch.float16)), dict(lse=lse.double()), dict(lse=lse[:, :1]),
                dict(q=q.transpose(1, 2).contiguous().transpose(1, 2))):
        args = dict(q=q, out=torch.empty_like(q), lse=lse)
        args.update(bad)
        with pytest.raises(ValueError):
            binding.scap_kv4_attend(c, args["q"], args["out"], 0.5, ws, lse=args["lse"], stream=0)
    assert not seen


def test_pages(seen):
    c, ws = cache(), torch.zeros(64, dtype=torch.uint8)
    i = torch.zeros(2, dtype=torch.int32)
    binding.scap_kv4_fork(c, i, i, None, ws, stream=0)
    binding.scap_kv4_free(c, i, stream=0)
    binding.scap_kv4_copy(c, i, i, stream=0)
    assert [(n, a[3] if n != "scap_kv4_free" else a[2]) for n, a in seen] == [("scap_kv4_fork", 2), ("scap_kv4_free", 2), ("scap_kv4_copy", 2)]
    with pytest.raises(ValueError):
        binding.scap_kv4_fork(c, i, i[:1], None, ws, stream=0)
    with pytest.raises(ValueError):
        binding.scap_kv4_free(c, i.long(), stream=0)
    with pytest.raises(ValueError):
        binding.scap_kv4_reserve(c, i, None, ws, stream=0)


def test_fc_act(seen):
    x, W, ws = torch.zeros(5, 12, dtype=torch.bfloat16), torch.zeros(12, 16, dtype=torch.bfloat16), torch.zeros(64, dtype=torch.uint8)
    y = torch.zeros(5, 24)[:, :16]
    binding.scap_fc_act(x, W, None, y, ws, act=binding.SCAP_ACT_GELU, res=y, stream=0)
    name, a = seen.pop()
    assert name == "scap_fc_act" and (a[1], a[4], a[6], a[8]) == (12, binding.SCAP_ACT_GELU, 24, 24) and a[9:14] == (5, 12, 16, binding.SCAP_BF16, binding.SCAP_F32)
    binding.scap_fc_act(x[:1], W, None, y[:1], ws, stream=0)
    assert (seen[-1][1][1], seen.pop()[1][8]) == (12, 24)
    for bad in (dict(W=W.half()), dict(W=W[:8]), dict(W=torch.zeros(16, 12, dtype=torch.bfloat16).t()), dict(y=y[:4]), dict(b=torch.zeros(8)), dict(b=torch.zeros(16).double()),
                dict(res=y.double()), dict(res=y[:4]), dict(x=torch.zeros(12, 5, dtype=torch.bfloat16).t())):
        args = dict(x=x, W=W, b=None, y=y, res=None)
        args.update(bad)
        with pytest.raises(ValueError):
            binding.scap_fc_act(args["x"], args["W"], args["b"], args["y"], ws, res=args["res"], stream=0)
    with pytest.raises(TypeError):
        binding.scap_fc_act(x, W, None, torch.zeros(5, 16, dtype=torch.int32), ws, stream=0)


@pytest.mark.parametrize("form", ["native", "ctypes"])
def test_the_number_reaches_its_place(form, monkeypatch):
    """scap_kv4_attend has a double among its arguments: 2e30 is refused as a scale, 0.5 is not (the missing workspace is)."""
    if form == "ctypes":
        monkeypatch.setattr(binding, "_call", binding._ctypes_call)
        monkeypatch.setattr(binding, "_entry", {n: getattr(binding.lib(), n) for n in binding.EXPORTS})
    c = cache()
    q = torch.zeros(3, 1, 4, 64, dtype=torch.float16)
    tiny = torch.zeros(16, dtype=torch.uint8)
    for scale, code in ((2e30, 1), (float("nan"), 1), (0.5, 5)):
        with pytest.raises(binding.ScapError) as e:
            binding.scap_kv4_attend(c, q, torch.empty_like(q), scale, tiny, stream=0)
        assert e.value.code == code
