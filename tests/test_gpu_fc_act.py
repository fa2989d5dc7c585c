"""scap_fc_act (the FC on the rows of a prompt) against the same formula in 64 bits."""
import numpy as np
import pytest
import torch

from scap_testlib import Guarded

ACTS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3, "gelu_tanh": 4}


def act64(u, act):
    if act == "relu":
        return u.clamp(min=0)
    if act == "silu":
        return u * torch.sigmoid(u)
    if act == "gelu":
        return 0.5 * u * torch.erfc(-u * 0.5 ** 0.5)
    if act == "gelu_tanh":
        return u * torch.sigmoid(2 * (2 / np.pi) ** 0.5 * (u + 0.044715 * u ** 3))
    return u


def run_case(M, K, N, dt, ydt, act="none", bias=True, res=False, ldx=None, ldy=None, in_place=False, seed=0):
    import paper_2412_07174_b200 as scap
    g = torch.Generator(device="cuda").manual_seed(1000 + seed)
    ldx, ldy = ldx or K, ldy or N
    xs = torch.randn(M, ldx, generator=g, device="cuda").to(dt)
    x = xs[:, :K]
    W = (0.05 * torch.randn(K, N, generator=g, device="cuda")).to(dt)
    b = 0.3 * torch.randn(N, generator=g, device="cuda") if bias else None
    buf = Guarded(M * ldy * ydt.itemsize)
    full = buf.view(ydt, (M, ldy))
    full.fill_(7.0)
    y = full[:, :N]
    r = None
    if res or in_place:
        r0 = torch.randn(M, N, generator=g, device="cuda").to(ydt)
        if in_place:
            y.copy_(r0)
            r = y
        else:
            r = r0
    ws = Guarded(scap.scap_fc_act_workspace(M, K, N, ldx))
    scap.scap_fc_act(x, W, b, y, ws.payload, act=ACTS[act], res=r)
    torch.cuda.synchronize()
    assert buf.intact() and ws.intact()
    if ldy > N:
        assert bool((full[:, N:] == 7.0).all())  # the columns between the rows are left as they were
    u = x.double() @ W.double()
    mag = x.double().abs() @ W.double().abs()
    if bias:
        u = u + b.double()
        mag = mag + b.double().abs()
    ref = act64(u, act)
    if r is not None:
        ref = ref + r0.double()
        mag = mag + r0.double().abs()
    # Products are exact in fp32; the tensor core adds with truncation, fewer than K / 8 additions into one accumulator, each off by at
    # most 2^-23 of the running sum of magnitudes; the activations have a slope below 1.2 and add a few units of 2^-23.  Then one
    # rounding to the type of y: half a step, eps / 2 of the value.
    bound = 1.2 * mag * (K / 8 + 16) * 2.0 ** -23 + ref.abs() * torch.finfo(ydt).eps / 2 * 1.001 + 1e-30
    if ydt is torch.float16:
        bound = bound + 2.0 ** -25  # half a step of the subnormal numbers
    err = (y.double() - ref).abs()
    assert bool((err <= bound).all()), float((err / bound).max())
    return y


BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1, 2, 15, 16, 17, 33, 64, 100, 129, 255, 256, 257, 500])
def test_row_counts(M):
    run_case(M, 512, 640, BF, F32, bias=True, seed=M)


@pytest.mark.gpu
@pytest.mark.parametrize("K,N", [(1, 8), (7, 8), (8, 8), (63, 72), (64, 128), (65, 136), (1000, 248), (4096, 264), (11008, 128), (129, 4104)])
@pytest.mark.parametrize("dt", [BF, HF])
def test_widths(K, N, dt):
    run_case(37, K, N, dt, dt, act="silu", res=True, seed=K + N)


@pytest.mark.gpu
@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("ydt", [BF, HF, F32])
def test_activations(act, ydt):
    dt = BF if ydt is BF else HF
    run_case(70, 192, 208, dt, ydt, act=act, res=True, seed=3)
    run_case(70, 192, 208, dt, ydt, act=act, bias=False, seed=4)


@pytest.mark.gpu
@pytest.mark.parametrize("M,K,N", [(1024, 512, 4096), (2048, 448, 2056), (700, 2048, 9000), (1111, 1024, 1032), (3000, 640, 2048)])
def test_many_tiles(M, K, N):
    run_case(M, K, N, BF, BF, act="gelu", res=True, seed=M)
    run_case(M, K, N, HF, F32, bias=False, seed=M + 1)


@pytest.mark.gpu
@pytest.mark.parametrize("M,K,N", [(1 << 20, 8, 8), (300001, 72, 16), (1, 1 << 20, 8), (20, 300001, 16), (3, 64, 1 << 18), (130, 24, 65544)])
def test_long_sides(M, K, N):
    run_case(M, K, N, BF, BF, act="silu", seed=7)
    run_case(M, K, N, HF, F32, bias=False, res=True, seed=8)


@pytest.mark.gpu
def test_slices_of_wider_matrices():
    import paper_2412_07174_b200 as scap
    wide = torch.randn(70, 400, device="cuda").to(BF)
    W = (0.05 * torch.randn(128, 64, device="cuda")).to(BF)
    ws = torch.empty(16, dtype=torch.uint8, device="cuda")
    out = torch.zeros(70, 400, device="cuda")
    scap.scap_fc_act(wide[:, 8:136], W, None, out[:, 104:168], ws)
    want = wide[:, 8:136].double() @ W.double()
    assert torch.allclose(out[:, 104:168].double(), want, atol=1e-4)
    assert bool((out[:, :104] == 0).all()) and bool((out[:, 168:] == 0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("M,K,N,ldx,ldy", [(5, 100, 64, 136, 64), (40, 100, 64, 101, 80), (300, 511, 520, 511, 521), (130, 256, 264, 300, 1000)])
def test_strides(M, K, N, ldx, ldy):
    run_case(M, K, N, BF, BF, act="relu", res=True, ldx=ldx, ldy=ldy, seed=ldx)
    run_case(M, K, N, HF, F32, in_place=True, ldx=ldx, ldy=ldy, seed=ldx + 1)


@pytest.mark.gpu
def test_same_bits_in_a_graph_and_on_another_stream():
    import paper_2412_07174_b200 as scap
    x = torch.randn(200, 1000, device="cuda").to(BF)[:, :999]
    x = x.contiguous()
    W = (0.05 * torch.randn(999, 520, device="cuda")).to(BF)
    b = torch.randn(520, device="cuda")
    y, y2 = torch.empty(200, 520, device="cuda"), torch.empty(200, 520, device="cuda")
    ws = torch.empty(scap.scap_fc_act_workspace(200, 999, 520), dtype=torch.uint8, device="cuda")
    scap.scap_fc_act(x, W, b, y, ws, act=3)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        scap.scap_fc_act(x, W, b, y2, ws, act=3)
    s.synchronize()
    assert torch.equal(y, y2)
    graph = torch.cuda.CUDAGraph()
    x2 = x.clone()
    with torch.cuda.graph(graph):
        scap.scap_fc_act(x2, W, b, y2, ws, act=3)
    x2.copy_(torch.randn_like(x2))
    graph.replay()
    scap.scap_fc_act(x2, W, b, y, ws, act=3)
    torch.cuda.synchronize()
    assert torch.equal(y, y2)
    scap.scap_device_status()


@pytest.mark.gpu
@pytest.mark.parametrize("M,K,N,ydt", [(600, 4096, 4096, BF), (600, 4096, 4096, F32), (5, 8192, 256, BF), (300, 1000, 520, F32)])
def test_a_wait_that_runs_out_is_reported(M, K, N, ydt):
    import paper_2412_07174_b200 as scap
    x, W = torch.randn(M, K, device="cuda").to(BF), (0.05 * torch.randn(K, N, device="cuda")).to(BF)
    y = torch.empty(M, N, dtype=ydt, device="cuda")
    ws = torch.empty(scap.scap_fc_act_workspace(M, K, N), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    scap.scap_tune("tc_spin", 1)
    try:
        scap.scap_fc_act(x, W, None, y, ws)
        try:
            scap.scap_device_status()
        except scap.ScapError as e:
            assert e.code == 7
    finally:
        scap.scap_tune("tc_spin", 0)
    run_case(M, K, N, BF, ydt, res=True, seed=5)  # and the next call is right
    scap.scap_device_status()


@pytest.mark.gpu
def test_non_finite_rows_stay_in_their_row():
    import paper_2412_07174_b200 as scap
    x = torch.randn(40, 128, device="cuda").to(BF)
    W = (0.05 * torch.randn(128, 64, device="cuda")).to(BF)
    y0, y = torch.empty(40, 64, device="cuda"), torch.empty(40, 64, device="cuda")
    ws = torch.empty(16, dtype=torch.uint8, device="cuda")
    scap.scap_fc_act(x, W, None, y0, ws)
    x[3, 5], x[17, 100] = float("nan"), float("inf")
    scap.scap_fc_act(x, W, None, y, ws)
    bad = ~torch.isfinite(y).all(1)
    assert bad.nonzero().flatten().tolist() == [3, 17]
    keep = [i for i in range(40) if i not in (3, 17)]
    assert torch.equal(y[keep], y0[keep])


def test_refusals():
    from paper_2412_07174_b200 import binding, build
    build.build()
    L = binding.lib()
    P = 0x10000  # a fake, 16-byte aligned, never dereferenced address
    base = dict(x=P, ldx=64, W=P, b=P, act=0, r=None, ldr=0, y=P, ldy=64, M=4, K=64, N=64, dt=1, ydt=2, ws=P, wsb=1 << 20, st=None)
    call = lambda **kw: L.scap_fc_act(*[kw.get(k, v) for k, v in base.items()])  # noqa: E731
    assert call(x=None) == 1 and call(W=None) == 1 and call(y=None) == 1 and call(ws=None) == 1
    assert call(act=5) == 1 and call(act=-1) == 1
    assert call(M=-1) == 2 and call(M=(1 << 20) + 1) == 2 and call(K=0) == 2 and call(K=(1 << 20) + 1) == 2 and call(N=0) == 2
    assert call(ldx=63) == 2 and call(ldy=63) == 2 and call(r=P, ldr=63) == 2
    assert call(dt=2) == 3 and call(dt=7) == 3 and call(ydt=0) == 3 and call(ydt=3) == 3
    assert call(N=60, ldy=64) == 4 and call(x=P + 2) == 4 and call(y=P + 4) == 4 and call(b=P + 4) == 4 and call(r=P + 2, ldr=64) == 4
    assert call(ldx=65, wsb=4 * 64 * 2 - 1) == 5
    assert call(M=0) == 0                                   # no rows: nothing to do
    assert call(M=0, x=None) == 0
    assert L.scap_fc_act_workspace(4, 64, 64, 63) == 0 and L.scap_fc_act_workspace(-1, 64, 64, 64) == 0
    assert L.scap_fc_act_workspace(4, 61, 64, 61) == 4 * 64 * 2


@pytest.mark.gpu
@pytest.mark.parametrize("M,K,N,ldy", [(1, 64, 24, 25), (2, 40, 8, 9), (31, 130, 136, 137), (300, 256, 520, 523), (1000, 128, 2056, 2059), (33, 2048, 264, 267)])
@pytest.mark.parametrize("dt", [BF, HF])
def test_rows_that_begin_between_two_words(M, K, N, ldy, dt):
    run_case(M, K, N, dt, dt, act="gelu", in_place=True, ldy=ldy, seed=M)       # y and the residual at odd strides
    run_case(M, K, N, dt, dt, act="relu", in_place=True, ldy=ldy + 1, seed=M)   # at even ones that are no multiple of eight


@pytest.mark.gpu
@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("dt,ydt", [(BF, BF), (HF, HF), (BF, F32), (HF, F32)])
@pytest.mark.parametrize("K", [8, 8192])  # (8192 of a few rows: a sum over ranks)
def test_activations_over_the_range_of_numbers(act, dt, ydt, K):
    """u = x[m, 0] alone, exactly: what is left is the activation and one rounding."""
    import paper_2412_07174_b200 as scap
    big = 3e38 if dt is BF else 6e4
    vals = [0.0, -0.0, 1e-7, -1e-7, 1e-3, -1e-3, 300.0, -300.0, big / 2, -big / 2, big, -big, float("inf"), float("nan")]
    vals += torch.linspace(-16, 16, 601).tolist()
    x = torch.zeros(len(vals), K, device="cuda").to(dt)
    x[:, 0] = torch.tensor(vals, device="cuda").to(dt)
    W = torch.zeros(K, 16, device="cuda").to(dt)
    W[0] = 1.0
    for rows in (slice(0, 10), slice(10, 21), slice(None)):  # few rows and many take different forms
        xs = x[rows].contiguous()
        y = torch.full((xs.shape[0], 16), 5.0, device="cuda").to(ydt)
        scap.scap_fc_act(xs, W, None, y, torch.empty(16, dtype=torch.uint8, device="cuda"), act=ACTS[act])
        u = xs[:, :1].double().expand(-1, 16)
        ref = act64(u, act)
        nan, inf = u.isnan(), u.isinf()
        assert bool(y[nan].isnan().all()) and bool((y[inf] == float("inf")).all())
        fine = ~(nan | inf)
        # The argument z of the exponential has at most four roundings, each 2^-24 of it, which make it wrong by so much of itself; the exponential,
        # the reciprocal and the polynomial add fewer than 16 units of 2^-24.  Then the rounding to the type of y, and what lies below its smallest
        # numbers (an exponential below 2^-126 is 0).
        z = {"silu": u.abs(), "gelu": u * u / 2, "gelu_tanh": 1.6 * (u.abs() + 0.045 * u.abs() ** 3)}.get(act, u * 0)
        rel = (4 * z + 16) * 2.0 ** -24 + torch.finfo(ydt).eps / 2
        least = {F32: 1e-36, BF: 1e-36, HF: 2.0 ** -25}[ydt]
        limit = torch.finfo(ydt).max
        want = torch.where(ref.abs() > limit, ref.sign() * float("inf"), ref)
        err = torch.where(want.isinf(), (y.double() != want).double(), (y.double() - ref).abs())
        bound = torch.where(ref.abs() > 0, ref.abs() * rel.clamp(max=4.0), 0.0) + least
        assert bool((err[fine] <= bound[fine]).all()), float((err / bound)[fine].max())
