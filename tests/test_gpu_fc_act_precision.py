"""scap_fc_act where the order and the rounding of the additions show: bounds made of what the kernel adds up, not of the sum of all magnitudes."""
import pytest
import torch

BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32


def call(x, W, ydt):
    import paper_2412_07174_b200 as scap
    M, K = x.shape
    y = torch.full((M, W.shape[1]), float("nan"), device="cuda").to(ydt)
    ws = torch.empty(scap.scap_fc_act_workspace(M, K, W.shape[1]), dtype=torch.uint8, device="cuda")
    scap.scap_fc_act(x, W, None, y, ws)
    torch.cuda.synchronize()
    scap.scap_device_status()
    return y


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [HF, BF])
@pytest.mark.parametrize("M,K,N", [(300, 1 << 18, 264), (5, 1 << 20, 136), (700, 140000, 1032)])  # pairs of CTAs; a cluster over the channels; several tiles
def test_long_sums_of_one_sign(dt, M, K, N):
    """A sum of one sign over many channels, in 16 bits: one rounding to the type, and what 512 channels of one accumulator are off by."""
    g = torch.Generator(device="cuda").manual_seed(K)
    x = (0.5 + 0.5 * torch.rand(M, K, generator=g, device="cuda")).to(dt)
    W = ((0.5 + 0.5 * torch.rand(K, N, generator=g, device="cuda")) * 2.0 ** -14).to(dt)
    y = call(x, W, dt).double()
    ref = torch.zeros(M, N, dtype=torch.float64, device="cuda")
    for k in range(0, K, 1 << 16):
        ref += x[:, k:k + (1 << 16)].double() @ W[k:k + (1 << 16)].double()
    # An accumulator takes 32 additions, each off by at most 2^-23 of it; the K / 512 sums of them are added up with half a step each, 2^-24 of what is
    # there.  Everything has one sign, so all of that is relative to the result.  Then half a step of the type.
    near(y, ref, dt, K)


def near(y, ref, dt, K):
    own = 32 * 2.0 ** -23 + K / 512 * 2.0 ** -24
    off = (y - ref) / ref
    assert float(off.abs().max()) <= torch.finfo(dt).eps / 2 + own
    # Rounding keeps order: the result lies between the roundings of the ends of that interval, so it is the rounded sum unless a tie lies in it.  (Its mean
    # over the elements says nothing: those of one case lie within one step of each other.)
    assert bool(((ref * (1 - own)).to(dt).double() <= y).all()) and bool((y <= (ref * (1 + own)).to(dt).double()).all())


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [HF, BF])
@pytest.mark.parametrize("M,K,N", [(1000, 1 << 18, 264), (16, 1 << 19, 512)])
def test_long_sums_of_every_size(dt, M, K, N):
    """The same with rows and columns of different size, so that results lie at all distances from a tie."""
    g = torch.Generator(device="cuda").manual_seed(K + 1)
    x = ((1 + torch.rand(M, 1, generator=g, device="cuda")) * (0.5 + 0.5 * torch.rand(1, K, generator=g, device="cuda"))).to(dt)
    W = ((0.5 + 0.5 * torch.rand(K, 1, generator=g, device="cuda")) * 2.0 ** -14 * (1 + torch.rand(1, N, generator=g, device="cuda"))).to(dt)
    y = call(x, W, dt).double()
    ref = torch.zeros(M, N, dtype=torch.float64, device="cuda")
    for k in range(0, K, 1 << 16):
        ref += x[:, k:k + (1 << 16)].double() @ W[k:k + (1 << 16)].double()
    near(y, ref, dt, K)


@pytest.mark.gpu
@pytest.mark.parametrize("M,K,N", [(333, 2560, 1032), (2000, 2560, 520), (200, 11008, 264), (7, 11008, 264), (1, 2560, 2048)])
@pytest.mark.parametrize("dt", [HF, BF])
def test_fp32_results_are_as_good_as_fp32(dt, M, K, N):
    """The sums of 512 channels are added up in fp32 outside the tensor core, which truncates."""
    g = torch.Generator(device="cuda").manual_seed(K + M)
    x, W = torch.randn(M, K, generator=g, device="cuda").to(dt), (0.05 * torch.randn(K, N, generator=g, device="cuda")).to(dt)
    off = call(x, W, F32).double() - x.double() @ W.double()
    rms = float((off + x.double() @ W.double()).square().mean().sqrt())
    # An addition to an accumulator takes off 0 .. 2^-23 of the partial sum, 0.72 2^-24 on the average over its size.  The partial sums of a chunk of 32 additions grow as the
    # root of their number: 32 2/3 of the last one, together 0.9e-6 of it; chunks of either sign add up as their own sizes do.  With as many roundings to
    # nearest in registers, 2^-25 each on the average: below 1.5e-6 of a result.  (One accumulator for all of K = 2560: 160 additions, 4.6e-6 by the same count.)
    assert float(off.square().mean().sqrt()) <= 1.5e-6 * rms


@pytest.mark.gpu
@pytest.mark.parametrize("M,K,N", [(1, 1 << 20, 8), (20, 300001, 16), (3, 64, 1 << 18), (130, 24, 65544), (257, 8192, 264), (600, 2560, 1032), (40, 30000, 136)])
@pytest.mark.parametrize("dt", [HF, BF])
def test_whole_numbers_are_exact(dt, M, K, N):
    """Sums of small whole numbers below 2^24: every addition is exact, in whatever order, so nothing may be missing or there twice."""
    g = torch.Generator(device="cuda").manual_seed(K + N)
    x = torch.randint(-2, 3, (M, K), generator=g, device="cuda").to(dt)
    W = torch.randint(-3, 4, (K, N), generator=g, device="cuda").to(dt)
    want = torch.zeros(M, N, dtype=torch.float64, device="cuda")
    for k in range(0, K, 1 << 16):
        want += x[:, k:k + (1 << 16)].double() @ W[k:k + (1 << 16)].double()
    assert torch.equal(call(x, W, F32).double(), want)
    assert torch.equal(call(x, W, dt), want.to(dt))


@pytest.mark.gpu
@pytest.mark.parametrize("M,K,N,ydt", [(600, 4096, 4096, BF), (600, 4096, 4096, F32), (5, 200000, 256, BF)])
def test_waits_that_run_out_are_reported(M, K, N, ydt):
    """One try of 4 us at most per wait: the epilogue's wait for sums of far longer than that runs out, and scap_device_status says so."""
    import paper_2412_07174_b200 as scap
    x, W = torch.randn(M, K, device="cuda").to(BF), (0.05 * torch.randn(K, N, device="cuda")).to(BF)
    y = torch.empty(M, N, dtype=ydt, device="cuda")
    ws = torch.empty(scap.scap_fc_act_workspace(M, K, N), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    scap.scap_tune("tc_spin", 1)
    try:
        scap.scap_fc_act(x, W, None, y, ws)
        with pytest.raises(scap.ScapError) as e:
            scap.scap_device_status()
        assert e.value.code == 7
    finally:
        scap.scap_tune("tc_spin", 0)
    scap.scap_device_status()  # and is done with it
    assert torch.allclose(call(x, W, F32).double(), x.double() @ W.double(), rtol=1e-4, atol=1e-3)
