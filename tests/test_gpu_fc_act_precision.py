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
