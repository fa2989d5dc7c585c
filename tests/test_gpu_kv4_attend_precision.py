"""scap_kv4_attend where rows differ much in size."""
import pytest
import torch

from test_gpu_kv4_attend import attend, check, filled, queries

BF = torch.bfloat16


@pytest.mark.gpu
@pytest.mark.parametrize("nq,g,heads,B", [(1, 8, 2, 3), (4, 2, 1, 2), (5, 4, 1, 2)])  # eight rows of one token and of several, sixteen
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
