"""The pruned layers with the cache between them, as a decoding program runs them: scap_fc_act on the prompts, then a captured step of scap_sparse_fc (query, key and value of a
token), scap_kv4_reserve, scap_kv4_append, scap_kv4_attend, scap_sparse_fc (output).  The FCs give fp32, the cache takes 16 bits: the rounding between them is the program's."""
import pytest
import torch

from kv4_testlib import starts, stored64

BF = torch.bfloat16


def sparse64(x, W, m, tau, b):
    d = x.double() - m.double()
    return torch.where(d.abs() >= tau.double(), d, 0.0) @ W.double() + b.double()


@pytest.mark.gpu
@pytest.mark.parametrize("B", [1, 3, 8])
def test_prompts_and_captured_steps(B):
    import paper_2412_07174_b200 as scap
    torch.manual_seed(B)
    heads, g, D, group, page, K, dev = 2, 4, 64, 32, 32, 512, "cuda"
    Hq, width = g * heads, (g + 2) * heads * D
    rand = lambda *s: torch.randn(*s, device=dev)  # noqa: E731
    W, Wo = (K ** -0.5 * rand(K, width)).to(BF), ((Hq * D) ** -0.5 * rand(Hq * D, K)).to(BF)
    b, mode = (0.1 * rand(width)).to(BF), 0.2 * rand(K)
    tau, tau_o = torch.full((1,), 0.4, device=dev), torch.full((1,), 0.05, device=dev)
    ws = torch.empty(1 << 24, dtype=torch.uint8, device=dev)
    bf, bo = torch.empty(width, device=dev), torch.zeros(K, device=dev)
    scap.scap_fold_bias(W, mode, b, bf, ws)
    prompt = [45, 1, 70, 32, 31, 33, 5, 64][:B]
    total, room = sum(prompt), 5
    pool = torch.zeros(B * room + 3, scap.scap_kv4_page_bytes(page, heads, D, group), dtype=torch.uint8, device=dev)
    table, lens, refs = (torch.full(s, f, dtype=torch.int32, device=dev) for s, f in (((B, room), -1), ((B,), 0), ((len(pool),), 0)))
    cache = scap.ScapKv4(pool, page, heads, D, group, table, lens, refs=refs)
    fail = torch.full((1,), 9, dtype=torch.int32, device=dev)

    def split(t):
        t = t.view(len(t), -1, D)
        return t[:, :Hq], t[:, Hq:Hq + heads], t[:, Hq + heads:]
    # the prompts: the same layer on all rows, its results in 16 bits
    x = rand(total, K).to(BF)
    qkv = torch.empty(total, width, dtype=BF, device=dev)
    scap.scap_fc_act(x, W, b.float(), qkv, ws)
    scap.scap_kv4_reserve(cache, torch.tensor(prompt, dtype=torch.int32, device=dev), fail, ws)
    _, k, v = split(qkv)
    at = starts(prompt)
    scap.scap_kv4_append(cache, k, v, at)
    assert int(fail) == 0
    past = [(k[int(at[i]):int(at[i + 1])].clone(), v[int(at[i]):int(at[i + 1])].clone()) for i in range(B)]
    # one token of every sequence
    x1, ones = torch.zeros(B, K, dtype=BF, device=dev), torch.ones(B, dtype=torch.int32, device=dev)
    y1, row = torch.empty(B, width, device=dev), torch.empty(B, width, dtype=BF, device=dev)
    out, y = torch.empty(B, 1, Hq, D, dtype=BF, device=dev), torch.empty(B, K, device=dev)
    q1, k1, v1 = split(row)

    def step():
        scap.scap_sparse_fc(x1, W, mode, tau, bf, y1, ws)
        row.copy_(y1)
        scap.scap_kv4_reserve(cache, ones, fail, ws)
        scap.scap_kv4_append(cache, k1, v1)
        scap.scap_kv4_attend(cache, q1[:, None], out, D ** -0.5, ws)
        scap.scap_sparse_fc(out.view(B, -1), Wo, None, tau_o, bo, y, ws)
    saved = [t.clone() for t in (table, lens, refs, pool)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    s.synchronize()
    for t, was in zip((table, lens, refs, pool), saved):
        t.copy_(was)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for n in range(36):  # over the end of a page of each
        x1.copy_(rand(B, K))
        graph.replay()
        torch.cuda.synchronize()
        assert int(fail) == 0 and lens.tolist() == [p + n + 1 for p in prompt]
        # scap_sparse_fc: fp32 products and sums of K terms, K 2^-24 of the sum of magnitudes; a channel on the border of the threshold is decided in fp32 as here
        d = (x1.float() - mode).abs()
        assert bool(((d - tau).abs() > 1e-6).all())
        mag = x1.double().abs() @ W.double().abs() + mode.double().abs() @ W.double().abs() + b.double().abs()
        assert bool(((y1.double() - sparse64(x1, W, mode, tau, bf)).abs() <= K * 2.0 ** -24 * mag).all())
        assert torch.equal(row, y1.to(BF))
        for i in range(B):
            past[i] = (torch.cat((past[i][0], k1[i:i + 1])), torch.cat((past[i][1], v1[i:i + 1])))
        if n % 9 == 8:
            for i in range(B):
                kk, vv = (torch.tensor(stored64(t, group), device=dev) for t in past[i])
                for h in range(heads):
                    qq = q1[i, h * g:(h + 1) * g].double()
                    p = torch.softmax(qq @ kk[:, h].T * D ** -0.5, -1)
                    want = p @ vv[:, h]
                    # 2^-11 for the rounding of p and its scale, 2^-8 for that of the result, and 2^-13 of the largest value for scores and sums in fp32
                    bound = (p @ vv[:, h].abs()) * 2.0 ** -11 + want.abs() * 2.0 ** -8 + vv[:, h].abs().amax() * 2.0 ** -13
                    assert bool(((out[i, 0, h * g:(h + 1) * g].double() - want).abs() <= bound).all())
        o = out.view(B, -1)
        mag = o.double().abs() @ Wo.double().abs()
        assert bool(((y.double() - sparse64(o, Wo, torch.zeros_like(o[0]).float(), tau_o, bo)).abs() <= Hq * D * 2.0 ** -24 * mag + 1e-6).all())
    scap.scap_device_status()
