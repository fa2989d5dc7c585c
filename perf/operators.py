"""What a decoding program runs around the pruned layers: the layers on the rows of a prompt, and attention over a cache in 4 bits.

A case is one pass of one of these paths, with the sizes of the models the repository is configured for (LLaMA-2-7B, LLaMA-3.1-8B
and MPT-7B shapes, Mamba2-2.7B projections, the 1024 x 1024 layer of the smoke test):

  fc      y = act(x W + b) + r on the rows of a prompt: scap_fc_act
  store   new keys and values into the cache, and the values it holds for them: scap_kv4_append, scap_kv4_read
  attend  attention of one or a few new tokens per sequence over the cache: scap_kv4_attend
  beam    a beam step on the cache's pages: scap_kv4_fork, scap_kv4_free, scap_kv4_reserve
  compact the used pages of a pool moved to its front: scap_kv4_compact

The 4-bit format, for a group of channels of one token and head with values x:  lo = min(0, min x), hi = max(0, max x),
s = (hi - lo) / 15 rounded to 20 significant bits, zero = round(-lo / s), code = min(15, max(0, round(x / s) + zero)), and the cache
stands for s (code - zero).
"""
import math

import torch

own = False  # False: elementary torch operations; True: the library's calls

ACTS = ("none", "relu", "silu", "gelu", "gelu_tanh")


def listed():
    return [
        # a short fp16 prompt through the small layer: launches and latency
        {"name": "fc_small_fp16_m37", "op": "fc", "M": 37, "K": 1024, "N": 1024, "dt": "fp16", "out": "fp16", "act": "gelu", "bias": True, "res": False},
        # Mamba2 in-projection (columns that fill no tile) on a ragged prompt
        {"name": "fc_inproj_bf16_m333", "op": "fc", "M": 333, "K": 2560, "N": 10576, "dt": "bf16", "out": "fp32", "act": "silu", "bias": False, "res": False},
        # LLaMA-2-7B down projection of a 2048-token prompt, residual added
        {"name": "fc_down_bf16_m2048", "op": "fc", "M": 2048, "K": 11008, "N": 4096, "dt": "bf16", "out": "bf16", "act": "none", "bias": True, "res": True},
        # MPT-7B up projection of a 4096-token chunk of prompts, with its GELU
        {"name": "fc_up_fp16_m4096", "op": "fc", "M": 4096, "K": 4096, "N": 16384, "dt": "fp16", "out": "fp16", "act": "gelu", "bias": True, "res": False},
        # one decode step: a token of each of 64 sequences
        {"name": "store_step_b64", "op": "store", "B": 64, "new": 64, "past": 4096, "Hkv": 8, "D": 128, "group": 64, "page": 64, "dt": "bf16"},
        # four prompts of together 8191 tokens, heads of 128 channels
        {"name": "store_prompt_8191", "op": "store", "B": 4, "new": 8191, "past": 100, "Hkv": 32, "D": 128, "group": 128, "page": 64, "dt": "fp16"},
        # one sequence at 1000 tokens: latency
        {"name": "attend_b1_1k", "op": "attend", "B": 1, "tokens": 1000, "Hkv": 8, "g": 4, "D": 128, "group": 128, "page": 64, "nq": 1, "window": 0, "dt": "bf16"},
        # 48 sequences of very different lengths
        {"name": "attend_b48_ragged", "op": "attend", "B": 48, "tokens": 196608, "Hkv": 8, "g": 4, "D": 128, "group": 64, "page": 64, "nq": 1, "window": 0, "dt": "bf16"},
        # one sequence with a long past
        {"name": "attend_b1_128k", "op": "attend", "B": 1, "tokens": 131001, "Hkv": 8, "g": 8, "D": 128, "group": 128, "page": 64, "nq": 1, "window": 0, "dt": "bf16"},
        # four guessed tokens per sequence verified at once, a key head for every query head, sliding window
        {"name": "attend_mha_nq4", "op": "attend", "B": 16, "tokens": 40000, "Hkv": 32, "g": 1, "D": 128, "group": 64, "page": 32, "nq": 4, "window": 4096, "dt": "fp16"},
        # 96 beams from 24 parents, the parents freed, room for a token in each beam; a page holds two layers
        {"name": "beam_24_to_96", "op": "beam", "parents": 24, "children": 96, "tokens": 1500, "pages": 2048, "stride": 147456, "page": 64},
        # a pool of which half the pages lie free
        {"name": "compact_half", "op": "compact", "seqs": 64, "tokens": 1024, "pages": 2048, "stride": 294912, "page": 64},
    ]


def _spread(rng, lo, hi, step=1):
    """A multiple of `step` between lo and hi, evenly spread over the logarithm."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return int(min(hi, max(lo, round(v / step) * step)))


def draw(rng):
    op = rng.choice(["fc", "fc", "fc", "store", "store", "attend", "attend", "attend", "attend", "beam", "compact"])
    dt = rng.choice(["bf16", "fp16"])
    if op == "fc":
        K, N = _spread(rng, 512, 11008, rng.choice([8, 8, 8, 1])), _spread(rng, 512, 16384, 8)
        M = min(_spread(rng, 1, 4096), (4096 * 4096 * 16384) // (K * N))
        return {"op": op, "M": M, "K": K, "N": N, "dt": dt, "out": rng.choice([dt, dt, "fp32"]), "act": rng.choice(ACTS),
                "bias": rng.random() < 0.7, "res": rng.random() < 0.5}
    if op in ("store", "attend"):
        D = rng.choice([64, 128, 128, 128, 256])
        case = {"op": op, "Hkv": rng.choice([1, 2, 4, 8, 8, 16, 32]), "D": D, "group": rng.choice([n for n in (32, 64, 128) if n <= D <= 4 * n]),
                "page": rng.choice([32, 64, 64, 128]), "dt": dt}
        if op == "store":
            case["B"] = _spread(rng, 1, 128)
            case["new"] = max(case["B"], min(_spread(rng, 1, 16384), 8192 * 4096 // (case["Hkv"] * D)))
            case["past"] = rng.choice([0, 1, 31, _spread(rng, 32, 8192)])
            return case
        case["nq"] = rng.choice([1, 1, 1, 2, 3, 4, 8, 16])
        case["g"] = rng.choice([n for n in (1, 2, 3, 4, 7, 8, 16) if n * case["Hkv"] <= 64])
        case["B"] = _spread(rng, 1, 64)
        most = 196608 * 1024 // (case["Hkv"] * D) // max(1, case["g"] * case["nq"] // 16)
        case["tokens"] = max(case["B"] * 32, min(_spread(rng, 64, 196608), most))
        case["window"] = rng.choice([0, 0, 0, _spread(rng, 16, 4096)])
        return case
    stride = 16 * _spread(rng, 256, 16384)
    pages = min(2048, 512 * 1024 * 1024 // stride)
    if op == "beam":
        parents = _spread(rng, 1, 24)
        return {"op": op, "parents": parents, "children": _spread(rng, parents, 96), "tokens": _spread(rng, 1, min(1500, 32 * (pages // 3) // parents)),
                "pages": pages, "stride": stride, "page": rng.choice([32, 64, 128])}
    return {"op": op, "seqs": _spread(rng, 1, 64), "tokens": _spread(rng, 32, 1024), "pages": pages, "stride": stride, "page": rng.choice([32, 64, 128])}


# ---- inputs -------------------------------------------------------------------------------------------------------

DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}


class _Maker:
    """Random tensors on the GPU, from the seed alone."""

    def __init__(self, case, seed):
        self.g = torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 29)
        self.dt = DTYPES[case.get("dt", "bf16")]

    def normal(self, *shape, std=1.0, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=self.g)

    def ints(self, lo, hi, *shape):
        return torch.randint(lo, hi, shape, generator=self.g, device="cuda")

    def share(self, total, parts, least):
        """`total` split into `parts` numbers of at least `least`, very different ones, as a list."""
        w = torch.exp(self.normal(parts))
        n = (w / w.sum() * max(0, total - parts * least)).long() + least
        n[0] += max(0, total - int(n.sum()))
        return n.tolist()

    def permutation(self, n):
        return torch.randperm(n, generator=self.g, device="cuda")


def _keys(mk, tokens, heads, D):
    """Keys: channels of different spread around different means, a few of them large."""
    spread = torch.exp(0.4 * mk.normal(heads, D))
    spread = torch.where(mk.normal(heads, D) > 2.0, 4.0 * spread, spread)
    mean = 0.5 * mk.normal(heads, D)
    k = torch.empty(tokens, heads, D, dtype=mk.dt, device="cuda")
    for i in range(0, tokens, 32768):
        n = min(32768, tokens - i)
        k[i:i + n] = (mean + spread * mk.normal(n, heads, D)).to(mk.dt)
    return k


def _paged(mk, lens, page):
    """A table that gives every sequence its pages, scattered over a pool with a few more than it needs."""
    need = [-(-n // page) for n in lens]
    width, total = max(max(need), 1), sum(need)
    pool = total + max(2, total // 16)
    ids = mk.permutation(pool).to(torch.int32)
    table = torch.full((len(lens), width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = ids[at:at + n]
        at += n
    return table, pool


def _starts(counts):
    return torch.tensor([0] + torch.tensor(counts).cumsum(0).tolist(), dtype=torch.int32, device="cuda")


def _kv_inputs(case, mk):
    """lens, rows of new tokens per sequence, and the keys and values of all tokens that a sequence holds."""
    B, D, H = case["B"], case["D"], case["Hkv"]
    if case["op"] == "store":
        new = mk.share(case["new"], B, 1)
        past = [case["past"] // 2 + int(n) for n in (mk.ints(0, case["past"] // 2 + 1, B)).tolist()]
        lens, rows = [n + p for n, p in zip(new, past)], new
    else:
        lens = mk.share(case["tokens"], B, case["nq"])
        rows = lens
    total = sum(rows)
    k = _keys(mk, total, H, D)
    v = torch.empty(total, H, D, dtype=mk.dt, device="cuda")
    for i in range(0, total, 32768):
        n = min(32768, total - i)
        v[i:i + n] = mk.normal(n, H, D).to(mk.dt)
    return lens, rows, k, v


def prepare(case, seed):
    mk, op = _Maker(case, seed), case["op"]
    st = {"case": case}
    if op == "fc":
        M, K, N = case["M"], case["K"], case["N"]
        st["x"], st["W"] = mk.normal(M, K).to(mk.dt), mk.normal(K, N, std=0.02, dtype=mk.dt)
        st["b"] = mk.normal(N, std=0.1) if case["bias"] else None
        st["r"] = mk.normal(M, N).to(DTYPES[case["out"]]) if case["res"] else None
        if own:
            import paper_2412_07174_b200 as scap
            st["y"] = torch.empty(M, N, dtype=DTYPES[case["out"]], device="cuda")
            st["ws"] = torch.empty(max(16, scap.scap_fc_act_workspace(M, K, N)), dtype=torch.uint8, device="cuda")
        return st
    if op in ("store", "attend"):
        H, D, group, page = case["Hkv"], case["D"], case["group"], case["page"]
        lens, rows, k, v = _kv_inputs(case, mk)
        table, pool = _paged(mk, lens, page)
        st.update(k=k, v=v, rows=rows, row_start=_starts(rows), lens_list=lens, lens=torch.tensor(lens, dtype=torch.int32, device="cuda"), table=table)
        if own:
            import paper_2412_07174_b200 as scap
            pages = torch.zeros(pool, scap.scap_kv4_page_bytes(page, H, D, group), dtype=torch.uint8, device="cuda")
            st["cache"] = scap.ScapKv4(pages, page, H, D, group, table, st["lens"])
        else:
            st["store"] = {n: (torch.zeros(pool * page, H, D // 2, dtype=torch.uint8, device="cuda"),
                               torch.zeros(pool * page, H, D // group, dtype=torch.float32, device="cuda"),
                               torch.zeros(pool * page, H, D // group, dtype=torch.uint8, device="cuda")) for n in "kv"}
        if op == "store":
            if own:
                st["ko"], st["vo"] = torch.empty_like(k), torch.empty_like(v)
            return st
        B, nq, Hq = case["B"], case["nq"], case["g"] * H
        st["q"] = mk.normal(B, nq, Hq, D).to(mk.dt)
        if own:
            scap.scap_kv4_append(st["cache"], k, v, st["row_start"])
            st["out"], st["lse"] = torch.empty_like(st["q"]), torch.empty(B, nq, Hq, dtype=torch.float32, device="cuda")
            st["ws"] = torch.empty(scap.scap_kv4_attend_workspace(B, nq, Hq, H, D), dtype=torch.uint8, device="cuda")
        else:
            _plain_append(st)
        del st["k"], st["v"]
        return st
    # a pool of pages with arbitrary contents, and the sequences that hold some of them
    P, page = case["pages"], case["page"]
    st["pool"] = mk.ints(0, 256, P, case["stride"]).to(torch.uint8) if P * case["stride"] < 1 << 27 else torch.empty(P, case["stride"], dtype=torch.uint8, device="cuda")
    if P * case["stride"] >= 1 << 27:
        for i in range(0, P, 128):
            n = min(128, P - i)
            st["pool"][i:i + n] = mk.ints(0, 256, n, case["stride"]).to(torch.uint8)
    if op == "beam":
        S = case["parents"] + case["children"]
        lens = [1 + int(n) for n in mk.ints(case["tokens"] // 2, case["tokens"], case["parents"]).tolist()] + [0] * case["children"]
        share, most = [0] * S, case["tokens"]
        st["src"] = mk.ints(0, case["parents"], case["children"]).to(torch.int32)
        st["dst"] = torch.arange(case["parents"], S, dtype=torch.int32, device="cuda")
        st["rows"] = torch.arange(case["parents"], dtype=torch.int32, device="cuda")
        st["add"] = torch.cat((torch.zeros(case["parents"]), torch.ones(case["children"]))).to(torch.int32).cuda()
    else:
        S = case["seqs"]
        least = max(1, P * page // (2 * S))  # about half the pool, where the tokens of a sequence allow it
        most = min(2 * least, case["tokens"])
        lens = [int(n) for n in mk.ints(max(1, most // 2), most + 1, S).tolist()]
        share = [0 if b % 4 else min(lens[b], lens[b - 1]) // page if b else 0 for b in range(S)]  # every fourth is a fork of its neighbour
    width = -(-(most + 1) // page) + 1
    table = torch.full((S, width), -1, dtype=torch.int32)
    ids = mk.permutation(P).to(torch.int32).cpu()
    refs = torch.zeros(P, dtype=torch.int32)
    at = 0
    for b, n in enumerate(lens):
        need = -(-n // page)
        if share[b]:
            table[b, :share[b]] = table[b - 1, :share[b]]
        table[b, share[b]:need] = ids[at:at + need - share[b]]
        at += need - share[b]
        refs[table[b, :need].long()] += 1
    st.update(table=table.cuda(), refs=refs.cuda(), lens=torch.tensor(lens, dtype=torch.int32, device="cuda"))
    st["count"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    if own:
        import paper_2412_07174_b200 as scap
        st["ws"] = torch.empty(scap.scap_kv4_pages_workspace(P, S), dtype=torch.uint8, device="cuda")
    return st


# ---- the plain forms ----------------------------------------------------------------------------------------------

def _activate(u, act):
    if act == "relu":
        return torch.where(u > 0, u, torch.zeros_like(u))
    if act == "silu":
        return u / (1 + torch.exp(-u))
    if act == "gelu":
        return 0.5 * u * (1 + torch.erf(u * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * u * (1 + torch.tanh(math.sqrt(2 / math.pi) * (u + 0.044715 * u * u * u)))
    return u


def _plain_codes(x, group):
    """Codes (two to a byte), scale and zero of [tokens, heads, D]: decided in 64 bits, a value may lie next to a border."""
    x = x.double().unflatten(-1, (-1, group))
    lo, hi = x.amin(-1).clamp(max=0.0), x.amax(-1).clamp(min=0.0)
    m, e = torch.frexp((hi - lo) / 15)
    s = torch.ldexp(torch.round(torch.ldexp(m, torch.full_like(e, 20))), e - 20)
    d = torch.where(s > 0, s, torch.ones_like(s))
    zero = torch.round(-lo / d).clamp(0, 15)
    q = (torch.round(x / d[..., None]) + zero[..., None]).clamp(0, 15).flatten(-2).to(torch.uint8)
    return q[..., 0::2] | (q[..., 1::2] << 4), s.float(), zero.to(torch.uint8)


def _plain_values(store, slots, group):
    codes, scale, zero = (t[slots] for t in store)
    q = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).float().unflatten(-1, (-1, group))
    return (scale[..., None] * (q - zero.float()[..., None])).flatten(-2)


def _plain_slots(st, b, first, last):
    page = st["case"]["page"]
    pos = torch.arange(first, last, device="cuda")
    return st["table"][b, pos // page].long() * page + pos % page


def _plain_append(st):
    slots = torch.cat([_plain_slots(st, b, n - r, n) for b, (n, r) in enumerate(zip(st["lens_list"], st["rows"]))])
    for name in "kv":
        for i in range(0, len(slots), 32768):
            for t, new in zip(st["store"][name], _plain_codes(st[name][i:i + 32768], st["case"]["group"])):
                t[slots[i:i + 32768]] = new
    return slots


def _plain_attend(st):
    case, q = st["case"], st["q"]
    H, g, D, nq = case["Hkv"], case["g"], case["D"], case["nq"]
    out, lse = torch.empty_like(q), torch.empty(q.shape[:3], dtype=torch.float32, device="cuda")
    for b, n in enumerate(st["lens_list"]):
        first = max(0, n - nq + 1 - case["window"]) if case["window"] else 0
        slots = _plain_slots(st, b, first, n)
        k, v = (_plain_values(st["store"][name], slots, case["group"]).transpose(0, 1) for name in "kv")  # [H, tokens, D]
        qb = q[b].float().view(nq, H, g, D).permute(1, 0, 2, 3).reshape(H, nq * g, D)
        s = (qb @ k.transpose(1, 2)) * D ** -0.5
        at = torch.arange(first, n, device="cuda")[None, :]
        own_pos = (n - nq + torch.arange(nq, device="cuda")).repeat_interleave(g)[:, None]
        seen = at <= own_pos
        if case["window"]:
            seen = seen & (at > own_pos - case["window"])
        s = torch.where(seen, s, torch.full_like(s, -math.inf))
        top = s.amax(-1, keepdim=True)
        p = torch.exp(s - top)
        total = p.sum(-1, keepdim=True)
        o = (p @ v) / total
        out[b] = o.view(H, nq, g, D).permute(1, 0, 2, 3).reshape(nq, H * g, D).to(q.dtype)
        lse[b] = (top + torch.log(total)).view(H, nq, g).permute(1, 0, 2).reshape(nq, H * g)
    return [out, lse]


def _plain_fork(table, refs, lens, pool, page, src, dst):
    """Full pages are shared, the last and partial one is copied to the lowest free page; a fork without one leaves its row empty."""
    src, dst = src.long(), dst.long()
    n = lens[src].long()
    part = (n % page) > 0
    free = (refs == 0).nonzero().flatten()
    rank = torch.cumsum(part.long(), 0) - 1
    fits = ~part | (rank < len(free))
    src, dst, n, part, rank = src[fits], dst[fits], n[fits], part[fits], rank[fits]
    full = n // page
    col = torch.arange(table.shape[1], device="cuda")[None, :]
    rows = torch.where(col < full[:, None], table[src], -1)
    shared = rows[rows >= 0].long()
    refs += torch.bincount(shared, minlength=len(refs)).to(torch.int32)
    new = free[rank[part]]
    pool[new] = pool[table[src[part], full[part]].long()]
    refs[new] = 1
    table[dst] = rows
    table[dst[part], full[part]] = new.to(torch.int32)
    lens[dst] = n.to(torch.int32)


def _plain_free(table, refs, lens, page, rows):
    rows = rows.long()
    held = table[rows]
    held = held[torch.arange(table.shape[1], device="cuda")[None, :] < ((lens[rows].long() + page - 1) // page)[:, None]].long()
    refs -= torch.bincount(held, minlength=len(refs)).to(torch.int32)
    table[rows] = -1
    lens[rows] = 0


def _plain_reserve(table, refs, lens, page, add):
    """Room for add[b] more tokens of every sequence: the lowest free pages, in the order of the sequences."""
    have, need = (lens.long() + page - 1) // page, (lens.long() + add.long() + page - 1) // page
    more = need - have
    free = (refs == 0).nonzero().flatten()
    end = torch.cumsum(more, 0)
    ok = (more == 0) | (end <= len(free))
    more = torch.where(ok, more, 0)
    for extra in range(int(more.max())):
        b = (more > extra).nonzero().flatten()
        page_id = free[end[b] - more[b] + extra]
        table[b, have[b] + extra] = page_id.to(torch.int32)
        refs[page_id] = 1
    lens += torch.where(ok, add, 0)


def _plain_compact(table, refs, pool):
    """The used pages beyond their number move, in ascending order, into the free ones before it."""
    used = int((refs > 0).sum())
    dst = (refs[:used] == 0).nonzero().flatten()
    src = (refs[used:] > 0).nonzero().flatten() + used
    pool[dst] = pool[src]
    place = torch.arange(len(refs), dtype=torch.int32, device="cuda")
    place[src] = dst.to(torch.int32)
    refs[dst] = refs[src]
    refs[src] = 0
    table[:] = torch.where(table >= 0, place[table.clamp(min=0).long()], table)
    return used


# ---- one pass -----------------------------------------------------------------------------------------------------

def _run_plain(st):
    case, op = st["case"], st["case"]["op"]
    if op == "fc":
        u = st["x"].float() @ st["W"].float()
        if st["b"] is not None:
            u = u + st["b"]
        y = _activate(u, case["act"])
        if st["r"] is not None:
            y = y + st["r"].float()
        return y.to(DTYPES[case["out"]])
    if op == "store":
        slots = _plain_append(st)
        return [_plain_values(st["store"][name], slots, case["group"]).to(st["k"].dtype) for name in "kv"]
    if op == "attend":
        return _plain_attend(st)
    table, refs, lens, page = st["table"].clone(), st["refs"].clone(), st["lens"].clone(), case["page"]
    if op == "beam":
        _plain_fork(table, refs, lens, st["pool"], page, st["src"], st["dst"])
        _plain_free(table, refs, lens, page, st["rows"])
        _plain_reserve(table, refs, lens, page, st["add"])
        return [table, refs, lens, st["pool"]]
    used = _plain_compact(table, refs, st["pool"])
    return [table, refs, torch.full((1,), used, dtype=torch.int32, device="cuda"), st["pool"]]


def _run_own(st):
    import paper_2412_07174_b200 as scap
    case, op = st["case"], st["case"]["op"]
    if op == "fc":
        act = (scap.SCAP_ACT_NONE, scap.SCAP_ACT_RELU, scap.SCAP_ACT_SILU, scap.SCAP_ACT_GELU, scap.SCAP_ACT_GELU_TANH)[ACTS.index(case["act"])]
        scap.scap_fc_act(st["x"], st["W"], st["b"], st["y"], st["ws"], act=act, res=st["r"])
        return st["y"]
    if op == "store":
        scap.scap_kv4_append(st["cache"], st["k"], st["v"], st["row_start"])
        scap.scap_kv4_read(st["cache"], st["ko"], st["vo"], st["row_start"])
        return [st["ko"], st["vo"]]
    if op == "attend":
        scap.scap_kv4_attend(st["cache"], st["q"], st["out"], case["D"] ** -0.5, st["ws"], window=case["window"], lse=st["lse"])
        return [st["out"], st["lse"]]
    table, refs, lens = st["table"].clone(), st["refs"].clone(), st["lens"].clone()
    cache = scap.ScapKv4(st["pool"], case["page"], 0, 0, 0, table, lens, refs=refs)  # the pages' bytes are all that these calls look at
    if op == "beam":
        scap.scap_kv4_fork(cache, st["src"], st["dst"], st["count"], st["ws"])
        scap.scap_kv4_free(cache, st["rows"])
        scap.scap_kv4_reserve(cache, st["add"], st["count"], st["ws"])
        return [table, refs, lens, st["pool"]]
    scap.scap_kv4_compact(cache, st["count"], st["ws"])
    return [table, refs, st["count"], st["pool"]]


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- what a pass cannot do without --------------------------------------------------------------------------------

def work(case):
    op = case["op"]
    if op == "fc":
        M, K, N = case["M"], case["K"], case["N"]
        wide = 4 if case["out"] == "fp32" else 2
        return {"bytes": 2.0 * (M * K + K * N) + (4.0 * N if case["bias"] else 0.0) + float(wide) * M * N * (2 if case["res"] else 1), "flops": 2.0 * M * K * N}
    if op in ("store", "attend"):
        D, H = case["D"], case["Hkv"]
        token = 2.0 * H * (D / 2 + 4.0 * D / case["group"])  # codes and a word of scale and zero per group, keys and values
        if op == "store":
            return {"bytes": case["new"] * (2 * 2 * 2.0 * H * D + 2 * token), "flops": 0.0}
        B, nq = case["B"], case["nq"]
        each = case["tokens"] / B
        seen = case["tokens"] if not case["window"] else B * min(each, case["window"] + nq - 1)  # of equal shares
        rows = nq * case["g"]
        return {"bytes": seen * token + 2 * 2.0 * B * nq * case["g"] * H * D + 4.0 * B * nq * case["g"] * H, "flops": 4.0 * seen * H * rows * D}
    if op == "beam":
        mean = 0.75 * case["tokens"] / case["page"]
        return {"bytes": 2.0 * case["children"] * case["stride"] + 4.0 * case["pages"] + 8.0 * case["children"] * mean, "flops": 0.0}
    S, P, page = case["seqs"], case["pages"], case["page"]
    each = 0.75 * min(2 * max(1, P * page // (2 * S)), case["tokens"])
    used = min(float(P), S * max(1.0, each / page) * 0.8)  # a fifth or so of the pages are shared
    return {"bytes": 2.0 * used * (1 - used / P) * case["stride"] + 8.0 * P + 8.0 * S * each / page, "flops": 0.0}


# ---- the same pass in 64 bits -------------------------------------------------------------------------------------

def _stored64(x, group):
    """What the cache stands for, by its definition, of [..., D]."""
    shape = x.shape
    x = x.double().reshape(-1, group)
    zeros = torch.zeros(len(x), 1, dtype=torch.float64, device=x.device)
    lo, hi = torch.minimum(x.min(1, keepdim=True).values, zeros), torch.maximum(x.max(1, keepdim=True).values, zeros)
    step = (hi - lo) / 15
    unit = torch.exp2(torch.floor(torch.log2(torch.where(step > 0, step, torch.ones_like(step)))) - 19)  # weight of the 20th bit
    step = torch.round(step / unit) * unit
    by = torch.where(step > 0, step, torch.ones_like(step))
    zero = torch.clamp(torch.round(-lo / by), 0, 15)
    return (step * (torch.clamp(torch.round(x / by) + zero, 0, 15) - zero)).reshape(shape)


def _attend64(case, mk):
    lens, _, k, v = _kv_inputs(case, mk)
    _paged(mk, lens, case["page"])  # takes its share of the random numbers
    H, g, D, nq = case["Hkv"], case["g"], case["D"], case["nq"]
    q = mk.normal(case["B"], nq, g * H, D).to(mk.dt).double()
    out, lse, end = torch.empty_like(q), torch.empty(q.shape[:3], dtype=torch.float64, device="cuda"), 0
    for b, n in enumerate(lens):
        kb, vb = k[end:end + n], v[end:end + n]
        end += n
        for h in range(H):
            kh, vh = _stored64(kb[:, h], case["group"]), _stored64(vb[:, h], case["group"])
            for i in range(nq):
                stop = n - nq + i + 1
                start = max(0, stop - case["window"]) if case["window"] else 0
                s = torch.einsum("gd,td->gt", q[b, i, h * g:(h + 1) * g], kh[start:stop]) / math.sqrt(D)
                lse[b, i, h * g:(h + 1) * g] = torch.logsumexp(s, -1)
                out[b, i, h * g:(h + 1) * g] = torch.einsum("gt,td->gd", torch.exp(s - torch.logsumexp(s, -1, keepdim=True)), vh[start:stop])
    return [out, lse]


def exact(case, seed):
    mk, op = _Maker(case, seed), case["op"]
    if op == "fc":
        st = prepare(case, seed)
        u = torch.matmul(st["x"].double(), st["W"].double())
        u = u if st["b"] is None else u + st["b"].double()
        if case["act"] == "gelu":
            u = 0.5 * u * torch.erfc(-u / math.sqrt(2.0))
        elif case["act"] == "gelu_tanh":  # 0.5 (1 + tanh a) = 1 / (1 + exp(-2 a))
            u = u / (1.0 + torch.exp(-2.0 * math.sqrt(2.0 / math.pi) * (u + 0.044715 * u ** 3)))
        elif case["act"] == "silu":
            u = u / (1.0 + torch.exp(-u))
        elif case["act"] == "relu":
            u = u.clamp(min=0.0)
        return u if st["r"] is None else u + st["r"].double()
    if op == "store":
        _, _, k, v = _kv_inputs(case, mk)
        return [_stored64(k, case["group"]), _stored64(v, case["group"])]
    if op == "attend":
        return _attend64(case, mk)
    return None  # whole numbers and bytes
