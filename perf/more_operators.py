"""The latent memory's operators: what they are timed on, and their plain forms.

A latent memory keeps, for every token, one vector that all heads share (its latent,
from which a head's key and value are linear maps) and one rotated key part.  Three
operators serve it: the append of new tokens (norm of the latent, rotation of the key
part and of the queries' parts), the attention of queries that were multiplied by the
key map already, over the latents themselves, and the expansion of latents into the
keys and values of an ordinary paged memory, for chunks that are better served so.
`own` selects the library's entry points; otherwise the same results are computed from
elementary tensor operations in 32 bits (angles in 64).
"""
import math

import torch

own = False

ROPE = 64                # values of the rotated part of a key or query
KEY = 64                 # values of an expanded key in front of its rotated part
VALUE = 128              # values of an expanded value
STD_EPS = 1e-6

# ---------------------------------------------------------------- the cases

# op       fields
# append   N sequences with M new tokens each behind up to L (ragged: fewer in some), heads, rank, type, page
# attend   the same; L counts the new tokens; causal: the chunk is the memory's last tokens
# expand   the last M tokens of each memory of up to L


def listed():
    return [
        # 64 environments, each remembers one more token; fp32 policy with the scale-up model's 8 heads
        dict(name="append_b64_token", op="append", N=64, M=1, L=1000, heads=8, rank=128, page=16, dtype="fp32", ragged=True),
        # 16 environments take in an observation of up to 1,025 image tokens
        dict(name="append_b16_chunk", op="append", N=16, M=1025, L=4500, heads=16, rank=512, page=64, dtype="bf16",
             ragged=True),
        # fp32 Push-T-shaped chunk of 16 action tokens behind a short memory, 3 environments
        dict(name="attend_f32_chunk", op="attend", N=3, M=16, L=333, heads=4, rank=128, page=16, dtype="fp32", causal=True,
             window=0, ragged=True),
        # 48 environments of an fp32 policy, one token each
        dict(name="attend_f32_token", op="attend", N=48, M=1, L=2050, heads=8, rank=256, page=32, dtype="fp32", causal=True,
             window=0, ragged=True),
        # one robot, one token, a long memory: latency, and the split of one sequence over the whole GPU
        dict(name="attend_b1_token", op="attend", N=1, M=1, L=16389, heads=8, rank=256, page=16, dtype="bf16", causal=True,
             window=0, ragged=False),
        # 64 environments, one token each, memories of up to 8,192 tokens
        dict(name="attend_b64_token", op="attend", N=64, M=1, L=8192, heads=16, rank=512, page=64, dtype="bf16", causal=True,
             window=0, ragged=True),
        # 32 environments, one token of many heads
        dict(name="attend_b32_heads", op="attend", N=32, M=1, L=8192, heads=64, rank=256, page=64, dtype="bf16", causal=True,
             window=0, ragged=True),
        # cross-attention of 16 action tokens of 64 environments over their observations
        dict(name="attend_b64_action", op="attend", N=64, M=16, L=2050, heads=8, rank=256, page=64, dtype="bf16",
             causal=False, window=0, ragged=True),
        # observation chunks of up to 250 tokens behind a memory, each token sees the last 4,096
        dict(name="attend_observe", op="attend", N=4, M=250, L=8000, heads=16, rank=256, page=128, dtype="bf16", causal=True,
             window=4096, ragged=True),
        # a short fp32 memory written out as keys and values
        dict(name="expand_f32", op="expand", N=3, M=333, L=333, heads=4, rank=128, page=16, dtype="fp32", ragged=True),
        # the newest observation of 16 environments
        dict(name="expand_new", op="expand", N=16, M=257, L=2050, heads=8, rank=512, page=32, dtype="bf16", ragged=True),
        # the memories of 4 environments before a long chunk
        dict(name="expand_b4", op="expand", N=4, M=8000, L=8000, heads=16, rank=256, page=64, dtype="bf16", ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "attend", "expand"])
    rank = rng.choice([128, 256, 512])
    heads = rng.choice([1, 2, 4, 5, 8, 16, 20, 32, 64])
    dtype = rng.choice(["fp32", "bf16", "bf16"])
    case = dict(op=op, heads=heads, rank=rank, page=rng.choice([16, 32, 64, 128]), dtype=dtype, ragged=rng.random() < 0.7)
    if op == "append":
        case["M"] = M = rng.choice([1, _log_int(rng, 1, 1100)])
        case["L"] = L = M + _log_int(rng, 1, 4000)
        case["N"] = _log_int(rng, 1, max(1, min(256, 16 * 1025 * 1600 // (M * (rank + ROPE + heads * ROPE)),
                                                16 * 4500 * 576 // (L * (rank + ROPE)))))
        return case
    if op == "expand":
        cells = 4 * 6000 * 16 * 192 * 256 // (heads * 192 * rank) // (8 if dtype == "fp32" else 1)
        case["M"] = M = max(1, min(_log_int(rng, 1, 8000), cells))
        case["L"] = L = max(M, min(M * rng.choice([1, 1, 2, 5]), 4 * 8000 * 16 // heads))
        case["N"] = _log_int(rng, 1, max(1, min(128, cells // M, 4 * 8000 * 16 // (heads * L))))
        return case
    case["M"] = M = rng.choice([1, 1, rng.choice([8, 16, 32]), _log_int(rng, 2, 512)])
    # bounds: the products of the scores, an eighth of them in fp32, and the values of the memories
    scores = 4 * 250 * 16 * 4000 * 576 // (2 * rank + ROPE) // (8 if dtype == "fp32" else 1)
    cells = 64 * 6000 * 576 // (rank + ROPE) // (2 if dtype == "fp32" else 1)
    L = max(1, min(_log_int(rng, 16, 20000), scores // (heads * M), cells))
    case["causal"] = rng.random() < 0.5
    case["L"] = L = max(L, M) if case["causal"] else L
    case["N"] = _log_int(rng, 1, max(1, min(256, scores // (heads * M * L), cells // L)))
    case["window"] = rng.choice([0, 0, 0, _log_int(rng, 1, L)])
    return case


# ---------------------------------------------------------------- sizes that follow from a case


def _news(case):
    """New tokens of each sequence: M, or between M/2 and M with an empty chunk among them."""
    N, M = case["N"], case["M"]
    m = [M - (n * 31) % (M // 2 + 1) if case["ragged"] else M for n in range(N)]
    if case["ragged"] and N > 4 and M > 1:
        m[1] = 0
    return m


def _lens(case):
    """Tokens of each memory, the new ones included: L, or between L/2 and L, a first chunk and an empty memory among them."""
    N, L, m = case["N"], case["L"], _news(case)
    lens = [L - (n * 7919) % (L // 2 + 1) if case["ragged"] else L for n in range(N)]
    grows = case["op"] != "attend" or case["causal"]
    if case["ragged"] and N > 4:
        lens[2] = m[2] if grows else 0
    return [max(a, b) for a, b in zip(lens, m)] if grows else lens


def _item(name):
    return {"fp32": 4, "bf16": 2}[name]


def work(case):
    H, R, b = case["heads"], case["rank"], _item(case["dtype"])
    news, lens = _news(case), _lens(case)
    rows = sum(news)
    if case["op"] == "append":
        return {"bytes": rows * (2 * (R + ROPE + H * ROPE) * b + 4 * ROPE), "flops": rows * (4 * R + 3 * (H + 1) * ROPE)}
    if case["op"] == "expand":
        return {"bytes": rows * (R + ROPE + H * (KEY + ROPE + VALUE)) * b + H * (KEY + VALUE) * R * b,
                "flops": 2.0 * rows * R * H * (KEY + VALUE)}
    cells, pairs = 0, 0
    for m, n in zip(news, lens):
        if m == 0:
            continue
        w = case["window"] if case["window"] else n
        if case["causal"]:
            pairs += sum(min(w, n - m + j + 1) for j in range(m))
            cells += min(n, w + m - 1)
        else:
            pairs += m * min(w, n)
            cells += min(w, n)
    return {"bytes": (rows * H * (2 * R + ROPE) + cells * (R + ROPE)) * b, "flops": 2.0 * (2 * R + ROPE) * H * pairs}


# ---------------------------------------------------------------- inputs

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def _pages(case, lens, g):
    """A table of pages in random order, with three pages that no sequence has, and their number."""
    P = case["page"]
    need = [-(-n // P) for n in lens]
    cols, pages = max(1, max(need)), sum(need) + 3
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32).cpu()
    table = torch.full((case["N"], cols), -1, dtype=torch.int32)
    at = 0
    for n, c in enumerate(need):
        table[n, :c] = order[at:at + c]
        at += c
    return table.cuda(), pages


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, dtype=torch.float32):
        return torch.randn(shape, generator=g, device="cuda", dtype=dtype)

    N, H, R, P, t = case["N"], case["heads"], case["rank"], case["page"], TYPES[case["dtype"]]
    news, lens = _news(case), _lens(case)
    table, pages = _pages(case, lens, g)
    starts = torch.zeros(N + 1, dtype=torch.int32)
    starts[1:] = torch.tensor(news).cumsum(0)
    rows = int(starts[-1])
    s = {"case": case, "table": table, "lens": torch.tensor(lens, dtype=torch.int32).cuda(), "starts": starts.cuda(),
         "rows": rows, "max_new": max(news), "max_len": max(lens)}
    # latents have the size that their norm leaves
    s["pages"] = normal(pages, P, R + ROPE).to(t)
    if case["op"] == "append":
        # one projection's output holds latent and key part; queries are [rows][heads][KEY + ROPE], of which the last are turned
        down = (normal(rows, R + ROPE) * 1.5).to(t)
        s["c"], s["k"] = down.split([R, ROPE], 1)
        s["q"] = normal(rows, H, KEY + ROPE).to(t)[:, :, KEY:]
        s["gain"] = 1 + 0.1 * normal(R)
        angle = (torch.arange(s["max_len"], device="cuda", dtype=torch.float64)[:, None]
                 * 10000.0 ** (-torch.arange(ROPE // 2, device="cuda", dtype=torch.float64) * 2 / ROPE))
        s["rotation"] = torch.cat([angle.cos(), angle.sin()], 1).float()
    elif case["op"] == "attend":
        s["q"] = normal(rows, H, R + ROPE).to(t)
        s["scale"] = (KEY + ROPE) ** -0.5
    else:
        s["w_k"], s["w_v"] = ((normal(H, d, R) * R ** -0.5).to(t) for d in (KEY, VALUE))
        s["to"], pages = _pages(case, lens, g)
        s["k_pages"], s["v_pages"] = (normal(pages, H, P, KEY + ROPE).to(t) for _ in range(2))
        s["first"] = s["lens"] - s["starts"].diff()
    if own:
        from paper_2607_20293_gb300 import binding
        s["latent"] = binding.LatentMemory(s["pages"], s["table"], s["lens"], H, starts=s["starts"])
        if case["op"] == "expand":
            s["memory"] = binding.Memory(s["k_pages"], s["v_pages"], s["to"], s["lens"], H, dtype=case["dtype"])
    return s


# ---------------------------------------------------------------- one pass


def run(s):
    return {"append": _append, "attend": _attend, "expand": _expand}[s["case"]["op"]](s)


def _rows(s):
    """Sequence and index within its chunk of every row."""
    n = torch.repeat_interleave(torch.arange(s["lens"].numel(), device="cuda"), s["starts"].diff().long(),
                                output_size=s["rows"])
    return n, torch.arange(s["rows"], device="cuda") - s["starts"].long()[n]


def _places(s):
    """Sequence and position within its memory of every row."""
    n, j = _rows(s)
    return n, s["lens"].long()[n] - s["starts"].diff().long()[n] + j


def _append(s):
    if own:
        return s["latent"].append(s["c"], s["k"], s["q"], c_gain=s["gain"], eps=STD_EPS, rotation=s["rotation"]), s["pages"]
    P = s["case"]["page"]
    n, pos = _places(s)
    cos, sin = s["rotation"][pos].split(ROPE // 2, 1)

    def turned(x, cos, sin):
        a, b = x.float().split(ROPE // 2, -1)
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)

    c = s["c"].float()
    c = c * torch.rsqrt(c.square().mean(-1, keepdim=True) + STD_EPS) * s["gain"]
    s["pages"][s["table"][n, pos // P].long(), pos % P] = torch.cat([c, turned(s["k"], cos, sin)], 1).to(s["pages"].dtype)
    return turned(s["q"], cos.unsqueeze(1), sin.unsqueeze(1)).to(s["q"].dtype), s["pages"]


def _attend(s):
    case = s["case"]
    if own:
        return s["latent"].attend(s["q"], s["scale"], causal=case["causal"], window=case["window"], max_new=s["max_new"],
                                  max_len=s["max_len"])
    N, H, R, M = case["N"], case["heads"], case["rank"], s["max_new"]
    c = s["pages"][s["table"].clamp(min=0).long()].flatten(1, 2).float()          # [N][tokens][R + ROPE]
    n, j = _rows(s)
    q = torch.zeros((N, M, H, R + ROPE), device="cuda")
    q[n, j] = s["q"].float()
    scores = (q.flatten(1, 2) @ c.transpose(1, 2)).unflatten(1, (M, H)) * s["scale"]
    key = torch.arange(scores.shape[-1], device="cuda")
    lens, news = s["lens"].long().view(N, 1, 1), s["starts"].diff().long().view(N, 1, 1)
    last = lens - news + torch.arange(M, device="cuda").view(1, M, 1) if case["causal"] else (lens - 1).expand(N, M, 1)
    hidden = key > last
    if case["window"]:
        hidden = hidden | (key <= last - case["window"])
    scores.masked_fill_(hidden.unsqueeze(2), float("-inf"))
    top = scores.amax(-1, keepdim=True).clamp(min=-3e38)
    p = torch.exp(scores - top)
    total = p.sum(-1, keepdim=True)
    del scores
    out = (p.flatten(1, 2) @ c[..., :R]).unflatten(1, (M, H)) / total.masked_fill(total == 0, 1.0)
    return out[n, j].to(s["q"].dtype)


def _expand(s):
    if own:
        s["latent"].expand(s["w_k"], s["w_v"], s["memory"], first=s["first"], max_len=s["max_len"], max_new=s["max_new"])
        return s["k_pages"], s["v_pages"]
    H, R, P = s["case"]["heads"], s["case"]["rank"], s["case"]["page"]
    n, pos = _places(s)
    x = s["pages"][s["table"][n, pos // P].long(), pos % P].float()
    c, turned = x.split([R, ROPE], 1)
    k = (c @ s["w_k"].float().flatten(0, 1).T).unflatten(1, (H, KEY))
    k = torch.cat([k, turned.unsqueeze(1).expand(-1, H, -1)], 2)
    v = (c @ s["w_v"].float().flatten(0, 1).T).unflatten(1, (H, VALUE))
    page, slot = s["to"][n, pos // P].long(), pos % P
    s["k_pages"][page, :, slot] = k.to(s["k_pages"].dtype)
    s["v_pages"][page, :, slot] = v.to(s["v_pages"].dtype)
    return s["k_pages"], s["v_pages"]


# ---------------------------------------------------------------- the definition, in 64 bits


def exact(case, seed):
    global own
    mine, own = own, False
    s = prepare(case, seed)
    own = mine
    H, R, P = case["heads"], case["rank"], case["page"]
    news, lens, table = _news(case), _lens(case), s["table"].long()
    at = 0
    if case["op"] == "append":
        pool = s["pages"].double()
        q_out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
        freq = 10000.0 ** (-2 * torch.arange(ROPE // 2, device="cuda", dtype=torch.float64) / ROPE)
        for n, m in enumerate(news):
            pos = torch.arange(lens[n] - m, lens[n], device="cuda")
            turn = torch.polar(torch.ones_like(freq).expand(m, -1), pos.double()[:, None] * freq)

            def rotated(x, turn):
                z = torch.complex(x[..., :ROPE // 2], x[..., ROPE // 2:]) * turn
                return torch.cat([z.real, z.imag], -1)

            c = s["c"][at:at + m].double()
            c = c / torch.sqrt((c * c).sum(-1, keepdim=True) / R + STD_EPS) * s["gain"].double()
            page, slot = table[n][pos // P], pos % P
            pool[page, slot, :R] = c
            pool[page, slot, R:] = rotated(s["k"][at:at + m].double(), turn)
            q_out[at:at + m] = rotated(s["q"][at:at + m].double(), turn[:, None])
            at += m
        return q_out, pool
    if case["op"] == "expand":
        k_pool, v_pool = s["k_pages"].double(), s["v_pages"].double()
        to = s["to"].long()
        for n, m in enumerate(news):
            pos = torch.arange(lens[n] - m, lens[n], device="cuda")
            x = s["pages"][table[n][pos // P], pos % P].double()
            for h in range(H):
                k_pool[to[n][pos // P], h, pos % P, :KEY] = x[:, :R] @ s["w_k"][h].double().T
                k_pool[to[n][pos // P], h, pos % P, KEY:] = x[:, R:]
                v_pool[to[n][pos // P], h, pos % P] = x[:, :R] @ s["w_v"][h].double().T
        return k_pool, v_pool
    out = torch.zeros((s["rows"], H, R), dtype=torch.float64, device="cuda")
    for n, (m, ln) in enumerate(zip(news, lens)):
        if m and ln:
            x = s["pages"][table[n, :-(-ln // P)]].double().flatten(0, 1)[:ln]
            key, row = torch.arange(ln, device="cuda"), torch.arange(m, device="cuda")[:, None]
            end = ln - m + row + 1 if case["causal"] else torch.full_like(row, ln)
            seen = (key < end) & (key >= (end - case["window"] if case["window"] else 0))
            for h in range(H):
                q = s["q"][at:at + m, h].double()
                a = torch.softmax((q @ x.T * s["scale"]).masked_fill(~seen, -math.inf), -1)
                out[at:at + m, h] = torch.nan_to_num(a) @ x[:, :R]
        at += m
    return out
