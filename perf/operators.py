"""The cache and memory operators: what they are timed on, and their plain forms.

Four operators serve policies that the built-in denoiser does not cover: a
refreshed unit's output written to its 8-bit cache (Eq. 1), the reuse of such
caches, the append of new tokens to a paged memory of keys and values (norm of
each head, rotation, quantisation), and the attention of a chunk of tokens over
that memory.  `own` selects the library's entry points; otherwise the same
results are computed from elementary tensor operations in 32 bits (angles in 64).

8-bit values are e4m3 codes with a power-of-two scale per group: the least
2^k, k >= -126, for which the group's largest magnitude is at most 448 * 2^k.
"""
import math

import torch

own = False

UNIT_GROUP = 32          # values that share a scale in a unit's cache (a memory row has one for the head)
STD_EPS = 1e-6

# ---------------------------------------------------------------- the cases

# op       fields
# write    N samples of H tokens of width E, the share of samples that refresh the unit, the type of r
# add      the same with U units in a run of skipped ones, and the share of (unit, sample) cells that reuse
# append   N sequences with M new tokens each behind up to L (ragged: fewer in some), heads, head size, type, format
# attend   the same; L counts the new tokens; causal: the chunk is the memory's last tokens


def listed():
    return [
        # one Push-T-shaped query: the smallest write, fp32 activations
        dict(name="write_pusht_b1", op="write", N=1, H=16, E=256, frac=1.0, dtype="fp32"),
        # the scale-up batch on per-sample lattices: half of the samples refresh the unit
        dict(name="write_scale_b1024", op="write", N=1024, H=32, E=512, frac=0.5, dtype="bf16"),
        # 64 environments of the manipulation policy, a run of 5 skipped units
        dict(name="add_manip_b64", op="add", U=5, N=64, H=16, E=256, frac=0.875),
        # the scale-up batch, 11 skipped units between two refreshed ones, one cell in eight refreshed instead
        dict(name="add_scale_b1024", op="add", U=11, N=1024, H=32, E=512, frac=0.875),
        # 64 environments, each remembers one more token; fp32 policy with the scale-up model's 8 heads of 64
        dict(name="append_b64_token", op="append", N=64, M=1, L=1000, heads=8, kv_heads=8, dim=64, page=16,
             dtype="fp32", format="e4m3", ragged=True),
        # 16 environments take in an observation of up to 1,025 image tokens, grouped heads of 128
        dict(name="append_b16_chunk", op="append", N=16, M=1025, L=4500, heads=16, kv_heads=4, dim=128, page=64,
             dtype="bf16", format="e4m3", ragged=True),
        # fp32 Push-T-shaped chunk of 16 action tokens behind a short memory, 3 environments
        dict(name="attend_f32_chunk", op="attend", N=3, M=16, L=333, heads=4, kv_heads=4, dim=64, page=16,
             dtype="fp32", format="fp32", causal=True, window=0, ragged=True),
        # one robot, one token, a long memory: latency, and the split of one sequence over the whole GPU
        dict(name="attend_b1_token", op="attend", N=1, M=1, L=16389, heads=8, kv_heads=8, dim=64, page=16,
             dtype="bf16", format="bf16", causal=True, window=0, ragged=False),
        # 64 environments, one token each, grouped heads of 128, 8-bit memory of up to 8,192 tokens
        dict(name="attend_b64_token", op="attend", N=64, M=1, L=8192, heads=32, kv_heads=8, dim=128, page=64,
             dtype="bf16", format="e4m3", causal=True, window=0, ragged=True),
        # cross-attention of 32 action tokens of 64 environments over their observations (scale-up heads)
        dict(name="attend_b64_action", op="attend", N=64, M=32, L=4099, heads=8, kv_heads=8, dim=64, page=64,
             dtype="bf16", format="e4m3", causal=False, window=0, ragged=True),
        # 64 candidates x 32 action tokens over one shared observation memory
        dict(name="attend_candidates", op="attend", N=1, M=2048, L=16384, heads=8, kv_heads=8, dim=64, page=128,
             dtype="bf16", format="bf16", causal=False, window=0, ragged=False),
        # observation chunks of up to 1,000 tokens behind a memory, each token sees the last 4,096
        dict(name="attend_observe", op="attend", N=4, M=1000, L=8000, heads=16, kv_heads=4, dim=128, page=64,
             dtype="bf16", format="bf16", causal=True, window=4096, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["write", "add", "append", "append", "attend", "attend", "attend", "attend"])
    if op in ("write", "add"):
        E = 32 * _log_int(rng, 2, 32)
        H = rng.choice([8, 16, 32, _log_int(rng, 1, 64)])
        U = 1 if op == "write" else _log_int(rng, 1, 24)
        N = _log_int(rng, 1, max(1, 1024 * 32 * 512 // (E * H * (1 if U == 1 else max(1, U // 11 + 1)))))
        case = dict(op=op, N=N, H=H, E=E, frac=round(rng.uniform(0.05, 1.0), 3))
        if op == "add":
            case["U"] = U
        else:
            case["dtype"] = rng.choice(["fp32", "bf16"])
        return case
    dim = rng.choice([64, 128])
    kv = rng.choice([1, 2, 4, 8])
    heads = kv * rng.choice([1, 1, 2, 4, 5])
    dtype = rng.choice(["fp32", "bf16", "bf16"])
    form = rng.choice([dtype, "e4m3"])
    page = rng.choice([16, 32, 64, 128])
    case = dict(op=op, heads=heads, kv_heads=kv, dim=dim, page=page, dtype=dtype, format=form, ragged=rng.random() < 0.7)
    if op == "append":
        case["M"] = rng.choice([1, _log_int(rng, 1, 1100)])
        case["N"] = _log_int(rng, 1, max(1, min(256, 16 * 1024 * 24 * 128 // (case["M"] * (heads + 2 * kv) * dim))))
        case["L"] = case["M"] + _log_int(rng, 1, 4000)
        return case
    case["M"] = M = rng.choice([1, 1, rng.choice([8, 16, 32]), _log_int(rng, 2, 2048)])
    # bounds: the scores (N * heads * M * L), the memory (N * kv_heads * L * dim), in fp32 a quarter of the products
    scores = 8 * 2048 * 16384 * 64 // dim // (8 if dtype == "fp32" else 1)
    cells = 64 * 8 * 6000 * 128 // 2
    L = _log_int(rng, 16, 20000)
    L = max(1, min(L, scores // (heads * M), cells // (kv * dim)))
    case["causal"] = rng.random() < 0.5
    case["L"] = L = max(L, M) if case["causal"] else L
    case["N"] = _log_int(rng, 1, max(1, min(256, scores // (heads * M * L), cells // (kv * dim * L))))
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
    grows = case["op"] == "append" or case["causal"]
    if case["ragged"] and N > 4:
        lens[2] = m[2] if grows else 0
    return [max(a, b) for a, b in zip(lens, m)] if grows else lens


def _count(case, share):
    return max(1, int(round(share * case["frac"])))


def _item(name):
    return {"fp32": 4, "bf16": 2, "e4m3": 1}[name]


def work(case):
    if case["op"] in ("write", "add"):
        each = case["H"] * case["E"]
        cached = each * (1 + 1 / UNIT_GROUP)
        if case["op"] == "write":
            k = _count(case, case["N"])
            return {"bytes": case["N"] * (8 * each + 1) + k * (each * _item(case["dtype"]) + cached), "flops": k * each}
        k = _count(case, case["N"] * case["U"])
        return {"bytes": case["N"] * (8 * each + case["U"]) + k * cached, "flops": 2 * k * each}
    Hq, Hk, D, b, f = case["heads"], case["kv_heads"], case["dim"], _item(case["dtype"]), _item(case["format"])
    news, lens = _news(case), _lens(case)
    rows, scale = sum(news), 1 if case["format"] == "e4m3" else 0
    if case["op"] == "append":
        return {"bytes": rows * ((2 * Hq + 2 * Hk) * D * b + 2 * Hk * (D * f + scale) + 4 * D),
                "flops": rows * (Hq + Hk) * D * 8}
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
    return {"bytes": 2 * rows * Hq * D * b + cells * Hk * 2 * (D * f + scale), "flops": 4.0 * D * Hq * pairs}


# ---------------------------------------------------------------- inputs

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def _quantise(x):
    """x [..., group] fp32 -> e4m3 codes (as bytes) and one scale byte (exponent + 127) a group."""
    amax = x.abs().amax(-1)
    e = torch.frexp(amax)
    k = (e.exponent - 9 + (e.mantissa > 0.875).int()).clamp(min=-126)
    k = torch.where(amax > 0, k, torch.full_like(k, -126))
    codes = torch.ldexp(x, -k.unsqueeze(-1)).to(torch.float8_e4m3fn)
    return codes.view(torch.uint8), (k + 127).to(torch.uint8)


def _values(codes, scales):
    """The fp32 values of e4m3 codes [..., group] with scale bytes [...]."""
    return torch.ldexp(codes.view(torch.float8_e4m3fn).float(), (scales.int() - 127).unsqueeze(-1))


def _gates(n, k, g):
    gate = torch.zeros(n, dtype=torch.uint8, device="cuda")
    gate[torch.randperm(n, generator=g, device="cuda")[:k]] = 1
    return gate


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, dtype=torch.float32):
        return torch.randn(shape, generator=g, device="cuda", dtype=dtype)

    if case["op"] in ("write", "add"):
        N, H, E = case["N"], case["H"], case["E"]
        s = {"case": case, "x": normal(N, H, E)}
        if case["op"] == "write":
            # residuals of one unit differ in size from token to token
            s["r"] = (normal(N, H, E) * torch.exp(0.5 * normal(N, H, 1))).to(TYPES[case["dtype"]])
            s["gate"] = _gates(N, _count(case, N), g)
            s["codes"], s["scales"] = _quantise(normal(N, H, E // UNIT_GROUP, UNIT_GROUP))
            s["codes"] = s["codes"].view(N, H, E)
        else:
            U = case["U"]
            s["gate"] = _gates(U * N, _count(case, U * N), g).view(U, N)
            s["codes"] = torch.empty((U, N, H, E), dtype=torch.uint8, device="cuda")
            s["scales"] = torch.empty((U, N, H, E // UNIT_GROUP), dtype=torch.uint8, device="cuda")
            for u in range(U):
                c, k = _quantise(0.3 * normal(N, H, E // UNIT_GROUP, UNIT_GROUP))
                s["codes"][u], s["scales"][u] = c.view(N, H, E), k
        return s

    N, Hq, Hk, D, P = case["N"], case["heads"], case["kv_heads"], case["dim"], case["page"]
    news, lens = _news(case), _lens(case)
    need = [-(-n // P) for n in lens]
    cols, pages = max(1, max(need)), sum(need) + 3
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    table = torch.full((N, cols), -1, dtype=torch.int32)
    at = 0
    order_host = order.cpu()
    for n, c in enumerate(need):
        table[n, :c] = order_host[at:at + c]
        at += c
    starts = torch.zeros(N + 1, dtype=torch.int32)
    starts[1:] = torch.tensor(news).cumsum(0)
    rows, t = int(starts[-1]), TYPES[case["dtype"]]
    s = {"case": case, "table": table.cuda(), "lens": torch.tensor(lens, dtype=torch.int32).cuda(),
         "starts": starts.cuda(), "max_new": max(news), "max_len": max(lens), "k_scales": None, "v_scales": None}
    # keys have the size that the norm of each head leaves, values differ from token to token
    for name, size in (("k", 1.0), ("v", 0.5)):
        x = normal(pages, Hk, P, D) * size
        if name == "v":
            x *= torch.exp(0.5 * normal(pages, Hk, P, 1))
        if case["format"] == "e4m3":
            s[name + "_pages"], s[name + "_scales"] = _quantise(x)
        else:
            s[name + "_pages"] = x.to(TYPES[case["format"]])
        del x
    if case["op"] == "append":
        # one fused projection's output: q, k and v are column ranges of its rows
        qkv = (normal(rows, (Hq + 2 * Hk) * D) * 1.5).to(t)
        s["q"], s["k"], s["v"] = (x.unflatten(1, (-1, D)) for x in qkv.split([Hq * D, Hk * D, Hk * D], 1))
        s["q_gain"], s["k_gain"] = 1 + 0.1 * normal(D), 1 + 0.1 * normal(D)
        angle = (torch.arange(s["max_len"], device="cuda", dtype=torch.float64)[:, None]
                 * 10000.0 ** (-torch.arange(D // 2, device="cuda", dtype=torch.float64) * 2 / D))
        s["rotation"] = torch.cat([angle.cos(), angle.sin()], 1).float()
    else:
        s["q"] = normal(rows, Hq, D).to(t)
        s["scale"] = D ** -0.5
    if own:
        from paper_2607_20293_gb300 import binding
        s["memory"] = binding.Memory(s["k_pages"], s["v_pages"], s["table"], s["lens"], Hq, k_scales=s["k_scales"],
                                     v_scales=s["v_scales"], starts=s["starts"], dtype=case["dtype"])
    return s


# ---------------------------------------------------------------- one pass


def run(s):
    return {"write": _write, "add": _add, "append": _append, "attend": _attend}[s["case"]["op"]](s)


def _eight_bits(codes, scales):
    # the values that codes and scale bytes are, each in its own 8-bit type
    return codes.view(torch.float8_e4m3fn), scales.view(torch.float8_e8m0fnu)


def _write(s):
    if own:
        from paper_2607_20293_gb300 import binding
        y = binding.cache_write(s["r"], s["codes"], s["scales"], s["x"], s["gate"])
        return (y, *_eight_bits(s["codes"], s["scales"]))
    r, gate = s["r"].float(), s["gate"].bool().view(-1, 1, 1)
    codes, scales = _quantise(r.unflatten(2, (-1, UNIT_GROUP)))
    s["codes"].copy_(torch.where(gate, codes.flatten(2), s["codes"]))
    s["scales"].copy_(torch.where(gate, scales, s["scales"]))
    return (torch.where(gate, s["x"] + r, s["x"]), *_eight_bits(s["codes"], s["scales"]))


def _add(s):
    if own:
        from paper_2607_20293_gb300 import binding
        return binding.cache_add(s["codes"], s["scales"], s["x"], s["gate"])
    c = _values(s["codes"].unflatten(3, (-1, UNIT_GROUP)), s["scales"]).flatten(3)
    return s["x"] + (c * s["gate"].float()[:, :, None, None]).sum(0)


def _rows(s):
    """Sequence and index within its chunk of every row."""
    n = torch.repeat_interleave(torch.arange(s["lens"].numel(), device="cuda"), s["starts"].diff().long(),
                                output_size=s["q"].shape[0])
    return n, torch.arange(s["q"].shape[0], device="cuda") - s["starts"].long()[n]


def _append(s):
    if own:
        q = s["memory"].append(s["q"], s["k"], s["v"], q_gain=s["q_gain"], k_gain=s["k_gain"], eps=STD_EPS,
                               rotation=s["rotation"], max_new=s["max_new"])
        return _appended(s, q)
    D, P = s["case"]["dim"], s["case"]["page"]
    n, j = _rows(s)
    pos = s["lens"].long()[n] - s["starts"].diff().long()[n] + j
    cos, sin = (x.unsqueeze(1) for x in s["rotation"][pos].split(D // 2, 1))

    def turned(x, gain):
        x = x.float()
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + STD_EPS) * gain
        a, b = x.split(D // 2, 2)
        return torch.cat([a * cos - b * sin, b * cos + a * sin], 2)

    page, slot = s["table"][n, pos // P].long(), pos % P
    for name, x in (("k", turned(s["k"], s["k_gain"])), ("v", s["v"].float())):
        if s["case"]["format"] == "e4m3":
            x, scale = _quantise(x)
            s[name + "_scales"][page, :, slot] = scale
        s[name + "_pages"][page, :, slot] = x.to(s[name + "_pages"].dtype)
    return _appended(s, turned(s["q"], s["q_gain"]).to(s["q"].dtype))


def _appended(s, q):
    if s["case"]["format"] == "e4m3":
        return (q, *_eight_bits(s["k_pages"], s["k_scales"]), *_eight_bits(s["v_pages"], s["v_scales"]))
    return q, s["k_pages"], s["v_pages"]


def _attend(s):
    case = s["case"]
    if own:
        return s["memory"].attend(s["q"], scale=s["scale"], causal=case["causal"], window=case["window"],
                                  max_new=s["max_new"], max_len=s["max_len"])
    N, Hq, Hk, D, M = case["N"], case["heads"], case["kv_heads"], case["dim"], s["max_new"]
    at = s["table"].clamp(min=0).long()

    def dense(name):           # [N][Hk][tokens][D]
        x = s[name + "_pages"][at]
        x = _values(x, s[name + "_scales"][at]) if case["format"] == "e4m3" else x.float()
        return x.transpose(1, 2).flatten(2, 3)

    n, j = _rows(s)
    q = torch.zeros((N, M, Hq, D), device="cuda")
    q[n, j] = s["q"].float()
    q = q.view(N, M, Hk, Hq // Hk, D).permute(0, 2, 3, 1, 4).flatten(2, 3)
    scores = (q @ dense("k").transpose(2, 3)).unflatten(2, (-1, M)) * s["scale"]
    key = torch.arange(scores.shape[-1], device="cuda")
    lens, news = s["lens"].long().view(N, 1, 1), s["starts"].diff().long().view(N, 1, 1)
    last = lens - news + torch.arange(M, device="cuda").view(1, M, 1) if case["causal"] else (lens - 1).expand(N, M, 1)
    hidden = key > last
    if case["window"]:
        hidden = hidden | (key <= last - case["window"])
    scores.masked_fill_(hidden.view(N, 1, 1, M, -1), float("-inf"))
    top = scores.amax(-1, keepdim=True).clamp(min=-3e38)
    p = torch.exp(scores - top)
    total = p.sum(-1, keepdim=True)
    del scores
    out = (p.flatten(2, 3) @ dense("v")).unflatten(2, (-1, M)) / total.masked_fill(total == 0, 1.0)
    return out.permute(0, 3, 1, 2, 4).flatten(2, 3)[n, j].to(s["q"].dtype)


# ---------------------------------------------------------------- the definition, in 64 bits


def _round_e4m3(x):
    """Nearest e4m3 value (ties to the even mantissa) of doubles with magnitude at most 448 (plus rounding)."""
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -20))).clamp(min=-6)
    step = torch.exp2(e - 3)
    return (torch.round(x / step) * step).clamp(-448.0, 448.0)


def _exact_groups(x):
    amax = x.abs().amax(-1)
    k = torch.ceil(torch.log2((amax / 448.0).clamp(min=2.0 ** -126))).clamp(min=-126)
    k = torch.where(amax > 448.0 * torch.exp2(k), k + 1, k)
    k = torch.where((amax <= 448.0 * torch.exp2(k - 1)) & (k > -126), k - 1, k)
    scale = torch.exp2(k)
    return _round_e4m3(x / scale.unsqueeze(-1)), scale


def _doubles(codes, scales=None):
    if scales is None:
        return codes.double()
    c = codes.int()
    e, m = (c >> 3) & 15, (c & 7).double()
    v = torch.where(e == 0, m * 2.0 ** -9, (8 + m) * torch.exp2(e.double() - 10))
    v = torch.where(c >= 128, -v, v)
    return v * torch.exp2(scales.double() - 127).unsqueeze(-1)


def exact(case, seed):
    global own
    mine, own = own, False
    s = prepare(case, seed)
    own = mine
    if case["op"] == "write":
        r, x, keep = s["r"].double(), s["x"].double(), s["gate"] == 0
        codes, scales = _exact_groups(r.reshape(*r.shape[:2], -1, UNIT_GROUP))
        codes, y = codes.reshape(r.shape), x + r
        old = torch.exp2(s["scales"].double() - 127)
        y[keep], scales[keep] = x[keep], old[keep]
        codes[keep] = _doubles(s["codes"], torch.full_like(s["scales"][..., :1], 127).squeeze(-1))[keep]
        return y, codes, scales
    if case["op"] == "add":
        y = s["x"].double()
        for u in range(case["U"]):
            shape = s["scales"][u].shape + (UNIT_GROUP,)
            y += _doubles(s["codes"][u].view(shape), s["scales"][u]).view(y.shape) * s["gate"][u].double().view(-1, 1, 1)
        return y
    Hq, Hk, D, P = case["heads"], case["kv_heads"], case["dim"], case["page"]
    news, lens, table = _news(case), _lens(case), s["table"].cpu()
    eight = case["format"] == "e4m3"
    if case["op"] == "append":
        pools = {}
        for name in "kv":
            one = torch.full_like(s[name + "_scales"], 127) if eight else None
            pools[name] = _doubles(s[name + "_pages"], one)
            pools[name + "s"] = torch.exp2(s[name + "_scales"].double() - 127) if eight else None
        freq = 10000.0 ** (-2 * torch.arange(D // 2, device="cuda", dtype=torch.float64) / D)
        q_out, at = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda"), 0
        for n, m in enumerate(news):
            pos = torch.arange(lens[n] - m, lens[n], device="cuda")
            turn = torch.polar(torch.ones_like(pos, dtype=torch.float64)[:, None], pos.double()[:, None] * freq)[:, None]

            def rotated(x, gain):
                x = x[at:at + m].double()
                x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / D + STD_EPS) * gain.double()
                z = torch.complex(x[..., :D // 2], x[..., D // 2:]) * turn
                return torch.cat([z.real, z.imag], -1)

            page, slot = table[n].cuda().long()[pos // P], pos % P
            q_out[at:at + m] = rotated(s["q"], s["q_gain"])
            for name, x in (("k", rotated(s["k"], s["k_gain"])), ("v", s["v"][at:at + m].double())):
                if eight:
                    x, pools[name + "s"][page, :, slot] = _exact_groups(x)
                pools[name][page, :, slot] = x
            at += m
        return (q_out, pools["k"], pools["ks"], pools["v"], pools["vs"]) if eight else (q_out, pools["k"], pools["v"])
    out, at = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda"), 0
    for n, (m, ln) in enumerate(zip(news, lens)):
        if m and ln:
            pages = table[n, :-(-ln // P)].cuda().long()
            k, v = (_doubles(s[x + "_pages"][pages], s[x + "_scales"][pages] if eight else None)
                    .transpose(0, 1).reshape(Hk, -1, D)[:, :ln] for x in "kv")
            q = s["q"][at:at + m].double().transpose(0, 1)
            key, row = torch.arange(ln, device="cuda"), torch.arange(m, device="cuda")[:, None]
            end = ln - m + row + 1 if case["causal"] else torch.full_like(row, ln)
            seen = (key < end) & (key >= (end - case["window"] if case["window"] else 0))
            for h in range(Hq):
                a = torch.softmax((q[h] @ k[h * Hk // Hq].T * s["scale"]).masked_fill(~seen, -math.inf), -1)
                out[at:at + m, h] = torch.nan_to_num(a) @ v[h * Hk // Hq]
        at += m
    return out
