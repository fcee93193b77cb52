"""The paged memory on the GPU against the float64 definitions.

Tolerances, for every output element by itself, from the roundings that the
documentation names (u = 2^-24; bf16 rounds by at most 2^-8 of the value):

append   norm and rotation are fewer than 32 fp32 operations on a value, each off by
         u of the pair's length, then one rounding to the row's type; an 8-bit value is
         off by 2^-4 of itself or 2^(k-10) more.
attend   a score is off by (D + 8) u of sum |q||k| scale, a weight by twice that (the
         maximum has it too) plus 2^-20 for the exponential, and by 2^-8 with bf16
         rows; a weight's error moves the output by at most that share of the
         weighted mean of |v|.  Sums of L terms add L u of it, the result one
         rounding to the row's type.
"""
import numpy as np
import pytest

from oracle import evo_memory as M

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def torch():
    import torch as _t
    if not _t.cuda.is_available():
        pytest.skip("no CUDA device")
    return _t


@pytest.fixture(scope="module")
def B(torch):
    from paper_2607_20293_gb300 import binding, build
    build.build()
    binding.load()
    return binding


class World:
    """A pool of pages with stale contents, a shuffled table and its float64 view."""

    def __init__(self, torch, lens, news, hq, hk, D, page, dtype, fmt, seed=0, stale="nan", spare_rows=0, max_pages=None):
        g = torch.Generator().manual_seed(seed)
        self.torch, self.D, self.hq, self.hk, self.page, self.dtype, self.fmt = torch, D, hq, hk, page, dtype, fmt
        self.lens, self.news = list(lens), list(news)
        need = [-(-n // page) for n in lens]
        pages = sum(need) + 2
        cols = max_pages or max(1, max(need))
        order = torch.randperm(pages, generator=g).to(torch.int32)
        self.table = torch.full((len(lens), cols), -7, dtype=torch.int32)
        at = 0
        for n, c in enumerate(need):
            self.table[n, :c] = order[at:at + c]
            at += c
        shape = (pages, hk, page, D)
        self.t = torch.float32 if dtype == "fp32" else torch.bfloat16
        val = [torch.randn(shape, generator=g).to(self.t).float() for _ in range(2)]
        val[1] *= torch.exp(torch.randn(shape[:3] + (1,), generator=g))
        live = torch.zeros(pages, page, dtype=torch.bool)
        for n, ln in enumerate(lens):
            for i in range(need[n]):
                live[int(self.table[n, i]), :max(0, min(page, ln - i * page))] = True
        dead = (~live)[:, None, :, None].expand(shape)
        self.scales = [None, None]
        if fmt == "e4m3":
            enc = [M.quantise(v.numpy().astype(np.float64)) for v in val]
            self.pages = [torch.from_numpy(c.copy()) for c, _ in enc]
            self.scales = [torch.from_numpy(s.copy()) for _, s in enc]
            if stale == "nan":
                for c, s in zip(self.pages, self.scales):
                    c[dead] = 0x7f
                    s[dead[..., 0]] = 255
        else:
            self.pages = [v.to(self.t) for v in val]
            if stale == "nan":
                for p in self.pages:
                    p[dead] = float("nan")
        self.starts = torch.tensor(np.concatenate([[0], np.cumsum(news)]), dtype=torch.int32)
        self.rows = int(self.starts[-1]) + spare_rows
        self.q = torch.randn(self.rows, hq, D, generator=g).to(self.t)
        self.k = (1.3 * torch.randn(self.rows, hk, D, generator=g)).to(self.t)
        self.v = torch.randn(self.rows, hk, D, generator=g).to(self.t)

    def device(self, B, starts=True):
        c = lambda t: None if t is None else t.cuda()  # noqa: E731
        self.dpages, self.dscales = [c(p) for p in self.pages], [c(s) for s in self.scales]
        self.dtable = self.table.cuda()
        self.dlens = self.torch.tensor(self.lens, dtype=self.torch.int32).cuda()
        self.status = self.torch.zeros(1, dtype=self.torch.int32).cuda()
        self.mem = B.Memory(self.dpages[0], self.dpages[1], self.dtable, self.dlens, self.hq, k_scales=self.dscales[0],
                            v_scales=self.dscales[1], starts=self.starts.cuda() if starts else None, status=self.status,
                            dtype=self.dtype)
        return self.mem

    def dense(self, n, pages=None, scales=None):
        """Keys and values [len][hk][D] of sequence n in float64 (from given device copies, or the initial contents)."""
        out = []
        for i in range(2):
            p = (pages or self.pages)[i].cpu()
            need = -(-self.lens[n] // self.page)
            at = self.table[n, :need].long()
            x = p[at]
            if self.fmt == "e4m3":
                x = M.dequantise(x.numpy(), (scales or self.scales)[i].cpu()[at].numpy())
            else:
                x = x.double().numpy()
            out.append(x.transpose(0, 2, 1, 3).reshape(-1, self.hk, self.D)[:self.lens[n]])
        return out

    def check_attend(self, got, q=None, scale=None, causal=True, window=0, pages=None, scales=None, only=None):
        scale = scale if scale is not None else self.D ** -0.5
        q = (self.q if q is None else q).double().cpu().numpy()
        got = got.double().cpu().numpy()
        for n in range(len(self.lens)):
            a, b = int(self.starts[n]), int(self.starts[n + 1])
            if only is not None and n not in only:
                continue
            k, v = self.dense(n, pages, scales)
            out, size, dots = M.attend(q[a:b], k, v, self.hk, scale, causal, window)
            half = 2.0 ** -8 if self.dtype == "bf16" else U
            weight = 2 * (self.D + 8) * U * dots + 2.0 ** -20 + (2.0 ** -8 if self.dtype == "bf16" else 0.0)
            tol = half * np.abs(out) + (1 + half) * (weight + self.lens[n] * U) * size + 1e-37
            bad = ~(np.abs(got[a:b] - out) <= tol) & ~(np.isnan(out) & np.isnan(got[a:b]))
            worst = np.nanmax(np.abs(got[a:b] - out) / tol) if out.size else 0
            assert not bad.any(), (n, int(bad.sum()), worst, np.argwhere(bad)[:4])


FORMATS = [("bf16", "bf16"), ("bf16", "e4m3"), ("fp32", "fp32"), ("fp32", "e4m3")]
HEADS = [(1, 1), (8, 8), (8, 2), (5, 1), (40, 2)]


# ---------------------------------------------------------------- append

def check_append(w, mem, q_out, q_gain, k_gain, eps, base, pos0=None):
    torch = w.torch
    pos = np.zeros(w.rows)
    at = 0
    for n, m in enumerate(w.news):
        pos[at:at + m] = np.arange(w.lens[n] - m, w.lens[n]) + (0 if pos0 is None else int(pos0[n]))
        at += m
    half = 2.0 ** -8 if w.dtype == "bf16" else U
    rows = at

    def want(x, gain):
        y = M.normed_and_turned(x.double().numpy()[:rows], gain, eps, pos[:rows], base)
        a = np.hypot(*np.split(y, 2, -1))
        return y, 32 * U * np.concatenate([a, a], -1) + 1e-37
    if q_out is not None:
        y, tol = want(w.q, q_gain)
        got = q_out.double().cpu().numpy()[:rows]
        assert (np.abs(got - y) <= tol + half * (np.abs(y) + tol)).all()
    pages = [p.cpu() for p in w.dpages]
    scales = [None if s is None else s.cpu() for s in w.dscales]
    touched = torch.zeros(pages[0].shape[:3], dtype=torch.bool)
    at = 0
    for x, i in ((want(w.k, k_gain), 0), ((w.v.double().numpy()[:rows], 0.0), 1)):
        y, tol = x
        at = 0
        for n, m in enumerate(w.news):
            for j in range(m):
                p = w.lens[n] - m + j
                page, slot = int(w.table[n, p // w.page]), p % w.page
                touched[page, :, slot] = True
                e, t = y[at], (tol[at] if i == 0 else 0.0)
                if w.fmt == "e4m3":
                    c, s = pages[i][page, :, slot].numpy(), scales[i][page, :, slot].numpy()
                    if i == 1:                                     # no arithmetic before the rounding: bit for bit
                        wc, ws = M.quantise(e)
                        assert np.array_equal(c, wc) and np.array_equal(s, ws)
                    k = s.astype(np.float64)[:, None] - 127
                    amax = np.abs(e).max(-1, keepdims=True)
                    assert (amax <= 448 * 2.0 ** k * (1 + 1e-4)).all() and ((amax > 448 * 2.0 ** (k - 1) * (1 - 1e-4)) | (k == -126)).all()
                    got = M.dequantise(c, s)
                    t = t + np.maximum(2.0 ** -4 * (np.abs(e) + t), 2.0 ** (k - 10))
                else:
                    got = pages[i][page, :, slot].double().numpy()
                    t = t + half * (np.abs(e) + t) if i == 0 else 0.0
                assert (np.abs(got - e) <= t).all(), (n, j, i)
                at += 1
    # nothing else was written
    for i in range(2):
        same = (pages[i].view(torch.uint8) == w.pages[i].view(torch.uint8)).flatten(3).all(-1)
        assert same[~touched].all()
        if w.fmt == "e4m3":
            assert (scales[i] == w.scales[i])[~touched].all()


@pytest.mark.parametrize("dtype,fmt", FORMATS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("hq,hk", HEADS)
def test_append(torch, B, dtype, fmt, D, hq, hk):
    w = World(torch, [37, 1, 0, 16, 130, 33], [5, 1, 0, 16, 65, 0], hq, hk, D, 16, dtype, fmt, seed=D + hq, spare_rows=2)
    mem = w.device(B)
    g = torch.Generator().manual_seed(1)
    qg, kg = 1 + 0.3 * torch.randn(D, generator=g), 1 + 0.3 * torch.randn(D, generator=g)
    rot = torch.from_numpy(B.rotation_table(256, D, 1e4)).cuda()
    out = torch.full((w.rows, hq, D), 7.0, dtype=w.t, device="cuda")
    q = mem.append(w.q.cuda(), w.k.cuda(), w.v.cuda(), qg.cuda(), kg.cuda(), 1e-6, rot, out=out)
    assert q is out and (out[-2:] == 7).all()                     # rows behind the last sequence
    check_append(w, mem, q, qg.double().numpy(), kg.double().numpy(), 1e-6, 1e4)
    assert int(w.status) == 0


@pytest.mark.parametrize("n_seq", [1, 2, 31, 32, 33, 64, 65, 1000])
def test_append_finds_every_row(torch, B, n_seq):
    news = [(n * 7) % 4 for n in range(n_seq)]
    news[-1] = 1
    w = World(torch, [m + n % 20 for n, m in enumerate(news)], news, 1, 1, 64, 16, "fp32", "fp32", seed=n_seq)
    mem = w.device(B)
    mem.append(None, w.k.cuda(), w.v.cuda())
    check_append(w, mem, None, None, None, 0, None)


@pytest.mark.parametrize("dtype,fmt", FORMATS)
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_append_equal_chunks_strided_rows_and_shifted_positions(torch, B, dtype, fmt, page):
    hq, hk, D = 4, 2, 64
    w = World(torch, [200, 130, 129], [3, 3, 3], hq, hk, D, page, dtype, fmt, seed=page)
    mem = w.device(B, starts=False)
    fused = torch.cat([w.q.flatten(1), w.k.flatten(1), w.v.flatten(1), torch.zeros(w.rows, 8, dtype=w.t)], 1).cuda()
    q, k, v = (fused[:, a:b].unflatten(1, (-1, D)) for a, b in ((0, 256), (256, 384), (384, 512)))
    pos0 = torch.tensor([0, 70000, 5], dtype=torch.int32)
    rot = torch.from_numpy(B.rotation_table(70200, D, 1e4)).cuda()
    got = mem.append(q, k, v, rotation=rot, pos0=pos0.cuda(), out=q)        # in place, rows of the fused projection
    assert got is q
    check_append(w, mem, q, None, None, 0, 1e4, pos0)
    assert int(w.status) == 0


def test_append_of_queries_or_keys_alone(torch, B):
    w = World(torch, [20, 9], [4, 2], 2, 1, 128, 16, "bf16", "e4m3")
    mem = w.device(B)
    gain = torch.linspace(0.5, 2, 128)
    q = mem.append(w.q.cuda(), None, None, q_gain=gain.cuda())
    assert torch.equal(w.dpages[0].cpu(), w.pages[0])
    y = M.normed_and_turned(w.q.double().numpy(), gain.double().numpy(), 1e-6, np.zeros(6), None)
    assert (np.abs(q.double().cpu().numpy() - y) <= (2.0 ** -8 + 64 * U) * np.abs(y)).all()
    assert mem.append(None, w.k.cuda(), w.v.cuda()) is None
    check_append(w, mem, None, None, None, 0, None)


def test_append_reports_what_it_cannot_place(torch, B):
    lens, news = [20, 40, 3, 18], [2, 2, 5, 1]
    w = World(torch, [20, 40, 5, 18], news, 2, 1, 64, 16, "bf16", "bf16", max_pages=3, stale="none")
    w.table[0, 1] = 10 ** 6                                        # its two tokens are 18 and 19: page 1
    mem = w.device(B)
    w.dlens.copy_(torch.tensor([20, 60, 3, 18], dtype=torch.int32))         # 60 is past 3 pages; 3 tokens of 5 new
    out = torch.full((w.rows, 2, 64), 7.0, dtype=w.t, device="cuda")
    rot = torch.from_numpy(B.rotation_table(18, 64)).cuda()
    mem.append(w.q.cuda(), w.k.cuda(), w.v.cuda(), rotation=rot, out=out)
    assert int(w.status) == B.ERR_CORRUPT
    o = out.cpu()
    assert (o[:4] == 7).all()                                      # bad page, past the table
    assert (o[4:6] == 7).all() and (o[6:9] != 7).any()             # tokens -2, -1 of sequence 2, then 0 .. 2
    assert (o[9] != 7).any()                                       # token 17, the last of the rotation table
    w.status.zero_()
    mem.append(w.q.cuda(), None, None, rotation=rot[:17], out=out)
    assert int(w.status) == B.ERR_CORRUPT


def test_append_of_values_that_are_not_numbers(torch, B):
    w = World(torch, [4], [4], 2, 2, 64, 16, "bf16", "e4m3")
    w.v[1, 0, 3], w.v[2, 1, 60], w.k[3, 0, 0] = float("nan"), float("-inf"), float("inf")
    mem = w.device(B)
    mem.append(None, w.k.cuda(), w.v.cuda())
    page = int(w.table[0, 0])
    s = w.dscales[1][page].cpu()
    assert s[0, 1] == 255 and s[1, 2] == 255 and (s[:, [0, 3]] != 255).all()
    assert w.dscales[0][page, 0, 3] == 255 and (w.dscales[0][page, 1, :4] != 255).all()


# ---------------------------------------------------------------- attend

@pytest.mark.parametrize("dtype,fmt", FORMATS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("hq,hk", HEADS)
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 7), (False, 70)])
def test_attend(torch, B, dtype, fmt, D, hq, hk, causal, window):
    w = World(torch, [37, 1, 0, 16, 130, 300, 9], [5, 1, 0, 16, 65, 3, 0], hq, hk, D, 16, dtype, fmt, seed=D + hq, spare_rows=3)
    mem = w.device(B)
    out = torch.full((w.rows, hq, D), 7.0, dtype=w.t, device="cuda")
    got = mem.attend(w.q.cuda(), causal=causal, window=window, max_new=65, max_len=300, out=out)
    assert got is out and (out[-3:] == 7).all()
    w.check_attend(got, causal=causal, window=window)
    assert int(w.status) == 0


@pytest.mark.parametrize("dtype,fmt", FORMATS)
@pytest.mark.parametrize("page", [32, 64, 128])
@pytest.mark.parametrize("m", [1, 2, 31, 64, 127, 128, 129, 200])
def test_attend_chunks(torch, B, dtype, fmt, page, m):
    w = World(torch, [m + 300, m], [m, m], 2, 1, 64, page, dtype, fmt, seed=m)
    mem = w.device(B, starts=False)
    w.check_attend(mem.attend(w.q.cuda()), causal=True)
    w.check_attend(mem.attend(w.q.cuda(), causal=False, scale=-0.3), causal=False, scale=-0.3)
    assert int(w.status) == 0


@pytest.mark.parametrize("dtype,fmt", FORMATS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("length", [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 255, 256, 257, 1023, 5000])
def test_attend_single_tokens(torch, B, dtype, fmt, D, length):
    w = World(torch, [length, max(1, length // 3), 1], [1, 1, 1], 4, 2, D, 16, dtype, fmt, seed=length)
    mem = w.device(B, starts=False)
    w.check_attend(mem.attend(w.q.cuda()))
    w.check_attend(mem.attend(w.q.cuda(), window=40), window=40)


@pytest.mark.parametrize("dtype,fmt", FORMATS)
@pytest.mark.parametrize("hq,hk,D,m,length", [(8, 8, 64, 32, 2100), (4, 4, 64, 300, 1500), (16, 4, 128, 150, 1300), (2, 2, 128, 520, 700)])
def test_attend_long(torch, B, dtype, fmt, hq, hk, D, m, length):
    w = World(torch, [length, length // 2 + m], [m, m - m // 3], hq, hk, D, 64, dtype, fmt, seed=m)
    mem = w.device(B)
    for causal, window in ((True, 0), (False, 0), (True, 333)):
        w.check_attend(mem.attend(w.q.cuda(), causal=causal, window=window, max_new=m), causal=causal, window=window)


@pytest.mark.parametrize("dtype,fmt", FORMATS)
@pytest.mark.parametrize("m", [3, 40, 200])
def test_attend_rows_without_keys_and_chunks_longer_than_the_memory(torch, B, dtype, fmt, m):
    w = World(torch, [2, 0], [m, m], 2, 2, 64, 16, dtype, fmt, seed=m)
    mem = w.device(B)
    got = mem.attend(w.q.cuda(), max_new=m)
    w.check_attend(got)
    assert (got[:m - 2] == 0).all() and (got[m:] == 0).all()
    assert int(w.status) == 0
    assert (mem.attend(w.q.cuda(), max_new=m, causal=False)[m:] == 0).all()


@pytest.mark.parametrize("dtype,fmt", FORMATS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("m,length", [(1, 90), (20, 90), (150, 400), (300, 900)])
def test_masked_tokens_that_are_not_numbers(torch, B, dtype, fmt, D, m, length):
    """NaN and infinite values of a token reach the rows that see it and no other."""
    w = World(torch, [length], [m], 2, 1, D, 16, dtype, fmt, seed=m)
    tok = length - m // 2 - 1
    for t, bad in ((tok, float("nan")), (3, float("inf"))):
        page, slot = int(w.table[0, t // 16]), t % 16
        for i in range(2):
            if fmt == "e4m3":
                w.scales[i][page, :, slot] = 255
            else:
                w.pages[i][page, :, slot] = bad
    mem = w.device(B)
    window = 30
    got = mem.attend(w.q.cuda(), causal=True, window=window, max_new=m).double().cpu().numpy()
    pos = np.arange(length - m, length)
    sees = ((pos >= tok) & (tok > pos - window)) | ((pos >= 3) & (3 > pos - window))
    assert np.isnan(got[sees]).all()
    assert np.isfinite(got[~sees]).all()
    ok = [p.clone() for p in w.pages]
    okv = [None if s is None else s.clone() for s in w.scales]
    for t in (tok, 3):                                            # their values do not matter to the others
        page, slot = int(w.table[0, t // 16]), t % 16
        for i in range(2):
            ok[i][page, :, slot] = 0
            if okv[i] is not None:
                okv[i][page, :, slot] = 127
    k, v = w.dense(0, ok, okv)
    out, size, dots = M.attend(w.q.double().numpy(), k, v, 1, D ** -0.5, True, window)
    half = 2.0 ** -8 if dtype == "bf16" else U
    tol = half * np.abs(out) + (1 + half) * (2 * (D + 8) * U * dots + 2.0 ** -20 + length * U + (half if dtype == "bf16" else 0)) * size + 1e-37
    assert (np.abs(got - out) <= tol)[~sees].all()


@pytest.mark.parametrize("dtype,fmt", [("bf16", "bf16"), ("fp32", "fp32")])
@pytest.mark.parametrize("m", [1, 20, 150])
def test_an_infinite_value_beside_finite_ones(torch, B, dtype, fmt, m):
    """One infinite entry of one value: that column of the rows that see it is infinite, all else stays."""
    length = m + 60
    w = World(torch, [length], [m], 1, 1, 64, 16, dtype, fmt, seed=m)
    tok = length - 1 - m // 2
    w.pages[1][int(w.table[0, tok // 16]), 0, tok % 16, 9] = float("-inf")
    mem = w.device(B)
    got = mem.attend(w.q.cuda(), max_new=m).double().cpu().numpy()
    pos = np.arange(length - m, length)
    assert (got[pos >= tok][..., 9] == -np.inf).all()
    got[pos >= tok, :, 9] = 0
    assert np.isfinite(got).all()


@pytest.mark.parametrize("dtype,fmt", FORMATS)
def test_attend_scores_of_every_size(torch, B, dtype, fmt):
    # one row's weights are one-hot, one's uniform, one's scores huge and negative; values of very different scale
    w = World(torch, [500], [70], 2, 2, 64, 16, dtype, fmt, seed=3)
    w.q[0] *= 60
    w.q[1] = 0
    w.q[2] *= -60
    for t, f in ((5, 1e-20), (6, 1e20), (7, 0.0)):
        page, slot = int(w.table[0, 0]), t
        v = (torch.randn(2, 64, generator=torch.Generator().manual_seed(t)) * f)
        if fmt == "e4m3":
            c, s = M.quantise(v.numpy().astype(np.float64))
            w.pages[1][page, :, slot], w.scales[1][page, :, slot] = torch.from_numpy(c), torch.from_numpy(s)
        else:
            w.pages[1][page, :, slot] = v.to(w.t)
    mem = w.device(B)
    w.check_attend(mem.attend(w.q.cuda(), max_new=70))


@pytest.mark.parametrize("dtype,fmt", FORMATS)
@pytest.mark.parametrize("m", [1, 12, 20, 45, 200])
def test_attend_scales(torch, B, dtype, fmt, m):
    """A scale of zero (the mean of the values), negative, tiny and large ones, at both head widths."""
    for D in (64, 128):
        w = World(torch, [m + 150, m // 2], [m, m], 4, 2, D, 16, dtype, fmt, seed=m + D)
        mem = w.device(B)
        q = w.q.cuda()
        for scale in (0.0, -0.125, 1e-30, 2.0):
            w.check_attend(mem.attend(q, scale=scale, max_new=m), scale=scale)
        w.check_attend(mem.attend(q, scale=-0.1, causal=False, window=33, max_new=m), scale=-0.1, causal=False, window=33)


def test_sequences_share_pages_and_strided_rows(torch, B):
    w = World(torch, [100, 100, 90], [8, 8, 8], 4, 2, 64, 16, "bf16", "e4m3")
    w.table[1] = w.table[0]
    mem = w.device(B)
    fused = torch.zeros(24, 4 * 64 + 64, dtype=w.t, device="cuda")
    fused[:, 64:] = w.q.flatten(1).cuda()
    out = torch.zeros(24, 6, 64, dtype=w.t, device="cuda")
    mem.attend(fused[:, 64:].unflatten(1, (4, 64)), causal=False, max_new=8, out=out[:, 1:5])
    w.check_attend(out[:, 1:5], causal=False)
    assert (out[:, 0] == 0).all() and (out[:, 5] == 0).all()


@pytest.mark.parametrize("dtype,fmt", FORMATS)
@pytest.mark.parametrize("m", [1, 70, 200])
def test_attend_reports_bad_entries(torch, B, dtype, fmt, m):
    w = World(torch, [260, 230, 240], [m, m, m], 2, 1, 64, 16, dtype, fmt, stale="none")
    mem = w.device(B)
    good = mem.attend(w.q.cuda(), max_new=m, max_len=260)
    assert int(w.status) == 0
    for bad in (10 ** 8, -1, w.pages[0].shape[0]):
        w.status.zero_()
        w.dtable.copy_(w.table)
        w.dtable[1, 3] = bad
        got = mem.attend(w.q.cuda(), max_new=m, max_len=260)
        assert int(w.status) == B.ERR_CORRUPT
        assert torch.equal(got[:m], good[:m]) and torch.equal(got[2 * m:], good[2 * m:])
    w.dtable.copy_(w.table)
    for n, ln in ((1, 261), (1, -5), (1, 2 ** 31 - 1)):
        w.status.zero_()
        w.dlens[n] = ln
        got = mem.attend(w.q.cuda(), max_new=m, max_len=260)
        assert int(w.status) == B.ERR_CORRUPT
        assert torch.equal(got[:m], good[:m]) and torch.equal(got[2 * m:], good[2 * m:])
        w.dlens[n] = w.lens[n]
    for starts in ([0, m, 2 * m, 3 * m + 1], [0, m, m - 1, 2 * m - 1], [-1, m - 1, 2 * m - 1, 3 * m - 1]):
        w.status.zero_()
        mem2 = B.Memory(w.dpages[0], w.dpages[1], w.dtable, w.dlens, 2, k_scales=w.dscales[0], v_scales=w.dscales[1],
                        starts=torch.tensor(starts, dtype=torch.int32).cuda(), status=w.status, dtype=dtype)
        mem2.attend(w.q.cuda(), max_new=m, max_len=260)
        mem2.append(w.q.cuda(), None, None)
        assert int(w.status) == B.ERR_CORRUPT


def test_offsets_past_32_bits(torch, B):
    """The last pages of pools of 8.6 GB each: 2^32 bytes and 2^32 / 2 values lie before them."""
    D, page, hk = 128, 128, 2
    n_pages = (1 << 32) // (D * page * hk) + 40
    k, v = (torch.empty((n_pages, hk, page, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    w = World(torch, [1000], [3], 4, hk, D, page, "bf16", "bf16", seed=8)
    far = torch.arange(n_pages - w.pages[0].shape[0], n_pages)
    k[far[0]:], v[far[0]:] = w.pages[0].cuda(), w.pages[1].cuda()
    table = (w.table + int(far[0])).to(torch.int32).cuda()
    mem = B.Memory(k, v, table, torch.tensor([1000], dtype=torch.int32).cuda(), 4)
    w.check_attend(mem.attend(w.q.cuda()))
    mem.append(None, w.k.cuda(), w.v.cuda())
    at = 997 + np.arange(3)
    page_i = torch.from_numpy(at // page)
    got = v[table.cpu()[0].long()[page_i].cuda(), :, torch.from_numpy(at % page).cuda()]
    assert torch.equal(got.cpu(), w.v)
    del k, v
    torch.cuda.empty_cache()


# ---------------------------------------------------------------- as they are used together

@pytest.mark.parametrize("dtype,fmt", FORMATS)
def test_a_policy_that_remembers(torch, B, dtype, fmt):
    """Observation chunks come in and are attended to causally, then action chunks cross-attend: after
    every append the outputs agree with the definition on what the pages hold."""
    hq, hk, D, page, N = 4, 2, 64, 16, 3
    g = torch.Generator().manual_seed(11)
    w = World(torch, [90, 90, 90], [1, 1, 1], hq, hk, D, page, dtype, fmt)
    rot = torch.from_numpy(B.rotation_table(128, D)).cuda()
    gain = (1 + 0.1 * torch.randn(D, generator=g)).cuda()
    lens = [0, 0, 0]
    for news in ([20, 7, 0], [1, 1, 1], [30, 0, 3], [1, 1, 1], [16, 70, 1]):
        lens = [a + b for a, b in zip(lens, news)]
        w.lens, w.news = lens, news
        w.starts = torch.tensor(np.concatenate([[0], np.cumsum(news)]), dtype=torch.int32)
        rows = sum(news)
        starts, dl = w.starts.cuda(), torch.tensor(lens, dtype=torch.int32).cuda()
        if lens == news:
            w.device(B)
        status = torch.zeros(1, dtype=torch.int32).cuda()
        mem = B.Memory(w.dpages[0], w.dpages[1], w.dtable, dl, hq, k_scales=w.dscales[0], v_scales=w.dscales[1], starts=starts,
                       status=status, dtype=dtype)
        q, k, v = (torch.randn(rows, h, D, generator=g).to(w.t).cuda() for h in (hq, hk, hk))
        q = mem.append(q, k, v, gain, gain, rotation=rot)
        w.check_attend(mem.attend(q, max_new=max(news)), q=q, pages=w.dpages, scales=w.dscales)
        cross = B.Memory(w.dpages[0], w.dpages[1], w.dtable, dl, hq, k_scales=w.dscales[0], v_scales=w.dscales[1], status=status,
                         dtype=dtype)
        act = torch.randn(N * 16, hq, D, generator=g).to(w.t).cuda()
        w.starts = torch.arange(N + 1, dtype=torch.int32) * 16
        w.check_attend(cross.attend(act, causal=False), q=act, causal=False, pages=w.dpages, scales=w.dscales)
        assert int(status) == 0


def test_token_by_token_gives_the_chunk(torch, B):
    """A chunk appended and attended to at once, and its tokens one by one, agree within both roundings."""
    hq, hk, D, m = 8, 2, 64, 24
    a = World(torch, [100 + m], [m], hq, hk, D, 16, "bf16", "e4m3", seed=2)
    mem = a.device(B)
    chunk_q = mem.append(a.q.cuda(), a.k.cuda(), a.v.cuda())
    chunk = mem.attend(chunk_q)
    b = World(torch, [100 + m], [m], hq, hk, D, 16, "bf16", "e4m3", seed=2)
    b.device(B)
    outs = []
    for j in range(m):
        dl = torch.tensor([100 + j + 1], dtype=torch.int32).cuda()
        one = B.Memory(b.dpages[0], b.dpages[1], b.dtable, dl, hq, k_scales=b.dscales[0], v_scales=b.dscales[1])
        q = one.append(b.q[j:j + 1].cuda(), b.k[j:j + 1].cuda(), b.v[j:j + 1].cuda())
        outs.append(one.attend(q))
    assert all(torch.equal(x, y) for x, y in zip(a.dpages + a.dscales, b.dpages + b.dscales))
    a.check_attend(chunk, pages=a.dpages, scales=a.dscales)
    a.check_attend(torch.cat(outs), pages=b.dpages, scales=b.dscales)


@pytest.mark.parametrize("dtype,fmt", FORMATS)
@pytest.mark.parametrize("m,length", [(1, 4000), (32, 1500), (200, 1500)])
def test_captured_replayed_and_repeated(torch, B, dtype, fmt, m, length):
    """Two captured calls with workspaces of their own replay on other contents and on two streams; repeats are bit-identical."""
    w = World(torch, [length, length // 2], [m, m], 4, 2, 64, 64, dtype, fmt, seed=m)
    mem = w.device(B, starts=False)
    q = w.q.cuda()
    first = mem.attend(q)
    assert all(torch.equal(first, mem.attend(q)) for _ in range(3))
    graphs, outs = [], []
    for _ in range(2):
        graph, st = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            with torch.cuda.graph(graph, stream=st):
                x = mem.append(q, None, None)
                outs.append(mem.attend(x))
        graphs.append((graph, st))
    q.copy_(-w.q.flip(0).cuda())
    w.dlens.copy_(torch.tensor([length - 7, length // 2 - 1], dtype=torch.int32))
    w.lens = [length - 7, length // 2 - 1]
    torch.cuda.synchronize()
    for _ in range(3):
        for graph, st in graphs:
            with torch.cuda.stream(st):
                graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1])
    w.check_attend(outs[0], q=q)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("m", [1, 20, 40, 200])
def test_a_key_at_minus_infinity_is_no_key(torch, B, dtype, D, m):
    """A key whose scores are all minus infinity has no weight: the others' attention is what is left."""
    w = World(torch, [333], [m], 2, 2, D, 32, dtype, dtype, seed=m)
    k, v = w.dense(0)
    tok = 100
    w.pages[0][int(w.table[0, tok // 32]), :, tok % 32, 3] = -float("inf")
    w.q[:, :, 3] = w.q[:, :, 3].abs() + 0.5
    mem = w.device(B)
    got = mem.attend(w.q.cuda(), causal=False, max_new=m).double().cpu().numpy()
    out, size, dots = M.attend(w.q.double().numpy(), np.delete(k, tok, 0), np.delete(v, tok, 0), 2, D ** -0.5, False, 0)
    half = 2.0 ** -8 if dtype == "bf16" else U
    weight = 2 * (D + 8) * U * dots + 2.0 ** -20 + (2.0 ** -8 if dtype == "bf16" else 0.0)
    assert (np.abs(got - out) <= half * np.abs(out) + (1 + half) * (weight + 333 * U) * size + 1e-37).all()


@pytest.mark.parametrize("dtype,fmt", FORMATS)
@pytest.mark.parametrize("m", [1, 20, 50, 130])
def test_rows_before_and_behind_the_sequences_stay(torch, B, dtype, fmt, m):
    """Starts begin behind the first rows, chunks may be empty, the table names far more pages than are used."""
    news = [m, 0, 3, m]
    w = World(torch, [m + 40, 17, 5, m], news, 4, 2, 64, 16, dtype, fmt, seed=m, max_pages=600)
    mem = w.device(B)
    front, back = 5, 4
    rows = front + sum(news) + back
    starts = (w.starts + front).to(torch.int32).cuda()
    pad = lambda t: torch.cat([torch.full((front,) + t.shape[1:], float("nan")).to(t), t,  # noqa: E731
                               torch.full((back,) + t.shape[1:], float("nan")).to(t)]).cuda()
    q, k, v = pad(w.q), pad(w.k), pad(w.v)
    mem = B.Memory(w.dpages[0], w.dpages[1], w.dtable, w.dlens, 4, k_scales=w.dscales[0], v_scales=w.dscales[1], starts=starts,
                   status=w.status, dtype=dtype)
    out = torch.full((rows, 4, 64), 7.0).to(w.t).cuda()
    got = mem.append(q, k, v, out=out)
    inner = slice(front, front + sum(news))
    assert torch.equal(got[inner], q[inner])
    assert (got[:front] == 7).all() and (got[rows - back:] == 7).all()
    out = torch.full((rows, 4, 64), 7.0).to(w.t).cuda()
    mem.attend(q, max_new=max(news), out=out)
    assert (out[:front] == 7).all() and (out[rows - back:] == 7).all() and int(w.status) == 0
    w.check_attend(out[inner], pages=w.dpages, scales=w.dscales)


@pytest.mark.parametrize("dtype,fmt", FORMATS)
@pytest.mark.parametrize("D", [64, 128])
def test_many_sequences_of_short_chunks(torch, B, dtype, fmt, D):
    """80 sequences of two key heads: chunks of up to 24 tokens, of which some see nothing, one is empty."""
    g = np.random.default_rng(D)
    news = g.integers(1, 25, 80).tolist()
    news[7], news[8] = 0, 24
    lens = (np.array(news) + g.integers(-5, 200, 80)).clip(0).tolist()
    w = World(torch, lens, news, 2, 2, D, 32, dtype, fmt, seed=D)
    mem = w.device(B)
    q = w.q.cuda()
    w.check_attend(mem.attend(q, max_new=24))
    w.check_attend(mem.attend(q, causal=False, window=50, max_new=24), causal=False, window=50)
    assert int(w.status) == 0


@pytest.mark.parametrize("dtype,fmt", [("bf16", "e4m3"), ("fp32", "fp32")])
def test_thousands_of_sequences(torch, B, dtype, fmt):
    g = np.random.default_rng(3)
    lens = g.integers(1, 40, 2500).tolist()
    w = World(torch, lens, [1] * 2500, 2, 1, 64, 16, dtype, fmt, seed=3)
    mem = w.device(B)
    got = mem.attend(w.q.cuda(), max_new=1, max_len=40)
    assert int(w.status) == 0
    w.check_attend(got)
    mem.append(None, w.k.cuda(), w.v.cuda())
    w.check_attend(mem.attend(w.q.cuda(), max_new=1), pages=w.dpages, scales=w.dscales)


@pytest.mark.parametrize("dtype,fmt", FORMATS)
def test_queries_in_place_and_outputs_beside_them(torch, B, dtype, fmt):
    """One buffer of rows holds queries, keys, values and outputs: queries are turned in place, outputs interleave."""
    hq, hk, D = 8, 2, 64
    w = World(torch, [300, 40], [70, 3], hq, hk, D, 32, dtype, fmt, seed=5)
    a, b = w.device(B), World(torch, [300, 40], [70, 3], hq, hk, D, 32, dtype, fmt, seed=5)
    rot = torch.from_numpy(B.rotation_table(300, D)).cuda()
    want = a.append(w.q.cuda(), w.k.cuda(), w.v.cuda(), rotation=rot)
    out = a.attend(want, max_new=70)
    wide = torch.cat([w.q, w.k, w.v, torch.zeros_like(w.q)], 1).cuda()
    q, k, v, o = wide[:, :hq], wide[:, hq:hq + hk], wide[:, hq + hk:hq + 2 * hk], wide[:, hq + 2 * hk:]
    mem = b.device(B)
    mem.append(q, k, v, rotation=rot, out=q)
    mem.attend(q, max_new=70, out=o)
    assert torch.equal(q, want) and torch.equal(o, out)
    assert torch.equal(k.cpu(), w.k) and torch.equal(v.cpu(), w.v)
    with pytest.raises(B.EvoError):
        mem.attend(q, max_new=70, out=q)


def test_appends_of_two_host_threads(torch, B):
    """Long chunks of different widths appended from two threads at once, each on its own stream."""
    import threading
    jobs = []
    for hq, hk, D in ((8, 2, 128), (2, 1, 128)):
        w = World(torch, [6400] * 2, [6400] * 2, hq, hk, D, 128, "bf16", "bf16", seed=hq, stale=None)
        mem, st = w.device(B), torch.cuda.Stream()
        args = [t.cuda() for t in (w.q, w.k, w.v)]
        want = mem.append(*args)
        jobs.append((mem, st, args, want, []))
    torch.cuda.synchronize()

    def run(mem, st, args, want, got):
        try:
            with torch.cuda.stream(st):
                for _ in range(200):
                    got[:] = [mem.append(*args)]
        except Exception as e:                                     # noqa: BLE001
            got[:] = [e]
    threads = [threading.Thread(target=run, args=j) for j in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for _, _, _, want, got in jobs:
        assert torch.is_tensor(got[0]) and torch.equal(got[0], want), got[0]


def test_a_stream_given_by_the_caller(torch, B):
    w = World(torch, [3000], [1], 4, 2, 64, 64, "bf16", "e4m3")
    mem = w.device(B, starts=False)
    q = w.q.cuda()
    torch.cuda.synchronize()
    for st in (torch.cuda.Stream(), torch.cuda.Stream().cuda_stream):
        got = mem.attend(q, stream=st)
        torch.cuda.synchronize()
        w.check_attend(got)


def test_a_call_on_another_stream_takes_nothing_from_the_current_ones_pool(torch, B):
    """Memory that pending work of the current stream may still use is neither output nor workspace of
    a call on another stream, and the call's own is not handed out on the current stream."""
    w = World(torch, [9000], [1], 4, 2, 64, 64, "bf16", "e4m3")
    mem, q, other = w.device(B, starts=False), w.q.cuda(), torch.cuda.Stream()
    nb = B.load().evo_memory_scratch_bytes(mem._ref, 1, 1, mem.max_len)
    assert nb > 1 << 12
    torch.cuda.synchronize()
    for st in (other, other.cuda_stream):
        gone = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in (512, nb, nb, 512, 512)]
        old = {t.data_ptr() for t in gone}
        del gone
        out = mem.attend(q, stream=st)
        assert out.data_ptr() not in old
        for n in (512, nb, nb, 512, 512):                          # nothing of this is the call's workspace
            torch.empty(n, dtype=torch.uint8, device="cuda").fill_(255)
        torch.cuda.synchronize()
        w.check_attend(out)
    x, y = torch.zeros(2, 2, 64, device="cuda"), torch.zeros(2, 2, 64, device="cuda").data_ptr()
    codes, scales = torch.zeros(1, 2, 2, 64, dtype=torch.uint8, device="cuda"), torch.ones(1, 2, 2, 2, dtype=torch.uint8, device="cuda")
    assert B.cache_add(codes, scales, x, stream=other).data_ptr() != y
    assert B.cache_write(x, codes[0], scales[0], x, stream=other).data_ptr() != y
    assert mem.append(q, None, None, stream=other).shape == q.shape
    torch.cuda.synchronize()


def test_sizes_of_a_growing_memory_are_forgotten(torch, B):
    w = World(torch, [3], [1], 4, 2, 64, 16, "bf16", "bf16", max_pages=100)
    mem, q = w.device(B, starts=False), w.q.cuda()
    for n in range(3, 1600):
        mem.attend(q, max_len=n)
    assert len(mem._scratch) <= 1024
    w.check_attend(mem.attend(q))


def test_binding_refuses(torch, B):
    w = World(torch, [30], [4], 4, 2, 64, 16, "bf16", "bf16")
    mem = w.device(B)
    q, k, v = w.q.cuda(), w.k.cuda(), w.v.cuda()
    for bad in (dict(q=q.float()), dict(q=q[:, :2]), dict(q=q.cpu()), dict(out=torch.empty_like(q)[:2])):
        with pytest.raises(ValueError):
            mem.attend(**(dict(q=q) | bad))
    for bad in (dict(max_new=5), dict(max_new=0), dict(max_len=1000), dict(window=-1), dict(scale=float("nan"))):
        with pytest.raises(B.EvoError) as e:
            mem.attend(q, **bad)
        assert e.value.code == B.ERR_ARG
    for bad in (dict(k=None), dict(q=None, k=None, v=None), dict(k=k[:2]), dict(q_gain=torch.ones(64)), dict(rotation=torch.ones(4, 32).cuda()),
                dict(v=v.float()), dict(pos0=torch.zeros(2, dtype=torch.int32).cuda())):
        with pytest.raises(ValueError):
            mem.append(**(dict(q=q, k=k, v=v) | bad))
    assert mem.attend(q[:0]).shape == (0, 4, 64)


# ---------------------------------------------------------------- scores past what fp32 resolves

def whole_numbers(torch, w, q_unit, k_unit):
    """Queries of -1, 0, 1 and keys of -3 .. 3, times a power of two: every score is exact in fp32, and two scores
    are equal or a unit apart."""
    g = torch.Generator().manual_seed(77)
    w.q = (torch.randint(-1, 2, w.q.shape, generator=g).float() * q_unit).to(w.t)
    k = torch.randint(-3, 4, w.pages[0].shape, generator=g).float() * k_unit
    k[..., 0] = 3 * k_unit
    if w.fmt == "e4m3":
        c, s = M.quantise(k.numpy().astype(np.float64))
        assert np.array_equal(M.dequantise(c, s), k.double().numpy())
        w.pages[0], w.scales[0] = torch.from_numpy(c.copy()), torch.from_numpy(s.copy())
    else:
        w.pages[0] = k.to(w.t)


@pytest.mark.parametrize("dtype,fmt", FORMATS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("m", [1, 3, 8, 14, 30, 40, 150])
def test_attend_scores_of_any_finite_size(torch, B, dtype, fmt, D, m):
    """Scores from 2^18 to 2^125: weights are equal for the keys with the largest score and zero for all others, so that
    the score's own rounding moves nothing, and what is left of the tolerance is that of the weights and the sums."""
    w = World(torch, [m + 300, m // 2 + 40], [m, m], 4, 2, D, 16, dtype, fmt, seed=m + D, stale="none")
    for q_unit, k_unit, scales in ((1.0, 1.0, (2.0 ** 12, 2.0 ** 21, -2.0 ** 26, 2.0 ** 60, 2.0 ** 118)),
                                   (2.0 ** 30, 2.0 ** 40, (2.0 ** -8, -2.0 ** -40))):
        whole_numbers(torch, w, q_unit, k_unit)
        mem = w.device(B)
        q = w.q.cuda()
        for scale in scales:
            for causal, window in ((True, 0), (False, 90)):
                got = mem.attend(q, scale=scale, causal=causal, window=window, max_new=m).double().cpu().numpy()
                for n in range(2):
                    k, v = w.dense(n)
                    a, b = int(w.starts[n]), int(w.starts[n + 1])
                    out, size, _ = M.attend(w.q[a:b].double().numpy(), k, v, 2, scale, causal, window)
                    half = 2.0 ** -8 if dtype == "bf16" else U
                    weight = 2.0 ** -20 + (2.0 ** -8 if dtype == "bf16" else 0.0)
                    tol = half * np.abs(out) + (1 + half) * (weight + w.lens[n] * U) * size + 1e-37
                    assert (np.abs(got[a:b] - out) <= tol).all(), (scale, causal, n)
        assert int(w.status) == 0


@pytest.mark.parametrize("dtype,fmt", FORMATS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("m", [1, 20, 40, 150, 300])
def test_pages_that_left_the_window(torch, B, dtype, fmt, D, m):
    """A memory whose oldest pages were dropped: their entries name no page, and no row of the call sees them."""
    window, lens, news = 100, [m + 700, m + 31, 450, 60], [m, m, 0, min(m, 60)]
    w = World(torch, lens, news, 4, 2, D, 16, dtype, fmt, seed=m + D)
    for causal in (True, False):
        mem = w.device(B)
        table = w.table.clone()
        for n, (ln, new) in enumerate(zip(lens, news)):
            first = max(0, ln - window - (new - 1 if causal else 0)) if new else ln
            table[n, :first // 16] = -1 - n
        w.dtable.copy_(table)
        got = mem.attend(w.q.cuda(), causal=causal, window=window, max_new=m)
        assert int(w.status) == 0
        w.check_attend(got, causal=causal, window=window)


@pytest.mark.parametrize("dtype,fmt", FORMATS)
@pytest.mark.parametrize("m,length", [(1, 9000), (6, 9000), (30, 3000), (100, 2000), (400, 1200)])
def test_windows_of_every_size_fit_the_workspace(torch, B, dtype, fmt, m, length):
    """A call stays in the bytes that its sizes ask for, whatever window cuts its pieces."""
    import ctypes
    w = World(torch, [length, length - 700], [m, m], 4, 2, 64, 16, dtype, fmt, seed=m)
    mem = w.device(B)
    q, out = w.q.cuda(), torch.empty(2 * m, 4, 64, dtype=w.t, device="cuda")
    nb = B.load().evo_memory_scratch_bytes(mem._ref, 2 * m, m, length)
    scratch = torch.full((nb + (8 << 20),), 85, dtype=torch.uint8, device="cuda")
    for causal, window in ((1, 0), (1, 1), (1, 17), (0, 300), (1, 1025), (0, 2500), (1, length), (0, 2 ** 31 - 1)):
        scratch.fill_(85)
        rc = B.load().evo_memory_attend(mem._ref, q.data_ptr(), 256, 2 * m, m, length, 0.125, causal, window, out.data_ptr(), 256,
                                        scratch.data_ptr(), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
        assert rc == B.OK
        assert (scratch[nb:] == 85).all() and int(w.status) == 0
        w.check_attend(out, causal=bool(causal), window=window)


# ---------------------------------------------------------------- append of thousands of rows (the kernel with a ring of rows)

def check_append_of_many(w, q_out, q_gain, k_gain, eps, base, pos0):
    """As check_append, all rows at once."""
    torch = w.torch
    n = np.repeat(np.arange(len(w.news)), w.news)
    at = np.concatenate([np.arange(ln - m, ln) for ln, m in zip(w.lens, w.news)])
    pos = at + np.asarray(pos0)[n]
    page, slot = w.table.numpy()[n, at // w.page], at % w.page
    half, rows = 2.0 ** -8 if w.dtype == "bf16" else U, len(n)

    def want(x, gain):
        y = M.normed_and_turned(x.double().numpy()[:rows], gain, eps, pos, base)
        a = np.hypot(*np.split(y, 2, -1))
        return y, 32 * U * np.concatenate([a, a], -1) + 1e-37
    y, tol = want(w.q, q_gain)
    assert (np.abs(q_out.double().cpu().numpy()[:rows] - y) <= tol + half * (np.abs(y) + tol)).all()
    y, tol = want(w.k, k_gain)
    v = w.v.double().numpy()[:rows]
    touched = torch.zeros(w.pages[0].shape[:3], dtype=torch.bool)
    touched[page, :, slot] = True
    for i, (e, t) in enumerate(((y, tol), (v, 0.0))):
        got = w.dpages[i].cpu()
        mine = got[page, :, slot]
        if w.fmt == "e4m3":
            s = w.dscales[i].cpu()
            c, k = mine.numpy(), s[page, :, slot].numpy().astype(np.float64)[..., None] - 127
            if i == 1:                                             # no arithmetic before the rounding: bit for bit
                wc, ws = M.quantise(e)
                assert np.array_equal(c, wc) and np.array_equal(k[..., 0] + 127, ws)
            amax = np.abs(e).max(-1, keepdims=True)
            assert (amax <= 448 * 2.0 ** k * (1 + 1e-4)).all() and ((amax > 448 * 2.0 ** (k - 1) * (1 - 1e-4)) | (k == -126)).all()
            mine = M.dequantise(c, (k[..., 0] + 127).astype(np.uint8))
            t = t + np.maximum(2.0 ** -4 * (np.abs(e) + t), 2.0 ** (k - 10))
            assert torch.equal(s[~touched], w.scales[i][~touched])
        else:
            mine = mine.double().numpy()
            t = t + half * (np.abs(e) + t) if i == 0 else 0.0
        assert (np.abs(mine - e) <= t).all(), i
        same = (got.view(torch.uint8) == w.pages[i].view(torch.uint8)).flatten(3).all(-1)
        assert same[~touched].all()


def many_rows(torch, hq, hk, D, dtype, fmt, page, seed, each=700):
    """Ragged chunks, 6,300 rows or more: first chunks of a memory, an empty one, one of a single token."""
    g = np.random.default_rng(seed)
    news = g.integers(each // 2, each + 400, 9).tolist() + [0, 1]
    while sum(news) < 6300:
        news.append(int(g.integers(1, each)))
    lens = [m + int(g.integers(0, 300)) for m in news]
    lens[0], lens[-1] = news[0], news[-1]
    return World(torch, lens, news, hq, hk, D, page, dtype, fmt, seed=seed, stale="none", spare_rows=3)


@pytest.mark.parametrize("dtype,fmt", FORMATS)
@pytest.mark.parametrize("hq,hk,D,page", [(2, 1, 64, 16), (3, 3, 64, 128), (5, 1, 128, 32), (16, 4, 128, 64)])
def test_append_of_thousands_of_rows(torch, B, dtype, fmt, hq, hk, D, page):
    w = many_rows(torch, hq, hk, D, dtype, fmt, page, seed=hq + D)
    mem = w.device(B)
    g = torch.Generator().manual_seed(1)
    qg, kg = 1 + 0.3 * torch.randn(D, generator=g), 1 + 0.3 * torch.randn(D, generator=g)
    pos0 = (torch.arange(len(w.news)) * 97 % 4000).to(torch.int32)
    rot = torch.from_numpy(B.rotation_table(5600, D, 1e4)).cuda()
    out = torch.full((w.rows, hq, D), 7.0, dtype=w.t, device="cuda")
    q = mem.append(w.q.cuda(), w.k.cuda(), w.v.cuda(), qg.cuda(), kg.cuda(), 1e-6, rot, pos0=pos0.cuda(), out=out)
    assert q is out and (out[-3:] == 7).all() and int(w.status) == 0     # rows behind the last sequence
    check_append_of_many(w, q, qg.double().numpy(), kg.double().numpy(), 1e-6, 1e4, pos0.numpy())


@pytest.mark.parametrize("dtype,fmt", [("bf16", "e4m3"), ("fp32", "fp32")])
def test_append_of_a_hundred_thousand_rows(torch, B, dtype, fmt):
    """More rows than all warps hold 32 of: blocks that start when others have ended."""
    g = np.random.default_rng(4)
    news = g.integers(1, 260, 800).tolist()
    assert sum(news) > 2 * 152 * 4 * 5 * 16 + 1000
    w = World(torch, [m + int(x) for m, x in zip(news, g.integers(0, 50, 800))], news, 1, 1, 64, 16, dtype, fmt, seed=4, stale="none")
    mem = w.device(B)
    rot = torch.from_numpy(B.rotation_table(320, 64, 1e4)).cuda()
    q = mem.append(w.q.cuda(), w.k.cuda(), w.v.cuda(), rotation=rot)
    assert int(w.status) == 0
    check_append_of_many(w, q, None, None, 0, 1e4, np.zeros(800, int))


@pytest.mark.parametrize("dtype,fmt", FORMATS)
@pytest.mark.parametrize("parts", ["all", "queries", "keys"])
@pytest.mark.parametrize("extras", [True, False])
def test_thousands_of_rows_are_those_of_small_calls(torch, B, dtype, fmt, parts, extras):
    """Rows of a fused projection, queries in place, bit for bit what calls of a sequence each leave; entries that name
    nothing, lengths past the table and rows outside the sequences are not touched."""
    hq, hk, D, page = 4, 2, 128, 32
    a, b = (many_rows(torch, hq, hk, D, dtype, fmt, page, seed=12) for _ in range(2))
    g = torch.Generator().manual_seed(2)
    gain = (1 + 0.3 * torch.randn(D, generator=g)).cuda() if extras else None
    rot = torch.from_numpy(B.rotation_table(1500, D, 1e4)).cuda() if extras else None
    pos0 = (torch.arange(len(a.news)) * 13 % 50).to(torch.int32).cuda() if extras else None
    front, back = 5, 3
    rows = front + a.rows + back
    fused = torch.cat([a.q.flatten(1), a.k.flatten(1), a.v.flatten(1), torch.zeros(a.rows, 8, dtype=a.t)], 1)
    fused = torch.cat([fused[:front], fused, fused[:back]]).cuda()
    two = fused.clone()
    states = []
    for w, buf in ((a, fused), (b, two)):
        w.table[2, (w.lens[2] - w.news[2] // 2) // page] = 10 ** 7       # a bad entry inside the chunk
        w.table[4, :] = -3
        w.device(B)
        w.dlens[5] = w.table.shape[1] * page + 40                       # the chunk's end is past the table
        cols = [buf[:, i:j].unflatten(1, (-1, D)) for i, j in ((0, hq * D), (hq * D, (hq + hk) * D), ((hq + hk) * D, (hq + 2 * hk) * D))]
        states.append(cols)
    starts = (a.starts + front).to(torch.int32).cuda()

    def call(w, cols, at, seqs, starts):
        mem = B.Memory(w.dpages[0], w.dpages[1], w.dtable[seqs].contiguous(), w.dlens[seqs].contiguous(), hq, k_scales=w.dscales[0],
                       v_scales=w.dscales[1], starts=starts, status=w.status, dtype=dtype)
        q, k, v = (x[at] for x in cols)
        p0 = None if pos0 is None else pos0[seqs].contiguous()
        if parts == "keys":
            mem.append(None, k, v, k_gain=gain, rotation=rot, pos0=p0)
        elif parts == "queries":
            mem.append(q, None, None, q_gain=gain, rotation=rot, pos0=p0, out=q)
        else:
            mem.append(q, k, v, gain, gain, rotation=rot, pos0=p0, out=q)
    call(a, states[0], slice(0, rows), slice(0, len(a.news)), starts)
    assert int(a.status) == B.ERR_CORRUPT
    for n, m in enumerate(b.news):
        first = front + int(b.starts[n])
        if m:
            call(b, states[1], slice(first, first + m), slice(n, n + 1), torch.tensor([0, m], dtype=torch.int32).cuda())
    assert int(b.status) == B.ERR_CORRUPT
    assert torch.equal(fused, two)
    raw = torch.cat([a.q.flatten(1), a.k.flatten(1), a.v.flatten(1), torch.zeros(a.rows, 8, dtype=a.t)], 1)
    assert torch.equal(fused[:front].cpu(), raw[:front]) and torch.equal(fused[rows - back - 3:rows - back].cpu(), raw[-3:])
    for x, y, z in zip(a.dpages + a.dscales, b.dpages + b.dscales, a.pages + a.scales):
        if x is not None:
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
            assert (parts == "queries") == torch.equal(x.cpu().view(torch.uint8), z.view(torch.uint8))


def test_numbers_past_32_bits(torch, B):
    """A window longer than any memory hides nothing; sizes that no table has are refused."""
    w = World(torch, [300], [4], 4, 2, 64, 16, "bf16", "bf16")
    mem, q = w.device(B), w.q.cuda()
    for window in (2 ** 31, 2 ** 32 + 5, 2 ** 40):
        w.check_attend(mem.attend(q, window=window))
    for bad in (dict(max_len=2 ** 32 + 300), dict(max_new=2 ** 32 + 4), dict(window=-2 ** 32 + 7)):
        with pytest.raises(B.EvoError) as e:
            mem.attend(q, **bad)
        assert e.value.code == B.ERR_ARG


@pytest.mark.parametrize("dtype,fmt", FORMATS)
@pytest.mark.parametrize("m", [1, 20, 70, 300])
def test_a_memory_without_a_status_word_reports_too(torch, B, dtype, fmt, m):
    w = World(torch, [m + 90, m], [m, m], 2, 1, 64, 16, dtype, fmt, seed=m, stale="none")
    w.device(B)
    mem = B.Memory(w.dpages[0], w.dpages[1], w.dtable, w.dlens, 2, k_scales=w.dscales[0], v_scales=w.dscales[1], dtype=dtype)
    q, k, v = w.q.cuda(), w.k.cuda(), w.v.cuda()
    w.check_attend(mem.attend(q))
    assert mem.status() == B.OK
    w.dtable[1, 0] = w.pages[0].shape[0]
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    for call in (lambda: mem.attend(q), lambda: mem.append(q, k, v), lambda: mem.attend(q, stream=other)):
        call()
        assert mem.status() == B.ERR_CORRUPT
        assert mem.status() == B.OK                                # read and cleared
    w.dtable.copy_(w.table)
    mem.attend(q)
    assert mem.status() == B.OK


# ---------------------------------------------------------------- calls at the edge of what is documented

@pytest.mark.parametrize("dtype,fmt", FORMATS)
def test_empty_memories_and_calls(torch, B, dtype, fmt):
    w = World(torch, [0, 0], [3, 3], 4, 2, 64, 16, dtype, fmt)
    mem = w.device(B)
    for m, news in ((3, [3, 3]), (60, [60, 60]), (300, [300, 300])):
        q = torch.randn(sum(news), 4, 64).to(w.t).cuda()
        starts = torch.tensor([0, m, 2 * m], dtype=torch.int32).cuda()
        mem = B.Memory(w.dpages[0], w.dpages[1], w.dtable, w.dlens, 4, k_scales=w.dscales[0], v_scales=w.dscales[1], starts=starts, dtype=dtype)
        for causal, window in ((False, 0), (True, 0), (True, 5)):
            assert (mem.attend(q, causal=causal, window=window, max_new=m, max_len=0) == 0).all()
            assert (mem.attend(q, causal=causal, window=window, max_new=m) == 0).all()
        assert mem.status() == B.OK
    empty = torch.empty(0, 4, 64, dtype=w.t, device="cuda")
    none = torch.zeros(0, 1, dtype=torch.int32, device="cuda")
    mem = B.Memory(w.dpages[0], w.dpages[1], none, none[:, 0].contiguous(), 4, k_scales=w.dscales[0], v_scales=w.dscales[1], dtype=dtype)
    assert mem.attend(empty).shape == empty.shape
    assert mem.append(empty, empty[:, :2], empty[:, :2]).shape == empty.shape


@pytest.mark.parametrize("dtype,fmt", FORMATS)
@pytest.mark.parametrize("hq,hk,D", [(256, 1, 64), (130, 2, 128), (1024, 1024, 64), (1024, 8, 64)])
def test_many_heads(torch, B, dtype, fmt, hq, hk, D):
    """One token's query heads fill several tiles; as many heads as a call may have."""
    w = World(torch, [77, 3], [2, 1], hq, hk, D, 16, dtype, fmt, seed=hq)
    mem = w.device(B)
    w.check_attend(mem.attend(w.q.cuda(), max_new=2))
    w.check_attend(mem.attend(w.q.cuda(), max_new=2, causal=False, window=20), causal=False, window=20)
    q = mem.append(w.q.cuda(), w.k.cuda(), w.v.cuda())
    assert torch.equal(q.cpu(), w.q) and mem.status() == B.OK
    check_append(w, mem, q, None, None, 0, None)


def test_streams_by_every_name(torch, B):
    w = World(torch, [9000], [1], 4, 2, 64, 64, "bf16", "e4m3")
    mem, q = w.device(B, starts=False), w.q.cuda()
    torch.cuda.synchronize()
    want = mem.attend(q)
    for st in (0, torch.cuda.default_stream(), torch.cuda.current_stream(), torch.cuda.current_stream().cuda_stream, torch.cuda.Stream()):
        got, turned = mem.attend(q, stream=st), mem.append(q, None, None, stream=st)
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(turned, q)


def test_one_memory_read_by_two_host_threads(torch, B):
    """Calls of different sizes on one memory at once, each thread on its stream: workspaces are a call's own."""
    import threading
    w = World(torch, [6000, 5000], [40, 40], 4, 2, 64, 64, "bf16", "e4m3")
    mem = w.device(B)
    q = w.q.cuda()
    calls = [dict(max_new=40), dict(max_new=41, window=900), dict(max_new=44, causal=False), dict(max_new=80, max_len=6016)]
    want = [mem.attend(q, **c) for c in calls]
    torch.cuda.synchronize()
    bad = []

    def run(first):
        st = torch.cuda.Stream()
        try:
            with torch.cuda.stream(st):
                for i in range(100):
                    c = (first + i) % len(calls)
                    if not torch.equal(mem.attend(q, **calls[c]), want[c]):
                        bad.append(c)
        except Exception as e:                                     # noqa: BLE001
            bad.append(e)
    threads = [threading.Thread(target=run, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not bad and int(w.status) == 0


@pytest.mark.parametrize("dtype,fmt", FORMATS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("m", [2, 7, 15, 30, 60, 200])
def test_queries_that_are_not_numbers(torch, B, dtype, fmt, D, m):
    """A NaN query gives NaN in its own row and head, and no other row knows of it."""
    w = World(torch, [m + 200, m], [m, m], 2, 2, D, 16, dtype, fmt, seed=m)
    w.q[0, 0, 5] = float("nan")
    w.q[m + 1, 1] = float("nan")
    mem = w.device(B)
    for window in (0, 50):
        got = mem.attend(w.q.cuda(), max_new=m, window=window).clone()
        assert got[0, 0].isnan().all() and got[m + 1, 1].isnan().all()
        sane = w.q.clone()
        sane[0, 0], sane[m + 1, 1] = 0, 0
        got[0, 0], got[m + 1, 1] = (mem.attend(sane.cuda(), max_new=m, window=window)[i] for i in ((0, 0), (m + 1, 1)))
        w.check_attend(got, q=sane, window=window)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("m", [1, 6, 14, 30, 200])
@pytest.mark.parametrize("size", [2.0 ** 8, 2.0 ** 14, 2.0 ** 30])
def test_one_large_value_beside_small_ones(torch, B, D, m, size):
    """8-bit pages, one token with a single large value: the others' columns are off by the weights' rounding, and by
    2^-25 of the largest weight times scale a key where the weights are fp16 (a code is at most 448)."""
    w = World(torch, [m + 250, m], [m, m], 2, 2, D, 16, "bf16", "e4m3", seed=m)
    page, slot = int(w.table[0, 0]), 3
    v = torch.zeros(2, D, dtype=torch.float64)
    v[:, 7] = size
    c, s = M.quantise(v.numpy())
    w.pages[1][page, :, slot], w.scales[1][page, :, slot] = torch.from_numpy(c), torch.from_numpy(s)
    mem = w.device(B)
    got = mem.attend(w.q.cuda(), causal=False, max_new=m).double().cpu().numpy()
    for n in range(2):
        k, v = w.dense(n)
        a, b = int(w.starts[n]), int(w.starts[n + 1])
        q = w.q[a:b].double().numpy()
        out, mean, dots = M.attend(q, k, v, 2, D ** -0.5, False, 0)
        p = np.exp(np.einsum("mhd,khd->mhk", q, k) * D ** -0.5)
        p /= p.sum(-1, keepdims=True)
        at = w.table[n, :-(-w.lens[n] // 16)].long()
        scales = 2.0 ** (w.scales[1][at].double().numpy() - 127).transpose(0, 2, 1).reshape(-1, 2)[:w.lens[n]]
        most = (p * scales.T[None]).max(-1)[..., None]
        tol = 2.0 ** -8 * np.abs(out) + (1 + 2.0 ** -8) * ((2 * (D + 8) * U * dots + 2.0 ** -20 + 2.0 ** -8 + w.lens[n] * U) * mean
                                                           + 2.0 ** -25 * 448 * w.lens[n] * most)
        assert (np.abs(got[a:b] - out) <= tol).all(), n
