"""The latent memory on the GPU against the float64 definitions.

Tolerances, for every output element by itself, from the roundings that the documentation
names (u = 2^-24; bf16 rounds by at most 2^-8 of the value):

append   the norm is a sum of `rank` squares (off by rank u / 32 at most in each of 32 lanes' chains, and 8 u
         in their join), a root and two products; the rotation four operations on a pair: fewer than
         rank / 16 + 32 fp32 operations on a value, each off by u of the pair's length, then one rounding.
attend   a score is off by (rank + 72) u of sum |q||x| scale, a weight by twice that (the maximum has it
         too) plus 2^-20 for the exponential, and by 2^-8 with bf16 rows; a weight's error moves the output
         by at most that share of the weighted mean of |c|.  Sums of L terms add L u of it, the result one
         rounding to the row's type.
expand   a sum of `rank` products is off by (rank + 8) u of sum |c||w|, the result one rounding.
"""
import threading

import numpy as np
import pytest

from oracle import evo_latent as L
from oracle import evo_memory as M

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
ROPE = 64


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


def half(dtype):
    return 2.0 ** -8 if dtype == "bf16" else U


class World:
    """A pool of pages with stale contents, a shuffled table and its float64 view."""

    def __init__(self, torch, lens, news, H, rank, page, dtype, seed=0, stale=True, spare_rows=0, max_pages=None):
        g = torch.Generator().manual_seed(seed)
        self.torch, self.H, self.rank, self.page, self.dtype = torch, H, rank, page, dtype
        self.t = torch.float32 if dtype == "fp32" else torch.bfloat16
        self.lens, self.news = list(lens), list(news)
        self.table, n_pages = self.shuffled(page, g, max_pages)
        self.pages = torch.randn(n_pages, page, rank + ROPE, generator=g).to(self.t)
        if stale:
            live = torch.zeros(n_pages, page, dtype=torch.bool)
            for n, ln in enumerate(self.lens):
                for i in range(-(-ln // page)):
                    live[int(self.table[n, i]), :max(0, min(page, ln - i * page))] = True
            self.pages[~live] = float("nan")
        self.starts = torch.tensor(np.concatenate([[0], np.cumsum(news)]), dtype=torch.int32)
        self.rows = int(self.starts[-1]) + spare_rows
        self.q = torch.randn(self.rows, H, rank + ROPE, generator=g).to(self.t)
        self.c = (1.3 * torch.randn(self.rows, rank, generator=g)).to(self.t)
        self.k = torch.randn(self.rows, ROPE, generator=g).to(self.t)
        self.scale = 128 ** -0.5
        self.gen = g

    def shuffled(self, page, g, max_pages=None):
        torch = self.torch
        need = [-(-n // page) for n in self.lens]
        order = torch.randperm(sum(need) + 2, generator=g).to(torch.int32)
        table, at = torch.full((len(need), max_pages or max(1, max(need))), -7, dtype=torch.int32), 0
        for n, c in enumerate(need):
            table[n, :c] = order[at:at + c]
            at += c
        return table, sum(need) + 2

    def device(self, B, starts=True, n_head=None):
        self.dpages, self.dtable = self.pages.cuda(), self.table.cuda()
        self.dlens = self.torch.tensor(self.lens, dtype=self.torch.int32).cuda()
        self.status = self.torch.zeros(1, dtype=self.torch.int32).cuda()
        self.mem = B.LatentMemory(self.dpages, self.dtable, self.dlens, n_head or self.H,
                                  starts=self.starts.cuda() if starts else None, status=self.status)
        return self.mem

    def dense(self, n, pages=None):
        at = self.table[n, :-(-self.lens[n] // self.page)].long()
        p = self.pages if pages is None else pages.cpu()
        return p[at].double().numpy().reshape(-1, self.rank + ROPE)[:self.lens[n]]

    def check_attend(self, got, q=None, scale=None, causal=True, window=0, pages=None):
        scale = self.scale if scale is None else scale
        q = (self.q if q is None else q).double().cpu().numpy()
        got = got.double().cpu().numpy()
        for n, ln in enumerate(self.lens):
            a, b = int(self.starts[n]), int(self.starts[n + 1])
            out, size, dots = L.attend(q[a:b], self.dense(n, pages), self.rank, scale, causal, window)
            h = half(self.dtype)
            weight = 2 * (self.rank + 72) * U * dots + 2.0 ** -20 + (2.0 ** -8 if self.dtype == "bf16" else 0.0)
            tol = h * np.abs(out) + (1 + h) * (weight + ln * U) * size + 1e-37
            bad = ~(np.abs(got[a:b] - out) <= tol) & ~(np.isnan(out) & np.isnan(got[a:b]))
            worst = np.nanmax(np.abs(got[a:b] - out) / tol) if out.size else 0
            assert not bad.any(), (n, int(bad.sum()), worst, np.argwhere(bad)[:4])


DTYPES = ["bf16", "fp32"]
RANKS = [128, 256, 512]
HEADS = [1, 5, 8, 16, 33, 64]


# ---------------------------------------------------------------- append

def check_append(w, q_in, q_out, gain, eps, base, pos0=None, tokens=True):
    torch = w.torch
    pos = np.concatenate([np.arange(ln - m, ln) + (0 if pos0 is None else int(pos0[n]))
                          for n, (ln, m) in enumerate(zip(w.lens, w.news))]).astype(np.float64)
    rows, h, ops = len(pos), half(w.dtype), (w.rank / 16 + 32) * U
    pairs = lambda y: np.concatenate(2 * [np.hypot(y[..., :32], y[..., 32:])], -1)  # noqa: E731
    if q_out is not None:
        y = L.turned(q_in.double().cpu().numpy()[:rows], pos, base)
        tol = (ops * pairs(y) if base is not None else 0.0) + h * np.abs(y) + 1e-37
        assert (np.abs(q_out.double().cpu().numpy()[:rows] - y) <= tol * (1 + h)).all()
    got = w.dpages.cpu()
    touched = torch.zeros(got.shape[:2], dtype=torch.bool)
    if tokens:
        c, k = L.normed(w.c.double().numpy()[:rows], gain, eps), L.turned(w.k.double().numpy()[:rows], pos, base)
        want = np.concatenate([c, k], 1)
        size = np.concatenate([ops * np.abs(c) if gain is not None else 0 * c, ops * pairs(k) if base is not None else 0 * k], 1)
        tol = (size + h * np.abs(want)) * (1 + h) + 1e-37
        at = 0
        for n, m in enumerate(w.news):
            for j in range(m):
                p = w.lens[n] - m + j
                page, slot = int(w.table[n, p // w.page]), p % w.page
                touched[page, slot] = True
                assert (np.abs(got[page, slot].double().numpy() - want[at]) <= tol[at]).all(), (n, j)
                at += 1
    same = (got.view(torch.uint8) == w.pages.view(torch.uint8)).all(-1)
    assert same[~touched].all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rank", RANKS)
@pytest.mark.parametrize("H", HEADS)
def test_append(torch, B, dtype, rank, H):
    w = World(torch, [37, 1, 0, 16, 130, 33], [5, 1, 0, 16, 65, 0], H, rank, 16, dtype, seed=rank + H, spare_rows=2)
    mem = w.device(B)
    gain = 1 + 0.3 * torch.randn(rank, generator=w.gen)
    rot = torch.from_numpy(B.rotation_table(256, ROPE, 1e4)).cuda()
    out = torch.full((w.rows, H, ROPE), 7.0, dtype=w.t, device="cuda")
    q = w.q.cuda()[..., rank:]
    got = mem.append(w.c.cuda(), w.k.cuda(), q, gain.cuda(), 1e-6, rot, out=out)
    assert got is out and (out[-2:] == 7).all()                   # rows behind the last sequence
    check_append(w, q, out, gain.double().numpy(), 1e-6, 1e4)
    assert int(w.status) == 0


@pytest.mark.parametrize("n_seq", [1, 2, 31, 32, 33, 64, 65, 1000])
def test_append_finds_every_row(torch, B, n_seq):
    news = [(n * 7) % 4 for n in range(n_seq)]
    news[-1] = 1
    w = World(torch, [m + n % 20 for n, m in enumerate(news)], news, 1, 128, 16, "fp32", seed=n_seq)
    w.device(B).append(w.c.cuda(), w.k.cuda())
    check_append(w, None, None, None, 0, None)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("H", [3, 20])
def test_append_to_absorbed_queries_from_one_projection(torch, B, dtype, page, H):
    """Equal chunks, shifted positions; latent and key part are columns of one tensor, queries the last columns of theirs,
    and go to the last columns of the absorbed ones."""
    rank = 256
    w = World(torch, [200, 130, 129], [3, 3, 3], H, rank, page, dtype, seed=page)
    mem = w.device(B, starts=False)
    down = torch.cat([w.c, w.k, torch.zeros(w.rows, 8, dtype=w.t)], 1).cuda()
    q = torch.randn(w.rows, H, 136, generator=w.gen).to(w.t).cuda()
    absorbed = torch.full((w.rows, H, rank + ROPE), 7.0, dtype=w.t, device="cuda")
    pos0 = torch.tensor([0, 70000, 5], dtype=torch.int32)
    rot = torch.from_numpy(B.rotation_table(70200, ROPE, 1e4)).cuda()
    got = mem.append(down[:, :rank], down[:, rank:rank + ROPE], q[..., 72:], None, 0.0, rot, pos0.cuda(), out=absorbed[..., rank:])
    check_append(w, q[..., 72:], got, None, 0, 1e4, pos0)
    assert (absorbed[..., :rank] == 7).all() and int(w.status) == 0
    w.device(B, starts=False)
    before = q.clone()
    same = mem.append(None, None, q[..., 72:], rotation=rot, pos0=pos0.cuda(), out=q[..., 72:])          # in place
    check_append(w, before[..., 72:], same, None, 0, 1e4, pos0, tokens=False)
    assert torch.equal(q[..., :72], before[..., :72])


@pytest.mark.parametrize("dtype", DTYPES)
def test_append_of_many_rows(torch, B, dtype):
    news = [700, 0, 1500, 1, 3000]
    w = World(torch, [900, 5, 1500, 77, 3100], news, 4, 512, 64, dtype, seed=5)
    mem = w.device(B)
    gain, rot = torch.linspace(0.5, 2, 512), torch.from_numpy(B.rotation_table(3200, ROPE, 1e4)).cuda()
    q = w.q.cuda()[..., 512:]
    got = mem.append(w.c.cuda(), w.k.cuda(), q, gain.cuda(), 1e-5, rot)
    check_append(w, q, got, gain.double().numpy(), 1e-5, 1e4)
    assert int(w.status) == 0


def test_append_reports_what_it_cannot_place(torch, B):
    w = World(torch, [20, 40, 5, 18], [2, 2, 5, 1], 2, 128, 16, "bf16", max_pages=3, stale=False)
    w.table[0, 1] = 10 ** 6                                        # its two tokens are 18 and 19: page 1
    mem = w.device(B)
    w.dlens.copy_(torch.tensor([20, 60, 3, 18], dtype=torch.int32))         # 60 is past 3 pages; 3 tokens of 5 new
    out = torch.full((w.rows, 2, ROPE), 7.0, dtype=w.t, device="cuda")
    rot = torch.from_numpy(B.rotation_table(18, ROPE)).cuda()
    q = w.q.cuda()[..., 128:]
    mem.append(w.c.cuda(), w.k.cuda(), q, rotation=rot, out=out)
    assert mem.status() == B.ERR_CORRUPT
    o = out.cpu()
    assert (o[:4] == 7).all()                                      # bad page, past the table
    assert (o[4:6] == 7).all() and (o[6:9] != 7).any()             # tokens -2, -1 of sequence 2, then 0 .. 2
    assert (o[9] != 7).any()                                       # token 17, the last of the rotation table
    mem.append(None, None, q, rotation=rot[:17], out=out)
    assert mem.status() == B.ERR_CORRUPT and mem.status() == B.OK


# ---------------------------------------------------------------- attend

@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rank", RANKS)
@pytest.mark.parametrize("H", HEADS)
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 7), (False, 70)])
def test_attend(torch, B, dtype, rank, H, causal, window):
    w = World(torch, [37, 1, 0, 16, 130, 300, 9], [5, 1, 0, 16, 33, 3, 0], H, rank, 16, dtype, seed=rank + H, spare_rows=3)
    mem = w.device(B)
    out = torch.full((w.rows, H, rank), 7.0, dtype=w.t, device="cuda")
    got = mem.attend(w.q.cuda(), w.scale, causal=causal, window=window, max_new=33, max_len=300, out=out)
    assert got is out and (out[-3:] == 7).all()
    w.check_attend(got, causal=causal, window=window)
    assert int(w.status) == 0


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("page", [32, 64, 128])
@pytest.mark.parametrize("m", [1, 2, 15, 16, 17, 31, 64, 65, 129])
def test_attend_chunks(torch, B, dtype, page, m):
    w = World(torch, [m + 300, m], [m, m], 4, 128, page, dtype, seed=m)
    mem = w.device(B, starts=False)
    w.check_attend(mem.attend(w.q.cuda(), w.scale), causal=True)
    w.check_attend(mem.attend(w.q.cuda(), -0.05, causal=False), causal=False, scale=-0.05)
    assert int(w.status) == 0


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rank", RANKS)
@pytest.mark.parametrize("length", [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 255, 256, 257, 1023, 5000])
def test_attend_single_tokens(torch, B, dtype, rank, length):
    w = World(torch, [length, max(1, length // 3), 1], [1, 1, 1], 8, rank, 16, dtype, seed=length)
    mem = w.device(B, starts=False)
    w.check_attend(mem.attend(w.q.cuda(), w.scale))
    w.check_attend(mem.attend(w.q.cuda(), w.scale, window=40), window=40)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rank,H,m,length", [(256, 8, 32, 2100), (128, 16, 100, 1500), (512, 16, 40, 900), (256, 64, 9, 1300)])
def test_attend_long(torch, B, dtype, rank, H, m, length):
    w = World(torch, [length, length // 2 + m], [m, m - m // 3], H, rank, 64, dtype, seed=m)
    mem = w.device(B)
    for causal, window in ((True, 0), (False, 0), (True, 333)):
        w.check_attend(mem.attend(w.q.cuda(), w.scale, causal=causal, window=window, max_new=m), causal=causal, window=window)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rank", RANKS)
@pytest.mark.parametrize("H", [1, 3])
def test_attend_again_and_again(torch, B, dtype, rank, H):
    """Chunks of one item and of several over memories of some tiles, whole and in pieces: every call gives the same."""
    news = [187, 156, 0, 125, 94, 180, 149, 118, 187, 33]
    w = World(torch, [2295 - 97 * n if n % 3 else 187 + n for n in range(len(news))], news, H, rank, 64, dtype, seed=rank)
    mem, q = w.device(B), w.q.cuda()
    want = mem.attend(q, w.scale, max_new=187)
    w.check_attend(want)
    for _ in range(50):
        assert torch.equal(mem.attend(q, w.scale, max_new=187), want)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rank", RANKS)
@pytest.mark.parametrize("N", [3, 40, 400])
def test_attend_many_sequences(torch, B, dtype, rank, N):
    w = World(torch, [1 + (n * 97) % 260 for n in range(N)], [1] * N, 4, rank, 32, dtype, seed=N)
    mem = w.device(B)
    w.check_attend(mem.attend(w.q.cuda(), w.scale, max_new=1, max_len=max(w.lens)))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m", [3, 40])
def test_attend_rows_without_tokens_and_chunks_longer_than_the_memory(torch, B, dtype, m):
    w = World(torch, [2, 0], [m, m], 4, 128, 16, dtype, seed=m)
    mem = w.device(B)
    got = mem.attend(w.q.cuda(), w.scale, max_new=m)
    w.check_attend(got)
    assert (got[:m - 2] == 0).all() and (got[m:] == 0).all()
    assert int(w.status) == 0
    assert (mem.attend(w.q.cuda(), w.scale, max_new=m, causal=False)[m:] == 0).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rank", RANKS)
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
def test_attend_what_masked_tokens_hold(torch, B, dtype, rank, value):
    """A value that is not finite reaches the rows that see it, and no others."""
    m, length = 12, 400
    w = World(torch, [length], [m], 4, rank, 16, dtype, seed=3)
    page, slot = int(w.table[0, (length - 5) // 16]), (length - 5) % 16    # row 7 is the first that sees it
    w.pages[page, slot, 3] = value
    far = int(w.table[0, 100 // 16])
    w.pages[far, 100 % 16, rank + 1] = value                               # outside every window of 200
    mem = w.device(B)
    got = mem.attend(w.q.cuda(), w.scale, window=200)
    x = w.dense(0)
    x[length - 5, 3] = 0
    out, size, dots = L.attend(w.q.double().numpy(), x, rank, w.scale, True, 200)
    weight = 2 * (rank + 72) * U * dots + 2.0 ** -20 + (2.0 ** -8 if dtype == "bf16" else 0.0)
    tol = half(dtype) * np.abs(out) + (1 + half(dtype)) * (weight + length * U) * size + 1e-37
    assert (np.abs(got.double().cpu().numpy() - out) <= tol)[:7].all()
    assert not torch.isfinite(got[7:, :, 3]).any()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rank", RANKS)
def test_attend_scores_that_grow(torch, B, dtype, rank):
    """Each run of tokens has larger scores than those before it, so that every reference is raised, and some scores are huge."""
    length = 700
    w = World(torch, [length], [1], 8, rank, 64, dtype, seed=9)
    growth = torch.linspace(0.01, 4, length)
    for n in range(length):
        w.pages[int(w.table[0, n // 64]), n % 64, rank:] = (growth[n] * torch.ones(ROPE)).to(w.t)
    w.q[..., rank:] = 1
    w.q[:, 3, rank:] = -1
    mem = w.device(B)
    for scale in (1.0, 0.1, 0.0, 1e-30):
        w.check_attend(mem.attend(w.q.cuda(), scale), scale=scale)


def test_attend_huge_scores(torch, B):
    """Scores of 2^100 and more: the largest weight is 1 and the others none."""
    for dtype in DTYPES:
        w = World(torch, [300], [1], 4, 128, 16, dtype, seed=4)
        w.pages[..., 128:] = 0
        w.pages[..., :128] = w.pages[..., :128].sign() * 0.5
        w.pages[int(w.table[0, 9]), 5, :128] = 1.0
        w.q[..., :128] = 2.0 ** 100
        mem = w.device(B)
        got = mem.attend(w.q.cuda(), 1.0)
        assert (got == 1).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_attend_strided_rows_and_bounds(torch, B, dtype):
    w = World(torch, [100, 260, 31], [4, 9, 1], 6, 128, 32, dtype, seed=8)
    mem = w.device(B)
    buf = torch.full((w.rows, 6 * (192 + 128) + 16), 7.0, dtype=w.t, device="cuda")
    q, out = buf[:, :6 * 192].unflatten(1, (6, 192)), buf[:, 6 * 192 + 8:-8].unflatten(1, (6, 128))
    q.copy_(w.q)
    mem.attend(q, w.scale, out=out)
    w.check_attend(out)
    assert (buf[:, 6 * 192:6 * 192 + 8] == 7).all() and (buf[:, -8:] == 7).all()
    exact = mem.attend(q, w.scale, max_new=9, max_len=260)
    w.check_attend(exact)
    assert torch.equal(exact, mem.attend(q, w.scale, max_new=9, max_len=260))


@pytest.mark.parametrize("dtype,rank", [("bf16", 128), ("bf16", 512), ("fp32", 256)])
def test_attend_chunks_far_below_their_bound(torch, B, dtype, rank):
    """max_new left to the number of rows: most of the launch's items are behind their sequences' rows."""
    news = [0, 1, 260, 0, 2] + [1] * 30 + [37]
    w = World(torch, [n + 7 * i % 140 for i, n in enumerate(news)], news, 64, rank, 16, dtype, seed=5)
    mem = w.device(B)
    w.check_attend(mem.attend(w.q.cuda(), w.scale))
    assert int(w.status) == 0


@pytest.mark.parametrize("dtype", DTYPES)
def test_attend_more_items_than_a_block_counts(torch, B, dtype):
    w = World(torch, [1 + (n * 37) % 200 for n in range(2100)], [1] * 2100, 3, 128, 32, dtype, seed=6)
    w.check_attend(w.device(B, starts=False).attend(w.q.cuda(), w.scale))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rank", RANKS)
@pytest.mark.parametrize("H", [129, 1000, 1024])
def test_attend_many_heads(torch, B, dtype, rank, H):
    w = World(torch, [170, 1, 300], [1, 1, 2], H, rank, 64, dtype, seed=H)
    mem = w.device(B)
    w.check_attend(mem.attend(w.q.cuda(), w.scale, max_new=2))
    w.check_attend(mem.attend(w.q.cuda(), w.scale, max_new=2, window=33), window=33)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rank", RANKS)
@pytest.mark.parametrize("strided", [False, True])
@pytest.mark.parametrize("window", [0, 60])
def test_attend_chunks_what_masked_tokens_hold(torch, B, dtype, rank, strided, window):
    """As above, with chunks of many rows, several items a sequence, and rows behind the last sequence that are no numbers."""
    m, length, H = 60, 700, 6
    w = World(torch, [length, length], [m, m], H, rank, 32, dtype, seed=3, spare_rows=30)
    w.q[2 * m:] = float("nan")
    for at, column in ((length - 20, 3), (length - 9, rank + 5)):          # rows 40 and 51 are the first that see them
        w.pages[int(w.table[0, at // 32]), at % 32, column] = float("nan")
    mem, q = w.device(B), w.q.cuda()
    buf = torch.full((w.rows, H * (2 * rank + ROPE) + 32), 7.0, dtype=w.t, device="cuda")
    out = buf[:, H * (rank + ROPE) + 16:-16].unflatten(1, (H, rank))
    if strided:
        buf[:, :H * (rank + ROPE)].copy_(q.flatten(1))
        q = buf[:, :H * (rank + ROPE)].unflatten(1, (H, rank + ROPE))
    mem.attend(q, w.scale, window=window, max_new=m, out=out)
    assert (buf[:, H * (rank + ROPE):H * (rank + ROPE) + 16] == 7).all() and (buf[:, -16:] == 7).all() and (out[2 * m:] == 7).all()
    got = out.double().cpu().numpy()
    for n in range(2):
        x, rows = w.dense(n), 40 if n == 0 else m
        x[np.isnan(x)] = 0
        want, size, dots = L.attend(w.q[n * m:(n + 1) * m].double().numpy(), x, rank, w.scale, True, window)
        weight = 2 * (rank + 72) * U * dots + 2.0 ** -20 + (2.0 ** -8 if dtype == "bf16" else 0.0)
        tol = half(dtype) * np.abs(want) + (1 + half(dtype)) * (weight + length * U) * size + 1e-37
        assert (np.abs(got[n * m:(n + 1) * m] - want) <= tol)[:rows].all()
    assert not np.isfinite(got[40:m, :, 3]).any() and not np.isfinite(got[51:m]).any()


EDGE = 2.0 ** 128 - 2.0 ** 116                                            # fp32 rows: from here on a number counts as infinite
BELOW = float(np.nextafter(np.float32(EDGE), np.float32(0)))
MOST = {"fp32": float(np.finfo(np.float32).max), "bf16": 2.0 ** 128 - 2.0 ** 120}


@pytest.mark.parametrize("rank", RANKS)
@pytest.mark.parametrize("dtype,value", [("fp32", v) for v in (MOST["fp32"], -MOST["fp32"], EDGE, -EDGE, BELOW)]
                         + [("bf16", v) for v in (MOST["bf16"], -MOST["bf16"])])
def test_attend_masked_tokens_of_the_largest_values(torch, B, dtype, rank, value):
    """Latents and key parts at the types' ends: what one row sees reaches no other, within an item and across them."""
    m, length = 12, 400
    w = World(torch, [length], [m], 4, rank, 16, dtype, seed=3)
    for at, column in ((length - 5, 3), (length - 3, rank + 1), (length - 2, rank - 1)):   # row 7 is the first that sees one
        w.pages[int(w.table[0, at // 16]), at % 16, column] = value
    assert w.pages.isinf().sum() == 0
    mem = w.device(B)
    for window in (0, 200):
        got = mem.attend(w.q.cuda(), w.scale, window=window).double().cpu().numpy()
        x = w.dense(0)
        x[length - 5:] = 0                                                 # rows 0 .. 6 do not see them
        out, size, dots = L.attend(w.q.double().numpy()[:7], x[:length - 5], rank, w.scale, True, window)
        weight = 2 * (rank + 72) * U * dots + 2.0 ** -20 + (2.0 ** -8 if dtype == "bf16" else 0.0)
        tol = half(dtype) * np.abs(out) + (1 + half(dtype)) * (weight + length * U) * size + 1e-37
        assert (np.abs(got[:7] - out) <= tol).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rank", RANKS)
@pytest.mark.parametrize("N,m", [(1, 1), (1, 20), (76, 1), (76, 20)])
def test_attend_scores_beyond_fp32_once_scaled(torch, B, dtype, rank, N, m):
    """Scores are fp32 numbers and so is the scale, their products are not: a few long memories in pieces and many whole ones.
    The token of the largest score has all of the weight, and tokens of one score share it equally."""
    H, length, page = 8, 3000 if N == 1 else 250, 64
    w = World(torch, [length] * N, [m] * N, H, rank, page, dtype, seed=4, stale=False)
    eighth = torch.arange(page) % 8 == 7
    w.q[...] = 0
    w.q[..., 1:rank] = 2.0 ** 100
    q = w.q.cuda()

    def attend(scale, best=None, q=q):                                     # tokens of 0.5, but one
        w.pages[..., :rank] = 0.5
        w.pages[..., 0] = eighth.to(w.t)
        if best is not None:
            for n in range(N):
                w.pages[int(w.table[n, (length - 9) // page]), (length - 9) % page, :rank] = best
        mem = w.device(B, starts=False)
        got = mem.attend(q, scale, causal=False).double().cpu()
        assert mem.status() == B.OK
        return got

    assert (attend(2.0 ** 60, 1.0) == 1).all()
    assert (attend(-2.0 ** 60, 0.25) == 0.25).all()                        # all scores far below zero
    assert (attend(2.0 ** 60, 0.25, -q) == 0.25).all()
    # the mean of 0 and 1 over the tokens, whose weights are 1 each: their count is exact
    mean = (length // 8) / length
    for scale in (2.0 ** 60, -2.0 ** 60):
        got = attend(scale)
        assert (got[..., 1:] == 0.5).all()
        assert ((got[..., 0] - mean).abs() <= (half(dtype) + 4 * U) * mean).all()   # a sum's reciprocal, a product and the result's rounding


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rank", RANKS)
@pytest.mark.parametrize("N,m", [(1, 1), (152, 1), (1, 20), (76, 20)])
def test_attend_scores_near_the_lowest_number(torch, B, dtype, rank, N, m):
    """The first 200 tokens have scores of -1.75 * 2^127, which a scale of 1e-37 makes -29.8 beside the others' 0."""
    H, length, page = 8, 600, 64
    w = World(torch, [length] * N, [m] * N, H, rank, page, dtype, seed=5, stale=False)
    tokens = torch.zeros(w.table.shape[1] * page, rank + ROPE)
    tokens[:200, 1], tokens[200:, 1] = 1, 2
    tokens[:200, rank + 3] = -1.75 * 2.0 ** 63
    for n in range(N):
        w.pages[w.table[n].long()] = tokens.to(w.t).unflatten(0, (-1, page))
    w.q[...] = 0
    w.q[..., rank + 3] = 2.0 ** 64
    mem = w.device(B, starts=False)
    w.check_attend(mem.attend(w.q.cuda(), 1e-37, causal=False), causal=False, scale=1e-37)
    w.check_attend(mem.attend(w.q.cuda(), 1e-37, causal=False, window=450), causal=False, scale=1e-37, window=450)
    w.lens = [200] * N                                                     # and no others
    w.check_attend(w.device(B, starts=False).attend(w.q.cuda(), 1e-37, causal=False), causal=False, scale=1e-37)


def test_attend_reports_bad_entries(torch, B):
    for dtype in DTYPES:
        w = World(torch, [40, 40, 40], [1, 1, 1], 4, 128, 16, dtype, max_pages=4, stale=False)
        good = w.device(B).attend(w.q.cuda(), w.scale)
        w.table[1, 2] = 10 ** 6
        mem = w.device(B)
        got = mem.attend(w.q.cuda(), w.scale)
        assert mem.status() == B.ERR_CORRUPT and torch.equal(got[[0, 2]], good[[0, 2]])
        w.table[1, 2] = -1
        mem = w.device(B)
        mem.attend(w.q.cuda(), w.scale)
        assert mem.status() == B.ERR_CORRUPT
        w.table[1, 2] = 0
        mem = w.device(B)
        w.dlens.copy_(torch.tensor([40, -3, 65], dtype=torch.int32))
        mem.attend(w.q.cuda(), w.scale)
        assert mem.status() == B.ERR_CORRUPT
        w.dlens.copy_(torch.tensor([40, 40, 40], dtype=torch.int32))
        mem.tensors[3].copy_(torch.tensor([0, 2, 1, 3], dtype=torch.int32))
        mem.attend(w.q.cuda(), w.scale, max_new=2)
        assert mem.status() == B.ERR_CORRUPT


# ---------------------------------------------------------------- expand

class Expanded:
    def __init__(self, w, B, page, format=None):
        torch = w.torch
        self.w, self.page = w, page
        self.table, pages = w.shuffled(page, w.gen)
        self.before = [torch.randn(pages, w.H, page, 128, generator=w.gen).to(w.t) for _ in range(2)]
        self.pages = [p.cuda() for p in self.before]
        self.w_k, self.w_v = (torch.randn(w.H, d, w.rank, generator=w.gen).mul(w.rank ** -0.5).to(w.t) for d in (64, 128))
        self.dtable = self.table.cuda()
        self.mem = B.Memory(*self.pages, self.dtable, w.dlens, w.H, starts=w.starts.cuda(), dtype=w.dtype)

    def check(self, first=None, skip=()):
        w, torch = self.w, self.w.torch
        got = [p.cpu() for p in self.pages]
        touched = torch.zeros(got[0].shape[0], self.page, dtype=torch.bool)
        wk, wv = self.w_k.double().numpy(), self.w_v.double().numpy()
        for n, ln in enumerate(w.lens):
            lo = 0 if first is None else int(first[n])
            if n in skip or ln <= lo:
                continue
            pos = torch.arange(lo, ln)
            at, slot = self.table[n][pos // self.page].long(), pos % self.page
            touched[at, slot] = True
            x = w.dense(n)[lo:]
            keys, values = L.expand(x, wk, wv)
            size = L.expand(np.abs(x), np.abs(wk), np.abs(wv))
            k, v = (p.transpose(1, 2)[at, slot].double().numpy() for p in got)
            assert np.array_equal(k[..., 64:], keys[..., 64:])             # copied
            for g, want, s in ((k[..., :64], keys[..., :64], size[0][..., :64]), (v, values, size[1])):
                tol = (half(w.dtype) * np.abs(want) + (w.rank + 8) * U * s) * (1 + half(w.dtype)) + 1e-37
                assert (np.abs(g - want) <= tol).all(), (n, float((np.abs(g - want) / tol).max()))
        for g, b in zip(got, self.before):
            same = (g.view(torch.uint8) == b.view(torch.uint8)).all(-1).transpose(1, 2).all(-1)
            assert same[~touched].all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rank", RANKS)
@pytest.mark.parametrize("H", [1, 3, 8])
@pytest.mark.parametrize("page,to", [(16, 16), (64, 16), (32, 128)])
def test_expand(torch, B, dtype, rank, H, page, to):
    w = World(torch, [130, 1, 0, 64, 300, 129], [1] * 6, H, rank, page, dtype, seed=rank + H)
    mem = w.device(B)
    e = Expanded(w, B, to)
    mem.expand(e.w_k.cuda(), e.w_v.cuda(), e.mem)
    e.check()
    assert mem.status() == B.OK


@pytest.mark.parametrize("dtype", DTYPES)
def test_expand_of_the_newest_tokens(torch, B, dtype):
    w = World(torch, [130, 1, 0, 640, 300, 129], [1] * 6, 4, 256, 32, dtype, seed=7)
    mem = w.device(B)
    e = Expanded(w, B, 64)
    first = torch.tensor([3, 1, 0, 500, 299, 0], dtype=torch.int32)
    mem.expand(e.w_k.cuda(), e.w_v.cuda(), e.mem, first=first.cuda(), max_new=140, max_len=640)
    e.check(first)
    assert mem.status() == B.OK


@pytest.mark.parametrize("dtype", DTYPES)
def test_expand_with_a_loose_bound_on_the_new_tokens(torch, B, dtype):
    w = World(torch, [130, 1, 0, 64], [1] * 4, 4, 128, 16, dtype, seed=7, max_pages=60)
    mem = w.device(B)
    e = Expanded(w, B, 64)
    mem.expand(e.w_k.cuda(), e.w_v.cuda(), e.mem, max_new=60 * 16, max_len=130)
    e.check()
    assert mem.status() == B.OK


@pytest.mark.parametrize("dtype", DTYPES)
def test_expand_long_memories(torch, B, dtype):
    w = World(torch, [2500, 777], [1, 1], 10, 128, 128, dtype, seed=2)
    mem = w.device(B)
    e = Expanded(w, B, 128)
    mem.expand(e.w_k.cuda(), e.w_v.cuda(), e.mem)
    e.check()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rank", RANKS)
def test_expand_few_tokens_of_many_sequences(torch, B, dtype, rank):
    w = World(torch, [(n * 31) % 90 for n in range(170)], [1] * 170, 5, rank, 16, dtype, seed=8)
    mem = w.device(B)
    e = Expanded(w, B, 32)
    for most in (3, 16, 17):
        for p, b in zip(e.pages, e.before):
            p.copy_(b)
        first = torch.tensor([max(0, ln - n % (most + 1)) for n, ln in enumerate(w.lens)], dtype=torch.int32)
        mem.expand(e.w_k.cuda(), e.w_v.cuda(), e.mem, first=first.cuda(), max_new=most)
        e.check(first)
    assert mem.status() == B.OK


@pytest.mark.parametrize("dtype", DTYPES)
def test_expand_reports_what_it_cannot_write(torch, B, dtype):
    w = World(torch, [100, 60, 60, 60, 60], [1] * 5, 2, 128, 16, dtype, seed=6, stale=False)
    mem = w.device(B)
    e = Expanded(w, B, 16)
    first = torch.tensor([0, -1, 61, 0, 50], dtype=torch.int32)           # too many; before the memory; behind it; fine; fine
    mem.expand(e.w_k.cuda(), e.w_v.cuda(), e.mem, first=first.cuda(), max_new=60)
    assert mem.status() == B.ERR_CORRUPT
    e.check(first, skip=(0, 1, 2))
    bad = w.table.clone()
    bad[3, 1] = 10 ** 6                                                   # tokens 16 .. 31 of sequence 3
    w.dtable.copy_(bad)
    e.dtable[4, 3] = -1                                                   # tokens 48 .. 59 of sequence 4
    for p, b in zip(e.pages, e.before):
        p.copy_(b)
    first = torch.tensor([100, 60, 60, 0, 45], dtype=torch.int32)
    mem.expand(e.w_k.cuda(), e.w_v.cuda(), e.mem, first=first.cuda())
    assert mem.status() == B.ERR_CORRUPT
    got, was = e.pages[0].cpu(), e.before[0]
    assert torch.equal(got[int(e.table[3, 1])], was[int(e.table[3, 1])])  # not written
    assert torch.equal(got[int(e.table[4, 3])], was[int(e.table[4, 3])])
    assert not torch.equal(got[int(e.table[3, 0])], was[int(e.table[3, 0])])
    assert not torch.equal(got[int(e.table[4, 2]), :, 13:], was[int(e.table[4, 2]), :, 13:])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rank", RANKS)
@pytest.mark.parametrize("most", [120, 16])
def test_expand_values_that_are_not_finite(torch, B, dtype, rank, most):
    """Infinities, NaN and the largest numbers in latents and maps: as the definition has it, product by product."""
    w = World(torch, [120, 40], [1, 1], 3, rank, 16, dtype, seed=21, stale=False)
    largest = MOST[dtype]
    special = [float("inf"), float("-inf"), float("nan"), largest, -largest, EDGE if dtype == "fp32" else largest, BELOW if dtype == "fp32" else -largest]
    at = [119 - 2 * i for i in range(len(special))]
    for i, v in zip(at, special):
        w.pages[int(w.table[0, i // 16]), i % 16, rank // 2] = v
    w.pages[int(w.table[1, 2]), 7, :2] = torch.tensor([float("inf"), float("-inf")])      # token 39: no number
    w.pages[int(w.table[1, 2]), 6, 1] = 0.25                              # token 38
    w.pages[:, :, 0] *= 0.125                                             # meets the largest weight: no product overflows
    mem = w.device(B)
    e = Expanded(w, B, 32)
    e.w_k[:, 3, rank // 2] = 0                                            # 0 * inf, and 0 * the largest
    e.w_v[1, 5, 0] = largest
    e.w_v[2, 9, 1] = float("inf")
    first = torch.tensor([max(0, ln - most) for ln in w.lens], dtype=torch.int32)
    mem.expand(e.w_k.cuda(), e.w_v.cuda(), e.mem, first=first.cuda(), max_new=most)
    assert mem.status() == B.OK
    wk, wv = e.w_k.double().numpy(), e.w_v.double().numpy()
    pages = [p.cpu() for p in e.pages]
    found = 0
    for n, ln in enumerate(w.lens):
        pos = torch.arange(int(first[n]), ln)
        where, slot = e.table[n][pos // 32].long(), pos % 32
        x = w.dense(n)[int(first[n]):]
        with np.errstate(invalid="ignore", over="ignore"):
            # the sums in the order of the dimensions, so that no infinity comes from elsewhere
            want = [np.zeros((len(x), 3, 64)), np.zeros((len(x), 3, 128))]
            size = [np.zeros_like(y) for y in want]
            for j in range(rank):
                for y, s, maps in zip(want, size, (wk, wv)):
                    y += x[:, j, None, None] * maps[None, :, :, j]
                    s += np.abs(x[:, j, None, None] * maps[None, :, :, j])
            for p, y, s, width in zip(pages, want, size, (64, 128)):
                got = p.transpose(1, 2)[where, slot].double().numpy()[..., :width]
                over = np.abs(y) > MOST[dtype] * (1 + half(dtype) / 2)     # an infinity of the type, or within a rounding of one
                odd = ~np.isfinite(y)
                assert np.array_equal(np.isnan(got), np.isnan(y))
                assert np.array_equal(got[np.isinf(y)], y[np.isinf(y)])
                fine = ~odd & ~over
                tol = (half(dtype) * np.abs(y) + (rank + 8) * U * s) * (1 + half(dtype)) + 1e-37
                assert (np.abs(got - y) <= tol)[fine].all()
                found += int(odd.sum())
    assert found > 100


# ---------------------------------------------------------------- as they are used

@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rank,H", [(128, 4), (256, 8), (512, 3)])
def test_a_policys_steps_absorbed_and_expanded(torch, B, dtype, rank, H):
    """Three observations are remembered and attended to, absorbed for the queries over latents and expanded to keys and
    values; both against one float64 run over what the memory holds."""
    N, news, page = 3, [[40, 7, 90], [1, 1, 1], [5, 64, 1]], 16
    lens, total = [0] * N, [46, 72, 92]
    w = World(torch, total, [1] * N, H, rank, page, dtype, seed=rank, stale=False)
    w.device(B)
    e = Expanded(w, B, page)
    g, rot = torch.Generator().manual_seed(1), torch.from_numpy(B.rotation_table(128, ROPE)).cuda()
    gain = 1 + 0.1 * torch.randn(rank, generator=g)
    wk, wv = e.w_k.cuda(), e.w_v.cuda()
    for new in news:
        lens = [a + b for a, b in zip(lens, new)]
        rows = sum(new)
        w.dlens.copy_(torch.tensor(lens, dtype=torch.int32))
        starts = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32)
        mem = B.LatentMemory(w.dpages, w.dtable, w.dlens, H, starts=starts.cuda(), status=w.status)
        full = B.Memory(*e.pages, e.dtable, w.dlens, H, starts=starts.cuda(), dtype=dtype)
        down = torch.randn(rows, rank + ROPE, generator=g).to(w.t).cuda()
        q = torch.randn(rows, H, 128, generator=g).to(w.t).cuda()
        absorbed = torch.empty(rows, H, rank + ROPE, dtype=w.t, device="cuda")
        absorbed[..., :rank] = torch.einsum("mhd,hdr->mhr", q[..., :64].float(), wk.float()).to(w.t)
        mem.append(down[:, :rank], down[:, rank:], q[..., 64:], gain.cuda(), 1e-6, rot, out=absorbed[..., rank:])
        got = mem.attend(absorbed, w.scale, max_new=max(new))
        first = w.dlens - starts.diff().cuda()
        mem.expand(wk, wv, full, first=first, max_new=max(new))           # the new tokens
        q[..., 64:] = absorbed[..., rank:]
        wide = full.attend(q, w.scale, max_new=max(new))
        w.lens, w.news, w.starts = lens, new, starts
        w.check_attend(got, q=absorbed, pages=w.dpages)
        for n in range(N):
            a, b = int(starts[n]), int(starts[n + 1])
            at = e.table[n, :-(-lens[n] // page)].long()
            k, v = (p.cpu()[at].double().numpy().transpose(0, 2, 1, 3).reshape(-1, H, 128)[:lens[n]] for p in e.pages)
            out, size, dots = M.attend(q[a:b].double().cpu().numpy(), k, v, H, w.scale, True, 0)
            h = half(dtype)
            tol = h * np.abs(out) + (1 + h) * (2 * 136 * U * dots + 2.0 ** -20 + h + lens[n] * U) * size
            assert (np.abs(wide[a:b].double().cpu().numpy() - out) <= tol).all()
        # the two ways round different things: the absorbed queries, the keys and the values, each by h.  A score of at
        # most `dots` moves by 2 h of it, a weight by twice that, and the value map adds h of its sums
        up = torch.einsum("mhr,hdr->mhd", got.double(), wv.double()).cpu().numpy()
        for n in range(N):
            a, b = int(starts[n]), int(starts[n + 1])
            x = w.dense(n, w.dpages)
            _, size, dots = L.attend(absorbed[a:b].double().cpu().numpy(), x, rank, w.scale, True, 0)
            move = (4 * half(dtype) * dots + 4 * half(dtype) + 2.0 ** -18 + 4 * (rank + 72) * U * dots)
            tol = move * np.einsum("mhr,hdr->mhd", size, np.abs(wv.double().cpu().numpy())) + 1e-6
            assert (np.abs(wide[a:b].double().cpu().numpy() - up[a:b]) <= tol).all()
    assert int(w.status) == 0


def test_calls_in_a_graph_follow_the_lengths(torch, B):
    """append and attend of one token, captured once and replayed as the memory grows."""
    w = World(torch, [200, 90], [1, 1], 8, 256, 16, "bf16", seed=11, stale=False)
    mem = w.device(B, starts=False)
    rot = torch.from_numpy(B.rotation_table(256, ROPE)).cuda()
    c, k, q, out = w.c.cuda(), w.k.cuda(), w.q.cuda(), torch.empty(2, 8, 256, dtype=torch.bfloat16, device="cuda")
    w.dlens.copy_(torch.tensor([150, 40], dtype=torch.int32))
    mem.append(c, k, rotation=rot)
    mem.attend(q, w.scale, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mem.append(c, k, rotation=rot)
        mem.attend(q, w.scale, out=out)
    for lens in ([151, 41], [160, 48], [200, 90]):
        w.dlens.copy_(torch.tensor(lens, dtype=torch.int32))
        c.normal_()
        graph.replay()
        w.lens = lens
        w.check_attend(out, pages=w.dpages)
        got = [w.dense(n, w.dpages)[-1, :256] for n in range(2)]
        assert np.array_equal(np.stack(got), c.double().cpu().numpy())
    assert mem.status() == B.OK


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m", [1, 40])
def test_two_graphs_of_split_memories(torch, B, dtype, m):
    """Two captured calls on streams of their own, replayed at once and in turn, over lengths that change in between."""
    worlds = [World(torch, [4000, 130, 900], [m] * 3, 4, 128, 64, dtype, seed=20 + i, stale=False) for i in range(2)]
    mems = [w.device(B, starts=False) for w in worlds]
    qs, outs, graphs = [w.q.cuda() for w in worlds], [None, None], [torch.cuda.CUDAGraph() for _ in range(2)]
    for mem, q, w in zip(mems, qs, worlds):
        mem.attend(q, w.scale)
    torch.cuda.synchronize()
    for i in range(2):
        with torch.cuda.graph(graphs[i]):
            outs[i] = mems[i].attend(qs[i], worlds[i].scale)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for lens in ([4000, 130, 900], [130, 100, 41], [60, 60, 60]):
        for w in worlds:
            w.lens = lens
            w.dlens.copy_(torch.tensor(lens, dtype=torch.int32))
        torch.cuda.synchronize()
        for _ in range(5):
            for s, g in zip(streams, graphs):
                with torch.cuda.stream(s):
                    g.replay()
        torch.cuda.synchronize()
        for w, out, mem in zip(worlds, outs, mems):
            w.check_attend(out)
            assert mem.status() == B.OK


@pytest.mark.parametrize("dtype", DTYPES)
def test_offsets_beyond_32_bits(torch, B, dtype):
    """Pools of more than 2^31 values: the same calls on their last pages give the same."""
    H, rank, page = 4, 512, 128
    w = World(torch, [300, 129, 40], [1, 60, 1], H, rank, page, dtype, seed=31, stale=False)
    mem = w.device(B)
    e = Expanded(w, B, page)
    far, far_to = 2 ** 31 // (page * (rank + ROPE)) + 5, 2 ** 31 // (page * H * 128) + 5
    pool = torch.empty(far + len(w.pages), page, rank + ROPE, dtype=w.t, device="cuda")
    pool[far:] = w.dpages
    keys, values = (torch.empty(far_to + len(p), H, page, 128, dtype=w.t, device="cuda") for p in e.pages)
    for big, p in ((keys, e.pages[0]), (values, e.pages[1])):
        big[far_to:] = p
    assert min(pool.numel(), keys.numel()) > 2 ** 31
    starts = w.starts.cuda()
    large = B.LatentMemory(pool, torch.where(w.dtable >= 0, w.dtable + far, w.dtable), w.dlens, H, starts=starts)
    to = B.Memory(keys, values, torch.where(e.dtable >= 0, e.dtable + far_to, e.dtable), w.dlens, H, starts=starts, dtype=dtype)
    c, k, q = w.c.cuda(), w.k.cuda(), w.q.cuda()
    for m, memory in ((mem, e.mem), (large, to)):
        m.append(c, k)
        m.expand(e.w_k.cuda(), e.w_v.cuda(), memory)
    assert torch.equal(pool[far:], w.dpages)
    assert torch.equal(keys[far_to:], e.pages[0]) and torch.equal(values[far_to:], e.pages[1])
    assert torch.equal(large.attend(q, w.scale, max_new=60), mem.attend(q, w.scale, max_new=60))
    w.check_attend(large.attend(q, w.scale, max_new=60), pages=w.dpages)
    assert large.status() == B.OK


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m", [1, 33])
def test_attend_very_long(torch, B, dtype, m):
    w = World(torch, [150001, m], [m, m], 3, 128, 128, dtype, seed=33)
    mem = w.device(B, starts=False)
    w.check_attend(mem.attend(w.q.cuda(), w.scale))


def test_streams_and_threads(torch, B):
    w = World(torch, [3000, 1700, 40], [1, 1, 1], 16, 256, 64, "bf16", seed=12)
    mem = w.device(B, starts=False)
    q = w.q.cuda()
    want = mem.attend(q, w.scale)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = mem.attend(q, w.scale, stream=side)
    other = mem.attend(q, w.scale, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(got, want) and torch.equal(other, want)
    found = [[], []]

    def work(i):
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            for _ in range(50):
                found[i].append(mem.attend(q, w.scale))
        s.synchronize()

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    assert all(torch.equal(x, want) for f in found for x in f)
    with pytest.raises(ValueError):
        mem.attend(w.q, w.scale)                                          # host queries


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rank", RANKS)
def test_calls_of_three_streams_at_once(torch, B, dtype, rank):
    """Chunks of several items while the GPU is shared: warps of a block lose their time to others', and wait for one another."""
    worlds = [World(torch, [1100 - 13 * n for n in range(40)], [m] * 40, 5, rank, page, dtype, seed=50 + m, stale=False)
              for m, page in ((32, 64), (20, 16), (3, 128))]
    mems, qs = [w.device(B, starts=False) for w in worlds], [w.q.cuda() for w in worlds]
    want = [m.attend(q, w.scale) for m, q, w in zip(mems, qs, worlds)]
    worlds[0].check_attend(want[0])
    streams = [torch.cuda.Stream() for _ in worlds]
    torch.cuda.synchronize()
    for _ in range(10):
        got = []
        for _ in range(20):
            for s, m, q, w, x in zip(streams, mems, qs, worlds, want):
                with torch.cuda.stream(s):
                    got.append((m.attend(q, w.scale), x))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in got)
    assert all(m.status() == B.OK for m in mems)


@pytest.mark.parametrize("rank", [128, 256])
@pytest.mark.parametrize("m,length", [(32, 100), (32, 128), (128, 250), (24, 1500)])
def test_items_of_a_tile_while_the_gpu_is_shared(torch, B, rank, m, length):
    """Items and pieces of 128 rows that end with the tile in which their reference is raised: a row's two threads, held up by
    other calls' blocks, take the same maximum before the sums of its weights are joined."""
    worlds = [World(torch, [length + 3 * i] * 40, [m] * 40, 5, rank, 64, "bf16", seed=70 + i, stale=False) for i in range(3)]
    mems, qs = [w.device(B, starts=False) for w in worlds], [w.q.cuda() for w in worlds]
    want = [m.attend(q, w.scale) for m, q, w in zip(mems, qs, worlds)]
    for w, x in zip(worlds, want):
        w.check_attend(x)
    streams = [torch.cuda.Stream() for _ in worlds]
    torch.cuda.synchronize()
    for _ in range(5):
        got = []
        for _ in range(20):
            for s, mem, q, w, x in zip(streams, mems, qs, worlds, want):
                with torch.cuda.stream(s):
                    got.append((mem.attend(q, w.scale), x))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in got)
    assert all(mem.status() == B.OK for mem in mems)


def test_calls_without_rows(torch, B):
    w = World(torch, [20], [0], 4, 128, 16, "bf16")
    mem = w.device(B)
    assert mem.attend(w.q.cuda(), 1.0).shape == (0, 4, 128)
    assert mem.append(w.c.cuda(), w.k.cuda(), w.q.cuda()[..., 128:]).shape == (0, 4, ROPE)
    assert mem.status() == B.OK
