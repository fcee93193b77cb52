"""The 8-bit unit caches on the GPU against the float64 definitions: codes, scales
and streams bit for bit (scaling by a power of two is exact, every other step is
one IEEE operation), over sizes, gates, types and extreme values."""
import numpy as np
import pytest

from oracle import evo_memory as M

pytestmark = pytest.mark.gpu


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


def make(torch, N, H, E, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    r = torch.randn(N, H, E, generator=g) * torch.exp(3 * torch.randn(N, H, E // 32, 1, generator=g)).expand(-1, -1, -1, 32).reshape(N, H, E)
    x = torch.randn(N, H, E, generator=g)
    gate = (torch.rand(N, generator=g) < 0.5).to(torch.uint8) * 3           # any value but zero refreshes
    codes = torch.randint(0, 256, (N, H, E), generator=g, dtype=torch.uint8)
    scales = torch.randint(100, 140, (N, H, E // 32), generator=g, dtype=torch.uint8)
    return r.to(torch.float32 if dtype == "fp32" else torch.bfloat16), x, gate, codes, scales


def check_write(torch, B, r, x, gate, codes, scales, in_place=False):
    c, s = codes.cuda(), scales.cuda()
    xd = x.cuda()
    y = B.cache_write(r.cuda(), c, s, xd, None if gate is None else gate.cuda(), out=xd if in_place else None)
    wc, ws = codes.numpy().copy(), scales.numpy().copy()
    rf = r.float().numpy()
    on = np.ones(len(rf), bool) if gate is None else gate.numpy() != 0
    with np.errstate(over="ignore", invalid="ignore"):
        want = np.where(on[:, None, None], x.numpy() + rf, x.numpy())       # fp32: one rounding
    M.cache_write(rf.astype(np.float64), x.numpy(), None if gate is None else gate.numpy(), wc, ws)
    assert np.array_equal(s.cpu().numpy(), ws)
    assert np.array_equal(c.cpu().numpy(), wc)
    assert np.array_equal(y.cpu().numpy(), want, equal_nan=True)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("N,H,E", [(1, 1, 32), (1, 16, 256), (3, 5, 96), (7, 8, 64), (33, 16, 256), (5, 32, 512), (129, 3, 1024)])
def test_write(torch, B, N, H, E, dtype):
    check_write(torch, B, *make(torch, N, H, E, dtype, N + E))


@pytest.mark.parametrize("in_place", [False, True])
def test_write_all_and_none(torch, B, in_place):
    r, x, gate, codes, scales = make(torch, 6, 8, 128, "fp32", 1)
    check_write(torch, B, r, x, None, codes, scales, in_place)
    check_write(torch, B, r, x, torch.zeros(6, dtype=torch.uint8), codes, scales, in_place)
    check_write(torch, B, r, x, gate, codes, scales, in_place)


def test_write_extreme_values(torch, B):
    # the borders of the scale, ties of the codes, subnormals, zeros, infinities and NaN, one group each
    rows = [[448.0, 1.0], [float(np.nextafter(np.float32(448), np.float32(449))), 1.0], [0.0, 0.0], [-0.0, 0.0], [1e-45, -1e-45],
            [1e-38, 3e-39], [3.4e38, -1.0], [np.inf, 1.0], [-np.inf, 1.0], [np.nan, 1.0], [np.nan, np.inf], [448.0, 2.0 ** -10],
            [448.0, 3 * 2.0 ** -10], [448.0, 17.0], [448.0, 19.0], [448.0, -2.0 ** -9], [1.75 * 2.0 ** 20, 1.0], [1.7500001 * 2.0 ** 20, 1.0]]
    r = torch.zeros(len(rows), 1, 32)
    for i, v in enumerate(rows):
        r[i, 0, 5], r[i, 0, 31] = v
    x = torch.ones_like(r)
    check_write(torch, B, r, x, None, torch.zeros(r.shape, dtype=torch.uint8), torch.zeros(len(rows), 1, 1, dtype=torch.uint8))


def test_write_without_a_stream(torch, B):
    r, x, gate, codes, scales = make(torch, 4, 8, 64, "bf16", 2)
    c, s = codes.cuda(), scales.cuda()
    assert B.cache_write(r.cuda(), c, s, refresh=gate.cuda()) is None
    wc, ws = codes.numpy().copy(), scales.numpy().copy()
    M.cache_write(r.double().numpy(), x.numpy(), gate.numpy(), wc, ws)
    assert np.array_equal(c.cpu().numpy(), wc) and np.array_equal(s.cpu().numpy(), ws)


def sequential(codes, scales, x, reuse):
    y = x.numpy().copy()
    for u in range(len(codes)):
        v = M.dequantise(codes[u].numpy().reshape(*scales[u].shape, 32), scales[u].numpy()).reshape(y.shape)
        on = np.ones(len(y), bool) if reuse is None else reuse[u].numpy() != 0
        y[on] = (y[on] + v[on].astype(np.float32)).astype(np.float32)
    return y


@pytest.mark.parametrize("U,N,H,E", [(0, 3, 4, 64), (1, 1, 1, 32), (1, 1, 16, 256), (5, 64, 16, 256), (11, 9, 32, 512), (36, 5, 7, 96), (3, 200, 1, 160)])
@pytest.mark.parametrize("gated", [True, False])
def test_add(torch, B, U, N, H, E, gated):
    g = torch.Generator().manual_seed(U + N)
    codes = torch.randint(0, 256, (U, N, H, E), generator=g, dtype=torch.uint8)
    codes[(codes & 127) == 127] = 5
    scales = torch.randint(90, 140, (U, N, H, E // 32), generator=g, dtype=torch.uint8)
    x = torch.randn(N, H, E, generator=g)
    reuse = (torch.rand(U, N, generator=g) < 0.6).to(torch.uint8) * 7 if gated else None
    want = sequential(codes, scales, x, reuse)
    args = (codes.cuda(), scales.cuda())
    gate = None if reuse is None else reuse.cuda()
    assert np.array_equal(B.cache_add(*args, x.cuda(), gate).cpu().numpy(), want)
    xd = x.cuda()
    assert B.cache_add(*args, xd, gate, out=xd) is xd
    assert np.array_equal(xd.cpu().numpy(), want)


def test_add_of_groups_that_are_not_numbers(torch, B):
    codes = torch.full((2, 1, 1, 64), 0x38, dtype=torch.uint8)
    scales = torch.full((2, 1, 1, 2), 127, dtype=torch.uint8)
    scales[1, 0, 0, 1] = 255
    y = B.cache_add(codes.cuda(), scales.cuda(), torch.zeros(1, 1, 64).cuda()).cpu()
    assert (y[..., :32] == 2).all() and y[..., 32:].isnan().all()
    # a unit that is not reused adds nothing, whatever it holds
    reuse = torch.tensor([[1], [0]], dtype=torch.uint8).cuda()
    y = B.cache_add(codes.cuda(), scales.cuda(), torch.zeros(1, 1, 64).cuda(), reuse).cpu()
    assert (y == 1).all()


def test_lattice_of_cells_as_a_policy_runs_them(torch, B):
    """Eq. 1 over a per-sample lattice of 4 units x 6 steps: each cell refreshes some samples and
    reuses the caches of the others; the stream against the float64 definition."""
    U, T, N, H, E = 4, 6, 9, 8, 128
    g = torch.Generator().manual_seed(9)
    S = (torch.rand(N, U, T, generator=g) < 0.4).to(torch.uint8)
    S[:, :, 0] = 1
    r = 0.2 * torch.randn(T, U, N, H, E, generator=g)
    x = torch.randn(N, H, E, generator=g)
    codes = torch.zeros(U, N, H, E, dtype=torch.uint8).cuda()
    scales = torch.zeros(U, N, H, E // 32, dtype=torch.uint8).cuda()
    wc, ws = codes.cpu().numpy(), scales.cpu().numpy()
    got, want = x.cuda(), x.double().numpy()
    for t in range(T):
        for u in range(U):
            gate = S[:, u, t].contiguous()
            B.cache_write(r[t, u].cuda(), codes[u], scales[u], got, gate.cuda(), out=got)
            B.cache_add(codes[u:u + 1], scales[u:u + 1], got, (1 - gate)[None].contiguous().cuda(), out=got)
            want = M.cache_write(r[t, u].double().numpy(), want, gate.numpy(), wc[u], ws[u])
            want = M.cache_add(wc[u:u + 1], ws[u:u + 1], want, (1 - gate.numpy())[None])
    assert np.array_equal(codes.cpu().numpy(), wc) and np.array_equal(scales.cpu().numpy(), ws)
    # 48 fp32 additions, each within half a step of a stream below 8
    assert np.abs(got.cpu().numpy() - want).max() <= 2 * U * T * 2.0 ** -24 * 8


def test_write_and_add_in_a_captured_graph_on_another_stream(torch, B):
    r, x, gate, codes, scales = make(torch, 6, 8, 128, "bf16", 5)
    dev = [t.cuda() for t in (r, x, gate, codes, scales)]
    y = torch.empty_like(dev[1])
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(st):
        with torch.cuda.graph(graph, stream=st):
            B.cache_write(dev[0], dev[3], dev[4], dev[1], dev[2], out=y)
            B.cache_add(dev[3][None], dev[4][None], y, out=y)
    r2 = (r.float() * 1.5).to(r.dtype)
    dev[0].copy_(r2)
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    wc, ws = codes.numpy().copy(), scales.numpy().copy()
    M.cache_write(r2.double().numpy(), x.numpy(), gate.numpy(), wc, ws)
    on = (gate.numpy() != 0)[:, None, None]
    want = np.where(on, x.numpy() + r2.float().numpy(), x.numpy())
    v = M.dequantise(wc.reshape(*ws.shape, 32), ws).reshape(want.shape).astype(np.float32)
    assert np.array_equal(dev[3].cpu().numpy(), wc)
    assert np.array_equal(y.cpu().numpy(), want + v, equal_nan=True)


def test_binding_refuses_other_layouts(torch, B):
    r, x, gate, codes, scales = (t.cuda() for t in make(torch, 4, 8, 64, "fp32", 6))
    for bad in (dict(r=r.double()), dict(codes=codes[:3]), dict(scales=scales.int()), dict(x=x.bfloat16()),
                dict(refresh=gate[:2]), dict(r=r.transpose(0, 1)), dict(codes=codes.cpu()), dict(x=None, out=x)):
        args = dict(r=r, codes=codes, scales=scales, x=x, refresh=gate) | bad
        with pytest.raises(ValueError):
            B.cache_write(**args)
    with pytest.raises(B.EvoError) as e:
        B.cache_write(torch.zeros(2, 2, 48, device="cuda"), torch.zeros(2, 2, 48, dtype=torch.uint8, device="cuda"),
                      torch.zeros(2, 2, 1, dtype=torch.uint8, device="cuda"))
    assert e.value.code == B.ERR_SHAPE
    with pytest.raises(ValueError):
        B.cache_add(codes[None], scales[None], x[:2])


def test_the_stream_takes_the_residuals_place(torch, B):
    r, x, gate, codes, scales = make(torch, 6, 8, 128, "fp32", 8)
    rd, c, s = r.cuda(), codes.cuda(), scales.cuda()
    assert B.cache_write(rd, c, s, x.cuda(), gate.cuda(), out=rd) is rd
    want = np.where((gate.numpy() != 0)[:, None, None], x.numpy() + r.numpy(), x.numpy())
    wc, ws = codes.numpy().copy(), scales.numpy().copy()
    M.cache_write(r.double().numpy(), x.numpy(), gate.numpy(), wc, ws)
    assert np.array_equal(rd.cpu().numpy(), want)
    assert np.array_equal(c.cpu().numpy(), wc) and np.array_equal(s.cpu().numpy(), ws)
    flat = torch.zeros(6 * 8 * 128 + 64, device="cuda")
    with pytest.raises(B.EvoError) as e:
        B.cache_write(flat[:-64].view(6, 8, 128), c, s, x.cuda(), out=flat[64:].view(6, 8, 128))
    assert e.value.code == B.ERR_ARG
