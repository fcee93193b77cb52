"""Argument checks of the latent memory: rejected on the host, before anything is
launched (CPU; the pointers are never read)."""
import ctypes

import pytest

P = 1 << 24                      # an aligned address that nothing dereferences


@pytest.fixture(scope="module")
def B():
    from paper_2607_20293_gb300 import binding, build
    build.build()
    binding.load()
    return binding


def view(B, **over):
    v = dict(dtype=1, n_head=8, rank=128, rope=64, page_tokens=16, n_pages=10, max_pages=4, n_seq=3, pages=P, table=P, lens=P,
             starts=P, status=None)
    v.update(over)
    m = B.LatentView()
    for k, x in v.items():
        setattr(m, k, x)
    return m


def append(B, m, c=2 * P, ldc=128, k=3 * P, ldk=64, q=4 * P, ldq=512, hdq=64, rows=6, gain=None, eps=1e-6, rotation=None, n_pos=0,
           pos0=None, out=5 * P, ldo=512, hdo=64):
    return B.load().evo_latent_append(ctypes.byref(m), c, ldc, k, ldk, q, ldq, hdq, rows, gain, eps, rotation, n_pos, pos0, out,
                                      ldo, hdo, None)


def attend(B, m, q=2 * P, ldq=8 * 192, rows=6, max_new=6, max_len=64, scale=0.125, causal=1, window=0, out=3 * P, ldo=8 * 128,
           scratch=P):
    return B.load().evo_latent_attend(ctypes.byref(m), q, ldq, rows, max_new, max_len, scale, causal, window, out, ldo, scratch,
                                      None)


def to_view(B, **over):
    v = dict(dtype=1, format=1, n_head=8, n_kv_head=8, head_dim=128, page_tokens=16, n_pages=10, max_pages=4, n_seq=3,
             k_pages=4 * P, v_pages=5 * P, table=P, lens=P)
    v.update(over)
    m = B.MemoryView()
    for k, x in v.items():
        setattr(m, k, x)
    return m


def expand(B, m, to, wk=2 * P, wv=3 * P, first=None, max_new=64, max_len=64):
    return B.load().evo_latent_expand(ctypes.byref(m), wk, wv, first, max_new, max_len, ctypes.byref(to), None)


@pytest.mark.parametrize("over,code", [
    (dict(dtype=2), "ARG"), (dict(dtype=-1), "ARG"), (dict(n_head=0), "ARG"), (dict(n_head=1025), "SHAPE"), (dict(rank=64), "SHAPE"),
    (dict(rank=192), "SHAPE"), (dict(rank=1024), "SHAPE"), (dict(rank=0), "SHAPE"), (dict(rope=32), "SHAPE"), (dict(rope=0), "SHAPE"),
    (dict(page_tokens=8), "SHAPE"), (dict(page_tokens=48), "SHAPE"), (dict(page_tokens=256), "SHAPE"), (dict(n_pages=0), "ARG"),
    (dict(max_pages=0), "ARG"), (dict(max_pages=(1 << 26) + 1), "SHAPE"), (dict(n_pages=1 << 27), "SHAPE"), (dict(n_seq=-1), "ARG"),
    (dict(pages=None), "ARG"), (dict(pages=P + 8), "ARG"), (dict(table=None), "ARG"), (dict(lens=None), "ARG")])
def test_latent_view_is_checked(B, over, code):
    m = view(B, **over)
    want = getattr(B, "ERR_" + code)
    assert append(B, m) == want and attend(B, m) == want and expand(B, m, to_view(B)) == want
    assert B.load().evo_latent_scratch_bytes(ctypes.byref(m), 6, 6, 64) == 0


def test_null_views(B):
    lib = B.load()
    assert lib.evo_latent_append(None, P, 128, P, 64, P, 512, 64, 6, None, 0.0, None, 0, None, P, 512, 64, None) == B.ERR_ARG
    assert lib.evo_latent_attend(None, P, 1536, 6, 6, 64, 1.0, 1, 0, P, 1024, P, None) == B.ERR_ARG
    assert lib.evo_latent_scratch_bytes(None, 6, 6, 64) == 0
    m, to = view(B), to_view(B)
    assert lib.evo_latent_expand(None, P, P, None, 1, 1, ctypes.byref(to), None) == B.ERR_ARG
    assert lib.evo_latent_expand(ctypes.byref(m), P, P, None, 1, 1, None, None) == B.ERR_ARG


@pytest.mark.parametrize("over,code", [
    (dict(rows=-1), "ARG"), (dict(c=None), "ARG"), (dict(k=None), "ARG"), (dict(q=None), "ARG"), (dict(out=None), "ARG"),
    (dict(ldc=120), "ARG"), (dict(ldc=132), "ARG"), (dict(ldc=1 << 31), "ARG"), (dict(ldk=56), "ARG"), (dict(ldk=65), "ARG"),
    (dict(ldq=504), "ARG"), (dict(hdq=56), "ARG"), (dict(hdq=66), "ARG"), (dict(hdq=128), "ARG"), (dict(hdq=1 << 31, ldq=1 << 35), "ARG"),
    (dict(ldo=0), "ARG"), (dict(hdo=-64), "ARG"), (dict(c=2 * P + 8), "ARG"), (dict(k=3 * P + 2), "ARG"), (dict(q=4 * P + 4), "ARG"),
    (dict(out=5 * P + 8), "ARG"), (dict(eps=-1.0), "ARG"), (dict(eps=float("nan")), "ARG"), (dict(rotation=P, n_pos=0), "ARG"),
    (dict(pos0=P), "ARG"), (dict(gain=P + 4), "ARG"), (dict(rotation=P + 4, n_pos=9), "ARG"), (dict(rows=1 << 28), "SHAPE"),
    (dict(c=P), "ARG"), (dict(k=P + 1024), "ARG"), (dict(q=P), "ARG"), (dict(out=P + 61440 - 16), "ARG")])
def test_append_arguments(B, over, code):
    assert append(B, view(B), **over) == getattr(B, "ERR_" + code)


def test_appended_queries_that_meet_what_is_read(B):
    """8 heads of 64 bf16 values: 128 bytes a head, 1,024 a row; 6 rows."""
    m = view(B)
    for over in (dict(out=4 * P + 16), dict(out=4 * P, ldo=520), dict(out=4 * P + 5 * 1024), dict(out=4 * P - 6 * 1024 + 16),
                 dict(out=4 * P, hdo=72, ldo=576), dict(out=2 * P), dict(out=3 * P + 16), dict(out=2 * P - 16),
                 dict(hdq=128, ldq=1024, out=4 * P + 64, hdo=128, ldo=1024), dict(hdq=128, ldq=1024, out=4 * P, hdo=64, ldo=1024),
                 dict(hdq=128, ldq=1024, c=4 * P + 1040, ldc=1024, k=4 * P + 1664, ldk=1024, out=4 * P + 128, hdo=128, ldo=1024)):
        assert append(B, m, **over) == B.ERR_ARG, over


@pytest.mark.parametrize("over,code", [
    (dict(rows=-1), "ARG"), (dict(q=None), "ARG"), (dict(out=None), "ARG"), (dict(ldq=1528), "ARG"), (dict(ldq=1537), "ARG"),
    (dict(ldo=1016), "ARG"), (dict(ldo=1 << 31), "ARG"), (dict(q=2 * P + 8), "ARG"), (dict(out=3 * P + 8), "ARG"), (dict(max_new=0), "ARG"),
    (dict(max_new=7), "ARG"), (dict(max_len=-1), "ARG"), (dict(max_len=65), "ARG"), (dict(scale=float("inf")), "ARG"),
    (dict(scale=float("nan")), "ARG"), (dict(scale=2.4e38), "ARG"), (dict(causal=2), "ARG"), (dict(window=-1), "ARG"),
    (dict(rows=1 << 28, max_new=1), "SHAPE"), (dict(out=2 * P), "ARG"), (dict(out=2 * P + 9216), "ARG"),
    (dict(out=P + 1024), "ARG"), (dict(ldq=2560, ldo=2560, out=2 * P + 2048), "ARG")])
def test_attend_arguments(B, over, code):
    assert attend(B, view(B), **over) == getattr(B, "ERR_" + code)


@pytest.mark.parametrize("to,over,code", [
    (dict(dtype=0, format=0), {}, "UNSUPPORTED"), (dict(format=2, k_scales=P, v_scales=P), {}, "UNSUPPORTED"), (dict(head_dim=64), {}, "SHAPE"),
    (dict(n_head=4, n_kv_head=4), {}, "SHAPE"), (dict(n_seq=2), {}, "SHAPE"), (dict(k_pages=None), {}, "ARG"), (dict(page_tokens=8), {}, "SHAPE"),
    ({}, dict(wk=None), "ARG"), ({}, dict(wv=None), "ARG"), ({}, dict(wk=2 * P + 8), "ARG"), ({}, dict(max_new=-1), "ARG"),
    ({}, dict(max_new=65), "ARG"), ({}, dict(max_len=65, max_new=1), "ARG"), ({}, dict(max_len=-1, max_new=-1), "ARG"),
    (dict(v_pages=4 * P), {}, "ARG"), (dict(v_pages=P), {}, "ARG"), (dict(k_pages=P + 1024), {}, "ARG"), ({}, dict(wk=4 * P), "ARG"),
    ({}, dict(wv=5 * P + 1024), "ARG")])
def test_expand_arguments(B, to, over, code):
    assert expand(B, view(B), to_view(B, **to), **over) == getattr(B, "ERR_" + code)


def test_equal_chunks_have_to_divide(B):
    m = view(B, starts=None)
    assert append(B, m, rows=7) == B.ERR_SHAPE
    assert attend(B, m, rows=7, max_new=3) == B.ERR_SHAPE
    assert attend(B, m, rows=6, max_new=1) == B.ERR_ARG


def test_a_split_memory_needs_scratch(B):
    for dtype in (0, 1):
        m = view(B, max_pages=4096, dtype=dtype)
        nb = B.load().evo_latent_scratch_bytes(ctypes.byref(m), 3, 1, 65536)
        assert nb > 0 and nb % 4 == 0
        assert attend(B, m, rows=3, max_new=1, max_len=65536, scratch=None) == B.ERR_ARG
        assert attend(B, m, rows=3, max_new=1, max_len=65536, scratch=P + 4) == B.ERR_ARG


def test_calls_that_do_nothing(B):
    assert append(B, view(B), rows=0) == B.OK and attend(B, view(B), rows=0) == B.OK
    assert append(B, view(B), c=None, k=None, q=None, out=None) == B.OK
    assert expand(B, view(B), to_view(B), max_new=0) == B.OK
    none = dict(n_seq=0, table=None, lens=None, starts=None)
    assert append(B, view(B, **none), rows=0) == B.OK and attend(B, view(B, **none), rows=0) == B.OK
    assert append(B, view(B, **none)) == B.ERR_ARG and attend(B, view(B, **none)) == B.ERR_ARG
    assert expand(B, view(B, **none), to_view(B, n_seq=0, table=None, lens=None)) == B.OK


def test_expansion_bounds_are_independent(B):
    """A bound on the written tokens may be looser than the one on the memories (nothing is launched here: no sequences)."""
    none = dict(n_seq=0, table=None, lens=None)
    m, to = view(B, **none, starts=None), to_view(B, **none)
    for max_new, max_len, code in ((64, 0, B.OK), (64, 17, B.OK), (3, 64, B.OK), (65, 64, B.ERR_ARG), (64, 65, B.ERR_ARG), (-1, 3, B.ERR_ARG)):
        assert expand(B, m, to, max_new=max_new, max_len=max_len) == code


def test_binding_checks_tensors(B):
    torch = pytest.importorskip("torch")
    pages = torch.zeros(4, 16, 192, dtype=torch.bfloat16)
    table, lens = torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    m = B.LatentMemory(pages, table, lens, 4)
    assert (m.view.dtype, m.view.rank, m.view.rope, m.view.n_pages, m.view.page_tokens, m.max_len) == (1, 128, 64, 4, 16, 32)
    assert B.LatentMemory(pages.float(), table, lens, 4).view.dtype == 0
    for bad in (dict(pages=pages.half()), dict(pages=pages.transpose(0, 1)), dict(table=table.long()), dict(lens=lens[:2]),
                dict(starts=lens), dict(status=lens)):
        with pytest.raises(ValueError):
            B.LatentMemory(**(dict(pages=pages, table=table, lens=lens, n_head=4) | bad))
    wide = torch.zeros(6, 4, 200, dtype=torch.bfloat16)
    assert m._parts(wide[..., 136:], "q", (6, 4, 64)) == (wide.data_ptr() + 272, 800, 200)
    assert m._heads(torch.zeros(6, 4, 192, dtype=torch.bfloat16), "q", (6, 4, 192))[1] == 768
    for bad in (wide, wide[:5, :, :64], wide[:, :3, :64], wide[..., :64].float(), wide.transpose(1, 2)[:, :64], wide[0]):
        with pytest.raises(ValueError):
            m._parts(bad, "q", (6, 4, 64))
    with pytest.raises(ValueError):
        m._heads(wide[..., :192], "q", (6, 4, 192))


def test_status_word(B):
    torch = pytest.importorskip("torch")
    with torch.inference_mode():
        m = B.LatentMemory(torch.zeros(4, 16, 192), torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32), 4)
        m.tensors[-1].fill_(B.ERR_CORRUPT)
    assert m.status() == B.ERR_CORRUPT and m.status() == B.OK
