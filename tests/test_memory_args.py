"""Argument checks of the 8-bit caches and the paged memory: rejected on the host,
before anything is launched (CPU; the pointers are never read)."""
import ctypes

import pytest

P = 1 << 20                      # an aligned address that nothing dereferences


@pytest.fixture(scope="module")
def B():
    from paper_2607_20293_gb300 import binding, build
    build.build()
    binding.load()
    return binding


def view(B, **over):
    v = dict(dtype=1, format=2, n_head=8, n_kv_head=2, head_dim=64, page_tokens=16, n_pages=10, max_pages=4, n_seq=3,
             k_pages=P, v_pages=P, k_scales=P, v_scales=P, table=P, lens=P, starts=P, status=None)
    v.update(over)
    m = B.MemoryView()
    for k, x in v.items():
        setattr(m, k, x)
    return m


def append(B, m, q=P, k=3 * P, v=4 * P, ldq=512, ldk=128, ldv=128, rows=6, eps=1e-6, rotation=None, n_pos=0, pos0=None, out=P,
           ldo=512, gain=None):
    return B.load().evo_memory_append(ctypes.byref(m), q, k, v, ldq, ldk, ldv, rows, gain, gain, eps, rotation, n_pos,
                                      pos0, out, ldo, None)


def attend(B, m, q=P, ldq=512, rows=6, max_new=6, max_len=64, scale=0.125, causal=1, window=0, out=2 * P, ldo=512,
           scratch=P):
    return B.load().evo_memory_attend(ctypes.byref(m), q, ldq, rows, max_new, max_len, scale, causal, window, out, ldo,
                                      scratch, None)


BAD_VIEWS = [
    (dict(dtype=2), "ARG"), (dict(format=3), "ARG"), (dict(format=0, k_scales=None, v_scales=None), "UNSUPPORTED"),
    (dict(dtype=0, format=1, k_scales=None, v_scales=None), "UNSUPPORTED"), (dict(head_dim=32), "SHAPE"),
    (dict(head_dim=96), "SHAPE"), (dict(n_head=7), "SHAPE"), (dict(n_head=0), "ARG"), (dict(n_kv_head=-1), "ARG"),
    (dict(n_head=2048, n_kv_head=1), "SHAPE"), (dict(page_tokens=8), "SHAPE"), (dict(page_tokens=48), "SHAPE"),
    (dict(page_tokens=256), "SHAPE"), (dict(n_pages=0), "ARG"), (dict(max_pages=0), "ARG"),
    (dict(max_pages=1 << 27), "SHAPE"), (dict(max_pages=(1 << 26) + 1), "SHAPE"), (dict(n_pages=1 << 27), "SHAPE"), (dict(n_seq=-1), "ARG"),
    (dict(k_pages=None), "ARG"), (dict(v_pages=P + 8), "ARG"), (dict(k_scales=None), "ARG"), (dict(table=None), "ARG"),
    (dict(lens=None), "ARG"), (dict(format=1), "ARG"),
]


@pytest.mark.parametrize("over,code", BAD_VIEWS)
def test_memory_view_is_checked(B, over, code):
    m = view(B, **over)
    want = getattr(B, "ERR_" + code)
    assert append(B, m) == want
    assert attend(B, m) == want
    assert B.load().evo_memory_scratch_bytes(ctypes.byref(m), 6, 6, 64) == 0


def test_null_view(B):
    assert B.load().evo_memory_append(None, P, P, P, 512, 128, 128, 6, None, None, 0.0, None, 0, None, P, 512, None) == B.ERR_ARG
    assert B.load().evo_memory_attend(None, P, 512, 6, 6, 64, 1.0, 1, 0, P, 512, P, None) == B.ERR_ARG
    assert B.load().evo_memory_scratch_bytes(None, 6, 6, 64) == 0


@pytest.mark.parametrize("over,code", [
    (dict(rows=-1), "ARG"), (dict(k=None), "ARG"), (dict(v=None), "ARG"), (dict(q=None), "ARG"), (dict(out=None), "ARG"),
    (dict(ldq=508), "ARG"), (dict(ldq=516), "ARG"), (dict(ldk=64), "ARG"), (dict(ldv=129), "ARG"), (dict(ldo=0), "ARG"),
    (dict(q=P + 4), "ARG"), (dict(out=P + 2), "ARG"), (dict(v=P + 8), "ARG"), (dict(eps=-1.0), "ARG"),
    (dict(eps=float("nan")), "ARG"), (dict(rotation=P, n_pos=0), "ARG"), (dict(pos0=P), "ARG"), (dict(gain=P + 4), "ARG"),
    (dict(rotation=P + 4, n_pos=9), "ARG"), (dict(rows=1 << 28), "SHAPE")])
def test_append_arguments(B, over, code):
    assert append(B, view(B), **over) == getattr(B, "ERR_" + code)


@pytest.mark.parametrize("over,code", [
    (dict(rows=-1), "ARG"), (dict(q=None), "ARG"), (dict(out=None), "ARG"), (dict(ldq=504 + 4), "ARG"), (dict(ldo=511), "ARG"),
    (dict(q=P + 8), "ARG"), (dict(out=P + 8), "ARG"), (dict(max_new=0), "ARG"), (dict(max_new=7), "ARG"),
    (dict(max_len=-1), "ARG"), (dict(max_len=65), "ARG"), (dict(scale=float("inf")), "ARG"), (dict(scale=float("nan")), "ARG"),
    (dict(causal=2), "ARG"), (dict(window=-1), "ARG"), (dict(rows=1 << 28, max_new=1), "SHAPE")])
def test_attend_arguments(B, over, code):
    assert attend(B, view(B), **over) == getattr(B, "ERR_" + code)


@pytest.mark.parametrize("scale", [2.4e38, -3e38, float("-inf")])
def test_a_scale_whose_base_2_form_is_infinite(B, scale):
    assert attend(B, view(B), scale=scale) == B.ERR_ARG


def test_outputs_that_overlap_what_is_read(B):
    """8 query heads of 64 bf16 are 1,024 bytes, 2 key heads 256; 6 rows."""
    m = view(B)
    for over in (dict(), dict(out=P + 16), dict(out=P + 5 * 1024), dict(out=P - 5 * 1024), dict(ldq=1024, ldo=1024, out=P + 1008),
                 dict(ldq=1024, ldo=1024, out=P - 1008), dict(ldq=520, ldo=512, out=P + 1024), dict(ldq=1024, out=P + 1024)):
        assert attend(B, m, **(dict(out=P) | over)) == B.ERR_ARG, over
    far = dict(k=P + 20480, v=P + 40960)
    for over in (dict(out=P + 1024), dict(out=P - 1024), dict(out=P, ldo=520), dict(out=P + 20480), dict(out=P + 40960 - 6 * 1024 + 16),
                 dict(ldq=768, ldk=768, ldv=768, k=P + 1024, v=P + 1280, out=P + 16, ldo=768)):
        assert append(B, m, **(far | over)) == B.ERR_ARG, over


def test_equal_chunks_have_to_divide(B):
    m = view(B, starts=None)
    assert append(B, m, rows=7) == B.ERR_SHAPE
    assert attend(B, m, rows=7, max_new=3) == B.ERR_SHAPE
    assert attend(B, m, rows=6, max_new=1) == B.ERR_ARG


def test_a_split_memory_needs_scratch(B):
    m = view(B, max_pages=4096)
    nb = B.load().evo_memory_scratch_bytes(ctypes.byref(m), 3, 1, 65536)
    assert nb > 0 and nb % 4 == 0
    assert attend(B, m, rows=3, max_new=1, max_len=65536, scratch=None) == B.ERR_ARG
    assert attend(B, m, rows=3, max_new=1, max_len=65536, scratch=P + 4) == B.ERR_ARG


def test_a_memory_of_the_most_tokens_is_planned(B):
    m = view(B, max_pages=1 << 26)
    assert B.load().evo_memory_scratch_bytes(ctypes.byref(m), 3, 1, 1 << 30) > 0
    assert attend(B, m, rows=3, max_new=1, max_len=1 << 30, scratch=None) == B.ERR_ARG


def test_calls_without_rows_do_nothing(B):
    assert append(B, view(B), rows=0) == B.OK
    assert append(B, view(B), q=None, k=None, v=None, out=None) == B.OK
    assert attend(B, view(B), rows=0) == B.OK
    assert append(B, view(B, n_seq=0), rows=0) == B.OK
    assert append(B, view(B, n_seq=0)) == B.ERR_ARG


def test_unit_cache_arguments(B):
    lib = B.load()

    def write(r=P, dtype=0, N=2, H=4, E=64, x=P, y=P, codes=P, scales=P):
        return lib.evo_cache_write(r, dtype, None, N, H, E, x, y, codes, scales, None)

    def add(U=2, N=2, H=4, E=64, x=P, y=P, codes=P, scales=P):
        return lib.evo_cache_add(codes, scales, None, U, N, H, E, x, y, None)

    for bad in (dict(dtype=2), dict(N=-1), dict(H=-1), dict(E=0), dict(r=None), dict(r=P + 8), dict(x=None), dict(y=None),
                dict(y=P + 16), dict(x=P + 4, y=P + 4), dict(codes=None), dict(scales=None), dict(codes=P + 4)):
        assert write(**bad) == B.ERR_ARG, bad
    for bad in (dict(U=-1), dict(N=-1), dict(E=0), dict(x=None, y=None), dict(x=None), dict(y=P + 4), dict(codes=None)):
        assert add(**bad) == B.ERR_ARG, bad
    for bad in (dict(E=48), dict(E=33), dict(N=1 << 20, H=1 << 10, E=1 << 10), dict(N=2, H=2147483647, E=2147483616)):
        assert write(**bad) == B.ERR_SHAPE, bad
        assert add(**bad) == B.ERR_SHAPE, bad
    assert write(N=0) == B.OK and write(H=0) == B.OK and add(N=0) == B.OK


def test_rotation_table_arguments(B):
    lib = B.load()
    buf = (ctypes.c_float * 8)()
    for n, d, base, out in [(0, 4, 1e4, buf), (2, 3, 1e4, buf), (2, 0, 1e4, buf), (2, 4, 0.0, buf), (2, 4, float("nan"), buf),
                            (2, 4, float("inf"), buf), (2, 4, 1e4, None)]:
        assert lib.evo_rotation_table(n, d, base, out) == B.ERR_ARG
    assert lib.evo_rotation_table(2, 4, 1e4, buf) == B.OK


def test_binding_checks_tensors(B):
    torch = pytest.importorskip("torch")
    pages = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    table, lens = torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    m = B.Memory(pages, pages, table, lens, 4)
    assert (m.view.format, m.view.n_pages, m.view.page_tokens, m.max_len) == (1, 4, 16, 32)
    for bad in (dict(k_pages=pages.float()), dict(v_pages=pages[:2]), dict(v_pages=pages.transpose(1, 2)),
                dict(table=table.long()), dict(lens=lens[:2]), dict(starts=lens), dict(status=lens), dict(k_scales=pages),
                dict(dtype="fp32"), dict(k_pages=pages.to(torch.uint8))):
        args = dict(k_pages=pages, v_pages=pages, table=table, lens=lens, n_head=4) | bad
        with pytest.raises(ValueError):
            B.Memory(**args)
    q = torch.zeros(6, 4, 64, dtype=torch.bfloat16)
    for bad in (q[:, :3], q.float(), q.transpose(0, 1), q[:5], q[..., :32], q[0], q.transpose(1, 2)):
        with pytest.raises(ValueError):
            m._rows(bad, "q", 6, 4)
    fused = torch.zeros(6, 8 * 64, dtype=torch.bfloat16)
    assert m._rows(fused[:, 128:384].unflatten(1, (4, 64)), "q", 6, 4) == (fused.data_ptr() + 256, 512)


def test_a_memory_has_a_status_word(B):
    torch = pytest.importorskip("torch")
    pages = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    table, lens, word = torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    m = B.Memory(pages, pages, table, lens, 4)
    assert m.view.status and m.status() == B.OK
    m = B.Memory(pages, pages, table, lens, 4, status=word)
    assert m.view.status == word.data_ptr()
    word.fill_(B.ERR_CORRUPT)
    assert m.status() == B.ERR_CORRUPT and int(word) == 0 and m.status() == B.OK


def test_status_of_a_memory_made_under_inference_mode(B):
    torch = pytest.importorskip("torch")
    with torch.inference_mode():
        pages = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
        m = B.Memory(pages, pages, torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32), 4)
        m.tensors[-1].fill_(B.ERR_TIMEOUT)
    assert m.status() == B.ERR_TIMEOUT and m.status() == B.OK


def test_unit_cache_buffers_that_overlap(B):
    """2 samples of 4 x 64: 512 values, 2,048 bytes of fp32, 512 of codes, 16 of scales; two units of them in the sum."""
    lib = B.load()
    at = dict(r=P, x=2 * P, y=3 * P, codes=4 * P, scales=5 * P)

    def write(dtype=0, **over):
        b = at | over
        return lib.evo_cache_write(b["r"], dtype, None, 2, 4, 64, b["x"], b["y"], b["codes"], b["scales"], None)

    def add(**over):
        b = at | over
        return lib.evo_cache_add(b["codes"], b["scales"], None, 2, 2, 4, 64, b["x"], b["y"], None)

    for over in (dict(y=P + 16), dict(y=P - 2032), dict(y=P, dtype=1), dict(codes=P + 2032), dict(codes=P - 496), dict(scales=P + 2047),
                 dict(scales=P - 15), dict(codes=2 * P), dict(codes=3 * P + 16), dict(scales=3 * P), dict(scales=4 * P + 511),
                 dict(scales=4 * P - 15), dict(x=2 * P, y=2 * P + 16), dict(r=P, y=P + 1008, dtype=1)):
        assert write(**over) == B.ERR_ARG, over
    for over in (dict(codes=2 * P), dict(codes=3 * P - 1008), dict(scales=2 * P + 2040), dict(scales=3 * P - 31), dict(scales=4 * P + 1023),
                 dict(y=4 * P + 1008), dict(x=5 * P + 16, y=5 * P + 16)):
        assert add(**over) == B.ERR_ARG, over


def test_a_memory_of_no_sequences_needs_no_table(B):
    m = view(B, n_seq=0, table=None, lens=None, starts=None)
    assert append(B, m, rows=0) == B.OK and attend(B, m, rows=0) == B.OK
    assert append(B, m) == B.ERR_ARG and attend(B, m) == B.ERR_ARG
