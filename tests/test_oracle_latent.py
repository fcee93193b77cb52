"""The float64 definitions of the latent memory against the paged memory's, and absorbed against expanded attention (CPU)."""
import numpy as np
import pytest

from oracle import evo_latent as L
from oracle import evo_memory as M


def test_rotation_and_norm_are_the_paged_memorys():
    r = np.random.default_rng(1)
    x, gain, pos = r.standard_normal((5, 3, 64)), r.standard_normal(64), np.array([0, 1, 7, 1000, 70000])
    assert np.allclose(L.turned(x, pos, 1e4), M.normed_and_turned(x, None, 0, pos, 1e4), rtol=0, atol=1e-12)
    assert np.allclose(L.normed(x[:, 0], gain, 1e-3), M.normed_and_turned(x[:, :1], gain, 1e-3, pos, None)[:, 0], rtol=0, atol=1e-14)
    assert np.array_equal(L.turned(x, pos, None), x) and np.array_equal(L.normed(x[:, 0], None, 0), x[:, 0])


@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 3), (False, 5)])
def test_attention_is_the_paged_memorys_with_one_shared_head(causal, window):
    r = np.random.default_rng(2)
    q, x = r.standard_normal((4, 3, 192)), r.standard_normal((9, 192))
    out, size, dots = L.attend(q, x, 128, 0.1, causal, window)
    o, s, d = M.attend(q, x[:, None], x[:, None], 1, 0.1, causal, window)
    assert np.allclose(out, o[..., :128], rtol=0, atol=1e-12) and np.allclose(size, s[..., :128], rtol=0, atol=1e-12)
    assert np.isclose(dots, d)


def test_a_row_that_sees_no_token_is_zero():
    out, size, _ = L.attend(np.ones((3, 2, 192)), np.ones((2, 192)), 128, 1.0, True, 0)
    assert (out[0] == 0).all() and (size[0] == 0).all() and (out[1:] == 1).all()


def test_absorbed_queries_give_the_expanded_heads_attention():
    r = np.random.default_rng(3)
    H, R = 3, 128
    x, wk, wv = r.standard_normal((11, R + 64)), r.standard_normal((H, 64, R)), r.standard_normal((H, 128, R))
    q = r.standard_normal((2, H, 128))
    keys, values = L.expand(x, wk, wv)
    expanded, _, _ = M.attend(q, keys, values, H, 0.02, True, 0)
    absorbed = np.concatenate([np.einsum("mhd,hdr->mhr", q[..., :64], wk), q[..., 64:]], -1)
    out, _, _ = L.attend(absorbed, x, R, 0.02, True, 0)
    assert np.allclose(np.einsum("mhr,hdr->mhd", out, wv), expanded, rtol=0, atol=1e-10)
