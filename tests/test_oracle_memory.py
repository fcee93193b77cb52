"""The float64 definitions of the 8-bit caches and the paged memory against
independent statements of the same things (CPU)."""
import numpy as np
import pytest

from oracle import evo_memory as M


def test_code_values_are_e4m3():
    torch = pytest.importorskip("torch")
    t = torch.arange(256, dtype=torch.int16).to(torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(t, M.CODES, equal_nan=True)


def test_codes_round_to_nearest_even():
    torch = pytest.importorskip("torch")
    x = np.concatenate([np.random.default_rng(0).standard_normal(4096) * 10.0 ** np.arange(-3, 3).repeat(4096 // 6 + 1)[:4096],
                        np.linspace(-448, 448, 897), [0.0, -0.0, 2.0 ** -10, 3 * 2.0 ** -10, 448.0]]).astype(np.float32)
    x = x[np.abs(x) <= 448]
    # with 448 in the group the scale is one: the codes are the values' own e4m3 rounding
    g = np.stack([x, np.full_like(x, 448.0)], 1)
    c, s = M.quantise(g)
    assert (s == 127).all()
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(c[:, 0], want)


@pytest.mark.parametrize("amax,byte", [(448.0, 127), (np.nextafter(np.float32(448), np.float32(1e3)), 128), (224.0, 126),
                                       (0.0, 1), (1e-45, 1), (3.4e38, 247), (np.inf, 255), (np.nan, 255), (1.0, 119)])
def test_scale_is_the_least_that_holds_the_group(amax, byte):
    x = np.zeros(32)
    x[7] = -amax
    assert M.scale_bytes(x) == byte


def test_values_are_within_half_a_step():
    x = np.random.default_rng(1).standard_normal((500, 32)) * np.exp(np.random.default_rng(2).standard_normal((500, 32)) * 4)
    c, s = M.quantise(x)
    k = s.astype(float)[:, None] - 127
    assert (np.abs(M.dequantise(c, s) - x) <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** (k - 10))).all()


def test_rotation_keeps_lengths_and_differences():
    rng = np.random.default_rng(3)
    q, k = rng.standard_normal((1, 1, 64)), rng.standard_normal((1, 1, 64))
    dots = [float((M.normed_and_turned(q, None, 0, [a], 1e4) * M.normed_and_turned(k, None, 0, [b], 1e4)).sum())
            for a, b in [(5, 2), (103, 100), (70003, 70000)]]
    assert np.allclose(dots, dots[0], rtol=0, atol=1e-9)


def test_rotation_table_of_the_library():
    from paper_2607_20293_gb300 import binding, build
    build.build()
    t = binding.rotation_table(5000, 128, 10000.0).astype(np.float64)
    ang = np.arange(5000)[:, None] * 10000.0 ** (-2.0 * np.arange(64) / 128)
    assert np.abs(t - np.concatenate([np.cos(ang), np.sin(ang)], 1)).max() <= 2.0 ** -25 + 1e-11


def test_attention_of_one_key_and_of_none():
    rng = np.random.default_rng(4)
    q, k, v = rng.standard_normal((3, 2, 64)), rng.standard_normal((2, 1, 64)), rng.standard_normal((2, 1, 64))
    out, _, _ = M.attend(q, k, v, 1, 0.125, True, 0)
    assert (out[0] == 0).all()                                   # token -1 sees nothing
    assert np.allclose(out[1], v[0], rtol=0, atol=1e-15)
    out, _, _ = M.attend(q, k, v, 1, 0.125, False, 1)            # the last token alone
    assert np.allclose(out, v[1], rtol=0, atol=1e-15)
