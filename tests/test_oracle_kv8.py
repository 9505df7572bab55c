"""Pins of the 8-bit cache's oracle: the code table against torch's own e4m3
type, rounding, block scales, what an append leaves, rotations and attention
worked by hand or against an independent form."""
import numpy as np
import pytest
import torch

from oracle import kv8


def test_code_values_match_the_type():
    v = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(kv8.e4m3_values(), v, equal_nan=True)


def test_rounding_matches_the_type_where_it_does_not_overflow():
    rng = np.random.default_rng(1)
    x = np.concatenate([rng.normal(0, 1, 20000), rng.uniform(-448, 448, 20000), rng.normal(0, 2.0 ** -8, 20000),
                        (kv8._POS[1:] + kv8._POS[:-1]) / 2, -kv8._POS, [0.0, -0.0, 2.0 ** -10, 3 * 2.0 ** -10]])
    x = x.astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(kv8.e4m3_round(x), want)


def test_rounding_saturates_and_keeps_nan():
    assert list(kv8.e4m3_round([449.0, 1e30, np.inf, -np.inf, -465.0, np.nan])) == [126, 126, 126, 254, 254, 255]


@pytest.mark.parametrize("amax,e", [(448.0, 0), (448.0001, 1), (224.0, -1), (1.75, -8), (1.7501, -7), (0.0, -64),
                                    (1e-30, -64), (3.3e38, 119)])
def test_block_exponent(amax, e):
    assert kv8.block_exponent([0.0, -amax, np.inf, np.nan]) == e


def test_append_requantizes_what_stays_only_when_the_scale_grows():
    s = kv8.Kv8Sequence(1, 2)
    s.append([[[1.0, -3.0]]])                       # 448 * 2^-7 = 3.5 holds 3
    assert s.scale[0, 0] == 2.0 ** -7 and np.array_equal(s.values()[0, 0], [1.0, -3.0])
    s.append([[[0.5, 0.25]]])
    assert s.scale[0, 0] == 2.0 ** -7
    s.append([[[500.0, 0.0]]])
    assert s.scale[0, 0] == 2.0                     # 1 and 3 are 0.5 and 1.5 scales: still exact
    assert np.array_equal(s.values()[:, 0], [[1.0, -3.0], [0.5, 0.25], [512.0, 0.0]])
    s.append(np.full((14, 1, 2), 7.0))              # 17 tokens: the last one opens a block of its own
    assert s.scale.shape == (2, 1) and s.scale[1, 0] == 2.0 ** -6


def test_rotation_is_a_turn_of_complex_numbers():
    rng = np.random.default_rng(2)
    x, pos = rng.normal(size=(5, 3, 20)), np.arange(5) * 7
    w, amp = kv8.frequencies(12, 1e4)
    assert amp == 1.0
    a = pos[:, None] * w
    for layout in ("half", "interleaved"):
        y = kv8.rotate(x, np.cos(a), np.sin(a), layout)
        lo = x[..., :6] if layout == "half" else x[..., 0:12:2]
        hi = x[..., 6:12] if layout == "half" else x[..., 1:12:2]
        z = (lo + 1j * hi) * np.exp(1j * a)[:, None]
        got = y[..., :6] + 1j * y[..., 6:12] if layout == "half" else y[..., 0:12:2] + 1j * y[..., 1:12:2]
        assert np.allclose(got, z, rtol=0, atol=1e-14) and np.array_equal(y[..., 12:], x[..., 12:])
        assert np.allclose(kv8.rotate(y, np.cos(a), np.sin(a), layout, inverse=True), x, rtol=0, atol=1e-14)


def test_scaled_frequencies():
    w, _ = kv8.frequencies(64, 1e4)
    lin, _ = kv8.frequencies(64, 1e4, "linear", 4.0)
    base, _ = kv8.frequencies(64, 1e4, "base", 4.0)
    band, amp = kv8.frequencies(64, 1e4, "bands", 4.0, 4096)
    assert np.allclose(lin, w / 4)
    assert base[0] == 1.0 and base[-1] == pytest.approx(w[-1] / 4, rel=1e-12)      # fastest kept, slowest interpolated
    turns = w * 4096 / (2 * np.pi)
    assert np.array_equal(band[turns >= 32], w[turns >= 32]) and np.allclose(band[turns <= 1], w[turns <= 1] / 4)
    assert np.all(band <= w) and np.all(band >= w / 4 - 1e-18) and amp == pytest.approx(1.1386294, rel=1e-7)


def test_attention_against_softmax():
    rng = np.random.default_rng(3)
    q, k, v = rng.normal(size=(3, 4, 8)), rng.normal(size=(9, 2, 8)), rng.normal(size=(9, 2, 8))
    o, mass, _ = kv8.attend(q, k, v, [8, -1, 3], 0.5)
    assert np.all(o[1] == 0)
    for r, p in ((0, 8), (2, 3)):
        for h in range(4):
            s = torch.softmax(torch.from_numpy(k[:p + 1, h // 2] @ q[r, h] * 0.5), 0).numpy()
            assert np.allclose(o[r, h], s @ v[:p + 1, h // 2], rtol=0, atol=1e-14)
            assert np.all(mass[r, h] + 1e-15 >= np.abs(o[r, h]))
