"""The oracle of the 8-bit cache and of a step's tables against hand-worked values, torch's own e4m3 numbers, and the bounds that the
cache's documentation states."""
import numpy as np
import pytest

from oracle import bwla_cache8_oracle as orc


def test_nearest_integers_and_ties():
    assert orc.nearest("i8", [0.5, 1.5, -2.5, 126.6, 300.0, -np.inf, np.nan]).tolist() == [0, 2, -2, 127, 127, -127, 0]


def test_nearest_e4m3_is_torchs():
    torch = pytest.importorskip("torch")
    x = np.concatenate([np.random.default_rng(0).standard_normal(4000) * s for s in (1e-3, 0.02, 1, 60, 200)] + [np.arange(-448, 449) / 32.0])
    x = np.clip(x, -448, 448).astype(np.float32)
    assert np.array_equal(orc.nearest("e4m3", x), torch.from_numpy(x).to(torch.float8_e4m3fn).double().numpy())
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    every = every[~np.isnan(every)]
    assert every.max() == 448 and np.array_equal(orc.nearest("e4m3", every), every)


@pytest.mark.parametrize("code", ["i8", "e4m3"])
def test_scales_double_until_they_hold(code):
    top = orc.TOP[code]
    assert orc.grow(code, 1.0, top, False) == (1.0, 0)
    assert orc.grow(code, 1.0, top * 1.01, False) == (2.0, 1)
    assert orc.grow(code, 1.0, top * 4, False) == (4.0, 2)
    assert orc.grow(code, 1.0, 3.0, True) == (3.0 / top, 0)
    assert orc.grow(code, 0.0, 3.0, False) == (3.0 / top, 0)
    assert orc.grow(code, 5.0, 0.0, True) == (0.0, 0)
    assert orc.grow(code, 5.0, 1e-44, True) == (2.0 ** -126, 0)


@pytest.mark.parametrize("code", ["i8", "e4m3"])
def test_a_value_is_off_by_a_step_of_the_last_scale_at_most(code):
    rng = np.random.default_rng(2)
    codes, scale, kept = np.zeros((64, 8)), 0.0, np.zeros((64, 8))
    for j in range(64):                                # tokens one by one, larger and larger ones
        kept[j] = rng.standard_normal(8) * 1.2 ** j
        scale, _ = orc.append(code, codes, scale, kept[j:j + 1], j)
        off = np.abs(codes[:j + 1] * scale - kept[:j + 1])
        # a half step when written, and a half, a quarter, .. of the last one for the doublings; e4m3: half a step at the value, and
        # below 2^-6 a half, a quarter .. of the smallest step
        step = scale if code == "i8" else scale * np.maximum(orc.step_of(code, kept[:j + 1] / scale), 2.0 ** -9)
        assert np.all(off <= step * (1 + 1e-12))


def test_tables_by_hand():
    got = orc.build([16, 3, 40], [1, 2, 5], [[4, -7, -7], [0, -7, -7], [1, 2, 3]], [9, 8, 5, 6, 7, 9], [2, 3], 16, 10, 10, 48, done=[0, 0, 1], shift=[0, 7, 0])
    # request 0 needs page 5 for its 17th token, request 1 none, request 2 starts anew with page 6; 1, 2, 3 go to the ring's end
    assert got["table"].tolist() == [[4, 5, -7], [0, -7, -7], [6, 2, 3]]
    assert got["length"].tolist() == [17, 5, 5] and got["first"].tolist() == [0, 1, 3, 8]
    assert got["ring"].tolist() == [2, 3, 5, 6, 7, 1] and got["state"].tolist() == [4, 4]
    assert got["slot"].tolist() == [80, 3, 4, 96, 97, 98, 99, 100, -1, -1]
    assert got["position"].tolist() == [16, 10, 11, 0, 1, 2, 3, 4, -1, -1]
    assert got["sequence"].tolist() == [0, 1, 1, 2, 2, 2, 2, 2, -1, -1] and got["status"].tolist() == [0, 0, 0, 8]


def test_norm_by_hand():
    assert np.allclose(orc.norm([3.0, 4.0], eps=1e-30), np.array([3, 4]) / np.sqrt(12.5))
    assert np.allclose(orc.norm([1.0, 3.0], [2.0, 1.0], 1e-30, centered=True), [-2, 1])
