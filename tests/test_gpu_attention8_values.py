"""Attention over a cache of 8-bit codes: what values and scales of one page make of the rows that do not see it, and scores of every size."""
import numpy as np
import pytest

from oracle import bwla_attention_oracle as orc
from test_gpu_attention8 import A, CODES, Case, call  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("page,n,new,far", [(16, 128, 128, 2), (8, 192, 192, 12), (16, 700, 200, 40), (8, 64, 24, 7), (16, 520, 20, 32)])
@pytest.mark.parametrize("names", [(), ("slopes",), ("runs",)])
def test_a_page_of_large_scales_costs_earlier_rows_nothing(A, code, dtype, page, n, new, far, names):  # noqa: F811
    """Rows that are computed together (16 or 32 of them) and all lie in front of a page have the same bits whatever its scales."""
    import torch
    c = Case(code, dtype, 64, 4, 2, page, [n], [new], seed=41)
    kw, _ = c.options(np.random.default_rng(1), names)
    want, lse0 = call(c, A, kw)
    p = int(c.table_np[0, far])
    c.vs[p] *= 2.0 ** 40
    c.ks[p] *= 2.0 ** 10
    out, lse = call(c, A, kw)
    together = 32 if 2 * new > 64 else 16              # (two heads of a token are rows)
    rows = (far * page - (n - new)) * 2 // together * together // 2
    assert rows > 0
    assert torch.equal(out[:rows], want[:rows]) and torch.equal(lse[:rows], lse0[:rows])
    assert not torch.equal(out[rows:], want[rows:]) and torch.isfinite(out.float()).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("n,new", [(96, 96), (400, 60), (300, 3)])
@pytest.mark.parametrize("size", [2.0 ** 3, 2.0 ** 9, 2.0 ** 12, -2.0 ** 14, 2.0 ** 17, -2.0 ** 19, 2.0 ** 19, 2.0 ** 21])
@pytest.mark.parametrize("form", ["plain", "cap", "bias"])
def test_equal_scores_weigh_as_their_values_scales_say(A, code, dtype, n, new, size, form):  # noqa: F811
    """Every key has the same score, of any size, in pages of different scales of values: outputs are means of the values.  A weight is off by the
    rounding of its term and, in bf16, by 2^-13 (bounds: test_gpu_attention8.py; the scores' own errors are the same for all keys), lse by
    roundings of the score."""
    import torch
    u = 2.0 ** -24
    c = Case(code, dtype, 64, 4, 2, 16, [n], [new], seed=51)
    one = torch.tensor([1.0]).to(torch.float8_e4m3fn).view(torch.uint8).item() if code == "e4m3" else 1
    k = c.k.view(torch.uint8)
    k.zero_()
    k[..., 0] = one
    c.ks.fill_(1.0)
    c.kv[0][0][:] = 0
    c.kv[0][0][..., 0] = 1.0
    c.q.zero_()
    c.q[..., 0] = 8.0 * size
    kw = {"plain": {}, "cap": {"cap": 2.0 ** 23}, "bias": {"slopes": torch.zeros(4, device="cuda")}}[form]
    out, lse = call(c, A, kw)
    want, lse_want, _, vabs, _, _ = orc.attend(c.q.double().numpy(), *c.kv[0], c.d ** -0.5, **({"cap": 2.0 ** 23} if form == "cap" else {}))
    bf = dtype == "bf16"
    weight = 2.0 ** -11 + 2.0 ** -13 if bf else 2.0 ** -22
    bound = vabs * (weight + (2 * n + 24) * u) + np.abs(want) * (2.0 ** -8 if bf else 4 * u) + n * 2.0 ** -35 * np.abs(c.kv[0][1]).max()
    assert np.all(np.abs(out.double().cpu().numpy() - want) <= bound), np.max(np.abs(out.double().cpu().numpy() - want) / bound)
    assert np.all(np.abs(lse.double().cpu().numpy() - lse_want) <= 16 * u * (np.abs(lse_want) + 1) + (2 * n + 24) * u + (2.0 ** -17 if bf else 0))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("d", [64, 128, 144, 256])
@pytest.mark.parametrize("new", [1, 90])
@pytest.mark.parametrize("cap", [50.0, 127.0, 300.0])
def test_caps_of_rows_that_see_one_key(A, code, dtype, d, new, cap):  # noqa: F811
    """Products of one column, without roundings of sums: lse is the capped score, off by a few units of itself, for heads of every width."""
    import torch
    u = 2.0 ** -24
    c = Case(code, dtype, d, 4, 2, 16, [100], [new], seed=52)
    one = torch.tensor([1.0]).to(torch.float8_e4m3fn).view(torch.uint8).item() if code == "e4m3" else 1
    c.k.view(torch.uint8).zero_()
    c.k.view(torch.uint8)[..., 0] = one
    c.ks.fill_(1.0)
    c.kv[0][0][:] = 0
    c.kv[0][0][..., 0] = 1.0
    first = c.q[..., 0].clone()
    c.q.zero_()
    c.q[..., 0] = 8 * first
    _, lse = call(c, A, {"cap": cap, "window": 1})
    _, want, _, _, _, _ = orc.attend(c.q.double().numpy(), *c.kv[0], np.float64(np.float32(d ** -0.5)), cap=cap, window=1)
    assert np.abs(want).max() > 0.3 and np.abs(want).max() < 0.25 * cap
    # scale, cap, change of base there and back, tanh (4 u), the logarithm of 1: below 12 u of the score; bf16 many rows: the factor of the values, 2^-20
    bound = 12 * u * np.abs(want) + 4 * u + (2.0 ** -20 if dtype == "bf16" else 0)
    assert np.all(np.abs(lse.double().cpu().numpy() - want) <= bound), np.max(np.abs(lse.double().cpu().numpy() - want) / bound)
