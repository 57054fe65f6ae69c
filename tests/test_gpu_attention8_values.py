"""Attention over a cache of 8-bit codes: what values and scales of one page make of the rows that do not see it, and scores of every size."""
import numpy as np
import pytest

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
