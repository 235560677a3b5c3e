"""Attention over latent rows at the ends of what a call may hold, against the 64-bit oracle."""
import numpy as np
import pytest
import torch

from oracle import ref_latent as R
from test_gpu_latent_cache import BF16, FP32, Case, attend_tolerance, check_attend, f64, lib  # noqa: F401 (lib is a fixture)

pytestmark = pytest.mark.gpu


# ---- tokens that are not there -------------------------------------------------
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("rows", [1, 3])
@pytest.mark.parametrize("page,gone", [(16, 4), (16, 9), (32, 2), (64, 1), (64, 3), (128, 1)])
def test_first_pages_that_are_not_there(lib, page, gone, rows, dtype):  # noqa: F811
    """A sequence's first 64 tokens and more do not exist, those behind them do."""
    from paper_2607_24787_b200 import binding as B
    c = Case(lib, 51, [page * gone + 70, 30], [rows, 1], 256, 32, page, dtype, fill=True)
    c.table[0, :gone] = -1
    c.dev_table.copy_(c.table)
    check_attend(c, 5)
    assert c.status.item() == B.KV_BAD_PAGE


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("latent,rope,length", [(128, 16, 20_000), (512, 64, 9600)])
def test_a_page_that_is_not_there_at_any_place(lib, latent, rope, length, dtype):  # noqa: F811
    """One page of a long context, each in turn: wherever the context is cut between CTAs, the result is that of the other tokens."""
    heads, page, scale = 2, 64, (128 + rope) ** -0.5
    c = Case(lib, 52, [length], [1], latent, rope, page, dtype, fill=True)
    q = c.randn(1, heads, latent + rope)
    rows = R.context(f64(c.start), c.table.numpy(), 0, length)[0]
    z = rows @ f64(q)[0].T * scale                                 # [tokens, heads]
    p, v = np.exp(z - z.max(0)), rows[:, :latent]
    reach = (np.abs(rows) @ np.abs(f64(q)[0]).T).max(0)[:, None] * scale
    whole = [(p.T @ v), (p.T @ np.abs(v)), p.sum(0)[:, None]]
    for at in range(-(-length // page)):
        here = slice(at * page, min((at + 1) * page, length))
        part = [p[here].T @ v[here], p[here].T @ np.abs(v[here]), p[here].sum(0)[:, None]]
        total, spread, weight = (a - b for a, b in zip(whole, part))
        kept = int(c.table[0, at])
        c.dev_table[0, at] = -1
        got = f64(c.cache.attend(c.batch, q, scale))[0]
        c.dev_table[0, at] = kept
        want, spread = total / weight, spread / weight
        tol = attend_tolerance(want, spread, reach, dtype, length, latent + rope)
        assert (np.abs(got - want) <= tol).all(), at


# ---- tokens that are not finite ------------------------------------------------
@pytest.mark.parametrize("scale", [0.1, -0.1])
@pytest.mark.parametrize("element", [0, 100, 255, 256, 287])
@pytest.mark.parametrize("token", [70, 196])                       # of a tile that all rows see whole, and one that some rows see
@pytest.mark.parametrize("what", [float("inf"), -float("inf"), float("nan")])
@pytest.mark.parametrize("form", ["bf16", "fp32", "expanded"])
def test_a_single_element_that_is_not_finite(lib, form, what, token, element, scale):  # noqa: F811
    """Of the latent vector or of the shared key, of either sign: NaN for every row that sees the token, all of it, and for no other."""
    c = Case(lib, 55, [200, 130], [6, 1], 256, 32, 16, FP32 if form == "fp32" else BF16, fill=True)
    w = torch.randn(3, 128, 256, generator=c.g).mul(0.1).to(BF16).cuda()
    q = c.randn(c.n_rows, 3, 96 if form == "expanded" else 288)
    if form != "expanded":
        q[:, 1] = q[:, 1].to(BF16)                                 # (fp32 numbers whose lower parts are zero)

    def run():
        if form == "expanded":
            return c.cache.attend_expanded(c.batch, q, w[:, :64], w[:, 64:], scale, 330)
        return c.cache.attend(c.batch, q, scale)

    good = run()
    assert good.isfinite().all()
    c.cache.pages[c.table[0, token // 16], token % 16, element] = what
    out = run()
    first = max(0, token - 194)                                    # the first row that sees it
    assert out[first:6].isnan().all()
    assert torch.equal(out[:first], good[:first]) and torch.equal(out[6], good[6])


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("token", [0, 63, 64, 4000, 8999])
def test_an_infinity_in_a_key_of_a_long_context(lib, token, dtype):  # noqa: F811
    c = Case(lib, 56, [9000, 9000], [1, 1], 128, 16, 64, dtype, fill=True)
    q = c.randn(2, 4, 144)
    good = c.cache.attend(c.batch, q, 0.1)
    for what in (float("inf"), -float("inf")):
        c.cache.pages[c.table[0, token // 64], token % 64, 140] = what
        out = c.cache.attend(c.batch, q, 0.1)
        assert out[0].isnan().all() and torch.equal(out[1], good[1])
