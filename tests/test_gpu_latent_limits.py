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
