"""Attention over the 4-bit cache at the ends of what a call may hold: scores far beyond any model's, queries that are not numbers."""
import numpy as np
import pytest
import torch

from oracle import ref_cache as R
from test_gpu_kv_cache import BF16, FP32, HALF, Case, attend_tolerance, kv  # noqa: F401

pytestmark = pytest.mark.gpu


def set_keys_and_values(c, key_codes, seed=0):
    """Every key becomes (code - 8) in element 0 and 0 elsewhere, `key_codes` [n_seq][tokens]; values get random codes and scales."""
    g = torch.Generator().manual_seed(seed)
    hd = c.hd
    pages = torch.randint(0, 256, c.start.shape, generator=g, dtype=torch.uint8)
    pages[..., 17 * hd:] = (torch.rand(*pages.shape[:3], hd // 2, generator=g) + 0.5).half().view(torch.uint8)
    pages[..., 16 * hd:17 * hd] = torch.ones(*pages.shape[:3], hd // 2).half().view(torch.uint8)
    pages[..., :8 * hd] = 0x88
    for s, codes in enumerate(key_codes):
        for t, code in enumerate(codes):
            page = int(c.table[s, t // c.page])
            pages[page, :, t % c.page // 16, t % 16 * 16] = 0x80 | int(code)
    c.start = pages.numpy().copy()
    c.cache.pages.copy_(pages)


# The best token's score is above every other one by at least the query's size times the scale, 2^18 and more: its probability is 1, all others
# are 0, and the result is its value. That value is a code less 8 times an fp16 scale, which fp32 holds exactly; the sum of probabilities is one
# power of two. What is left are the roundings of the quotient and the last product (fp32, two each, and the fast division's two), of the
# value to fp16 where many bf16 rows meet, and of the result.
@pytest.mark.parametrize("power", [19, 24, 27, 28, 30, 33, 40, 55, 90])
@pytest.mark.parametrize("dtype,hd,lengths,rows,heads", [
    (BF16, 128, [900, 40], [1, 1], 32), (FP32, 128, [900, 40], [1, 1], 32), (FP32, 256, [6000], [2], 8), (BF16, 64, [6000, 77], [3, 5], 16),
    (BF16, 128, [600, 300], [300, 300], 16), (BF16, 64, [300, 1100], [130, 260], 16), (FP32, 64, [333], [50], 4),
])
def test_scores_of_any_size(kv, dtype, hd, lengths, rows, heads, power):  # noqa: F811
    c = Case(kv, 41, lengths, rows, 1, hd, 32, dtype, 1, fill=True)
    g = torch.Generator().manual_seed(power)
    tops, codes = [], []
    for n in lengths:                          # eight tokens, each above the ones before it
        at = sorted([0] + (torch.randperm(n - 1, generator=g)[:7] + 1).tolist())
        row = np.zeros(n, int)
        row[at] = np.arange(8) + 8
        tops.append(at)
        codes.append(row)
    set_keys_and_values(c, codes)
    q = torch.zeros(c.n_rows, heads, hd, dtype=dtype)
    q[..., 0] = torch.ldexp(1 + torch.randint(0, 128, (c.n_rows, heads), generator=g) / 128, torch.tensor(power)).to(dtype)
    where = R.places(c.lengths, c.row_start, c.n_rows)
    tol = HALF[dtype] * (1 + 2.0 ** -8) + 8 * HALF[FP32] + (2.0 ** -11 if dtype is BF16 and max(rows) > 64 else 0)
    for scale in (0.7, -0.3):
        out = c.cache.attend(c.batch, (q if scale > 0 else -q).cuda(), scale).double().cpu().numpy()
        for i, at in enumerate(where):
            if at is None:
                continue
            best = max(t for t in tops[at[0]] if t <= at[1])
            want = R.get(c.start, int(c.table[at[0], best // c.page]), 0, best % c.page, 1)
            assert (np.abs(out[i] - want) <= tol * np.abs(want)).all(), (scale, i, at, best)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dtype,hd,lengths,rows,heads", [
    (BF16, 128, [20], [1], 8), (FP32, 64, [1], [1], 2),                       # one tile, one token
    (BF16, 128, [100], [1], 8), (FP32, 128, [100, 30], [1, 1], 8),            # cut between warps
    (BF16, 128, [5000], [1], 8), (FP32, 128, [5000], [1], 3), (FP32, 256, [3000], [2], 4), (BF16, 256, [3000, 9], [1, 1], 4),   # and CTAs
    (BF16, 128, [300, 200], [300, 200], 16), (BF16, 64, [385, 1], [280, 1], 16),                                                 # prompts
])
def test_queries_that_are_not_finite(kv, dtype, hd, lengths, rows, heads, bad):  # noqa: F811
    """A head whose query holds a NaN or an infinity gives NaN, however its tokens are shared out; the other heads give what they give."""
    c = Case(kv, 42, lengths, rows, 1, hd, 16, dtype, 1, fill=True)
    q = c.randn(c.n_rows, heads, hd)
    clean, spread, reach, span = R.attend(q.double().cpu().numpy(), c.start, c.table.numpy(), c.lengths, c.row_start, hd ** -0.5)
    n = c.row_start[-1]
    hit = np.zeros((n, heads), bool)
    for i, h in {(0, 0), (n - 1, heads - 1), (n // 2, heads // 2)}:
        q[i, h, (5 * i + h) % hd] = bad
        hit[i, h] = True
    got = c.cache.attend(c.batch, q).double().cpu().numpy()[:n]
    assert np.isnan(got[hit]).all()
    tol = attend_tolerance(clean, spread, reach, span, dtype, max(lengths))[:n]
    assert (np.abs(got - clean[:n]) <= tol)[~hit].all()


def test_a_query_that_is_not_finite_and_sees_nothing(kv):  # noqa: F811
    for dtype, rows, heads in ((BF16, [3], 4), (FP32, [3], 4), (BF16, [280], 16)):
        c = Case(kv, 43, [2], rows, 1, 128, 16, dtype, fill=True)
        q = torch.full((c.n_rows, heads, 128), float("nan"), dtype=dtype, device="cuda")
        out = c.cache.attend(c.batch, q)
        assert (out[:-2] == 0).all() and out[-2:].isnan().all()


@pytest.mark.parametrize("dtype,hd,lengths,rows,heads", [
    (BF16, 128, [900, 40], [1, 1], 8), (FP32, 64, [900], [4], 4), (BF16, 256, [20], [1], 2), (BF16, 128, [5000] * 70, [1] * 70, 8),
    (BF16, 128, [600, 300], [300, 300], 16), (BF16, 64, [385, 1], [280, 1], 16), (BF16, 64, [20], [300], 16),
])
def test_a_wait_that_runs_out(kv, dtype, hd, lengths, rows, heads):  # noqa: F811
    """An arrival that nobody makes: the kernels give up after the limit and say so, and the next call is what it was."""
    from paper_2607_24787_b200 import binding as B
    c = Case(kv, 44, lengths, rows, 1, hd, 16, dtype, fill=True)
    q = c.randn(c.n_rows, heads, hd)
    want = c.cache.attend(c.batch, q)
    assert c.status.item() == 0
    try:
        B.spm_test_kv_waits(1, 1000)
        c.cache.attend(c.batch, q)
        torch.cuda.synchronize()
    finally:
        B.spm_test_kv_waits(0, 0)
    assert c.status.item() == B.KV_TIMEOUT
    c.status.zero_()
    assert torch.equal(c.cache.attend(c.batch, q), want) and c.status.item() == 0


# Ordinary inputs, in the 2-norm, where independent roundings add up as squares. A bf16 result's own rounding is half a step at most, and the root
# mean square of a rounding is its step over sqrt(12): 2^-8 / sqrt(3) = 0.00226 of a number just above a power of two and half of that below the
# next, 0.00166 for normal numbers. What else bf16 calls round, probabilities and their products with scales (or probabilities, keys and values of
# prompts), has fp16's 11 bits: 2^-11 / sqrt(3) = 0.00028 each at most, three of them 0.0005. Together 0.0018; one more rounding to bf16 on the way,
# of probabilities say, would be 0.0023 and more. fp32 calls: two operands of 23 bits each a product, a score of some units, sums: ten halves of a
# step of 2^-24, 6e-7; three of 2^-22 would be over it.
@pytest.mark.parametrize("dtype,hd,lengths,rows,heads,page", [
    (BF16, 128, [700, 333], [1, 1], 16, 64), (BF16, 64, [500, 90], [5, 3], 8, 16), (BF16, 256, [400], [2], 4, 32),
    (BF16, 128, [600, 300], [280, 250], 16, 64), (BF16, 64, [300, 900], [300, 100], 24, 32),
    (FP32, 128, [700, 333], [1, 1], 16, 64), (FP32, 64, [500, 90], [5, 3], 4, 16), (FP32, 256, [400], [30], 4, 32),
])
def test_errors_of_ordinary_calls(kv, dtype, hd, lengths, rows, heads, page):  # noqa: F811
    c = Case(kv, 45, lengths, rows, 2, hd, page, dtype, fill=True)
    q = c.randn(c.n_rows, heads, hd)
    rows64, want, group = q.double().cpu().numpy(), np.zeros((c.n_rows, heads, hd)), heads // 2
    for s, n in enumerate(rows):
        at = slice(c.row_start[s], c.row_start[s + 1])
        hidden = np.arange(lengths[s])[None] > np.arange(lengths[s] - n, lengths[s])[:, None]
        for h in range(heads):
            if h % group == 0:
                k, v = R.context(c.start, c.table.numpy(), s, lengths[s], page, h // group)[:2]
            z = np.where(hidden, -np.inf, rows64[at, h] @ k.T * hd ** -0.5)
            p = np.exp(z - z.max(-1, keepdims=True))
            want[at, h] = p @ v / p.sum(-1, keepdims=True)
    got = c.cache.attend(c.batch, q).double().cpu().numpy()
    assert np.linalg.norm(got - want) <= (2.1e-3 if dtype is BF16 else 6e-7) * np.linalg.norm(want)


def want_of(c, q, heads, lengths, rows):
    """Results of a whole batch in 64 bits (rows and heads of a sequence at a time)."""
    rows64, want, group = q.double().cpu().numpy(), np.zeros((c.n_rows, heads, c.hd)), heads // c.hk
    for s, n in enumerate(rows):
        at = slice(c.row_start[s], c.row_start[s + 1])
        for h in range(heads):
            if h % group == 0:
                k, v, there = R.context(c.start, c.table.numpy(), s, min(lengths[s], c.table.shape[1] * c.page), c.page, h // group)[:3]
            hidden = (np.arange(len(k))[None] > np.arange(lengths[s] - n, lengths[s])[:, None]) | ~there
            z = np.where(hidden, -np.inf, rows64[at, h] @ k.T * c.hd ** -0.5)
            p = np.exp(z - np.maximum(z.max(-1, keepdims=True, initial=-np.inf), -1e30))
            want[at, h] = p @ v / np.maximum(p.sum(-1, keepdims=True), 1e-30)
    return want


@pytest.mark.parametrize("hd,lengths,rows,heads,hk", [
    (128, [300, 9000, 9, 8600, 0, 9500], [300, 1, 1, 3, 1, 0], 16, 1),       # a prompt beside decoded and drafted tokens of long contexts
    (64, [9000, 260, 270, 40], [2, 260, 200, 1], 24, 2),
    (128, [700] * 40, [10] * 40, 16, 1),                                     # none is longer than the others
    (64, [30] * 99 + [8800], [5] * 99 + [5], 16, 1),
])
def test_batches_of_prompts_and_long_contexts(kv, hd, lengths, rows, heads, hk):  # noqa: F811
    c = Case(kv, 46, lengths, rows, hk, hd, 16, BF16, 2, wide_table=600, fill=True)
    q = c.randn(c.n_rows, heads, hd)
    out = torch.full_like(q, 9.0)
    c.cache.attend(c.batch, q, out=out)
    n = c.row_start[-1]
    want = want_of(c, q, heads, lengths, rows)[:n]
    got = out.double().cpu().numpy()
    assert (got[n:] == 9).all() and c.status.item() == 0
    for i in range(n):                         # the norm of a row: twice what all of it may be off by (see above), a row being few numbers
        assert np.linalg.norm(got[i] - want[i]) <= 4.2e-3 * np.linalg.norm(want[i]), i
    assert torch.equal(c.cache.attend(c.batch, q)[:n], out[:n])


def test_a_prompt_does_not_slow_long_contexts_down(kv):  # noqa: F811
    """One prompt and seven sequences of 100 000 tokens, together and in two calls. One after another's tokens in one place would be 14 times."""
    lengths, rows = [2048] + [100_000] * 7, [2048] + [1] * 7
    need = [-(-n // 64) for n in lengths]
    table = torch.full((8, max(need)), -1, dtype=torch.int32)
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = torch.arange(at, at + n)
        at += n
    pages = torch.randint(0, 256, (at, 4, 4, 18 * 128), dtype=torch.uint8, device="cuda")
    pages[..., 16 * 128:] = torch.rand(at, 4, 4, 128, device="cuda").half().view(torch.uint8)
    cache = kv.KVCache(pages)
    q = torch.randn(sum(rows), 32, 128, device="cuda").bfloat16()

    def batch(a, b):
        ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        starts = np.cumsum([0] + rows[a:b]).tolist()
        return kv.KVBatch(table[a:b].cuda(), ints(lengths[a:b]), ints(starts), n_rows=starts[-1], max_rows=max(rows[a:b]))

    def took(*calls):
        best = 1e9
        for _ in range(6):
            begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            begin.record()
            for b, x in calls:
                cache.attend(b, x)
            end.record()
            torch.cuda.synchronize()
            best = min(best, begin.elapsed_time(end))
        return best

    whole, prompt, rest = batch(0, 8), batch(0, 1), batch(1, 8)
    together, apart = took((whole, q)), took((prompt, q[:2048]), (rest, q[2048:]))
    assert together < 3 * apart, (together, apart)
