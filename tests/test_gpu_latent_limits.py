"""Attention over latent rows at the ends of what a call may hold, against the 64-bit oracle."""
import numpy as np
import pytest
import torch

from oracle import ref_latent as R
from oracle.ref_cache import places
from test_gpu_latent_cache import BF16, FP32, HALF, Case, attend_tolerance, check_attend, f64, lib  # noqa: F401 (lib is a fixture)

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


# ---- scores of any size, expanded ----------------------------------------------
# The best token's score is above every other one by at least the query's size times the scale, 2^18 and more: its probability is 1, all others
# are 0, and the result is its value: a sum of 128 fp32 products (each addition off by 2^-23 at most), rounded to fp16 (2^-11; 2^-25 where the
# largest value of its 32 tokens is 2^9 or more: 2^-34 of the largest) and to bf16, with a handful of fp32 roundings between.
@pytest.mark.parametrize("power", [8, 13, 19, 24, 27, 28, 30, 33, 40, 55, 90])
@pytest.mark.parametrize("lengths,rows,heads,head,rope,unit", [
    ([600, 300], [300, 300], 3, 128, 64, 0), ([300, 1100], [130, 260], 2, 64, 16, 0), ([20, 40], [20, 1], 2, 64, 16, 0), ([700], [200], 2, 128, 16, -30),
    ([700], [200], 2, 64, 32, 100),
])
def test_expanded_scores_of_any_size(lib, lengths, rows, heads, head, rope, unit, power):  # noqa: F811
    c = Case(lib, 53, lengths, rows, 128, rope, 32, BF16, 1, fill=True)
    g = torch.Generator().manual_seed(power)
    tops = []
    c.start[..., 128:] = c.start[..., 128:] * 0                    # (what is not a number behind a sequence's end stays)
    for s, n in enumerate(lengths):                # eight tokens, each above the ones before it; others far below, some of them small by themselves
        at = sorted([0] + (torch.randperm(n - 1, generator=g)[:7] + 1).tolist())
        tops.append(at)
        for t in range(n):
            key = at.index(t) + 1.0 if t in at else -8.0 if t // 32 % 2 else -2.0 ** -10
            c.start[c.table[s, t // 32], t % 32, 128] = key * 2.0 ** unit
    c.cache.pages.copy_(c.start)
    q = torch.zeros(c.n_rows, heads, head + rope, dtype=BF16)
    q[..., head] = torch.ldexp(1 + torch.randint(0, 128, (c.n_rows, heads), generator=g) / 128, torch.tensor(power - unit)).to(BF16)
    w_k = torch.zeros(heads, head, 128, dtype=BF16, device="cuda")
    w_v = torch.randn(heads, head, 128, generator=g).mul(0.1).to(BF16)
    values = [np.einsum("tc,hdc->thd", R.context(f64(c.start), c.table.numpy(), s, n)[0][:, :128], f64(w_v)) for s, n in enumerate(lengths)]
    made = [np.einsum("tc,hdc->thd", np.abs(R.context(f64(c.start), c.table.numpy(), s, n)[0][:, :128]), np.abs(f64(w_v))) for s, n in enumerate(lengths)]
    # (below 2^13 the others are not all zero: only that it is near)
    others = {8: 2.0 ** -8, 13: 0.0}.get(power, 0.0)
    for scale in (0.7, -0.3):
        got = f64(c.cache.attend_expanded(c.batch, (q if scale > 0 else -q).cuda(), w_k, w_v.cuda(), scale, sum(lengths)))
        for i, at in enumerate(places(lengths, c.row_start, c.n_rows)):
            if at is None:
                continue
            best = max(t for t in tops[at[0]] if t <= at[1])
            want, largest = values[at[0]][best], np.abs(values[at[0]]).max()
            tol = (2.0 ** -11 + HALF[BF16] * (1 + 2.0 ** -8) + 16 * HALF[FP32]) * np.abs(want) + 128 * 2.0 ** -23 * made[at[0]][best] + (2.0 ** -34 + others) * largest
            assert (np.abs(got[i] - want) <= tol).all(), (scale, i, at, best)


@pytest.mark.parametrize("part", ["key", "made"])
@pytest.mark.parametrize("power,finite", [(100, True), (113, False), (120, False)])
def test_expanded_keys_too_large_for_a_call(lib, part, power, finite):  # noqa: F811
    """An element of a key of 2^109 and more counts as one that is not finite: NaN for the rows that see it, and for no other."""
    c = Case(lib, 54, [200, 130], [60, 1], 128, 32, 16, BF16, fill=True)
    q = c.randn(c.n_rows, 2, 96).mul(2.0 ** -20)
    w = torch.randn(2, 128, 128, generator=c.g).mul(0.1).to(BF16).cuda()
    w_k, w_v = w[:, :64], w[:, 64:]
    w_v[..., 5], w_k[..., 5] = 0, 1
    good = c.cache.attend_expanded(c.batch, q, w_k, w_v, 2.0 ** -90, 330)
    c.cache.pages[c.table[0, 170 // 16], 170 % 16, 128 + 7 if part == "key" else 5] = 2.0 ** power
    out = c.cache.attend_expanded(c.batch, q, w_k, w_v, 2.0 ** -90, 330)
    assert torch.equal(out[:30], good[:30]) and torch.equal(out[60], good[60])
    if finite:                                                     # scores are all but zero
        assert (out[30:60] - good[30:60]).abs().max() <= 2.0 ** -5 * good.abs().max()
    else:
        assert out[30:60].isnan().all()


# ---- products of heads ---------------------------------------------------------
# Terms of one sign, 1/4 to 9/4 each, so that what is cut off a sum adds up. Of the first parts a product has its last bit at 2^-16 and 64 of them are below
# 2^8: exact in 24 bits. The other parts are 2^-7 of the result at most; a product of 16 elements is off by 17 steps of 2^-23 at most of what
# is there (16 terms and the sum, cut off at one place). In units of 2^-24 of the result:
# few rows: sums of 16 elements (transposed 32) begin with the other parts (two to four products, half a unit), which the first parts cut off at most twice (four units),
# and are added up in fp32, half a step each of what is there so far; the warps' sums by three additions more. `warps`: a CTA's, which share them out;
# 64 rows (warps 1): first parts' sums of 64 elements are added up in fp32; the other parts' products stay in one sum, two for each 16 elements.
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("n,heads,size,to,warps", [(3, 2, 8192, 128, 8), (3, 150, 8192, 128, 4), (40, 3, 8192, 64, 8), (17, 2, 4096, 192, 8), (1, 5, 576, 64, 8),
                                                   (64, 100, 2048, 128, 1)])
def test_fp32_products_of_one_sign(lib, n, heads, size, to, warps, transposed):  # noqa: F811
    g = torch.Generator().manual_seed(57)
    x = torch.rand(n, heads, size, generator=g).add(0.5).cuda()
    w = torch.rand(heads, to, size, generator=g).add(0.5).to(BF16).cuda()
    y = lib.head_product(x, w if transposed else w.transpose(1, 2).contiguous(), transposed=transposed)
    want = torch.stack([x[:, h].double() @ w[h].double().T for h in range(heads)], 1)
    added = size // 64 if warps == 1 else -(-size // (32 if transposed else 16) // warps)
    other = 17 * 2 * 2.0 ** -7 * (2 * size // 16 + 1) / 2 if warps == 1 else 4.5
    bound = (added + 1) / 2 + other + 3
    assert ((y.double() - want).abs() <= bound * 2.0 ** -24 * want).all()


# ---- rows on their way into the cache --------------------------------------------
# fp32 roundings of a sum of 256 squares, a root and two products, then the one to bf16 (of the smallest numbers: half a step of 2^-133)
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("size,eps", [(1.0, 1e-6), (1e17, 1e-6), (1e19, 1e-6), (1e30, 0.0), (1e38, 1e-6), (1e-18, 0.0), (1e-25, 0.0), (1e-37, 0.0), (1e-25, 1e-6), (0.0, 1e-6)])
def test_norms_of_rows_of_any_size(lib, size, eps, dtype):  # noqa: F811
    c = Case(lib, 58, [40, 9], [11, 3], 256, 32, 16, dtype)
    x, key = torch.randn(c.n_rows, 256, generator=c.g).clamp(-3, 3).mul(size).to(dtype).cuda(), c.randn(c.n_rows, 32)
    x[3] = c.randn(256)                                            # one row is an ordinary one
    gamma = 1 + 0.2 * torch.randn(256, generator=c.g)
    rope = lib.kv.Rope(torch.ones(16).cuda(), k_gamma=gamma.cuda(), eps=eps)
    c.cache.write(c.batch, x, key, positions=torch.zeros(c.n_rows, dtype=torch.int32, device="cuda"), rope=rope)
    want = R.norm(f64(x), gamma.numpy(), float(np.float32(eps))) if size else np.where(np.arange(c.n_rows)[:, None] == 3, R.norm(f64(x), gamma.numpy(), eps), 0)
    got = np.stack([f64(c.cache.pages[int(c.table[s, p // 16]), p % 16, :256]) for s, p in places(c.lengths, c.row_start, c.n_rows)])
    assert (np.abs(got - want) <= (256 + 8) * HALF[FP32] * np.abs(want) + HALF[BF16] * np.abs(want) + 2.0 ** -134).all()
    assert c.status.item() == 0


# ---- pools without pages ---------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_a_pool_without_pages(lib, dtype):  # noqa: F811
    """No token exists: nothing is written, rows that see only such tokens give zeros, and the status says why."""
    from paper_2607_24787_b200 import binding as B
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    cache = lib.LatentCache(torch.zeros(0, 32, 144, dtype=BF16, device="cuda"), 128, status)
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    batch = lib.kv.KVBatch(torch.zeros(2, 9, dtype=torch.int32, device="cuda"), ints(200, 30), ints(0, 5, 6), n_rows=7, max_rows=5)
    g = torch.Generator().manual_seed(59)
    rows = torch.randn(7, 144, generator=g).to(dtype).cuda()
    cache.write(batch, rows[:, :128], rows[:, 128:])
    assert status.item() == B.KV_BAD_PAGE
    out = cache.attend(batch, torch.randn(7, 5, 144, generator=g).to(dtype).cuda(), 0.1, out=torch.full((7, 5, 128), 9.0, dtype=dtype, device="cuda"))
    assert (out[:6] == 0).all() and (out[6] == 9).all()
    if dtype is BF16:
        w = torch.randn(5, 128, 128, generator=g).to(BF16).cuda()
        out = cache.attend_expanded(batch, torch.randn(7, 5, 80, generator=g).to(BF16).cuda(), w[:, :64], w[:, 64:], 0.1, 230,
                                    out=torch.full((7, 5, 64), 9.0, dtype=BF16, device="cuda"))
        assert (out[:6] == 0).all() and (out[6] == 9).all()
    # and a table without pages
    status.zero_()
    batch = lib.kv.KVBatch(torch.zeros(2, 0, dtype=torch.int32, device="cuda"), ints(200, 30), ints(0, 5, 6), n_rows=7, max_rows=5)
    cache.write(batch, rows[:, :128], rows[:, 128:])
    out = cache.attend(batch, torch.randn(7, 5, 144, generator=g).to(dtype).cuda(), 0.1)
    assert (out[:6] == 0).all() and status.item() == B.KV_TOO_LONG


# ---- long sums of fp32 calls -------------------------------------------------------
def test_long_sums_of_one_sign(lib):  # noqa: F811
    """8000 tokens in one CTA, all of the same probability, 1: results are means. Values of 8 bits from 2^-8 to 1 end at 2^-15, and 256 of them are below 2^8: exact
    in 24 bits. Up to 32 such sums are added up in fp32, half a step of 2^-24 each of what is there so far (half as many, and a half), then up to two parts
    joined, divided by their sum: six roundings more."""
    n, heads, latent, rope, page = 8000, 1024, 128, 16, 64
    g = torch.Generator(device="cuda").manual_seed(60)
    pages = torch.rand(3 * n // page, page, latent + rope, device="cuda", generator=g).mul(-8).exp2().to(BF16)
    cache = lib.LatentCache(pages, latent)
    table = torch.randperm(3 * n // page, device="cuda", generator=g).to(torch.int32).view(3, -1)
    batch = lib.kv.KVBatch(table, torch.full((3,), n, dtype=torch.int32, device="cuda"))
    out = cache.attend(batch, torch.zeros(3, heads, latent + rope, device="cuda"), 0.1).double()
    want = pages[table.long()].flatten(1, 2)[..., :latent].double().mean(1)[:, None]
    assert ((out - want).abs() <= ((32 + 1) / 2 + 6) * 2.0 ** -24 * want).all()


# ---- values of any size, absorbed --------------------------------------------------
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("size", [-100, 40, 70, 99])
def test_latent_vectors_of_any_size(lib, size, dtype):  # noqa: F811
    """As many sequences as CTAs. Scores come from the shared keys alone and go up by some 50 powers of two from tile to tile."""
    lengths = [320] * 160
    c = Case(lib, 61, lengths, [1] * 160, 128, 16, 64, dtype, fill=True)
    ramp = torch.arange(320).div(64, rounding_mode="floor") * 12.0 * 0.693 + torch.arange(320) % 3
    for s in range(160):
        for p in range(5):
            c.start[c.table[s, p], :, 128:] = ramp[64 * p:64 * p + 64, None].to(BF16)
    c.start[..., :128] *= 2.0 ** size
    c.cache.pages.copy_(c.start)
    q = torch.zeros(c.n_rows, 6, 144, dtype=dtype)
    q[..., 130] = torch.linspace(-1, 1, 6).to(dtype)
    check_attend(c, 6, 1.0, q.cuda())


# ---- ordinary calls ----------------------------------------------------------------
# In the 2-norm, where independent roundings add up as squares. A rounding to bf16 is uniform within its step, half a step at most: its root mean square is
# 2^-8 / sqrt(3) = 0.00226 of a number just above a power of two and half of that below the next, 0.00166 over normal numbers. That is the result's. One
# more of probabilities, whose products with values of either sign add up as squares too, makes 0.00235 of it: calls of 64 columns (heads times new
# rows, in equal blocks). Probabilities of two parts are off by 2^-17 and leave it as it is.
@pytest.mark.parametrize("lengths,rows,heads,latent,rope,limit", [
    ([700, 333], [1, 1], 16, 512, 64, 0.0018), ([900], [1], 10, 256, 32, 0.0018), ([500, 90], [5, 3], 16, 512, 64, 0.0018), ([600, 300], [1, 1], 33, 128, 64, 0.0018),
    ([800, 333], [2, 2], 10, 384, 48, 0.0018), ([700, 333], [1, 1], 128, 512, 64, 0.0024), ([700], [4], 16, 256, 64, 0.0024),
])
def test_errors_of_ordinary_calls(lib, lengths, rows, heads, latent, rope, limit):  # noqa: F811
    c = Case(lib, 62, lengths, rows, latent, rope, 32, BF16, fill=True)
    q = c.randn(c.n_rows, heads, latent + rope)
    got = f64(c.cache.attend(c.batch, q, (128 + rope) ** -0.5))
    want = R.attend(f64(q), f64(c.start), c.table.numpy(), lengths, c.row_start, (128 + rope) ** -0.5, latent)[0]
    assert np.linalg.norm(got - want) <= limit * np.linalg.norm(want)


# ---- queries that are not finite, waits that run out ---------------------------------
SHARED = [  # form, lengths, new rows, heads: one tile; several; cut between CTAs; columns of 16, 32, 48 and 64; prompts
    ("bf16", [20], [1], 8), ("fp32", [1], [1], 2), ("bf16", [300, 40], [2, 1], 16), ("fp32", [300, 40], [2, 1], 16), ("bf16", [5000], [1], 8), ("fp32", [9000], [1], 3),
    ("bf16", [3000, 9], [5, 1], 16), ("bf16", [3000, 200], [1, 1], 64), ("fp32", [700], [3], 20), ("expanded", [300, 200], [300, 200], 3), ("expanded", [20], [20], 2),
    ("expanded", [500, 1], [280, 1], 2),
]


def form_of(form, lengths, rows, heads):
    c = Case(form_of.lib, 63, lengths, rows, 256, 32, 16, FP32 if form == "fp32" else BF16, 1, fill=True)
    w = torch.randn(heads, 128, 256, generator=c.g).mul(0.1).to(BF16).cuda()
    q = c.randn(c.n_rows, heads, 96 if form == "expanded" else 288)

    def run():
        if form == "expanded":
            return c.cache.attend_expanded(c.batch, q, w[:, :64], w[:, 64:], 0.1, sum(lengths))[:c.n]
        return c.cache.attend(c.batch, q, 0.1)[:c.n]
    return c, q, run


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("form,lengths,rows,heads", SHARED)
def test_queries_that_are_not_finite(lib, form, lengths, rows, heads, bad):  # noqa: F811
    """A head whose query holds a NaN or an infinity gives NaN, however its tokens are shared out; the other heads give the same bits."""
    form_of.lib = lib
    c, q, run = form_of(form, lengths, rows, heads)
    good = run()
    assert good.isfinite().all()
    hit = {(0, 0), (c.n - 1, heads - 1), (c.n // 2, heads // 2)}
    for i, h in hit:
        q[i, h, (5 * i + 37 * h) % q.shape[2]] = bad
    out = run()
    for i, h in hit:
        assert out[i, h].isnan().all()
        out[i, h] = good[i, h]
    assert torch.equal(out, good)


@pytest.mark.parametrize("form,lengths,rows,heads", SHARED)
def test_a_wait_that_runs_out(lib, form, lengths, rows, heads):  # noqa: F811
    """An arrival that nobody makes: the kernels give up after the limit and say so, and the next call is what it was."""
    from paper_2607_24787_b200 import binding as B
    form_of.lib = lib
    c, q, run = form_of(form, lengths, rows, heads)
    want = run()
    assert c.status.item() == 0
    try:
        B.spm_test_kv_waits(1, 1000)
        run()
        torch.cuda.synchronize()
    finally:
        B.spm_test_kv_waits(0, 0)
    assert c.status.item() == B.KV_TIMEOUT
    c.status.zero_()
    assert torch.equal(run(), want) and c.status.item() == 0


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_a_score_that_is_not_finite_behind_others(lib, dtype):  # noqa: F811
    """An infinity in a query meets keys of one sign first and of the other later: its head gives NaN, the heads beside it the same bits."""
    c = Case(lib, 64, [320] * 160, [1] * 160, 128, 16, 64, dtype, fill=True)
    for s in range(160):
        c.start[c.table[s, 0], :, 130] = -1.0
        c.start[c.table[s, 1:5].long(), :, 130] = 1.0
    c.cache.pages.copy_(c.start)
    q = c.randn(160, 6, 144)
    good = c.cache.attend(c.batch, q, 0.3)
    q[:, 2, 130] = float("inf")
    out = c.cache.attend(c.batch, q, 0.3)
    assert out[:, 2].isnan().all()
    out[:, 2] = good[:, 2]
    assert torch.equal(out, good)
