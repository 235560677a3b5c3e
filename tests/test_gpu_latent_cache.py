"""Attention over latent rows on the GPU (the cache, products of heads, the absorbed form), against the 64-bit oracle."""
import numpy as np
import pytest
import torch

from oracle import ref_latent as R
from oracle.ref_cache import page_of, places

pytestmark = pytest.mark.gpu

BF16, FP32 = torch.bfloat16, torch.float32
HALF = {BF16: 2.0 ** -8, FP32: 2.0 ** -24}        # one rounding, relative


@pytest.fixture(scope="module")
def lib():
    from paper_2607_24787_b200 import kv_cache, latent_cache
    from paper_2607_24787_b200.build import build
    build()
    latent_cache.kv = kv_cache
    return latent_cache


def f64(x):
    return x.double().cpu().numpy()


class Case:
    """A ragged batch over a pool whose pages are handed out in random order; new rows are the last ones of each sequence."""

    def __init__(self, lib, seed, lengths, rows, latent=512, rope=64, page=32, dtype=BF16, pad_rows=0, wide_table=0, fill=False, max_rows=None):
        self.g = torch.Generator().manual_seed(seed)
        self.lengths, self.rows, self.latent, self.rope, self.page, self.dtype = lengths, rows, latent, rope, page, dtype
        self.row_start = [0]
        for n in rows:
            self.row_start.append(self.row_start[-1] + n)
        self.n, self.n_rows = self.row_start[-1], self.row_start[-1] + pad_rows
        need = [-(-n // page) for n in lengths]
        pool = sum(need) + 2
        order = torch.randperm(pool, generator=self.g).to(torch.int32)
        table = torch.full((len(need), max(need + [1]) + wide_table), -1, dtype=torch.int32)
        first = 0
        for i, n in enumerate(need):
            table[i, :n] = order[first:first + n]
            first += n
        shape = pool, page, latent + rope
        pages = torch.randn(shape, generator=self.g) if fill else torch.full(shape, 3.0)
        if fill:                                   # what is behind a sequence's end may be anything
            for s, n in enumerate(lengths):
                if n % page:
                    pages[table[s, n // page], n % page:] = float("nan")
        self.table = table
        self.start = pages.to(BF16)
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.cache = lib.LatentCache(self.start.cuda(), latent, self.status)
        self.dev_table, self.dev_lengths = table.cuda(), torch.tensor(lengths, dtype=torch.int32, device="cuda")
        self.batch = lib.kv.KVBatch(self.dev_table, self.dev_lengths, torch.tensor(self.row_start, dtype=torch.int32, device="cuda"),
                                    n_rows=self.n_rows, max_rows=max(rows + [0]) if max_rows is None else max_rows)

    def randn(self, *shape, scale=1.0):
        return (torch.randn(*shape, generator=self.g) * scale).to(self.dtype).cuda()


def rope_of(lib, c, gamma=True, rot=None, neighbours=False, axes=1):
    rot = c.rope if rot is None else rot
    inv = (1e4 ** (-torch.arange(rot // 2, dtype=torch.float64) / (rot // 2))).float()
    axis = torch.arange(rot // 2) % axes
    g = 1 + 0.2 * torch.randn(c.latent, generator=c.g) if gamma else None
    rope = lib.kv.Rope(inv.cuda(), axis_of=axis.to(torch.uint8).cuda(), k_gamma=None if g is None else g.cuda(), eps=1e-6, neighbours=neighbours)
    return rope, inv.numpy(), axis.numpy(), None if g is None else g.numpy()


def turn_tolerance(x, rot, neighbours, dtype):
    """Two products, a sum and a cosine and a sine of 24 bits: four fp32 roundings of the pair's length; then the result's."""
    pairs = x[..., :rot]
    a, b = (pairs[..., 0::2], pairs[..., 1::2]) if neighbours else (pairs[..., :rot // 2], pairs[..., rot // 2:])
    length = np.sqrt(a * a + b * b)
    both = np.stack((length, length), -1).reshape(pairs.shape) if neighbours else np.concatenate((length, length), -1)
    return np.concatenate((both, np.abs(x[..., rot:])), -1) * 4 * HALF[FP32]


# lengths, new rows, heads, latent, rope, turned, page, padded rows, neighbours, gamma
WRITES = [
    ([1], [1], 1, 128, 16, 16, 16, 0, True, True),
    ([17, 33, 16], [1, 1, 1], 16, 512, 64, 64, 16, 0, True, True),
    ([5, 40, 0, 70], [5, 9, 0, 70], 9, 256, 32, 32, 32, 4, False, True),
    ([48, 200], [31, 130], 128, 384, 48, 32, 48, 3, False, False),
    ([7, 0, 12], [9, 2, 12], 33, 512, 64, 48, 64, 1, True, True),        # more rows than tokens: the first ones have no place
    ([1300], [1300], 3, 512, 64, 64, 128, 0, False, True),
]


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("lengths,rows,heads,latent,rope,rot,page,pad,neighbours,gamma", WRITES)
def test_write(lib, lengths, rows, heads, latent, rope, rot, page, pad, neighbours, gamma, dtype):
    c = Case(lib, 3, lengths, rows, latent, rope, page, dtype, pad)
    turn, inv, axis, g = rope_of(lib, c, gamma, rot, neighbours, axes=2)
    x, key, q = c.randn(c.n_rows, latent, scale=3.0), c.randn(c.n_rows, rope), c.randn(c.n_rows, heads, rope)
    pos = torch.randint(0, 200_000, (2, c.n_rows), generator=c.g, dtype=torch.int32)
    out = torch.full_like(q, 7.0)
    assert c.cache.write(c.batch, x, key, q=q, positions=pos.cuda(), rope=turn, q_out=out) is out
    assert (out[c.n:] == 7).all()
    want = R.turn(f64(q), pos.numpy(), inv, axis, neighbours)[:c.n]
    tol = turn_tolerance(f64(q), rot, neighbours, dtype)[:c.n] + HALF[dtype] * np.abs(want)
    assert (np.abs(f64(out)[:c.n] - want) <= tol).all()
    # the pool: exact up to the norm's fp32 roundings (a sum of up to 512 squares, a root, two products) and the one to bf16; nothing else touched
    row = np.concatenate((R.norm(f64(x), g, 1e-6), R.turn(f64(key), pos.numpy(), inv, axis, neighbours)), -1)
    tol = np.concatenate((np.abs(row[:, :latent]) * (512 + 8) * HALF[FP32], turn_tolerance(f64(key), rot, neighbours, dtype)), -1) + HALF[BF16] * np.abs(row)
    want, limit = f64(c.start), np.zeros(c.start.shape)
    for i, at in enumerate(places(lengths, c.row_start, c.n_rows)):
        p = None if at is None else page_of(c.start, c.table.numpy(), *at, page)
        if p is not None:
            want[p, at[1] % page], limit[p, at[1] % page] = row[i], tol[i]
    assert (np.abs(f64(c.cache.pages) - want) <= limit).all()
    assert c.status.item() == 0


def test_write_without_rotation_and_in_place(lib):
    c = Case(lib, 4, [40, 9], [11, 3], 256, 32, 16, FP32, pad_rows=2)
    x, key = c.randn(c.n_rows, 256), c.randn(c.n_rows, 32)
    assert c.cache.write(c.batch, x, key) is None
    want = c.start.clone()
    for i, at in enumerate(places(c.lengths, c.row_start, c.n_rows)):
        if at is not None:
            want[page_of(c.start, c.table.numpy(), *at, 16), at[1] % 16] = torch.cat((x[i], key[i])).to(BF16).cpu()
    assert torch.equal(c.cache.pages.cpu(), want)
    rope, *_ = rope_of(lib, c)
    q = c.randn(c.n_rows, 5, 32)
    pos = torch.arange(c.n_rows, dtype=torch.int32).cuda()
    out = c.cache.write(c.batch, x, key, q=q, positions=pos, rope=rope)
    same = q.clone()
    c.cache.write(c.batch, x, key, q=same, positions=pos, rope=rope, q_out=same)
    assert torch.equal(same[:c.n], out[:c.n]) and torch.equal(same[c.n:], q[c.n:])


def test_write_takes_slices(lib):
    """Latent vector and key side by side in one projection, queries' parts in another, results into the absorbed queries."""
    c = Case(lib, 5, [40, 90], [11, 30], 512, 64, 16, BF16)
    rope, *_ = rope_of(lib, c)
    kv, wide = c.randn(c.n_rows, 576), c.randn(c.n_rows, 7, 192)
    pos = torch.arange(c.n_rows, dtype=torch.int32).cuda()
    apart = c.cache.write(c.batch, kv[:, :512].contiguous(), kv[:, 512:].contiguous(), q=wide[..., 128:].contiguous(), positions=pos, rope=rope)
    pages = c.cache.pages.clone()
    c.cache.pages.fill_(3.0)
    q = torch.zeros(c.n_rows, 7, 576, dtype=BF16, device="cuda")
    c.cache.write(c.batch, kv[:, :512], kv[:, 512:], q=wide[..., 128:], positions=pos, rope=rope, q_out=q[..., 512:])
    assert torch.equal(c.cache.pages, pages) and torch.equal(q[..., 512:], apart) and (q[..., :512] == 0).all()


def test_write_notes_what_it_cannot_place(lib):
    from paper_2607_24787_b200 import binding as B
    c = Case(lib, 6, [40, 40], [2, 2], 128, 16, 16, FP32)
    x, key = c.randn(4, 128), c.randn(4, 16)
    for change, bit in ((lambda: c.dev_table[0, 2].fill_(1000), B.KV_BAD_PAGE), (lambda: c.dev_lengths[1].fill_(500), B.KV_TOO_LONG),
                        (lambda: x[3, 5].fill_(float("inf")), 0), (lambda: c.dev_lengths[1].fill_(40), B.KV_NONFINITE)):
        change()
        c.status.zero_()
        c.cache.write(c.batch, x, key)
        assert c.status.item() & bit == bit
    x[3, 5] = 3.4e38                                   # finite, but not in bf16
    c.dev_table[0, 2] = int(c.table[0, 2])
    c.status.zero_()
    c.cache.write(c.batch, x, key)
    assert c.status.item() == B.KV_NONFINITE


# ---- products of heads -------------------------------------------------------
PRODUCTS = [(1, 16, 128, 512), (3, 1, 64, 64), (16, 5, 512, 128), (17, 10, 64, 256), (32, 2, 384, 128), (33, 33, 128, 128), (200, 3, 512, 64), (64, 128, 512, 128),
            (7, 2, 1024, 320), (70, 60, 64, 320), (130, 40, 320, 64)]


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("n,heads,size,to", PRODUCTS)
def test_head_product(lib, n, heads, size, to, dtype, transposed):
    g = torch.Generator().manual_seed(9)
    x = torch.randn(n, heads, size, generator=g).to(dtype).cuda()
    w = torch.randn(heads, size, to, generator=g).to(BF16)
    y = lib.head_product(x, (w.transpose(1, 2).contiguous() if transposed else w).cuda(), transposed=transposed)
    want = np.einsum("nhi,hio->nho", f64(x), f64(w))
    span = np.einsum("nhi,hio->nho", np.abs(f64(x)), np.abs(f64(w)))
    # exact products, fp32 sums of `size` (three parts: three times as many), a truncated one off by 2^-23
    tol = (3 if dtype is FP32 else 1) * size * 2.0 ** -23 * span + HALF[dtype] * np.abs(want)
    off = np.abs(f64(y) - want)
    assert (off <= tol).all()
    assert np.linalg.norm(off) <= (3e-3 if dtype is BF16 else 1e-6) * np.linalg.norm(want)


def test_head_product_of_slices(lib):
    g = torch.Generator().manual_seed(10)
    both = torch.randn(6, 256, 512, generator=g).to(BF16).cuda()
    x = torch.randn(9, 6, 192, generator=g).to(BF16).cuda()
    q = torch.zeros(9, 6, 576, dtype=BF16, device="cuda")
    lib.head_product(x[..., :128], both[:, :128], out=q[..., :512])
    assert torch.equal(q[..., :512], lib.head_product(x[..., :128].contiguous(), both[:, :128].contiguous())) and (q[..., 512:] == 0).all()
    o = torch.randn(9, 6, 512, generator=g).to(BF16).cuda()
    assert torch.equal(lib.head_product(o, both[:, 128:], transposed=True), lib.head_product(o, both[:, 128:].contiguous(), transposed=True))
    assert lib.head_product(x[:0, :, :128], both[:, :128]).shape == (0, 6, 512)


def test_head_product_of_what_is_not_finite(lib):
    w = torch.ones(2, 64, 64, dtype=BF16, device="cuda")
    for dtype in (BF16, FP32):
        x = torch.ones(5, 2, 64, dtype=dtype, device="cuda")
        x[1, 0, 3], x[2, 1, 9] = float("nan"), float("inf")
        y = lib.head_product(x, w)
        assert y[1, 0].isnan().all() and not y[2, 1].isfinite().any()
        y[1, 0], y[2, 1] = 64, 64
        assert (y == 64).all()
    x = torch.full((3, 2, 64), 3e38, device="cuda")    # rounds to an infinity in bf16; its parts do not
    assert torch.allclose(lib.head_product(x, w / 64), x, rtol=1e-6)


# ---- attention, absorbed -----------------------------------------------------
# A score is the sum of latent + rope products in fp32, each addition off by 2^-23 of the terms' sum at most (truncated), and is scaled with
# another rounding: a probability moves by as much relative to itself, twice (its row's sum too). The probabilities' and the sums' own
# additions are one for every 16 tokens, and a few joins. bf16 calls round a probability and the result once more.
def attend_tolerance(want, spread, reach, dtype, tokens, width):
    probability = 2 * ((width / 16 * 3 + 16) * 2.0 ** -23 * (reach + 1)) + (tokens / 16 * 3 + 40) * 2.0 ** -23
    if dtype is BF16:
        probability = probability + HALF[BF16]
    return probability * spread + HALF[dtype] * np.abs(want) + 1e-30


def check_attend(c, heads, scale=None, q=None, out=None):
    width = c.latent + c.rope
    scale = (128 + c.rope) ** -0.5 if scale is None else scale
    q = c.randn(c.n_rows, heads, width) if q is None else q
    out = torch.full((c.n_rows, heads, c.latent), 9.0, dtype=c.dtype, device="cuda") if out is None else out
    c.cache.attend(c.batch, q, scale, out=out)
    want, spread, reach = R.attend(f64(q), f64(c.start), c.table.numpy(), c.lengths, c.row_start, scale, c.latent)
    got = f64(out)
    assert (got[c.n:] == 9).all()
    off = np.abs(got[:c.n] - want[:c.n])
    tol = attend_tolerance(want, spread, reach, c.dtype, max(c.lengths), width)[:c.n]
    assert (off <= tol).all(), (off.max(), np.unravel_index((off - tol).argmax(), off.shape))
    size = np.linalg.norm(want[:c.n])
    if size:
        assert np.linalg.norm(off) <= (4e-3 if c.dtype is BF16 else 4e-6) * size
    return out


ATTENDS = [
    # lengths, new rows, heads, latent, rope, page, padded rows
    ([1], [1], 16, 512, 64, 16, 0),
    ([2, 15, 16, 17], [1, 1, 1, 1], 1, 128, 16, 16, 0),
    ([300], [1], 16, 512, 64, 64, 1),
    ([31, 0, 129, 64, 333], [1, 0, 1, 1, 1], 10, 256, 32, 32, 2),
    ([700, 1], [1, 1], 33, 384, 48, 48, 0),
    ([100, 77], [3, 5], 16, 512, 64, 16, 0),
    ([40, 65, 3], [40, 20, 3], 5, 128, 64, 32, 3),
    ([9, 4], [11, 4], 8, 256, 16, 16, 1),               # rows before position 0 see nothing
    ([150, 33], [50, 30], 7, 512, 64, 64, 0),
    ([260], [1], 128, 512, 64, 128, 0),
    ([65, 64, 63, 128, 127], [1, 2, 1, 1, 2], 64, 384, 64, 256, 0),
]


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("lengths,rows,heads,latent,rope,page,pad", ATTENDS)
def test_attend(lib, lengths, rows, heads, latent, rope, page, pad, dtype):
    c = Case(lib, 8, lengths, rows, latent, rope, page, dtype, pad, wide_table=1, fill=True)
    check_attend(c, heads)
    assert c.status.item() == 0


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("lengths,heads,latent,rope", [([9000], 16, 512, 64), ([20_000], 3, 128, 32), ([3000, 70, 2500, 1], 20, 256, 64)])
def test_attend_over_long_contexts(lib, lengths, heads, latent, rope, dtype):
    """Items cut between many CTAs, and their parts joined; the same bits again."""
    c = Case(lib, 9, lengths, [1] * len(lengths), latent, rope, 64, dtype, fill=True)
    q = c.randn(c.n_rows, heads, latent + rope)
    out = check_attend(c, heads, q=q)
    for _ in range(3):
        assert torch.equal(c.cache.attend(c.batch, q, (128 + rope) ** -0.5), out)


def test_attend_of_many_sequences(lib):
    r = np.random.default_rng(1)
    lengths = [int(x) for x in r.integers(0, 90, 300)]
    c = Case(lib, 10, lengths, [min(1, n) for n in lengths], 128, 16, 16, BF16, fill=True)
    check_attend(c, 6)


@pytest.mark.parametrize("max_rows", [0, 1, 50])
def test_the_rows_hint_changes_no_result(lib, max_rows):
    c = Case(lib, 11, [200, 90], [9, 4], 256, 64, 32, BF16, fill=True, max_rows=max_rows)
    check_attend(c, 12)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("size,scale", [(300.0, 0.1), (1.0, -0.2), (1.0, 0.0), (1e4, 1.0), (1e-20, 1e18), (1e15, 1e-16)])
def test_attend_scores_of_any_size(lib, size, scale, dtype):
    """The running maximum moves often, or nothing does. Scores so large leave one token, and which is decided by their fp32 sums: where two
    are within those sums' error the tolerance is the values themselves."""
    c = Case(lib, 12, [400, 90], [1, 2], 128, 32, 16, dtype, fill=True)
    q = c.randn(c.n_rows, 4, 160, scale=size)
    check_attend_norm = size * scale <= 1
    if check_attend_norm:
        check_attend(c, 4, scale, q)
        return
    out = f64(c.cache.attend(c.batch, q, scale))
    want, spread, reach = R.attend(f64(q), f64(c.start), c.table.numpy(), c.lengths, c.row_start, scale, 128)
    slack = 2 * (160 / 16 * 3 + 16) * 2.0 ** -23 * reach
    tol = attend_tolerance(want, spread, 0 * reach, dtype, 400, 160) + np.minimum(np.expm1(np.minimum(slack, 30)), 2) * 5
    assert (np.abs(out - want) <= tol).all()


def test_growing_scores_move_the_maximum(lib):
    """Each tile's scores are far above those before."""
    c = Case(lib, 13, [640], [1], 128, 16, 64, BF16, fill=True)
    ramp = torch.arange(640).div(64, rounding_mode="floor").float() * 40.0
    for t in range(640):
        c.start[c.table[0, t // 64], t % 64, 128] = ramp[t]
    c.cache.pages.copy_(c.start)
    q = torch.zeros(1, 16, 144, dtype=BF16)
    q[..., :128] = torch.randn(1, 16, 128, generator=c.g) * 0.1
    q[..., 128] = torch.arange(16).float() * 0.5 - 2           # some go up by up to 220 a tile, some down, one stays
    check_attend(c, 16, 1.0, q.cuda())


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_bad_queries_stay_by_themselves(lib, dtype):
    c = Case(lib, 14, [100, 0, 70], [2, 1, 1], 256, 32, 16, dtype, fill=True)
    q = c.randn(c.n_rows, 6, 288)
    good = c.cache.attend(c.batch, q, 0.1)
    q[0, 2, 7], q[1, 3, 280], q[3, 0], q[2, 1] = float("nan"), float("inf"), -float("inf"), float("nan")
    out = c.cache.attend(c.batch, q, 0.1)
    for row, head in ((0, 2), (1, 3), (3, 0)):
        assert out[row, head].isnan().all()
        out[row, head] = good[row, head]
    assert torch.equal(out, good) and (good[2] == 0).all()     # (a row that sees nothing stays zero)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("what", [float("nan"), float("inf"), -float("inf")])
def test_bad_tokens_reach_only_rows_that_see_them(lib, what, dtype):
    c = Case(lib, 15, [200, 130], [6, 1], 256, 32, 16, dtype, fill=True)
    q = c.randn(c.n_rows, 3, 288)
    good = c.cache.attend(c.batch, q, 0.1)
    page = c.table[0, 196 // 16]
    c.cache.pages[page, 196 % 16] = what                       # row 2 of sequence 0 is the first to see it
    out = c.cache.attend(c.batch, q, 0.1)
    assert out[2:6].isnan().all()
    assert torch.equal(out[:2], good[:2]) and torch.equal(out[6], good[6])


def test_pages_that_are_not_there(lib):
    from paper_2607_24787_b200 import binding as B
    c = Case(lib, 16, [200, 90, 64], [1, 3, 1], 128, 16, 16, BF16, fill=True)
    for s, p, to in ((0, 3, -1), (0, 12, 10 ** 6), (1, 0, -5), (2, 0, 99), (2, 1, 99), (2, 2, 99), (2, 3, 99)):
        c.table[s, p] = to
    c.dev_table.copy_(c.table)
    check_attend(c, 16)                                        # (the last sequence sees nothing)
    assert c.status.item() == B.KV_BAD_PAGE
    c.status.zero_()
    c.dev_lengths[1] = 10 ** 6
    q = c.randn(c.n_rows, 2, 144)
    c.cache.attend(c.batch, q, 0.1)
    assert c.status.item() == B.KV_BAD_PAGE | B.KV_TOO_LONG


def test_attend_takes_strided_rows(lib):
    c = Case(lib, 17, [150, 60], [4, 1], 256, 32, 32, BF16, fill=True)
    wide = c.randn(c.n_rows, 8, 300 + 20)
    q = wide[:, 1:6, 16:304]
    want = c.cache.attend(c.batch, q.contiguous(), 0.07)
    assert torch.equal(c.cache.attend(c.batch, q, 0.07), want)
    first = c.randn(8, c.n_rows, 256)
    c.cache.attend(c.batch, q, 0.07, out=first.transpose(0, 1)[:, 2:7])
    assert torch.equal(first.transpose(0, 1)[:, 2:7], want)


def test_a_step_and_its_replay(lib):
    """Absorbed decode as a program runs it, against attention in its whole form, then captured and replayed with other lengths; two captured
    graphs and another stream."""
    heads, head, latent, rope = 6, 64, 256, 32
    c = Case(lib, 18, [70, 33, 5], [1, 1, 1], latent, rope, 16, BF16, wide_table=2, fill=True)
    w = torch.randn(heads, 2 * head, latent, generator=c.g).mul(latent ** -0.5).to(BF16).cuda()
    w_k, w_v = w[:, :head], w[:, head:]
    turn, inv, axis, gamma = rope_of(lib, c)
    x, q_in = c.randn(3, latent + rope), c.randn(3, heads, head + rope)
    pos = (c.dev_lengths - 1).clone()
    scale = (head + rope) ** -0.5

    def step():
        q = torch.empty(3, heads, latent + rope, dtype=BF16, device="cuda")
        lib.head_product(q_in[..., :head], w_k, out=q[..., :latent])
        c.cache.write(c.batch, x[:, :latent], x[:, latent:], q=q_in[..., head:], positions=pos, rope=turn, q_out=q[..., latent:])
        return lib.head_product(c.cache.attend(c.batch, q, scale), w_v, transposed=True)

    out = step()
    # roundings on the way: queries, results and the cache's rows (as they are read back) are bf16
    q64 = np.concatenate((f64(q_in[..., :head]), R.turn(f64(q_in[..., head:]), pos[None].cpu().numpy(), inv, axis, False)), -1)
    want = R.attend(q64, f64(c.cache.pages), c.table.numpy(), c.lengths, c.row_start, scale, latent, f64(w_k), f64(w_v))[0]
    assert np.linalg.norm(f64(out) - want) <= 2e-2 * np.linalg.norm(want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        assert torch.equal(step(), out)
    torch.cuda.current_stream().wait_stream(side)
    graphs, outs = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(step())
        graphs.append(g)
    c.dev_lengths.copy_(torch.tensor([64, 30, 1]))
    pos.copy_(c.dev_lengths - 1)
    x.copy_(c.randn(3, latent + rope))
    want = step()
    for g, o in zip(graphs, outs):
        o.zero_()
        g.replay()
        assert torch.equal(o, want)


def test_pools_beyond_4_gigabytes(lib):
    """Rows whose byte offsets do not fit into 32 bits, signed or not: written, attended to and expanded as in a small pool."""
    heads, head, page, n = 4, 64, 256, 16_500
    small = Case(lib, 34, [700], [3], 512, 64, page, BF16)
    rows = small.randn(700, 576)
    table = torch.tensor([[2, 0, 1]], dtype=torch.int32)
    big = lib.LatentCache(torch.empty(n, page, 576, dtype=BF16, device="cuda"), 512)      # 4.9 GB
    outs = []
    q, qe, w = small.randn(700, heads, 576), small.randn(700, heads, head + 64), torch.randn(heads, 2 * head, 512, generator=small.g).mul(0.05).to(BF16).cuda()
    for cache, first in ((lib.LatentCache(torch.empty(3, page, 576, dtype=BF16, device="cuda"), 512), 0), (big, n - 3)):
        start = torch.tensor([0, 700], dtype=torch.int32, device="cuda")
        batch = lib.kv.KVBatch((table + first).int().cuda(), torch.tensor([700], dtype=torch.int32, device="cuda"), start, n_rows=700, max_rows=700)
        cache.write(batch, rows[:, :512], rows[:, 512:])
        outs.append((cache.attend(batch, q, 0.05), cache.attend_expanded(batch, qe, w[:, :head], w[:, head:], 0.1, 700), cache.pages[first:first + 3].clone()))
    for a, b in zip(*outs):
        assert torch.equal(a, b)


def test_waits_that_run_out(lib):
    """Copies that never count as landed: the call ends with the status bit, and the next one is right."""
    from paper_2607_24787_b200 import binding as B
    c = Case(lib, 19, [300, 90], [1, 2], 512, 64, 16, BF16, fill=True)
    q = c.randn(c.n_rows, 16, 576)
    want = c.cache.attend(c.batch, q, 0.1)
    B.spm_test_kv_waits(1, 3000)
    try:
        c.cache.attend(c.batch, q, 0.1)
        torch.cuda.synchronize()
        assert c.status.item() & B.KV_TIMEOUT
    finally:
        B.spm_test_kv_waits(0, 0)
    assert torch.equal(c.cache.attend(c.batch, q, 0.1), want)
