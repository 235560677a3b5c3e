"""Rotary positions, the 4-bit key/value cache and attention over it on the GPU, against the 64-bit oracle."""
import numpy as np
import pytest
import torch

from oracle import ref_cache as R

pytestmark = pytest.mark.gpu

BF16, FP32 = torch.bfloat16, torch.float32
HALF = {BF16: 2.0 ** -8, FP32: 2.0 ** -24}        # one rounding, relative


@pytest.fixture(scope="module")
def kv():
    from paper_2607_24787_b200 import kv_cache
    from paper_2607_24787_b200.build import build
    build()
    return kv_cache


class Case:
    """A ragged batch over a pool whose pages are handed out in random order; new rows are the last ones of each sequence."""

    def __init__(self, kv, seed, lengths, rows, kv_heads=2, hd=128, page=32, dtype=BF16, pad_rows=0, wide_table=0, fill=False):
        self.g = torch.Generator().manual_seed(seed)
        self.lengths, self.rows, self.hd, self.page, self.hk, self.dtype = lengths, rows, hd, page, kv_heads, dtype
        self.row_start = [0]
        for n in rows:
            self.row_start.append(self.row_start[-1] + n)
        self.n_rows = self.row_start[-1] + pad_rows
        need = [-(-n // page) for n in lengths]
        pool = sum(need) + 2
        order = torch.randperm(pool, generator=self.g).to(torch.int32)
        table = torch.full((len(need), max(need + [1]) + wide_table), -1, dtype=torch.int32)
        first = 0
        for i, n in enumerate(need):
            table[i, :n] = order[first:first + n]
            first += n
        if fill:
            pages = torch.randint(0, 256, (pool, kv_heads, page // 16, 18 * hd), generator=self.g, dtype=torch.uint8)
            scale = (torch.rand(pool, kv_heads, page // 16, hd, generator=self.g) * 0.3 - 0.15).half()
            pages[..., 16 * hd:] = scale.view(torch.uint8)
        else:
            pages = torch.full((pool, kv_heads, page // 16, 18 * hd), 0xab, dtype=torch.uint8)
        self.table = table
        self.start = pages.numpy().copy()
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.cache = kv.KVCache(pages.cuda(), self.status)
        self.dev_lengths = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        self.batch = kv.KVBatch(table.cuda(), self.dev_lengths, torch.tensor(self.row_start, dtype=torch.int32, device="cuda"),
                                n_rows=self.n_rows, max_rows=max(rows + [0]))

    def randn(self, *shape, scale=1.0):
        return (torch.randn(*shape, generator=self.g) * scale).to(self.dtype).cuda()

    def pages(self):
        return self.cache.pages.cpu().numpy()


def expected_pages(c, k, v):
    """The pool after the rows k, v (fp32, on the host) have been written."""
    pages = c.start.copy()
    table = c.table.numpy()
    for i, at in enumerate(R.places(c.lengths, c.row_start, c.n_rows)):
        if at is None:
            continue
        page = R.page_of(pages, table, at[0], at[1], c.page)
        if page is None:
            continue
        for h in range(c.hk):
            for part, x in ((0, k), (1, v)):
                R.put(pages, page, h, at[1] % c.page, part, *R.quantise(x[i, h]))
    return pages


WRITES = [
    # lengths, new rows, kv heads, head size, page, dtype, padded rows
    ([1], [1], 1, 64, 16, BF16, 0),
    ([17, 33, 16], [1, 1, 1], 2, 128, 16, FP32, 0),
    ([5, 40, 0, 70], [5, 9, 0, 70], 3, 128, 32, BF16, 4),
    ([48, 200], [31, 130], 1, 256, 48, FP32, 3),
    ([7, 0, 12], [9, 2, 12], 2, 64, 64, BF16, 1),        # more rows than tokens: the first ones have no place
]


@pytest.mark.parametrize("lengths,rows,hk,hd,page,dtype,pad", WRITES)
def test_write_is_exact(kv, lengths, rows, hk, hd, page, dtype, pad):
    c = Case(kv, 3, lengths, rows, hk, hd, page, dtype, pad)
    k, v = c.randn(c.n_rows, hk, hd), c.randn(c.n_rows, hk, hd, scale=30.0)
    k[0, 0, :32] = 0                       # a group of zeros
    v[0, 0, 3], v[0, 0, 7] = 99.0, -99.0   # two of equal magnitude: the first one's sign counts
    assert c.cache.write(c.batch, k, v) is None
    got = c.pages()
    want = expected_pages(c, k.float().cpu().numpy(), v.float().cpu().numpy())
    assert np.array_equal(got, want)       # byte for byte, and nothing else touched
    assert c.status.item() == 0


def test_many_rows(kv):
    """More rows than one block a row takes: written, read back and turned as in small calls."""
    c = Case(kv, 17, [2500, 900, 17], [2400, 900, 10], 1, 64, 16, BF16, 3)
    k, v = c.randn(c.n_rows, 1, 64), c.randn(c.n_rows, 1, 64)
    rope, plain = rope_of(kv, 64)
    pos = torch.randint(0, 9000, (3, c.n_rows), generator=c.g, dtype=torch.int32).cuda()
    c.cache.write(c.batch, k, v)
    assert np.array_equal(c.pages(), expected_pages(c, k.float().cpu().numpy(), v.float().cpu().numpy()))
    back = [torch.full((c.n_rows, 1, 64), 4.0, device="cuda") for _ in range(2)]
    c.cache.read(c.batch, k_out=back[0], v_out=back[1])
    n = c.row_start[-1]
    for x, y in ((k, back[0]), (v, back[1])):
        codes, d = R.quantise(x.float().cpu().numpy())
        want = (codes.astype(np.float64) - 8) * np.repeat(d.astype(np.float64), 32, axis=-1)
        assert np.array_equal(y.double().cpu().numpy()[:n], want[:n]) and (y[n:] == 4).all()
    big = torch.randn(20_001, 3, 64, generator=c.g).cuda()          # and enough for blocks of many rows, in both calls
    at = torch.randint(0, 9000, (3, 20_001), generator=c.g, dtype=torch.int32)
    want = plain(big, at, 0)
    off = np.abs(kv.rotate_heads(big, at.cuda(), rope).double().cpu().numpy() - want)
    assert (off <= turn_tolerance(want, 64, False, FP32)).all()
    whole = Case(kv, 18, [19_500, 33], [19_500, 33], 1, 64, 16, BF16, fill=True)
    got = whole.cache.read(whole.batch, FP32)
    for i in list(range(0, 19_500, 977)) + [19_499, 19_500, 19_532]:
        seq, p = (0, i) if i < 19_500 else (1, i - 19_500)
        page = R.page_of(whole.start, whole.table.numpy(), seq, p, 16)
        for part in range(2):
            assert np.array_equal(got[part][i, 0].double().cpu().numpy(), R.get(whole.start, page, 0, p % 16, part))


@pytest.mark.parametrize("layout", ["projection", "heads_first", "wide_rows"])
def test_write_takes_strided_rows(kv, layout):
    c = Case(kv, 4, [40, 9], [11, 3], 2, 128, 16, BF16)
    k, v = c.randn(c.n_rows, 2, 128), c.randn(c.n_rows, 2, 128)
    if layout == "projection":
        both = torch.cat((k.flatten(1), v.flatten(1)), dim=1)
        sk, sv = (x.unflatten(1, (2, 128)) for x in both.split(256, dim=1))
    elif layout == "heads_first":
        sk, sv = (x.transpose(0, 1).contiguous().transpose(0, 1) for x in (k, v))
    else:
        wide = torch.zeros(c.n_rows, 5, 160, dtype=BF16, device="cuda")
        wide[:, 1:3, 8:136] = k
        wide[:, 3:5, 16:144] = v
        sk, sv = wide[:, 1:3, 8:136], wide[:, 3:5, 16:144]
    c.cache.write(c.batch, sk, sv)
    assert np.array_equal(c.pages(), expected_pages(c, k.float().cpu().numpy(), v.float().cpu().numpy()))


def test_numbers_that_are_not_finite(kv):
    c = Case(kv, 5, [4], [4], 1, 64, 16, FP32)
    k, v = c.randn(4, 1, 64), c.randn(4, 1, 64)
    k[1, 0, 5], k[2, 0, 40], v[3, 0, 0] = float("nan"), float("inf"), -1e30
    c.cache.write(c.batch, k, v)
    assert np.array_equal(c.pages(), expected_pages(c, k.cpu().numpy(), v.cpu().numpy()))
    assert c.status.item() == 4
    got = c.cache.read(c.batch, FP32)
    assert got[0][1, 0, 5] == 0 and got[0][2, 0, 40] == 8 * 65504 and got[1][3, 0, 0] == -8 * 65504
    assert all(x.isfinite().all() for x in got)


def rope_of(kv, hd, rot=None, axes=3, gammas=True, neighbours=False, seed=0):
    g = torch.Generator().manual_seed(seed)
    half = (hd if rot is None else rot) // 2
    inv = (1e4 ** (-torch.arange(half, dtype=torch.float64) / max(half, 1))).float()
    axis = torch.arange(half, dtype=torch.uint8) % axes
    gq, gk = (1 + 0.2 * torch.randn(hd, generator=g) for _ in range(2))
    rope = kv.Rope(inv.cuda(), axis_of=axis.cuda(), q_gamma=gq.cuda() if gammas else None, k_gamma=gk.cuda() if gammas else None,
                   eps=1e-6, neighbours=neighbours)
    plain = lambda x, pos, which: R.rotate(x.float().cpu().numpy(), pos.cpu().numpy(), inv.numpy(), axis.numpy().astype(int),  # noqa: E731
                                           (gq, gk)[which].numpy() if gammas else None, 1e-6, neighbours)
    return rope, plain


# The norm's factor is one rounding and its two products two; a turned element is two products of these with a cosine or sine of one
# rounding each, and their sum: six roundings relative to |a| + |b| of the pair, which are at most sqrt(2) times the pair's length. A row's
# rounding comes on top, relative to the value.
def turn_tolerance(want, rot, neighbours, dtype):
    pair = np.abs(want).copy()
    half = rot // 2
    if neighbours:
        both = np.hypot(want[..., 0:rot:2], want[..., 1:rot:2])
        pair[..., 0:rot:2], pair[..., 1:rot:2] = both, both
    else:
        both = np.hypot(want[..., :half], want[..., half:rot])
        pair[..., :half], pair[..., half:rot] = both, both
    return 6 * np.sqrt(2) * HALF[FP32] * pair + (HALF[dtype] * np.abs(want) * (1 + 1e-6) if dtype is BF16 else 0) + 1e-30


@pytest.mark.parametrize("hd,rot,axes,gammas,neighbours", [(64, 64, 3, True, False), (128, 128, 2, False, False), (128, 64, 4, True, True),
                                                           (256, 32, 1, True, False), (128, 0, 1, True, False), (256, 256, 3, False, True)])
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("n", [1, 37])
def test_rotation(kv, hd, rot, axes, gammas, neighbours, dtype, n):
    g = torch.Generator().manual_seed(hd + n)
    rope, plain = rope_of(kv, hd, rot, axes, gammas, neighbours)
    x = torch.randn(n, 5, hd, generator=g).to(dtype).cuda()
    pos = torch.randint(-50, 70, (axes, n), generator=g, dtype=torch.int32)
    pos[0, 0] = 2 ** 31 - 1                # as far as a position goes
    want = plain(x, pos, 0)
    got = kv.rotate_heads(x, pos.cuda(), rope)
    assert got.dtype is dtype
    off = np.abs(got.double().cpu().numpy() - want)
    assert (off <= turn_tolerance(want, rot, neighbours, dtype)).all(), off.max()
    y = x.clone()                          # in place
    kv.rotate_heads(y, pos.cuda(), rope, out=y)
    assert torch.equal(y, got)


def deq(cd):
    codes, d = cd
    return (codes.astype(np.float64) - 8) * np.repeat(d.astype(np.float64), 32)


@pytest.mark.parametrize("hd,dtype,neighbours", [(64, FP32, False), (128, BF16, False), (256, BF16, True)])
def test_write_with_rotation(kv, hd, dtype, neighbours):
    c = Case(kv, 6, [90, 3, 41], [33, 1, 8], 2, hd, 32, dtype, pad_rows=2)
    rope, plain = rope_of(kv, hd, neighbours=neighbours)
    q, k, v = c.randn(c.n_rows, 6, hd), c.randn(c.n_rows, 2, hd), c.randn(c.n_rows, 2, hd)
    pos = torch.randint(0, 200_000, (3, c.n_rows), generator=c.g, dtype=torch.int32)
    out = torch.full_like(q, 7.0)
    got_q = c.cache.write(c.batch, k, v, q=q, positions=pos.cuda(), rope=rope, q_out=out)
    assert got_q is out
    n = c.row_start[-1]
    assert (out[n:] == 7.0).all()          # rows behind the last sequence
    want_q = plain(q, pos, 0)
    assert (np.abs(out.double().cpu().numpy() - want_q)[:n] <= turn_tolerance(want_q, hd, neighbours, dtype)[:n]).all()
    # keys: codes of the exact rotation, but where it lies within the rotation's error of a border between two codes
    want_k = plain(k, pos, 1)
    pages, table = c.pages(), c.table.numpy()
    far = 0
    for i, (seq, p) in enumerate(R.places(c.lengths, c.row_start, c.n_rows)[:n]):
        page = R.page_of(pages, table, seq, p, c.page)
        for h in range(2):
            assert np.array_equal(R.get(pages, page, h, p % c.page, 1), deq(R.quantise(v[i, h].float().cpu().numpy())))
            have = R.get(pages, page, h, p % c.page, 0)
            codes, d = R.quantise(want_k[i, h].astype(np.float32))
            same = have == deq((codes, d))
            step = np.repeat(np.abs(d.astype(np.float64)), 32)
            # a group whose scale rounds the other way is off by 8 times the scale's step, a code at a border by one step
            assert (np.abs(have - deq((codes, d)))[~same] <= 1.01 * step[~same] + 8 * step[~same] * 2.0 ** -10).all()
            far += (~same).sum()
    assert far <= 1e-3 * n * 2 * hd


@pytest.mark.parametrize("hd,hk,page,dtype", [(64, 3, 16, FP32), (128, 2, 48, BF16), (256, 1, 64, FP32), (128, 1, 256, BF16)])
def test_read(kv, hd, hk, page, dtype):
    c = Case(kv, 7, [50, 0, 3, 120], [50, 0, 4, 20], hk, hd, page, dtype, pad_rows=3, fill=True)
    outs = [torch.full((c.n_rows, hk, hd), 5.0, dtype=dtype, device="cuda") for _ in range(2)]
    c.cache.read(c.batch, k_out=outs[0], v_out=outs[1])
    for part, out in enumerate(outs):
        for i, at in enumerate(R.places(c.lengths, c.row_start, c.n_rows)):
            for h in range(hk):
                if at is None:
                    assert (out[i, h] == 5).all()
                    continue
                page_no = R.page_of(c.start, c.table.numpy(), *at, c.page)
                want = np.zeros(hd) if page_no is None else R.get(c.start, page_no, h, at[1] % c.page, part)
                assert torch.equal(out[i, h].cpu(), torch.tensor(want).to(dtype)), (i, h, part)


# fp32 calls: products of split operands are short of 2^-17 of a probability times a value, and the sums of a few hundred terms add a
# rounding each at worst; a score is off by a few roundings of its terms' sum, which moves a probability by as much. bf16 calls round a
# probability, a value and the result once, and a key once (with many rows), which moves a score by a rounding of its terms' sum.
# On top, for both: products are summed in fp32 with codes of up to 15 (or both nibbles of a byte, up to 255) less 8 (136) times the
# probability and scale, where an element may be nearly zero. Two products for every 16 tokens and a few joins go into a sum, each leaves
# at most 2^-23 (a truncated fp32 sum) of the largest: 15 / 8, or 255 / (16 * 8) = 2 times the sum of p 8 |scale|.
SUMS = 2 * 2 ** -23


def attend_tolerance(want, spread, reach, span, dtype, tokens):
    sums = SUMS * (2 * (tokens + 15) // 16 + 8) * span
    if dtype is FP32:
        return (2.0 ** -17 + 300 * HALF[FP32] + 2 * 40 * HALF[FP32] * (1 + reach)) * spread + sums + 1e-30
    return HALF[BF16] * np.abs(want) + (2 * HALF[BF16] + 2 * HALF[BF16] * reach) * spread + sums + 1e-30


def check_attend(c, heads, scale=None, q=None):
    q = c.randn(c.n_rows, heads, c.hd) if q is None else q
    out = torch.full_like(q, 9.0)
    c.cache.attend(c.batch, q, scale, out=out)
    want, spread, reach, span = R.attend(q.double().cpu().numpy(), c.start, c.table.numpy(), c.lengths, c.row_start,
                                   c.hd ** -0.5 if scale is None else scale)
    got = out.double().cpu().numpy()
    n = c.row_start[-1]
    assert (got[n:] == 9).all()
    off = np.abs(got[:n] - want[:n])
    tol = attend_tolerance(want, spread, reach, span, c.dtype, max(c.lengths))[:n]
    assert (off <= tol).all(), (off.max(), np.unravel_index((off - tol).argmax(), off.shape))
    # the 2-norm is far below what single elements may be off
    norm = np.linalg.norm(want[:n])
    if norm:
        assert np.linalg.norm(got[:n] - want[:n]) <= (5e-3 if c.dtype is BF16 else 5e-6) * norm
    return out


ATTENDS = [
    # lengths, new rows, query heads, kv heads, head size, page, padded rows
    ([1], [1], 8, 1, 128, 16, 0),
    ([2, 15, 16, 17], [1, 1, 1, 1], 4, 2, 64, 16, 0),
    ([300], [1], 32, 4, 128, 64, 1),
    ([31, 0, 129, 64, 333], [1, 0, 1, 1, 1], 16, 2, 128, 32, 2),
    ([700, 1], [1, 1], 5, 1, 256, 48, 0),
    ([100, 77], [3, 5], 10, 10, 128, 16, 0),
    ([40, 65, 3], [40, 20, 3], 8, 4, 64, 32, 3),
    ([9, 4], [11, 4], 8, 2, 128, 16, 1),               # rows before position 0 see nothing
    ([150, 33], [150, 30], 16, 2, 128, 64, 0),
    ([90], [70], 6, 2, 256, 16, 0),
    ([210, 140], [17, 130], 24, 1, 64, 128, 0),
    ([260], [1], 48, 2, 128, 32, 0),
]


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("lengths,rows,hq,hk,hd,page,pad", ATTENDS)
def test_attend(kv, lengths, rows, hq, hk, hd, page, pad, dtype):
    c = Case(kv, 8, lengths, rows, hk, hd, page, dtype, pad, wide_table=1, fill=True)
    check_attend(c, hq)
    assert c.status.item() == 0


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("lengths,rows,hq,hk,hd,page,pad", [
    ([900, 333, 0, 128], [300, 333, 0, 128], 8, 1, 128, 32, 3),
    ([640], [256], 4, 2, 128, 256, 0),
    ([257, 700], [257, 90], 8, 2, 64, 16, 5),
    ([130, 20], [150, 31], 16, 1, 64, 48, 0),          # more rows than tokens
    ([385], [129], 3, 1, 128, 16, 0),
    # enough columns for the tensor cores
    ([640], [256], 16, 2, 128, 256, 0),
    ([257, 700, 9], [257, 90, 9], 16, 2, 64, 16, 5),
    ([130, 20], [150, 31], 32, 1, 64, 48, 0),
    ([385], [129], 33, 1, 128, 16, 0),
    ([70] * 9, [60] * 9, 8, 1, 128, 16, 1),
])
def test_prompts(kv, lengths, rows, hq, hk, hd, page, pad, dtype):
    c = Case(kv, 21, lengths, rows, hk, hd, page, dtype, pad, wide_table=2, fill=True)
    check_attend(c, hq)
    assert c.status.item() == 0


@pytest.mark.parametrize("hd", [64, 128, 256])
@pytest.mark.parametrize("size,scale", [(1e-38, 1.0), (1e-30, 1e28), (1e30, 1e-31), (1e37, 0.0), (1.0, -0.3), (1e-3, 1e-35), (1e-37, 1e36)])
def test_queries_of_any_size(kv, hd, size, scale):
    """fp32 queries from the smallest to the largest numbers, heads and elements of a head 2^20 apart."""
    c = Case(kv, 26, [333, 40], [2, 1], 2, hd, 16, FP32, 1, fill=True)
    q = c.randn(c.n_rows, 10, hd) * torch.logspace(-6, 0, 10, dtype=torch.float32, device="cuda")[None, :, None]
    q[..., ::7] *= 1e-6
    check_attend(c, 10, scale=scale, q=q * size)


@pytest.mark.parametrize("rows", [2, 200, 300])
@pytest.mark.parametrize("size,scale", [(1e-9, 1e8), (1e18, 1e-19), (1e15, 1e-31), (1e-30, 1e28), (1e36, 1e-37), (1e36, 0.0)])
def test_bf16_queries_and_scales_of_any_size(kv, rows, size, scale):
    c = Case(kv, 27, [333], [rows], 1, 128, 16, BF16, 1, fill=True)
    q = (c.randn(c.n_rows, 16, 128).float() * size).bfloat16()
    check_attend(c, 16, scale=scale, q=q)


@pytest.mark.parametrize("n_seq,most", [(31, 90), (32, 400), (40, 90), (70, 200)])
def test_prompts_of_many_sequences(kv, n_seq, most):
    """Items go by their tokens over up to 32 sequences and by sequence beyond: every row is somebody's, empty sequences and rows before
    position 0 among them."""
    g = torch.Generator().manual_seed(n_seq)
    lengths = torch.randint(0, most, (n_seq,), generator=g).tolist()
    rows = torch.randint(0, 50, (n_seq,), generator=g).tolist()
    lengths[0], rows[0], lengths[1], rows[1], lengths[2], rows[2] = 0, 33, most, 0, most, 47
    c = Case(kv, 25, lengths, rows, 1, 64, 16, BF16, 2, wide_table=1, fill=True)
    check_attend(c, 16)
    assert c.status.item() == 0


@pytest.mark.parametrize("rows,heads", [([1, 1], 4), ([200, 64], 4), ([200, 64], 16)])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_values_and_keys_of_any_size(kv, rows, heads, dtype):
    """Scales of values grow by ten decades along the context, and then fall; keys are large in one stretch, queries tiny and large."""
    c = Case(kv, 22, [900, 400], rows, 1, 128, 16, dtype, fill=True)
    g = torch.Generator().manual_seed(5)
    pages = torch.from_numpy(c.start)
    for seq in range(2):
        for t in range(0, c.lengths[seq], 16):
            block = pages[c.table[seq, t // 16], 0, 0]
            at = t / c.lengths[seq]
            size = 10.0 ** (-6 + 10 * (at / 0.7 if at < 0.7 else (1 - at) / 0.3))
            block[17 * 128:] = ((torch.rand(64, generator=g) + 0.5) * size).half().view(torch.uint8)
            key = 9000.0 if 0.4 < at < 0.5 else 0.1
            block[16 * 128:17 * 128] = ((torch.rand(64, generator=g) - 0.5) * key).half().view(torch.uint8)
    c.start = pages.numpy().copy()
    c.cache.pages.copy_(pages)
    q = c.randn(c.n_rows, heads, 128)
    for size in (1e-6, 1e-20):
        check_attend(c, heads, q=(q * size))
    c.start[:, :, :, 16 * 128:17 * 128] = 0            # keys of 0 and the largest queries
    c.cache.pages.copy_(torch.from_numpy(c.start))
    check_attend(c, heads, q=q * 1e15)


@pytest.mark.parametrize("rows,heads", [([4], 4), ([200], 16)])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_small_values_beside_large_ones_that_a_row_does_not_see(kv, rows, heads, dtype):
    """The last three tokens' values are 2^13 times the others': rows before them hold what the others give, as exactly as without them."""
    c = Case(kv, 24, [325], rows, 1, 128, 16, dtype, fill=True)
    g = torch.Generator().manual_seed(6)
    pages = torch.from_numpy(c.start)
    for t in range(0, 325, 16):
        block = pages[c.table[0, t // 16], 0, 0]
        size = torch.full((16, 4), 0.0625)
        size[max(0, 322 - t):] = 512.0
        block[17 * 128:] = ((torch.rand(16, 4, generator=g) + 0.5) * size).half().view(torch.uint8).flatten()
        block[16 * 128:17 * 128] = ((torch.rand(64, generator=g) - 0.5) * 0.1).half().view(torch.uint8)
    c.start = pages.numpy().copy()
    c.cache.pages.copy_(pages)
    check_attend(c, heads)


@pytest.mark.parametrize("heads", [4, 12])
def test_bad_pages_in_a_prompt(kv, heads):
    c = Case(kv, 23, [600, 300], [200, 300], 1, 64, 16, BF16, fill=True)
    c.table[0, 3], c.table[0, 20], c.table[1, 0], c.table[1, 18] = -1, 10 ** 6, -2, c.start.shape[0]
    c.batch = kv.KVBatch(c.table.cuda(), c.dev_lengths, c.batch._keep[2], n_rows=c.n_rows, max_rows=300)
    check_attend(c, heads)
    assert c.status.item() == 1
    c.status.zero_()
    c.table = c.table[:, :10].contiguous()             # and contexts beyond the table
    c.batch = kv.KVBatch(c.table.cuda(), c.dev_lengths, c.batch._keep[2], n_rows=c.n_rows, max_rows=300)
    check_attend(c, heads)
    assert c.status.item() == 3


@pytest.mark.parametrize("max_rows", [0, 1, 10 ** 6])
@pytest.mark.parametrize("heads", [8, 24])
def test_max_rows_is_a_hint(kv, max_rows, heads):
    c = Case(kv, 24, [150, 33, 90], [150, 1, 30], 2, 128, 16, BF16, fill=True)
    c.batch = kv.KVBatch(c.batch._keep[0], c.dev_lengths, c.batch._keep[2], n_rows=c.n_rows, max_rows=max_rows)
    check_attend(c, heads)


@pytest.mark.parametrize("n_seq", [64, 65, 300, 1024])
@pytest.mark.parametrize("rows", ["one", "ragged"])
def test_many_sequences(kv, n_seq, rows):
    """Sequences are found by a warp for itself up to 64 of them, by the block beyond; some have no rows, some no tokens."""
    g = torch.Generator().manual_seed(n_seq)
    new = [1] * n_seq if rows == "one" else torch.randint(0, 3, (n_seq,), generator=g).tolist()
    lengths = torch.randint(0, 45, (n_seq,), generator=g).tolist()
    lengths[n_seq // 2] = 400
    c = Case(kv, 20, lengths, new, 1, 64, 16, BF16, 2, fill=True)
    check_attend(c, 4)
    assert c.status.item() == 0


def test_one_row_a_sequence_without_row_start(kv):
    c = Case(kv, 9, [20, 0, 57], [1, 1, 1], 2, 128, 16, BF16, fill=True)
    q = c.randn(3, 8, 128)
    want = check_attend(c, 8, q=q)
    batch = kv.KVBatch(c.batch._keep[0], c.dev_lengths)
    assert torch.equal(c.cache.attend(batch, q), want)
    assert (want[1] == 0).all()


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("rows,heads", [([1, 1], 8), ([40, 25], 8), ([260, 100], 16)])
def test_sharp_and_flat_scores(kv, rows, heads, dtype):
    """One token far above the rest, later than many others; and every score alike."""
    c = Case(kv, 10, [260, 100], rows, 1, 128, 32, dtype, fill=True)
    check_attend(c, heads, scale=3.0)
    check_attend(c, heads, scale=0.0)
    check_attend(c, heads, scale=-0.05)


def test_bad_pages_and_lengths(kv):
    c = Case(kv, 11, [100, 60, 80], [1, 1, 1], 2, 128, 16, BF16, fill=True)
    c.table[0, 2], c.table[0, 4], c.table[1, 0] = -1, 10 ** 6, c.start.shape[0]
    c.batch = kv.KVBatch(c.table.cuda(), c.dev_lengths, torch.tensor(c.row_start, dtype=torch.int32, device="cuda"), n_rows=3)
    check_attend(c, 16)
    assert c.status.item() == 1
    # every page of a sequence is bad: nothing to attend to
    c.table[2] = -5
    c.status.zero_()
    c.batch = kv.KVBatch(c.table.cuda(), c.dev_lengths, n_rows=3)
    out = check_attend(c, 16)
    assert (out[2] == 0).all() and c.status.item() == 1
    k, v = c.cache.read(c.batch)
    assert (k[2] == 0).all() and (v[2] == 0).all() and (k[0] != 0).any()
    # a sequence that is longer than its row of the table
    short = c.table[:, :3].contiguous()
    c.status.zero_()
    c.table, c.lengths = short, [100, 60, 30]
    c.batch = kv.KVBatch(short.cuda(), torch.tensor(c.lengths, dtype=torch.int32, device="cuda"), n_rows=3)
    check_attend(c, 16)
    assert c.status.item() & 2
    before = c.pages()
    c.cache.write(c.batch, c.randn(3, 2, 128), c.randn(3, 2, 128))
    assert np.array_equal(c.pages(), before)           # the first two rows are beyond the table, the third one's page is bad


def test_steps_as_a_decoder_takes_them(kv):
    """A prompt goes in, then tokens one by one: write, attend, against the oracle fed with the same rows."""
    hk, hq, hd, page, steps = 2, 8, 128, 16, 6
    rope, plain = rope_of(kv, hd)
    g = torch.Generator().manual_seed(12)
    prompt = [19, 5, 32]
    table = torch.randperm(12, generator=g).to(torch.int32).reshape(3, 4)
    cache = kv.KVCache.empty(12, page, hk, hd)
    lengths = torch.tensor(prompt, dtype=torch.int32, device="cuda")
    start = torch.tensor([0, 19, 24, 56], dtype=torch.int32, device="cuda")
    for step in range(steps):
        rows = prompt if step == 0 else [1, 1, 1]
        n = sum(rows)
        batch = kv.KVBatch(table.cuda(), lengths, start if step == 0 else None, n_rows=n, max_rows=max(rows))
        qkv = torch.randn(n, (hq + 2 * hk) * hd, generator=g).cuda()
        q, k, v = (x.unflatten(1, (-1, hd)) for x in qkv.split((hq * hd, hk * hd, hk * hd), dim=1))
        pos = torch.randint(0, 500, (3, n), generator=g, dtype=torch.int32)
        turned = cache.write(batch, k, v, q=q, positions=pos.cuda(), rope=rope)
        out = cache.attend(batch, turned)
        edges = np.cumsum([0] + rows)
        want, spread, reach, span = R.attend(plain(q, pos, 0), cache.pages.cpu().numpy(), table.numpy(), lengths.tolist(), edges, hd ** -0.5)
        assert (np.abs(out.double().cpu().numpy() - want) <= attend_tolerance(want, spread, reach, span, FP32, 64)).all(), step
        lengths += 1


def test_captured_calls_follow_the_lengths(kv):
    """One graph of write and attend serves every step: lengths, positions and rows change in their buffers. A call on another stream and
    eager calls of the same cache in between leave it as it is."""
    hk, hq, hd = 2, 16, 128
    rope, _ = rope_of(kv, hd)
    g = torch.Generator().manual_seed(13)
    table = torch.arange(24, dtype=torch.int32, device="cuda").reshape(2, 12)
    lengths = torch.tensor([3, 100], dtype=torch.int32, device="cuda")
    qkv = torch.zeros(2, (hq + 2 * hk) * hd, dtype=BF16, device="cuda")
    pos = torch.zeros(3, 2, dtype=torch.int32, device="cuda")
    pools = [kv.KVCache.empty(24, 16, hk, hd) for _ in range(2)]

    def step(cache):
        q, k, v = (x.unflatten(1, (-1, hd)) for x in qkv.split((hq * hd, hk * hd, hk * hd), dim=1))
        batch = kv.KVBatch(table, lengths)
        return cache.attend(batch, cache.write(batch, k, v, q=q, positions=pos, rope=rope))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(pools[0])
    torch.cuda.current_stream().wait_stream(side)
    pools[0].pages.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(pools[0])
    for i in range(40):
        qkv.copy_(torch.randn(qkv.shape, generator=g))
        pos.copy_(torch.randint(0, 1000, pos.shape, generator=g))
        graph.replay()
        assert torch.equal(out, step(pools[1])), i
        lengths += 1
    assert torch.equal(pools[0].pages, pools[1].pages)


def test_two_streams_at_once(kv):
    c = Case(kv, 14, [900, 40, 2000], [1, 1, 1], 2, 128, 64, BF16, fill=True)
    q = [c.randn(3, 16, 128) for _ in range(2)]
    want = [c.cache.attend(c.batch, x) for x in q]
    streams = [torch.cuda.Stream() for _ in q]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(c.cache.attend(c.batch, q[i]))
    torch.cuda.synchronize()
    assert all(torch.equal(x, want[i]) for i in range(2) for x in got[i])


def test_refusals(kv):
    c = Case(kv, 15, [20, 9], [1, 1], 2, 128, 16, BF16)
    k = c.randn(2, 2, 128)
    rope, _ = rope_of(kv, 128)
    pos = torch.zeros(3, 2, dtype=torch.int32, device="cuda")
    bad = [
        lambda: c.cache.write(c.batch, k[:1], k),
        lambda: c.cache.write(c.batch, k, k.float()),
        lambda: c.cache.write(c.batch, k.half(), k.half()),
        lambda: c.cache.write(c.batch, k.cpu(), k.cpu()),
        lambda: c.cache.write(c.batch, k.transpose(1, 2), k),
        lambda: c.cache.write(c.batch, k, k, q=k),                                  # nothing to turn q by
        lambda: c.cache.write(c.batch, k, k, rope=rope),                            # no positions
        lambda: c.cache.write(c.batch, k, k, rope=rope, positions=pos.long()),
        lambda: c.cache.write(c.batch, k, k, rope=rope, positions=pos[:, :1]),
        lambda: c.cache.attend(c.batch, c.randn(2, 3, 128)),                        # 3 query heads on 2 cache heads
        lambda: c.cache.attend(c.batch, c.randn(2, 4, 64)),
        lambda: c.cache.attend(c.batch, c.randn(3, 4, 128)),
        lambda: c.cache.attend(c.batch, c.randn(2, 4, 130)[..., 2:]),               # not on 16-byte boundaries
        lambda: c.cache.read(c.batch, torch.float16),
        lambda: kv.KVCache(torch.zeros(2, 2, 1, 18 * 96, dtype=torch.uint8, device="cuda")),
        lambda: kv.KVBatch(c.table.cuda(), c.dev_lengths.long()),
        lambda: kv.KVBatch(c.table.cuda(), c.dev_lengths[:1]),
        lambda: kv.rotate_heads(c.randn(2, 2, 64), pos, rope),                      # gammas of 128
    ]
    for i, call in enumerate(bad):
        with pytest.raises((ValueError, RuntimeError)):
            call()
            pytest.fail(f"call {i} was taken")


@pytest.mark.parametrize("rows,heads", [([1, 1], 8), ([300, 270], 16)])
def test_pages_beyond_32_bits(kv, rows, heads):
    """A pool of over 4 GB, sequences in its last pages: written, read, attended as in a small one."""
    small = Case(kv, 25, [300, 270], rows, 2, 128, 64, BF16, fill=True)
    n, need = 61_000, small.start.shape[0]                  # 61000 pages of 2 * 4 * 2304 bytes and some
    pages = torch.empty(n * 4, 2, 4, 18 * 128, dtype=torch.uint8, device="cuda")
    assert pages.numel() > 2 ** 32
    pages[-need:] = small.cache.pages
    table = torch.where(small.table >= 0, small.table + (pages.shape[0] - need), small.table).to(torch.int32).cuda()
    big = kv.KVCache(pages)
    batch = kv.KVBatch(table, small.dev_lengths, small.batch._keep[2], n_rows=small.n_rows, max_rows=max(rows))
    k, v = small.randn(small.n_rows, 2, 128), small.randn(small.n_rows, 2, 128)
    q = small.randn(small.n_rows, heads, 128)
    for cache, b in ((small.cache, small.batch), (big, batch)):
        cache.write(b, k, v)
    assert torch.equal(pages[-need:], small.cache.pages)
    assert all(torch.equal(x, y) for x, y in zip(big.read(batch), small.cache.read(small.batch)))
    assert torch.equal(big.attend(batch, q), small.cache.attend(small.batch, q))


def test_nothing_to_do(kv):
    c = Case(kv, 16, [20], [0], 2, 128, 16, BF16, pad_rows=2, fill=True)
    q = c.randn(2, 4, 128)
    out = torch.full_like(q, 3.0)
    c.cache.attend(c.batch, q, out=out)
    assert (out == 3).all()
    empty = kv.KVBatch(torch.zeros(0, 4, dtype=torch.int32, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda"))
    assert c.cache.attend(empty, q[:0]).shape == (0, 4, 128)
    c.cache.write(empty, c.randn(0, 2, 128), c.randn(0, 2, 128))
    assert np.array_equal(c.pages(), c.start)
