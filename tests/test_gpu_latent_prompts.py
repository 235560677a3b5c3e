"""Attention of prompts over latent rows in the expanded form, on the GPU, against the 64-bit oracle; and both forms together."""
import numpy as np
import pytest
import torch

from oracle import ref_latent as R
from test_gpu_latent_cache import BF16, FP32, HALF, Case, f64, lib, rope_of  # noqa: F401 (lib is a fixture)

pytestmark = pytest.mark.gpu


# Keys' first parts and values are sums of `latent` fp32 products (each addition off by 2^-23 at most, truncated) rounded to fp16 (2^-11); scores
# sums of head + rope; a probability moves by twice what scores are off, and is rounded once; sums of values add once for 16 tokens. Numbers
# below fp16's smallest normal ones are off by 2^-25 where the largest of their 32 tokens are 2^9 (keys, values) and probabilities are up to
# 2^4: 2^-34 of the largest key for each element, 2^-29 of a probability, which is less than the sums' part of them.
FP16 = 2.0 ** -11


def tolerance(want, spread, reach, made, reach_made, latent, width, tokens):
    score = FP16 * reach + (latent * 2.0 ** -23) * reach_made + (width / 16 + 8) * 2.0 ** -23 * (reach + 1)
    probability = 2 * score + FP16 + (tokens / 16 + 40) * 2.0 ** -23
    return (probability + FP16) * spread + latent * 2.0 ** -23 * made + HALF[BF16] * np.abs(want) + 1e-30


def matrices(c, heads, head):
    both = torch.randn(heads, 2 * head, c.latent, generator=c.g).mul(c.latent ** -0.5).to(BF16).cuda()
    return both[:, :head], both[:, head:]


def check(c, heads, head, scale=None, q=None, w=None, n_tokens=None):
    scale = (head + c.rope) ** -0.5 if scale is None else scale
    q = c.randn(c.n_rows, heads, head + c.rope) if q is None else q
    w_k, w_v = matrices(c, heads, head) if w is None else w
    out = torch.full((c.n_rows, heads, head), 9.0, dtype=BF16, device="cuda")
    c.cache.attend_expanded(c.batch, q, w_k, w_v, scale, sum(c.lengths) if n_tokens is None else n_tokens, out=out)
    want, spread, reach, made, reach_made = R.attend(f64(q), f64(c.start), c.table.numpy(), c.lengths, c.row_start, scale, c.latent, f64(w_k), f64(w_v))
    got = f64(out)
    assert (got[c.n:] == 9).all()
    off = np.abs(got[:c.n] - want[:c.n])
    tol = tolerance(want, spread, reach, made, reach_made, c.latent, head + c.rope, max(c.lengths))[:c.n]
    assert (off <= tol).all(), (off.max(), np.unravel_index((off - tol).argmax(), off.shape))
    size = np.linalg.norm(want[:c.n])
    if size:
        assert np.linalg.norm(off) <= 3e-3 * size
    return out


PROMPTS = [
    # lengths, new rows, heads, latent, rope, head, page, padded rows
    ([1], [1], 1, 128, 16, 64, 16, 0),
    ([128], [128], 2, 512, 64, 128, 128, 0),
    ([129, 64], [129, 64], 3, 512, 64, 128, 16, 2),
    ([300, 0, 77], [300, 0, 20], 5, 256, 32, 64, 32, 3),
    ([9, 4], [11, 4], 4, 384, 48, 128, 16, 1),               # rows before position 0 see nothing
    ([700], [260], 2, 512, 64, 64, 64, 0),
    ([257, 256, 255, 400], [257, 1, 255, 129], 2, 256, 64, 128, 48, 0),
    ([513], [513], 16, 128, 32, 128, 256, 0),
]


@pytest.mark.parametrize("lengths,rows,heads,latent,rope,head,page,pad", PROMPTS)
def test_prompts(lib, lengths, rows, heads, latent, rope, head, page, pad):  # noqa: F811
    c = Case(lib, 20, lengths, rows, latent, rope, page, BF16, pad, wide_table=1, fill=True)
    check(c, heads, head)
    assert c.status.item() == 0


def test_many_sequences(lib):  # noqa: F811
    r = np.random.default_rng(3)
    lengths = [int(x) for x in r.integers(0, 60, 70)]
    rows = [int(r.integers(0, n + 1)) for n in lengths]
    c = Case(lib, 21, lengths, rows, 128, 16, 16, BF16, fill=True)
    check(c, 2, 64)


def test_more_blocks_of_rows_than_warps_that_look_for_them(lib):  # noqa: F811
    """As many sequences as a batch has, and 60000 rows of one, most of them before position 0."""
    r = np.random.default_rng(4)
    lengths = [int(x) for x in r.integers(0, 20, 1024)]
    rows = [int(r.integers(0, n + 1)) for n in lengths]
    lengths[900], rows[900] = 700, 60000
    c = Case(lib, 34, lengths, rows, 128, 16, 16, BF16, fill=True)
    check(c, 1, 64)


@pytest.mark.parametrize("size,scale", [(1.0, -0.2), (1.0, 0.0), (30.0, 0.3), (1e-20, 1e18)])
def test_scores_of_any_size(lib, size, scale):  # noqa: F811
    c = Case(lib, 22, [400, 90], [130, 60], 128, 32, 16, BF16, fill=True)
    q = c.randn(c.n_rows, 2, 96, scale=size)
    if size * scale <= 1:
        check(c, 2, 64, scale, q)
        return
    # scores so large that keys' roundings decide: results are of the values' size, and most rows are right
    w = matrices(c, 2, 64)
    out = f64(c.cache.attend_expanded(c.batch, q, *w, scale, 490))
    want, spread, *_ = R.attend(f64(q), f64(c.start), c.table.numpy(), c.lengths, c.row_start, scale, 128, f64(w[0]), f64(w[1]))
    assert np.isfinite(out).all() and np.median(np.abs(out - want) / (spread + 1e-30)) < 0.05


def test_growing_scores_move_the_maximum(lib):  # noqa: F811
    c = Case(lib, 23, [640], [640], 128, 16, 64, BF16, fill=True)
    for t in range(640):
        c.start[c.table[0, t // 64], t % 64, 128] = t // 128 * 80.0
    c.cache.pages.copy_(c.start)
    q = torch.randn(640, 4, 80, generator=c.g).mul(0.1).to(BF16)
    q[..., 64] = torch.tensor([-2.0, 0.0, 1.0, 2.0])
    check(c, 4, 64, 1.0, q.cuda())


@pytest.mark.parametrize("order", ["up", "down", "mixed"])
def test_values_of_any_size(lib, order):  # noqa: F811
    """Tokens' values lie far apart in size, some are zero: the larger ones keep their bits, and all tokens' probabilities count. An error of a
    probability is at most 2^-25 in fp16's smallest steps, where it and its values stand times 2^4 and 2^(10 - largest): 2^-28 of the largest value."""
    c = Case(lib, 32, [640], [640], 128, 16, 64, BF16, fill=True)
    step = torch.arange(640) // 32
    power = {"up": step * 5.0 - 50, "down": 50 - step * 5.0, "mixed": (step * 7 % 20) * 6.0 - 60}[order]
    zero = (step % 7 == 3) | (step % 11 == 0)
    for t in range(640):
        c.start[c.table[0, t // 64], t % 64, :128] *= 0.0 if zero[t] else 2.0 ** power[t].item()
    c.cache.pages.copy_(c.start)
    q, w = torch.randn(640, 2, 80, generator=c.g).to(BF16).cuda(), matrices(c, 2, 64)
    w[0].zero_()                                                  # (keys' first parts would be as far apart)
    got = f64(c.cache.attend_expanded(c.batch, q, *w, 0.25, 640))
    want, spread, reach, made, _ = R.attend(f64(q), f64(c.start), c.table.numpy(), c.lengths, c.row_start, 0.25, 128, f64(w[0]), f64(w[1]))
    largest = np.array([np.abs(f64(c.start)[c.table[0, : -(-(i + 1) // 64)]][..., :128]).max() for i in range(640)])[:, None, None] * 12
    tol = tolerance(want, spread, reach, made, 0 * reach, 128, 80, 640) + 640 * 2.0 ** -28 * largest
    assert (np.abs(got - want) <= tol).all()


@pytest.mark.parametrize("small,large", [(-40, 0), (0, 40), (-30, 30)])
def test_keys_of_any_size(lib, small, large):  # noqa: F811
    """Some tokens' keys are far from fp16's range, in tiles with ordinary ones beside them: scores are of one size by the queries, or zero."""
    c = Case(lib, 33, [500, 130], [500, 30], 128, 32, 16, BF16, fill=True)
    for seq in range(2):
        for t in range(c.lengths[seq]):
            size = [0, small, 0, large, 0, 0, large][t // 32 % 7]
            c.start[c.table[seq, t // 16], t % 16] *= 2.0 ** size
    c.cache.pages.copy_(c.start)
    q, w = c.randn(c.n_rows, 3, 96), matrices(c, 3, 64)
    w[1].mul_(2.0 ** -large if large else 1.0)
    for scale in (0.1 * 2.0 ** -large, 0.0):
        out = f64(c.cache.attend_expanded(c.batch, q, *w, scale, 630))
        want, spread, reach, made, reach_made = R.attend(f64(q), f64(c.start), c.table.numpy(), c.lengths, c.row_start, scale, 128, f64(w[0]), f64(w[1]))
        largest = np.nanmax(np.abs(f64(c.start)[..., :128])) * np.abs(f64(w[1])).sum(-1).max()
        tol = tolerance(want, spread, reach, made, reach_made, 128, 96, 500) + 500 * 2.0 ** -28 * largest
        assert (np.abs(out - want) <= tol)[:c.n].all()


def test_bad_queries_stay_by_themselves(lib):  # noqa: F811
    c = Case(lib, 24, [200, 0, 70], [150, 1, 3], 256, 32, 16, BF16, fill=True)
    w = matrices(c, 3, 64)
    q = c.randn(c.n_rows, 3, 96)
    good = c.cache.attend_expanded(c.batch, q, *w, 0.1, 270)
    q[0, 2, 7], q[140, 1, 80], q[151, 0], q[150, 1] = float("nan"), float("inf"), -float("inf"), float("nan")
    out = c.cache.attend_expanded(c.batch, q, *w, 0.1, 270)
    for row, head in ((0, 2), (140, 1), (151, 0)):
        assert out[row, head].isnan().all()
        out[row, head] = good[row, head]
    assert torch.equal(out, good) and (good[150] == 0).all()     # (a row that sees nothing stays zero)


@pytest.mark.parametrize("what", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("whole", [True, False])
def test_bad_tokens_reach_only_rows_that_see_them(lib, what, whole):  # noqa: F811
    c = Case(lib, 25, [200, 130], [60, 1], 256, 32, 16, BF16, fill=True)
    w = matrices(c, 3, 64)
    q = c.randn(c.n_rows, 3, 96)
    good = c.cache.attend_expanded(c.batch, q, *w, 0.1, 330)
    row = c.cache.pages[c.table[0, 170 // 16], 170 % 16]          # row 30 of sequence 0 is the first to see it
    if whole:
        row.fill_(what)
    else:
        row[17] = what
    out = c.cache.attend_expanded(c.batch, q, *w, 0.1, 330)
    assert out[30:60].isnan().all()
    assert torch.equal(out[:30], good[:30]) and torch.equal(out[60], good[60])


def test_a_bad_token_at_any_place_of_a_tile(lib):  # noqa: F811
    """Token i of sequence i, whose rows all see the whole tile that it is in."""
    c = Case(lib, 33, [200] * 33, [40] * 33, 128, 16, 16, BF16, fill=True)
    w = matrices(c, 2, 64)
    q = c.randn(c.n_rows, 2, 80)
    good = c.cache.attend_expanded(c.batch, q, *w, 0.1, 200 * 33)
    for i in range(32):
        c.cache.pages[c.table[i, i // 16], i % 16] = float("nan")
    out = c.cache.attend_expanded(c.batch, q, *w, 0.1, 200 * 33)
    assert out[:32 * 40].isnan().all() and torch.equal(out[32 * 40:], good[32 * 40:])


def test_pages_that_are_not_there(lib):  # noqa: F811
    from paper_2607_24787_b200 import binding as B
    c = Case(lib, 26, [200, 90, 64], [30, 90, 9], 128, 16, 16, BF16, fill=True)
    for s, p, to in ((0, 3, -1), (0, 12, 10 ** 6), (1, 0, -5), (2, 0, 99), (2, 1, 99), (2, 2, 99), (2, 3, 99)):
        c.table[s, p] = to
    c.dev_table.copy_(c.table)
    check(c, 2, 64)                                               # (the last sequence sees nothing)
    assert c.status.item() == B.KV_BAD_PAGE
    c.status.zero_()
    c.dev_lengths[1] = 10 ** 6
    c.cache.attend_expanded(c.batch, c.randn(c.n_rows, 2, 80), *matrices(c, 2, 64), 0.1, 400)
    assert c.status.item() & B.KV_TOO_LONG


def test_room_for_fewer_tokens_than_there_are(lib):  # noqa: F811
    """Tokens beyond n_tokens (rounded up by sequence) do not exist, and a status bit says so; the rows before are right."""
    from paper_2607_24787_b200 import binding as B
    c = Case(lib, 27, [300, 500], [300, 500], 128, 16, 16, BF16, fill=True)
    w = matrices(c, 2, 64)
    q = c.randn(c.n_rows, 2, 80)
    good = c.cache.attend_expanded(c.batch, q, *w, 0.1, 800)
    assert c.status.item() == 0
    out = c.cache.attend_expanded(c.batch, q, *w, 0.1, 400)
    assert c.status.item() == B.KV_TOO_LONG
    room = (400 + 2 * 127) // 128 * 128 - 384                     # of the second sequence, behind the first one's three tiles
    assert torch.equal(out[:300 + room], good[:300 + room]) and out.isfinite().all() and not torch.equal(out, good)
    assert torch.equal(c.cache.attend_expanded(c.batch, q, *w, 0.1, 5000), good)


def test_strided_rows_and_rounds_of_heads(lib, monkeypatch):  # noqa: F811
    c = Case(lib, 28, [150, 60], [150, 10], 256, 32, 32, BF16, fill=True)
    wide = c.randn(c.n_rows, 8, 200)
    q = wide[:, 1:6, 16:176]
    w = matrices(c, 5, 128)
    want = c.cache.attend_expanded(c.batch, q.contiguous(), w[0].contiguous(), w[1].contiguous(), 0.07, 210)
    assert torch.equal(c.cache.attend_expanded(c.batch, q, *w, 0.07, 210), want)
    first = c.randn(8, c.n_rows, 128)
    c.cache.attend_expanded(c.batch, q, *w, 0.07, 210, out=first.transpose(0, 1)[:, 2:7])
    assert torch.equal(first.transpose(0, 1)[:, 2:7], want)
    # so much room that a head by itself takes what several do not: one round a head
    big = 1_100_000
    from paper_2607_24787_b200 import binding as B
    assert B.spm_latent_attend_expanded_workspace(c.cache.c, c.batch.c, 5, 128, big, B.DTYPE_BF16) < 2 * big * 128 * 4
    assert torch.equal(c.cache.attend_expanded(c.batch, q, *w, 0.07, big), want)


def test_prompt_then_steps(lib):  # noqa: F811
    """A layer as a program runs it: a prompt in the expanded form, drafts and single tokens in the absorbed one, against one attention over all of it
    in 64 bits, from the rows as the cache holds them; and a captured prompt, replayed."""
    heads, head, latent, rope, page = 4, 128, 512, 64, 16
    scale = (head + rope) ** -0.5
    c = Case(lib, 29, [200, 90], [200, 90], latent, rope, page, BF16, wide_table=2, fill=True)
    pool = iter(range(c.start.shape[0] - 2, c.start.shape[0]))
    for s, n in enumerate((200, 90)):                             # pages that later tokens need
        c.table[s, -(-n // page)] = next(pool)
    c.dev_table.copy_(c.table)
    w_k, w_v = matrices(c, heads, head)
    turn, inv, axis, gamma = rope_of(lib, c, neighbours=True)
    kv = lib.kv

    def run(lengths, rows):
        start = [0, rows[0], sum(rows)]
        batch = kv.KVBatch(c.dev_table, torch.tensor(lengths, dtype=torch.int32, device="cuda"), torch.tensor(start, dtype=torch.int32, device="cuda"),
                           n_rows=start[-1], max_rows=max(rows))
        x, q = c.randn(start[-1], latent + rope), c.randn(start[-1], heads, head + rope)
        pos = torch.cat([torch.arange(n - r, n) for n, r in zip(lengths, rows)]).int().cuda()
        turned = R.turn(f64(q[..., head:]), pos[None].cpu().numpy(), inv, axis, True)
        if max(rows) > 16:
            c.cache.write(batch, x[:, :latent], x[:, latent:], q=q[..., head:], positions=pos, rope=turn, q_out=q[..., head:])
            out = c.cache.attend_expanded(batch, q, w_k, w_v, scale, sum(lengths))
        else:
            full = torch.empty(start[-1], heads, latent + rope, dtype=BF16, device="cuda")
            lib.head_product(q[..., :head], w_k, out=full[..., :latent])
            c.cache.write(batch, x[:, :latent], x[:, latent:], q=q[..., head:], positions=pos, rope=turn, q_out=full[..., latent:])
            out = lib.head_product(c.cache.attend(batch, full, scale), w_v, transposed=True)
        q64 = np.concatenate((f64(q[..., :head]), turned), -1)
        want = R.attend(q64, f64(c.cache.pages), c.table.numpy(), lengths, start, scale, latent, f64(w_k), f64(w_v))[0]
        # queries (twice in the absorbed form), keys or sums, probabilities and results are rounded to bf16: a few of 2^-9 in the mean
        assert np.linalg.norm(f64(out) - want) <= 1e-2 * np.linalg.norm(want)
        return batch, q, out

    batch, q, out = run([200, 90], [200, 90])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        again = c.cache.attend_expanded(batch, q, w_k, w_v, scale, 290)
    run([204, 93], [4, 3])
    run([205, 94], [1, 1])
    again.zero_()
    graph.replay()
    assert torch.equal(again, out)                                # (the prompt's rows are as they were)
    assert c.status.item() == 0


def test_waits_that_run_out(lib):  # noqa: F811
    """Copies that never count as landed: the calls end with the status bit, and the next one is right."""
    from paper_2607_24787_b200 import binding as B
    c = Case(lib, 30, [300, 90], [300, 20], 512, 64, 16, BF16, fill=True)
    q, w = c.randn(c.n_rows, 3, 192), matrices(c, 3, 128)
    want = c.cache.attend_expanded(c.batch, q, *w, 0.1, 390)
    B.spm_test_kv_waits(1, 3000)
    try:
        c.cache.attend_expanded(c.batch, q, *w, 0.1, 390)
        torch.cuda.synchronize()
        assert c.status.item() & B.KV_TIMEOUT
    finally:
        B.spm_test_kv_waits(0, 0)
    c.status.zero_()
    assert torch.equal(c.cache.attend_expanded(c.batch, q, *w, 0.1, 390), want)
    assert c.status.item() == 0


def test_fp32_rows_are_refused(lib):  # noqa: F811
    from paper_2607_24787_b200 import binding as B
    c = Case(lib, 31, [20], [20], 128, 16, 16, FP32, fill=True)
    with pytest.raises(B.SpmError, match="absorbed"):
        c.cache.attend_expanded(c.batch, c.randn(20, 2, 80), *matrices(c, 2, 64), 0.1, 20)
