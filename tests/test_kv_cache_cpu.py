"""Refusals of the attention block's entry points (nothing is enqueued, so no GPU is needed) and pins of its oracle."""
import numpy as np
import pytest

from oracle import ref_cache as R

SPM_FP32, SPM_BF16, SPM_Q4 = 0, 1, 2
AT = 1 << 20                # an address that is never read


@pytest.fixture(scope="module")
def B():
    from paper_2607_24787_b200 import binding
    from paper_2607_24787_b200.build import build
    build()
    return binding


def cache(B, **kw):
    d = dict(pages=AT, status=None, n_pages=4, page_size=32, n_kv_heads=2, head_dim=128)
    d.update(kw)
    return B.KvCache(**d)


def batch(B, **kw):
    d = dict(page_table=AT, lengths=AT, row_start=AT, n_seq=3, table_stride=2, n_rows=5, max_rows=2)
    d.update(kw)
    return B.KvBatch(**d)


def rope(B, **kw):
    d = dict(inv_freq=AT, axis_of=AT, q_gamma=None, k_gamma=None, n_axes=3, rot_dim=128, neighbours=0, eps=1e-6)
    d.update(kw)
    return B.Rope(**d)


def rows(B, p=AT, row=1024, head=128):
    return B.Rows(p, row, head)


def refused(B, code, call):
    with pytest.raises(B.SpmError) as e:
        call()
    assert e.value.code == code and len(str(e.value)) > 20


INVALID, CONFIG = -1, -2


@pytest.mark.parametrize("kw,code", [
    (dict(pages=None), INVALID), (dict(pages=AT + 8), INVALID), (dict(status=AT + 2), INVALID), (dict(n_pages=-1), INVALID),
    (dict(page_size=0), CONFIG), (dict(page_size=24), CONFIG), (dict(page_size=1 << 17), CONFIG), (dict(n_kv_heads=0), CONFIG),
    (dict(head_dim=96), CONFIG), (dict(head_dim=0), CONFIG)])
def test_caches_that_are_refused(B, kw, code):
    kv, b, r = cache(B, **kw), batch(B), rows(B)
    refused(B, code, lambda: B.spm_kv_read(kv, b, r, r, SPM_BF16))
    refused(B, code, lambda: B.spm_kv_write(kv, b, None, None, 0, None, None, 0, r, r, SPM_BF16))
    refused(B, code, lambda: B.spm_kv_attend(kv, b, r, 8, r, 1.0, SPM_BF16, AT, 1 << 40))


@pytest.mark.parametrize("kw", [
    dict(n_seq=-1), dict(n_seq=1025), dict(n_rows=-1), dict(max_rows=-1), dict(table_stride=-1), dict(table_stride=1 << 26),
    dict(lengths=None), dict(page_table=None), dict(row_start=AT + 1), dict(page_table=AT + 2), dict(row_start=None, n_rows=2)])
def test_batches_that_are_refused(B, kw):
    kv, b, r = cache(B), batch(B, **kw), rows(B)
    refused(B, INVALID, lambda: B.spm_kv_read(kv, b, r, r, SPM_BF16))
    refused(B, INVALID, lambda: B.spm_kv_write(kv, b, None, None, 0, None, None, 0, r, r, SPM_BF16))
    refused(B, INVALID, lambda: B.spm_kv_attend(kv, b, r, 8, r, 1.0, SPM_BF16, AT, 1 << 40))
    refused(B, INVALID, lambda: B.spm_kv_attend_workspace(kv, b, 8, SPM_BF16))


@pytest.mark.parametrize("bad", [dict(p=None), dict(p=AT + 4), dict(row=1028), dict(head=130)])
def test_rows_that_are_refused(B, bad):
    kv, b, r, x = cache(B), batch(B), rows(B), rows(B, **bad)
    refused(B, INVALID, lambda: B.spm_kv_read(kv, b, x, r, SPM_BF16))
    refused(B, INVALID, lambda: B.spm_kv_read(kv, b, r, x, SPM_BF16))
    refused(B, INVALID, lambda: B.spm_kv_write(kv, b, None, None, 0, None, None, 0, x, r, SPM_BF16))
    refused(B, INVALID, lambda: B.spm_kv_write(kv, b, None, None, 0, None, None, 0, r, x, SPM_BF16))
    refused(B, INVALID, lambda: B.spm_kv_write(kv, b, rope(B), AT, 5, x, r, 8, r, r, SPM_BF16))
    refused(B, INVALID, lambda: B.spm_kv_write(kv, b, rope(B), AT, 5, r, x, 8, r, r, SPM_BF16))
    refused(B, INVALID, lambda: B.spm_kv_attend(kv, b, x, 8, r, 1.0, SPM_BF16, AT, 1 << 40))
    refused(B, INVALID, lambda: B.spm_kv_attend(kv, b, r, 8, x, 1.0, SPM_BF16, AT, 1 << 40))
    refused(B, INVALID, lambda: B.spm_rotate_heads(rope(B), AT, 5, x, r, 5, 8, 128, SPM_BF16))
    refused(B, INVALID, lambda: B.spm_rotate_heads(rope(B), AT, 5, r, x, 5, 8, 128, SPM_BF16))


@pytest.mark.parametrize("kw,code", [
    (dict(rot_dim=-8), CONFIG), (dict(rot_dim=136), CONFIG), (dict(rot_dim=4), CONFIG), (dict(n_axes=0), INVALID), (dict(n_axes=5), INVALID),
    (dict(inv_freq=None), INVALID), (dict(inv_freq=AT + 2), INVALID), (dict(q_gamma=AT + 4), INVALID), (dict(k_gamma=AT + 8), INVALID)])
def test_ropes_that_are_refused(B, kw, code):
    r, x = rope(B, **kw), rows(B)
    refused(B, code, lambda: B.spm_rotate_heads(r, AT, 5, x, x, 5, 8, 128, SPM_BF16))
    refused(B, code, lambda: B.spm_kv_write(cache(B), batch(B), r, AT, 5, None, None, 0, x, x, SPM_BF16))


def test_calls_that_are_refused(B):
    kv, b, r, x = cache(B), batch(B), rope(B), rows(B)
    for dtype in (SPM_Q4, 7, -1):
        refused(B, CONFIG, lambda: B.spm_kv_read(kv, b, x, x, dtype))
        refused(B, CONFIG, lambda: B.spm_kv_write(kv, b, None, None, 0, None, None, 0, x, x, dtype))
        refused(B, CONFIG, lambda: B.spm_kv_attend(kv, b, x, 8, x, 1.0, dtype, AT, 1 << 40))
        refused(B, CONFIG, lambda: B.spm_rotate_heads(r, AT, 5, x, x, 5, 8, 128, dtype))
        refused(B, CONFIG, lambda: B.spm_kv_attend_workspace(kv, b, 8, dtype))
    refused(B, INVALID, lambda: B.spm_rotate_heads(r, None, 5, x, x, 5, 8, 128, SPM_BF16))          # no positions
    refused(B, INVALID, lambda: B.spm_rotate_heads(r, AT, 4, x, x, 5, 8, 128, SPM_BF16))            # axes closer than the rows
    refused(B, INVALID, lambda: B.spm_rotate_heads(None, AT, 5, x, x, 5, 8, 128, SPM_BF16))
    refused(B, INVALID, lambda: B.spm_rotate_heads(r, AT, 5, x, x, -1, 8, 128, SPM_BF16))
    refused(B, INVALID, lambda: B.spm_rotate_heads(r, AT, 5, x, x, 5, -8, 128, SPM_BF16))
    refused(B, CONFIG, lambda: B.spm_rotate_heads(r, AT, 5, x, x, 5, 8, 80, SPM_BF16))
    refused(B, INVALID, lambda: B.spm_kv_write(kv, b, None, None, 0, x, x, 8, x, x, SPM_BF16))      # q, but nothing to turn it by
    refused(B, INVALID, lambda: B.spm_kv_write(kv, b, r, AT, 5, x, None, 8, x, x, SPM_BF16))
    refused(B, INVALID, lambda: B.spm_kv_read(kv, b, None, None, SPM_BF16))
    refused(B, INVALID, lambda: B.spm_kv_read(kv, None, x, x, SPM_BF16))
    need = B.spm_kv_attend_workspace(kv, b, 8, SPM_BF16)
    for at, size in ((None, need), (AT + 8, need), (AT, need - 1), (AT, 0)):
        refused(B, INVALID, lambda: B.spm_kv_attend(kv, b, x, 8, x, 1.0, SPM_BF16, at, size))
    refused(B, INVALID, lambda: B.spm_kv_attend(kv, batch(B, n_rows=1 << 28), x, 16, x, 1.0, SPM_BF16, AT, 1 << 40))      # 2^32 columns
    for heads in (0, -2, 3):
        refused(B, CONFIG, lambda: B.spm_kv_attend(kv, b, x, heads, x, 1.0, SPM_BF16, AT, 1 << 40))
        refused(B, CONFIG, lambda: B.spm_kv_attend_workspace(kv, b, heads, SPM_BF16))


def test_nothing_to_do_needs_no_gpu(B):
    kv, x = cache(B), rows(B)
    for b in (batch(B, n_rows=0, row_start=AT), batch(B, n_seq=0)):
        B.spm_kv_read(kv, b, x, x, SPM_BF16)
        B.spm_kv_write(kv, b, rope(B), AT, 5, x, x, 8, x, x, SPM_FP32)
        B.spm_kv_attend(kv, b, x, 8, x, 1.0, SPM_BF16, AT, 1 << 40)
    B.spm_rotate_heads(rope(B), AT, 0, x, x, 0, 8, 128, SPM_BF16)


def test_cache_bytes(B):
    assert B.spm_kv_cache_bytes(cache(B, pages=None)) == 4 * 2 * 2 * 18 * 128
    assert B.spm_kv_cache_bytes(cache(B, n_pages=1 << 20, page_size=256, n_kv_heads=8)) == (1 << 20) * 8 * 16 * 2304


# ---- the oracle ---------------------------------------------------------------
def test_codes_are_nearest():
    rng = np.random.default_rng(0)
    x = (rng.standard_normal((50, 128)) * 10.0 ** rng.integers(-3, 3, (50, 1))).astype(np.float32)
    codes, d = R.quantise(x)
    step = np.repeat(d.astype(np.float64), 32, axis=1)
    value = (codes.astype(np.float64) - 8) * step
    grid = (np.arange(16)[:, None, None] - 8) * step
    best = np.abs(grid - x).min(0)
    assert (np.abs(value - x) <= best + 1e-5 * np.abs(step)).all()
    top = np.abs(x.reshape(50, 4, 32)).argmax(-1)
    assert (np.take_along_axis(codes.reshape(50, 4, 32), top[..., None], -1) == 0).all()      # the largest takes the far end


def test_rows_come_back():
    rng = np.random.default_rng(1)
    pages = np.zeros((3, 2, 2, 18 * 64), np.uint8)
    want = {}
    for page, head, at, part in [(0, 0, 0, 0), (0, 0, 0, 1), (2, 1, 31, 0), (2, 1, 30, 1), (1, 0, 16, 0)]:
        codes, d = rng.integers(0, 16, 64).astype(np.uint8), rng.standard_normal(2).astype(np.float16)
        R.put(pages, page, head, at, part, codes, d)
        want[page, head, at, part] = (codes.astype(float) - 8) * np.repeat(d.astype(float), 32)
    for key, w in want.items():
        assert np.array_equal(R.get(pages, *key), w)
    assert np.count_nonzero(pages) <= 5 * (32 + 4)


def test_rotation_keeps_distances():
    rng = np.random.default_rng(2)
    inv, axis = 1e4 ** (-np.arange(32) / 32), np.arange(32) % 3
    q, k = rng.standard_normal((1, 1, 64)), rng.standard_normal((1, 1, 64))
    for neighbours in (False, True):
        def dot(p, r):
            a = R.rotate(q, np.array(p)[:, None], inv, axis, neighbours=neighbours)
            b = R.rotate(k, np.array(r)[:, None], inv, axis, neighbours=neighbours)
            return (a * b).sum()
        assert abs(dot((5, 7, 9), (2, 3, 4)) - dot((105, 57, 10), (102, 53, 5))) < 1e-9     # only the axes' differences count
        assert np.isclose((R.rotate(q, np.array([[3], [4], [5]]), inv, axis, neighbours=neighbours) ** 2).sum(), (q ** 2).sum())


# ---- the block of a decode step -------------------------------------------------
def test_attention_blocks_that_are_refused(B):
    cfg = B.make_cfg(2, 512, 8, 128, 2, 0, 4, B.DTYPE_BF16, max_batch=4)

    def block(kv=None, n=2, **kw):
        caches = (B.KvCache * n)(*[kv or cache(B)] * n)
        d = dict(caches=caches, batch=batch(B, row_start=None, n_seq=4, n_rows=4), rope=rope(B), positions=AT, pos_stride=4, rms_gamma=AT, w_qkv=AT,
                 w_o=AT, n_q_heads=8, scale=0.1, workspace=AT, workspace_bytes=1 << 40)
        d.update(kw)
        return B.Attention(**d)

    nb, hd = 4, 128
    least = 8 * 1024 * 6 + nb * (8 + 4) * hd * 4 + nb * 8 * hd * 4
    assert B.spm_attention_workspace(cfg, block()) >= least
    refused(B, INVALID, lambda: B.spm_attention_workspace(cfg, block(caches=None)))
    refused(B, CONFIG, lambda: B.spm_attention_workspace(cfg, block(n_q_heads=0)))
    refused(B, CONFIG, lambda: B.spm_attention_workspace(cfg, block(n_q_heads=3)))
    refused(B, INVALID, lambda: B.spm_attention_workspace(cfg, block(batch=batch(B, n_seq=0))))
    refused(B, INVALID, lambda: B.spm_attention_workspace(cfg, block(batch=batch(B, lengths=None))))
    refused(B, INVALID, lambda: B.spm_attention_workspace(cfg, block(kv=cache(B, pages=AT + 8))))
    refused(B, CONFIG, lambda: B.spm_attention_workspace(cfg, block(kv=cache(B, head_dim=96))))
    mixed = (B.KvCache * 2)(cache(B), cache(B, page_size=16))
    refused(B, CONFIG, lambda: B.spm_attention_workspace(cfg, block(caches=mixed)))
    refused(B, CONFIG, lambda: B.spm_attention_workspace(B.make_cfg(2, 500, 8, 128, 2, 0, 4, B.DTYPE_BF16, max_batch=4), block()))
