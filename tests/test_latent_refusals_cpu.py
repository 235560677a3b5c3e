"""Calls of the latent cache that are refused ahead of the device (no GPU is needed for that)."""
import ctypes as C

import pytest
import torch

AT = 1 << 20                # an address that is never read


@pytest.fixture(scope="module")
def B():
    from paper_2607_24787_b200 import binding
    from paper_2607_24787_b200.build import build
    build()
    return binding


def cache(B, **kw):
    d = dict(rows=AT, status=None, n_pages=4, page_size=32, latent_dim=512, rope_dim=64)
    d.update(kw)
    return B.LatentRows(**d)


def batch(B, **kw):
    d = dict(page_table=AT, lengths=AT, row_start=AT, n_seq=2, table_stride=2, n_rows=3, max_rows=2)
    d.update(kw)
    return B.KvBatch(**d)


def refused(B, call, code, word):
    with pytest.raises(B.SpmError) as e:
        call()
    assert e.value.code == code and word in str(e.value), str(e.value)


SHAPES = [(dict(latent_dim=500), -2, "latent_dim"), (dict(latent_dim=640), -2, "latent_dim"), (dict(latent_dim=0), -2, "latent_dim"),
          (dict(rope_dim=0), -2, "rope_dim"), (dict(rope_dim=24), -2, "rope_dim"), (dict(rope_dim=80), -2, "rope_dim"),
          (dict(page_size=8), -2, "page_size"), (dict(page_size=24), -2, "page_size"), (dict(page_size=65552), -2, "page_size"),
          (dict(n_pages=-1), -1, "n_pages"), (dict(n_pages=2 ** 26, page_size=32), -2, "tokens")]
POINTERS = [(dict(rows=None), -1, "rows"), (dict(rows=AT + 8), -1, "aligned"), (dict(status=AT + 2), -1, "aligned")]
BATCHES = [(dict(n_seq=-1), "n_seq"), (dict(n_seq=1025), "n_seq"), (dict(n_rows=-1), "negative"), (dict(table_stride=2 ** 26), "tokens"),
           (dict(lengths=None), "null"), (dict(page_table=None), "null"), (dict(lengths=AT + 2), "aligned"), (dict(row_start=None, n_rows=1), "rows")]


def calls(B, kv, b, heads=16, dtype=1, scale=0.1, rows=None, out=None, work=AT, size=1 << 40):
    rows, out = rows or B.Rows(AT, 16 * 576, 576), out or B.Rows(2 * AT, 16 * 576, 576)
    rope = B.Rope(AT, None, None, None, 1, 64, 0, 1e-6)
    return (lambda: B.spm_latent_write(kv, b, rope, AT, 3, rows, out, heads, rows, rows, dtype),
            lambda: B.spm_latent_attend(kv, b, rows, heads, out, scale, dtype, work, size))


@pytest.mark.parametrize("change,code,word", SHAPES + POINTERS)
def test_caches(B, change, code, word):
    for call in calls(B, cache(B, **change), batch(B)):
        refused(B, call, code, word)
    if (change, code, word) in SHAPES:
        refused(B, lambda: B.spm_latent_attend_workspace(cache(B, **change), batch(B), 16, 1), code, word)


@pytest.mark.parametrize("change,word", BATCHES)
def test_batches(B, change, word):
    for call in calls(B, cache(B), batch(B, **change)):
        refused(B, call, -1, word)


def test_nothing_is_no_error(B):
    for b in (batch(B, n_rows=0, n_seq=0), batch(B, n_rows=0), batch(B, n_seq=0)):
        for call in calls(B, cache(B), b):
            call()
    B.spm_head_product(None, None, 0, 0, 0, None, 0, 1, 64, 64, 1)


def test_null_structs(B):
    lib, n = B.load(), C.c_size_t()
    assert lib.spm_latent_attend(None, batch(B), None, 1, None, 1.0, 1, None, 0, None) == -1
    assert lib.spm_latent_attend(cache(B), None, None, 1, None, 1.0, 1, None, 0, None) == -1
    assert lib.spm_latent_write(None, batch(B), None, None, 0, None, None, 0, None, None, 1, None) == -1
    assert lib.spm_latent_attend_workspace(None, batch(B), 1, 1, n) == -1
    assert lib.spm_latent_attend_workspace(cache(B), batch(B), 1, 1, None) == -1


@pytest.mark.parametrize("kw,code,word", [
    (dict(dtype=2), -2, "fp32 or bf16"), (dict(heads=0), -2, "heads"), (dict(heads=1025), -2, "heads"),
    (dict(scale=float("nan")), -1, "scale"), (dict(scale=float("inf")), -1, "scale"), (dict(scale=3e38), -1, "scale"),
    (dict(work=None), -1, "workspace"), (dict(work=AT + 8), -1, "workspace"), (dict(size=1000), -1, "workspace"),
])
def test_attend(B, kw, code, word):
    refused(B, calls(B, cache(B), batch(B), **kw)[1], code, word)


def test_rows(B):
    good, elsewhere = B.Rows(AT, 16 * 576, 576), B.Rows(2 * AT, 16 * 576, 576)
    for bad in (B.Rows(None, 9216, 576), B.Rows(AT + 8, 9216, 576), B.Rows(AT, 9217, 576), B.Rows(AT, 9216, 580)):
        for call in calls(B, cache(B), batch(B), rows=bad) + calls(B, cache(B), batch(B), out=bad):
            refused(B, call, -1, "null" if bad.p is None else "boundaries")
    refused(B, calls(B, cache(B), batch(B), rows=good, out=good)[1], -1, "place")
    refused(B, calls(B, cache(B), batch(B), rows=good, out=B.Rows(AT, 2 * 9216, 576))[0], -1, "place")
    refused(B, calls(B, cache(B), batch(B, n_rows=2 ** 27), heads=16)[1], -1, "n_rows")
    assert elsewhere.p == 2 * AT


def test_write_ropes(B):
    kv, b, rows = cache(B), batch(B), B.Rows(AT, 9216, 576)
    good = (AT, None, None, None, 1, 64, 0, 1e-6)

    def call(rope, q=rows, positions=AT):
        return lambda: B.spm_latent_write(kv, b, rope, positions, 3, q, B.Rows(2 * AT, 9216, 576), 16, rows, rows, 1)
    refused(B, call(None), -1, "without rope")
    refused(B, call(B.Rope(AT, None, AT, None, 1, 64, 0, 1e-6)), -1, "q_gamma")
    refused(B, call(B.Rope(AT, None, None, None, 1, 80, 0, 1e-6)), -2, "rot_dim")
    refused(B, call(B.Rope(AT, None, None, None, 1, 24, 0, 1e-6)), -2, "rot_dim")
    refused(B, call(B.Rope(AT, None, None, None, 5, 64, 0, 1e-6)), -1, "n_axes")
    refused(B, call(B.Rope(AT, None, None, AT + 4, 1, 64, 0, 1e-6)), -1, "aligned")
    refused(B, call(B.Rope(*good), positions=None), -1, "positions")


def expanded(B, kv=None, b=None, heads=16, head=128, n_tokens=100, dtype=1, scale=0.1, q=None, out=None, w_k=None, w_v=None, work=AT, size=1 << 50):
    q, out = q or B.Rows(AT, 16 * 192, 192), out or B.Rows(2 * AT, 16 * 128, 128)
    w_k, w_v = w_k or B.Matrices(AT, 256 * 512, 512), w_v or B.Matrices(AT, 256 * 512, 512)
    return lambda: B.spm_latent_attend_expanded(kv or cache(B), b or batch(B), q, w_k, w_v, heads, head, out, scale, n_tokens, dtype, work, size)


@pytest.mark.parametrize("kw,code,word", [
    (dict(dtype=0), -2, "absorbed"), (dict(dtype=2), -2, "fp32 or bf16"), (dict(heads=0), -2, "heads"), (dict(head=96), -2, "head_dim"), (dict(head=256), -2, "head_dim"),
    (dict(n_tokens=-1), -1, "n_tokens"), (dict(n_tokens=2 ** 30 + 1), -1, "n_tokens"), (dict(scale=float("inf")), -1, "scale"),
    (dict(work=None), -1, "workspace"), (dict(work=AT + 128), -1, "workspace"), (dict(size=1000), -1, "workspace"),
])
def test_expanded(B, kw, code, word):
    refused(B, expanded(B, **kw), code, word)


def test_expanded_structs(B):
    for change, code, word in SHAPES + POINTERS:
        refused(B, expanded(B, kv=cache(B, **change)), code, word)
    for change, word in BATCHES:
        refused(B, expanded(B, b=batch(B, **change)), -1, word)
    for bad in (B.Rows(None, 9216, 576), B.Rows(AT + 8, 9216, 576), B.Rows(AT, 9217, 576)):
        refused(B, expanded(B, q=bad), -1, "null" if bad.p is None else "boundaries")
        refused(B, expanded(B, out=bad), -1, "null" if bad.p is None else "boundaries")
    refused(B, expanded(B, out=B.Rows(AT, 16 * 192, 192)), -1, "place")
    for bad in (B.Matrices(None, 65536, 512), B.Matrices(AT + 8, 65536, 512), B.Matrices(AT, 65540, 512), B.Matrices(AT, 65536, 516), B.Matrices(AT, 65536, 0),
                B.Matrices(AT, -65536, 512)):
        refused(B, expanded(B, w_k=bad), -1, "w_k")
        refused(B, expanded(B, w_v=bad), -1, "w_v")
    expanded(B, b=batch(B, n_rows=0))()
    with pytest.raises(B.SpmError):
        B.spm_latent_attend_expanded_workspace(cache(B), batch(B), 16, 100, 10, 1)
    assert B.spm_latent_attend_expanded_workspace(cache(B), batch(B), 16, 128, 1000, 1) >= 1000 * 16 * 128 * 4


@pytest.mark.parametrize("size,to,code,word", [(0, 64, -2, "in_dim"), (96, 64, -2, "in_dim"), (64, 96, -2, "out_dim"), (64, 8256, -2, "out_dim")])
def test_product_sizes(B, size, to, code, word):
    x, y = B.Rows(AT, 9216, 576), B.Rows(2 * AT, 9216, 576)
    refused(B, lambda: B.spm_head_product(x, AT, 512, 64, 0, y, 3, 16, size, to, 1), code, word)


def test_products(B):
    x, y = B.Rows(AT, 9216, 576), B.Rows(2 * AT, 9216, 576)

    def call(x=x, w=AT, head=65536, row=512, y=y, n=3, heads=16, dtype=1):
        return lambda: B.spm_head_product(x, w, head, row, 0, y, n, heads, 128, 512, dtype)
    refused(B, call(dtype=2), -2, "fp32 or bf16")
    refused(B, call(heads=0), -2, "heads")
    refused(B, call(n=-1), -1, "negative")
    refused(B, call(n=2 ** 31 - 1), -1, "many rows")
    refused(B, call(w=None), -1, "weights")
    refused(B, call(w=AT + 8), -1, "weights")
    refused(B, call(row=516), -1, "weights")
    refused(B, call(head=65540), -1, "weights")
    refused(B, call(y=x), -1, "place")
    refused(B, call(x=B.Rows(AT + 4, 9216, 576)), -1, "boundaries")


def test_tensors_that_are_refused(B):
    from paper_2607_24787_b200 import latent_cache as L
    for pages in (torch.zeros(4, 32, 576, dtype=torch.bfloat16), torch.zeros(4, 32, 576), torch.zeros(4, 576, dtype=torch.bfloat16)):
        with pytest.raises(ValueError, match="pages"):
            L.LatentCache(pages, 512)
    for x, w in ((torch.zeros(3, 2, 64), torch.zeros(2, 64, 64, dtype=torch.bfloat16)),):
        with pytest.raises(ValueError, match="CUDA"):
            L.head_product(x, w)
