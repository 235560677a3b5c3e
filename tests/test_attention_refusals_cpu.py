"""Tensors that OffloadedMoE.set_attention refuses before it takes an address of any (no context and no GPU are needed for that)."""
from types import SimpleNamespace

import pytest
import torch

L, D, HD, HK, HQ, N = 2, 512, 64, 2, 4, 3


@pytest.fixture(scope="module")
def model():
    from paper_2607_24787_b200 import binding as B
    from paper_2607_24787_b200.build import build
    from paper_2607_24787_b200.model import OffloadedMoE
    build()
    here = torch.device("meta")                # of the context: a device that nothing reads from
    ctx = SimpleNamespace(cfg=B.make_cfg(L, D, 8, 128, 2, 0, 4, B.DTYPE_BF16, max_batch=N), L=L, D=D, device=here, ctx=None)

    def call(**kw):
        on = lambda dt, *shape: torch.empty(*shape, dtype=dt, device=here)  # noqa: E731
        cache = SimpleNamespace(head_dim=HD, kv_heads=HK, device=here, c=B.KvCache(1 << 20, None, 4, 16, HK, HD))
        rope = SimpleNamespace(device=here, gamma_sizes=(None, None), for_axes=lambda n: B.Rope(1 << 20, None, None, None, n, HD, 0, 1e-6))
        d = dict(caches=[cache] * L, page_table=on(torch.int32, N, 4), lengths=on(torch.int32, N), rope=rope, positions=on(torch.int32, 3, N),
                 rms_gamma=on(torch.float32, L, D), w_qkv=on(torch.bfloat16, L, (HQ + 2 * HK) * HD, D), w_o=on(torch.bfloat16, L, D, HQ * HD))
        d.update({k: v(d[k]) for k, v in kw.items()})
        OffloadedMoE.set_attention(ctx, **d)
    return call


def elsewhere(x):
    return SimpleNamespace(**{**vars(x), "device": torch.device("cuda", 7)})


@pytest.mark.parametrize("name,change", [
    ("positions", lambda x: torch.zeros(3, N, dtype=torch.int32)),             # in host memory
    ("positions", lambda x: torch.empty(5, N, dtype=torch.int32, device="meta")),
    ("page_table", lambda x: torch.zeros(N, 4, dtype=torch.int32)),
    ("page_table", lambda x: x[0]),
    ("lengths", lambda x: torch.zeros(N, dtype=torch.int32)),
    ("rms_gamma", lambda x: torch.zeros(L, D)),
    ("w_qkv", lambda x: torch.zeros(x.shape, dtype=x.dtype)),
    ("w_o", lambda x: torch.zeros(x.shape, dtype=x.dtype)),
    ("w_o", lambda x: x[0]),
    ("rope", elsewhere),
    ("caches", lambda x: [x[0], elsewhere(x[1])]),
    ("caches", lambda x: x[:1]),
    ("caches", lambda x: []),
])
def test_tensors_that_are_refused(model, name, change):
    with pytest.raises(ValueError, match=name.rstrip("s")):
        model(**{name: change})


@pytest.mark.parametrize("h", [torch.zeros(N, D), torch.empty(N, D, dtype=torch.bfloat16, device="meta"), torch.empty(N, D - 32, device="meta"),
                               torch.empty(D, device="meta"), torch.empty(N, 2 * D, device="meta")[:, ::2], torch.empty(N, 2 * D, device="meta")[:, :D]])
def test_rows_that_a_block_refuses(h):
    from paper_2607_24787_b200.model import OffloadedMoE
    with pytest.raises(ValueError, match="h_inout"):
        OffloadedMoE.attention_block(SimpleNamespace(D=D, device=torch.device("meta"), ctx=None), 0, h)


def test_limits_that_are_refused():
    from paper_2607_24787_b200 import binding as B
    from paper_2607_24787_b200.build import build
    build()
    for us in (-1, 1, 999):
        with pytest.raises(B.SpmError):
            B.spm_test_kv_waits(0, us)


KV_AT = 1 << 20             # an address that is never read


def kv_structs(B, **kw):
    d = dict(page_table=KV_AT, lengths=KV_AT, row_start=None, n_seq=1, table_stride=2, n_rows=1, max_rows=1)
    d.update(kw)
    return B.KvCache(KV_AT, None, 4, 32, 2, 128), B.KvBatch(**d), B.Rows(KV_AT, 1024, 128)


@pytest.mark.parametrize("scale", [float("nan"), float("inf"), -float("inf"), 1e39])
def test_scales_that_are_refused(scale):
    from paper_2607_24787_b200 import binding as B
    kv, batch, rows = kv_structs(B)
    with pytest.raises(B.SpmError) as e:
        B.spm_kv_attend(kv, batch, rows, 8, rows, scale, B.DTYPE_BF16, KV_AT, 1 << 40)
    assert e.value.code == -1 and "scale" in str(e.value)
    cfg = B.make_cfg(L, D, 8, 128, 2, 0, 4, B.DTYPE_BF16, max_batch=N)
    block = B.Attention((B.KvCache * L)(kv, kv), batch, B.Rope(KV_AT, None, None, None, 1, 128, 0, 1e-6), KV_AT, N, KV_AT, KV_AT, KV_AT, 8, scale, None, 0)
    with pytest.raises(B.SpmError) as e:
        B.spm_attention_workspace(cfg, block)
    assert e.value.code == -1 and "scale" in str(e.value)


def test_tables_whose_tokens_kernels_could_not_count():
    """Tiles of 128 tokens are counted in 32 bits: 2^31 - 4096 tokens a sequence are taken, more are not."""
    from paper_2607_24787_b200 import binding as B
    for stride, ok in ((2 ** 26 - 128, True), (2 ** 26 - 127, False), (2 ** 26 - 1, False)):
        kv, batch, rows = kv_structs(B, table_stride=stride)
        if ok:
            assert B.spm_kv_attend_workspace(kv, batch, 8, B.DTYPE_BF16) > 0
            continue
        with pytest.raises(B.SpmError) as e:
            B.spm_kv_attend_workspace(kv, batch, 8, B.DTYPE_BF16)
        assert e.value.code == -1


def test_results_on_top_of_what_other_rows_still_read():
    """Attention's results in its queries' place, and turned heads in their own place with other strides."""
    from paper_2607_24787_b200 import binding as B
    kv, batch, rows = kv_structs(B)
    other = B.Rows(KV_AT, 2048, 256)
    for out in (rows, other):
        with pytest.raises(B.SpmError) as e:
            B.spm_kv_attend(kv, batch, rows, 8, out, 0.1, B.DTYPE_BF16, KV_AT, 1 << 40)
        assert e.value.code == -1 and "place" in str(e.value)
    rope = B.Rope(KV_AT, None, None, None, 1, 128, 0, 1e-6)
    for call in (lambda: B.spm_rotate_heads(rope, KV_AT, 1, rows, other, 1, 8, 128, B.DTYPE_BF16),
                 lambda: B.spm_kv_write(kv, batch, rope, KV_AT, 1, rows, other, 8, B.Rows(2 * KV_AT, 256, 128), B.Rows(3 * KV_AT, 256, 128), B.DTYPE_BF16)):
        with pytest.raises(B.SpmError) as e:
            call()
        assert e.value.code == -1 and "place" in str(e.value)
