"""Decode steps with the attention block: what a refused step leaves as it was, the block's part of the overlap window."""
import pytest
import torch

from oracle import ref_math as M
from test_gpu_attention_block import Block, build, config

pytestmark = pytest.mark.gpu


def resident(m, cfg):
    for l in range(cfg.n_layers):
        assert m.prefetch_async(l, list(range(cfg.n_experts))) == cfg.n_experts
    m.synchronize()


@pytest.mark.parametrize("kind", ["offloaded", "resident"])
def test_a_refused_step_changes_nothing(kind):
    """Four rows for three sequences, before and after steps that are taken: outputs, caches and bookkeeping are as without that call."""
    from paper_2607_24787_b200.binding import SpmError
    runs = []
    for refuse in (False, True):
        cfg = config("bf16", 4, slots=8 if kind == "resident" else 4)
        m = build(cfg)
        if kind == "resident":
            resident(m, cfg)
        block = Block(m, cfg, 3)
        g, outs = torch.Generator().manual_seed(4), []
        wide, host = torch.randn(4, cfg.hidden, generator=g), torch.full((4, cfg.hidden), 5.0).pin_memory()
        wide_in, wide_out = wide.cuda(), torch.full((4, cfg.hidden), 7.0, device="cuda")
        torch.cuda.synchronize()
        for step in range(12):
            h = torch.randn(3, cfg.hidden, generator=g).cuda()
            block.step(g)
            if refuse:
                with pytest.raises(SpmError):
                    m.decode_step(wide_in, wide_out)
                with pytest.raises(SpmError):
                    m.decode_step_host(wide.pin_memory(), host)
                m.synchronize()
                assert (wide_out == 7).all() and (host == 5).all()
            outs.append(m.decode_step(h))
            m.synchronize()
        st = m.stats()
        assert (st["host_free_steps"] == 12) == (kind == "resident")
        runs.append((outs, [c.pages.clone() for c in block.caches], m.events(), st["kernel_launches"], st["steps"]))
        m.close()
    assert runs[0][2:] == runs[1][2:]
    assert all(torch.equal(a, b) for i in range(2) for a, b in zip(runs[0][i], runs[1][i]))


@pytest.mark.parametrize("name,nb,n_seq", [("bf16", 1, 1), ("q4", 16, 16), ("tiny", 4, 3)])
def test_the_window_holds_the_block(name, nb, n_seq):
    """The profiled window of a model with the block is longer by it, and profiling leaves the caches as they are."""
    cfg = config(name, nb)
    m = build(cfg)
    for _ in range(2):                         # (the first profile of a process has kernels to load)
        without = m.profile_window()[0]
    block = Block(m, cfg, n_seq, pages_each=600)
    block.lengths.fill_(9000)
    block.table[-1, 7] = -1                    # (a page outside the pool is nobody's error here)
    torch.cuda.synchronize()
    state = [c.pages.clone() for c in block.caches] + [block.lengths.clone(), block.table.clone(), block.positions.clone()]
    torch.cuda.synchronize()
    W, t, raw = m.profile_window()
    assert raw == M.window_budget(W, t) and m.get_profile() == (W, t, raw)
    h = torch.randn(n_seq, cfg.hidden).cuda()
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    times = []
    now = [c.pages.clone() for c in block.caches] + [block.lengths.clone(), block.table.clone(), block.positions.clone()]
    assert all(torch.equal(a, b) for a, b in zip(state, now))
    block.table[-1, 7] = 0
    torch.cuda.synchronize()
    for i in range(9):
        with torch.cuda.stream(m.compute):
            begin.record()
            m.attention_block(i % cfg.n_layers, h)
            end.record()
        m.compute.synchronize()
        times.append(begin.elapsed_time(end) * 1e3)
    took = sorted(times)[4]
    assert W > without + 0.5 * took, (W, without, took)
    m.set_attention(None, None, None, None, None, None, None, None)
    assert m.profile_window()[0] < W - 0.4 * took
    m.close()


@pytest.mark.parametrize("kind", ["offloaded", "resident", "block"])
@pytest.mark.parametrize("fault,code", [("page", -1), ("length", -1), ("finite", -7), (None, 0)])
def test_what_goes_wrong_in_a_step_is_reported(kind, fault, code):
    """Caches without a status word: the next synchronize says it, once, and the context goes on. With one, it is there."""
    from paper_2607_24787_b200 import binding as B
    bits = dict(page=B.KV_BAD_PAGE, length=B.KV_TOO_LONG, finite=B.KV_NONFINITE)
    cfg = config("bf16", 3, slots=8 if kind == "resident" else 4)
    m = build(cfg)
    if kind == "resident":
        resident(m, cfg)
    block = Block(m, cfg, 3)
    g = torch.Generator().manual_seed(6)
    words = [torch.zeros(1, dtype=torch.int32, device="cuda") for _ in block.caches]

    def one():
        h = torch.randn(3, cfg.hidden, generator=g).cuda()
        block.step(g)
        if kind == "block":
            m.attention_block(1, h)
        else:
            m.decode_step(h)

    def broken(on):
        if fault == "page":
            block.table[1, 0] = 10 ** 6 if on else keep[1, 0]
        elif fault == "length":
            block.lengths[2] = 97 if on else 5
        elif fault == "finite":                # of one value's row of weights: infinite values, finite hidden rows
            block.w_qkv[1, -1] = 3e38 if on else 0.01
        torch.cuda.synchronize()

    keep = block.table.clone()
    block.lengths.clamp_(max=5)
    one()
    m.synchronize()
    for own in (False, True):
        if own:
            for c, w in zip(block.caches, words):
                c.c.status = w.data_ptr()
            m.set_attention(block.caches, block.table, block.lengths, block.rope, block.positions, block.gamma, block.w_qkv, block.w_o)
        for _ in range(2):
            broken(True)
            one()
            if fault and not own:
                with pytest.raises(B.SpmError) as e:
                    m.synchronize()
                assert e.value.code == code and "attention" in str(e.value)
            m.synchronize()
            broken(False)
            one()
            m.synchronize()
    assert words[1].item() == (bits[fault] if fault else 0)
    m.close()


def test_a_step_whose_copies_do_not_land_is_reported():
    from paper_2607_24787_b200 import binding as B
    cfg = config("bf16", 3, slots=4)
    m = build(cfg)
    block = Block(m, cfg, 3)
    g = torch.Generator().manual_seed(7)
    h = torch.randn(3, cfg.hidden, generator=g).cuda()
    block.step(g)
    try:
        B.spm_test_kv_waits(1, 1000)
        m.decode_step(h)
    finally:
        B.spm_test_kv_waits(0, 0)
    with pytest.raises(B.SpmError) as e:
        m.synchronize()
    assert e.value.code == -4
    m.decode_step(h)
    m.synchronize()
    m.close()


def test_addresses_that_a_step_would_refuse():
    """What the calls of a step refuse is refused when the block is set, and what was set before stays."""
    from paper_2607_24787_b200 import binding as B
    cfg = config("bf16", 3)
    m = build(cfg)
    block = Block(m, cfg, 3)
    work = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    caches = (B.KvCache * cfg.n_layers)(*[c.c for c in block.caches])

    def attention(rope_kw={}, **kw):
        r = block.rope.for_axes(3)
        rope = B.Rope(*(rope_kw.get(f, getattr(r, f)) for f, _ in B.Rope._fields_))
        batch = B.KvBatch(block.table.data_ptr(), block.lengths.data_ptr(), None, 3, block.table.shape[1], 3, 1)
        d = dict(caches=caches, batch=batch, rope=rope, positions=block.positions.data_ptr(), pos_stride=3, rms_gamma=block.gamma.data_ptr(),
                 w_qkv=block.w_qkv.data_ptr(), w_o=block.w_o.data_ptr(), n_q_heads=block.hq, scale=0.1, workspace=work.data_ptr(),
                 workspace_bytes=work.numel())
        d.update(kw)
        return B.Attention(**d)

    at = block.positions.data_ptr()
    for bad in (dict(positions=at + 2), dict(positions=None), dict(pos_stride=2), dict(rope_kw=dict(inv_freq=block.inv.data_ptr() + 2)),
                dict(rope_kw=dict(inv_freq=None)), dict(rope_kw=dict(rot_dim=8)), dict(rope_kw=dict(n_axes=5)), dict(rope_kw=dict(q_gamma=at + 4))):
        with pytest.raises(B.SpmError):
            B.spm_set_attention(m.ctx, attention(**bad))
    B.spm_set_attention(m.ctx, attention())
    block.step(torch.Generator().manual_seed(1))
    m.decode_step(torch.randn(3, cfg.hidden).cuda())
    m.synchronize()
    m.close()
