"""The attention block inside decode steps: projections, rotation, the 4-bit cache, attention, against the 64-bit oracle and call by call."""
import numpy as np
import pytest
import torch

import synth
from oracle import ref_cache as R, ref_math as M

pytestmark = pytest.mark.gpu

HK, HD, PAGE = 2, 64, 16


def build(cfg):
    from paper_2607_24787_b200.build import build as b
    from paper_2607_24787_b200.synth_model import build_from_synth
    b()
    return build_from_synth(cfg)


class Block:
    """Weights of the block, and the caches and sequence state of one context."""

    def __init__(self, m, cfg, n_seq, hq=6, seed=0, pages_each=6, hd=HD, gammas=True):
        from paper_2607_24787_b200 import kv_cache as kv
        g = torch.Generator().manual_seed(seed)
        dt = torch.float32 if cfg.dtype == "fp32" else torch.bfloat16
        L, D, self.hq, self.hd = cfg.n_layers, cfg.hidden, hq, hd
        self.w_qkv = (torch.randn(L, (hq + 2 * HK) * hd, D, generator=g) * D ** -0.5).to(dt).cuda()
        self.w_o = (torch.randn(L, D, hq * hd, generator=g) * (hq * hd) ** -0.5).to(dt).cuda()
        self.gamma = (1 + 0.1 * torch.randn(L, D, generator=g)).cuda()
        self.gq, self.gk = ((1 + 0.1 * torch.randn(L * hd, generator=g)).cuda() if gammas else None for _ in range(2))
        self.inv = (1e4 ** (-torch.arange(hd // 2, dtype=torch.float64) / (hd // 2))).float()
        self.axis = torch.arange(hd // 2, dtype=torch.uint8) % 3
        self.rope = kv.Rope(self.inv.cuda(), axis_of=self.axis.cuda(), q_gamma=self.gq, k_gamma=self.gk)
        self.caches = [kv.KVCache.empty(n_seq * pages_each + 1, PAGE, HK, hd) for _ in range(L)]
        self.table = torch.randperm(n_seq * pages_each, generator=g).to(torch.int32).reshape(n_seq, pages_each).cuda()
        self.lengths = torch.randint(0, 20, (n_seq,), generator=g).to(torch.int32).cuda()
        self.positions = torch.zeros(3, n_seq, dtype=torch.int32, device="cuda")
        for c in self.caches:                  # some context before the first step
            c.pages.copy_(torch.randint(0, 256, c.pages.shape, generator=g, dtype=torch.uint8))
            c.pages[..., 16 * hd:] = (torch.rand(*c.pages.shape[:3], hd, generator=g) * 0.4 - 0.2).half().view(torch.uint8).cuda()
        m.set_attention(self.caches, self.table, self.lengths, self.rope, self.positions, self.gamma, self.w_qkv, self.w_o)

    def step(self, g):
        """The caller's part of a step: the new tokens are counted and have positions."""
        self.lengths += 1
        self.positions.copy_(torch.randint(0, 1000, self.positions.shape, generator=g))
        torch.cuda.synchronize()

    def want(self, layer, h, nb):
        """The block's result for rows h from the oracle, with the codes that the GPU left in the cache."""
        f = lambda t: t.double().cpu().numpy()  # noqa: E731
        hd, hq = self.hd, self.hq
        x = h / np.sqrt((h * h).mean(-1, keepdims=True) + 1e-6) * f(self.gamma[layer])
        qkv = x @ f(self.w_qkv[layer]).T
        q, k, v = (qkv[:, a:b].reshape(nb, -1, hd) for a, b in ((0, hq * hd), (hq * hd, (hq + HK) * hd), ((hq + HK) * hd, None)))
        turn = lambda t, gamma: R.rotate(t, self.positions[:, :nb].cpu().numpy(), self.inv.numpy(), self.axis.numpy().astype(int),  # noqa: E731
                                         None if gamma is None else f(gamma[layer * hd:(layer + 1) * hd]))
        pages, lengths = self.caches[layer].pages.cpu().numpy(), self.lengths.tolist()
        for s in range(nb):                    # what is in the cache are the codes of k and v, or next to them
            at = lengths[s] - 1
            for part, rows in ((0, turn(k, self.gk)), (1, v)):
                for head in range(HK):
                    have = R.get(pages, int(self.table[s, at // PAGE]), head, at % PAGE, part)
                    step = np.abs(R.scales(pages, int(self.table[s, at // PAGE]), head, at % PAGE, part))
                    assert (np.abs(have - rows[s, head]) <= 1.01 * step + 1e-6).all()
        out = R.attend(turn(q, self.gq), pages, self.table.cpu().numpy(), lengths[:nb], list(range(nb + 1)), hd ** -0.5)[0]
        return h + out.reshape(nb, -1) @ f(self.w_o[layer]).T


def config(name, nb, slots=8, **kw):
    if name == "tiny":
        return synth.get_config("tiny", batch=nb, slots=2 * slots, **kw)
    d = dict(n_layers=2, hidden=512, n_experts=8, inter=128, top_k=2, slots=slots, budget=1, batch=nb, dtype=name)
    d.update(kw)
    return synth.get_config("qwen3", **d)


@pytest.mark.parametrize("name,nb,hd,gammas", [("tiny", 1, 64, True), ("tiny", 11, 128, False), ("bf16", 1, 64, True), ("bf16", 7, 128, True),
                                               ("bf16", 16, 64, False), ("q4", 30, 64, True), ("bf16", 64, 64, True)])
def test_block(name, nb, hd, gammas):
    cfg = config(name, nb)
    m = build(cfg)
    block = Block(m, cfg, nb, hd=hd, gammas=gammas)
    g = torch.Generator().manual_seed(7)
    for step in range(2):
        block.step(g)
        for layer in range(cfg.n_layers):
            h = torch.randn(nb, cfg.hidden, generator=g).cuda()
            start = h.double().cpu().numpy()
            torch.cuda.synchronize()
            m.attention_block(layer, h)
            m.synchronize()
            want = block.want(layer, start, nb)
            for t in range(nb):
                assert M.rel_linf(h[t].double().cpu().numpy(), want[t]) < 4e-5, (step, layer, t)
    m.close()


@pytest.mark.parametrize("nb", [1, 8, 9, 31, 40])
def test_block_of_many_heads(nb):
    """w_qkv of 2816 rows and w_o of 512: more row tiles than SMs, and fewer."""
    cfg = config("bf16", nb, n_layers=1)
    m = build(cfg)
    block = Block(m, cfg, nb, hq=40, seed=3)
    g = torch.Generator().manual_seed(8)
    block.step(g)
    h = torch.randn(nb, cfg.hidden, generator=g).cuda()
    start = h.double().cpu().numpy()
    torch.cuda.synchronize()
    m.attention_block(0, h)
    m.synchronize()
    want = block.want(0, start, nb)
    for t in range(nb):
        assert M.rel_linf(h[t].double().cpu().numpy(), want[t]) < 4e-5, t
    m.close()


@pytest.mark.parametrize("name,nb", [("tiny", 1), ("bf16", 1), ("bf16", 5), ("q4", 1), ("bf16", 64)])
def test_steps_with_the_block(name, nb):
    """A decode step is the calls one after another; with every expert resident it is the same bits, also when replayed from a graph; and
    without the block the step is what it was."""
    runs = {}
    for kind in ("calls", "offloaded", "resident"):
        cfg = config(name, nb, slots=8 if kind == "resident" else 4)
        m = build(cfg)
        g, outs = torch.Generator().manual_seed(9), []
        plain = torch.randn(nb, cfg.hidden, generator=g).cuda()
        torch.cuda.synchronize()
        if kind == "resident":
            for l in range(cfg.n_layers):
                assert m.prefetch_async(l, list(range(cfg.n_experts))) == cfg.n_experts
            m.synchronize()
        before = m.decode_step(plain)
        m.synchronize()
        block = Block(m, cfg, nb)
        for step in range(6):
            h = torch.randn(nb, cfg.hidden, generator=g).cuda()
            block.step(g)
            if kind == "calls":
                for l in range(cfg.n_layers):
                    m.attention_block(l, h)
                    x, ids, w, _ = m.router_topk(l, h)
                    m.moe_ffn(l, x, ids, w, h)
                out = h
            else:
                out = m.decode_step(h)
            m.synchronize()
            outs.append(out.clone())
        if kind == "resident":
            assert m.stats()["host_free_steps"] > 0
        m.set_attention(None, None, None, None, None, None, None, None)
        after = m.decode_step(plain)
        m.synchronize()                        # (steps run on a stream of their own)
        assert torch.equal(after, before)
        runs[kind] = (outs, [c.pages.clone() for c in block.caches])
        m.close()
    for a, b in zip(runs["offloaded"][0], runs["resident"][0]):
        assert torch.equal(a, b)
    for a, b in zip(runs["offloaded"][1], runs["resident"][1]):
        assert torch.equal(a, b)
    for a, b in zip(runs["calls"][0], runs["offloaded"][0]):
        # (batches round activations to bf16 where the call chain and the step both do: the same kernels)
        assert (a - b).abs().max() <= 1e-5 * b.abs().max()


def test_refusals_of_the_block():
    from paper_2607_24787_b200.binding import SpmError
    cfg = config("bf16", 4)
    m = build(cfg)
    h = torch.randn(4, cfg.hidden).cuda()
    with pytest.raises(SpmError):
        m.attention_block(0, h)                # not set
    block = Block(m, cfg, 3)
    with pytest.raises(SpmError):
        m.attention_block(0, h)                # four rows, three sequences
    with pytest.raises(SpmError):
        m.decode_step(h)
    with pytest.raises(SpmError):
        m.attention_block(2, h[:3])
    with pytest.raises(ValueError):
        m.set_attention(block.caches[:1], block.table, block.lengths, block.rope, block.positions, block.gamma, block.w_qkv, block.w_o)
    with pytest.raises(ValueError):
        m.set_attention(block.caches, block.table, block.lengths, block.rope, block.positions, block.gamma, block.w_qkv.float(), block.w_o)
    with pytest.raises(ValueError):
        m.set_attention(block.caches, block.table, block.lengths, block.rope, block.positions[:, :2], block.gamma, block.w_qkv, block.w_o)
    block.step(torch.Generator().manual_seed(0))
    out = m.decode_step(h[:3])
    m.synchronize()
    assert out.isfinite().all()
    m.close()
