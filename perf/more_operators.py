"""Attention with keys and values from one latent vector a token, which all heads share.

A token's row in the cache is [latent | rope]: `latent` elements that were normed as they went in, and a key of `rope` elements,
turned by the token's position. Rows are bf16 in pages [pages, page_size, latent + rope]. A head has two matrices: w_k [head, latent]
makes its key's first part from the latent vector, w_v [head, latent] its value:

    key = [w_k c | r],  value = w_v c,  out = sum of softmax(scale q . key) value.

The absorbed form never makes them: q' = [q w_k | q_rope] meets the cache's rows as they are, o' = sum of p c, out = o' w_v^T (two
products a head around the attention). The expanded form makes them for a prompt's whole context. Row i of a sequence's `n` new rows
stands at position length - n + i and sees the positions up to its own.

With `own` false, `run` computes all of this from elementary tensor operations; with `own` true it calls the library.
"""
from __future__ import annotations

import math
import random

import torch

own = False

MODES = ("write", "product", "attend", "attend", "expanded")
EPS = 1e-6
# (heads, latent, rope, head): few and many heads over a wide latent vector, odd numbers of heads over narrow ones
HEADS = ((16, 512, 64, 128), (128, 512, 64, 128), (10, 256, 32, 64), (20, 384, 48, 128), (33, 128, 64, 64))


def _case(name, mode, heads, dtype, page=64, seqs=1, rows=1, length=1, lens=0, flag=True):
    """rows: most new rows of a sequence; length: tokens of its longest sequence; lens: seed of the others' (0: all alike).
    flag: write: pairs are neighbours; product: with w_v's transpose, not with w_k."""
    c = dict(mode=mode, heads=heads[0], latent=heads[1], rope=heads[2], head=heads[3], dtype=dtype, page=page, seqs=seqs, rows=rows,
             length=length, lens=lens, flag=flag)
    return c if name is None else dict(name=name, **c)


def listed():
    return [
        # one token of one sequence goes into the cache: nothing but latency
        _case("write_1", "write", HEADS[0], "fp32", 64, 1, 1, 1025),
        # prompts go into the cache: ragged, pages that end inside a prompt
        _case("write_prompts", "write", HEADS[0], "bf16", 16, 9, 4099, 4099, 5),
        # a decode step's queries of one sequence are brought into the latent space
        _case("product_1", "product", HEADS[0], "bf16", seqs=1, flag=False),
        # a full batch's results are brought out of it, with fp32 activations as this library's decode steps have
        _case("product_64_fp32", "product", HEADS[1], "fp32", seqs=64),
        # one sequence decodes over a short context, and over one of a quarter of a million tokens
        _case("attend_1", "attend", HEADS[0], "bf16", 64, 1, 1, 1025),
        _case("attend_1_long", "attend", HEADS[0], "bf16", 128, 1, 1, 262145),
        # a full batch over ragged contexts
        _case("attend_64", "attend", HEADS[0], "bf16", 64, 64, 1, 16001, 7),
        # many heads over one latent vector: as much arithmetic as memory
        _case("attend_wide", "attend", HEADS[1], "bf16", 64, 32, 1, 8190, 11),
        # fp32 activations, a narrow latent vector, small pages
        _case("attend_16_fp32", "attend", HEADS[2], "fp32", 16, 16, 1, 4099, 8),
        # a few drafted tokens a sequence are checked in one call
        _case("attend_drafts", "attend", HEADS[0], "bf16", 64, 8, 5, 8193, 9),
        # a short prompt, and prompts that attend to themselves and to what stands before them
        _case("expanded_short", "expanded", HEADS[2], "bf16", 16, 3, 101, 250, 3),
        _case("expanded_prompts", "expanded", HEADS[0], "bf16", 64, 4, 2049, 4097, 10),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    mode = rng.choice(MODES)
    heads = rng.choice(HEADS)
    dtype = rng.choice(("bf16", "bf16", "fp32"))
    page = rng.choice((16, 32, 64, 128, 256))
    seqs = _log_int(rng, 1, 64)
    lens, flag = rng.randint(1, 10 ** 6), rng.random() < 0.5
    if mode == "product":
        return _case(None, mode, heads, dtype, seqs=_log_int(rng, 1, 8000 // heads[0]), flag=flag)
    if mode == "write":
        rows = _log_int(rng, 1, max(2, min(4000, 20_000 // seqs)))
        return _case(None, mode, heads, dtype, page, seqs, rows, rows + _log_int(rng, 1, 2000) - 1, lens, flag)
    if mode == "attend":
        rows = 1 if rng.random() < 0.6 else rng.randint(2, 8)
        length = _log_int(rng, 1, max(2, min(250_000, 400_000 // seqs, 16_000_000 // (seqs * rows * heads[0]))))
        return _case(None, mode, heads, dtype, page, seqs, min(rows, length), length, lens)
    length = _log_int(rng, 60, 4000)
    rows = max(2, int(length * rng.uniform(0.2, 1.0)))
    seqs = min(seqs, 16, max(1, 250_000_000 // (rows * length * heads[0])))
    if rows * length * heads[0] > 250_000_000:
        rows = max(2, 250_000_000 // (length * heads[0]))
    return _case(None, mode, heads, "bf16", page, seqs, rows, length, lens)


def _sizes(case):
    """(tokens, new rows) of each sequence: functions of the case alone."""
    n, lens = case["seqs"], case["lens"]
    if case["mode"] == "product":
        return [1] * n, [1] * n
    if lens == 0:
        return [case["length"]] * n, [case["rows"]] * n
    r = random.Random(lens)
    lengths = [case["length"]] + [max(1, int(case["length"] * r.random())) for _ in range(n - 1)]
    if case["rows"] == 1:
        return lengths, [1] * n
    return lengths, [case["rows"]] + [max(1, min(t, int(case["rows"] * (0.3 + 0.7 * r.random())))) for t in lengths[1:]]


DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    host = random.Random(seed)
    h, lat, rope, head, page = (case[k] for k in ("heads", "latent", "rope", "head", "page"))
    dtype, mode = DTYPES[case["dtype"]], case["mode"]
    lengths, rows = _sizes(case)
    total = sum(rows)

    def randn(*shape):
        return torch.randn(*shape, device="cuda", generator=g)

    s = dict(case)
    s["dtype"] = dtype
    s["scale"] = (head + rope) ** -0.5
    if mode in ("product", "expanded"):
        # one matrix of a checkpoint: of each head the rows that make its key, then those that make its value
        both = (randn(h, 2 * head, lat) * lat ** -0.5).bfloat16()
        s["w_k"], s["w_v"] = both[:, :head], both[:, head:]
    if mode == "product":
        s["x"] = randn(total, h, lat if case["flag"] else head).to(dtype)
        return s

    s["max_rows"], s["max_len"], s["n_tokens"] = max(rows), max(lengths), sum(lengths)
    starts = [0]
    for n in rows:
        starts.append(starts[-1] + n)
    s["row_start"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
    s["lengths"] = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    # for every new row its sequence and its position there, as a program that lays out a batch has them
    s["row_seq"] = torch.repeat_interleave(torch.arange(len(rows), device="cuda"), torch.tensor(rows, device="cuda"))
    before = s["lengths"].long() - torch.tensor(rows, device="cuda")
    s["row_pos"] = torch.arange(total, device="cuda") - s["row_start"].long()[s["row_seq"]] + before[s["row_seq"]]
    need = [(n + page - 1) // page for n in lengths]
    pool = sum(need) + 3
    order = torch.randperm(pool, device="cuda", generator=g).to(torch.int32)
    table = torch.full((len(need), max(need)), -1, dtype=torch.int32, device="cuda")
    first = 0
    for i, n in enumerate(need):
        table[i, :n] = order[first:first + n]
        first += n
    s["page_table"] = table

    if mode == "write":
        s["positions"] = (s["row_pos"] + host.choice((0, 1000, 100_000))).to(torch.int32)
        s["inv_freq"] = (1e4 ** (-torch.arange(rope // 2, device="cuda", dtype=torch.float64) / (rope // 2))).float()
        s["gamma"] = 1 + 0.1 * randn(lat)
        # rows of one projection: the latent vector and the shared key side by side; queries of another, their two parts side by side
        s["kv"] = randn(total, lat + rope).to(dtype)
        s["q"] = randn(total, h, head + rope).to(dtype)
        s["pages"] = torch.zeros(pool, page, lat + rope, dtype=torch.bfloat16, device="cuda")
        return s
    pages = torch.empty(pool, page, lat + rope, dtype=torch.bfloat16, device="cuda")
    channel = 1 + 2 * torch.rand(lat + rope, device="cuda", generator=g) ** 4        # some channels are wide
    for i in range(0, pool, 1024):
        part = pages[i:i + 1024]
        part.copy_(randn(*part.shape) * channel)
    s["pages"] = pages
    s["q"] = (randn(total, h, (lat if mode == "attend" else head) + rope)).to(dtype)
    return s


# ---- the plain form ---------------------------------------------------------
def _turn(s, x):
    """Rows [rows, ..., rope] turned by their positions; the angles in 64 bits (far positions)."""
    x = x.float()
    angle = s["positions"].double()[:, None] * s["inv_freq"].double()
    c, w = angle.cos().float(), angle.sin().float()
    if x.dim() == 3:
        c, w = c[:, None], w[:, None]
    if s["flag"]:
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack((a * c - b * w, b * c + a * w), dim=-1).flatten(-2)
    a, b = x.chunk(2, dim=-1)
    return torch.cat((a * c - b * w, b * c + a * w), dim=-1)


def _plain_write(s):
    lat, page = s["latent"], s["page"]
    x = s["kv"][:, :lat].float()
    x = x * (x.square().mean(-1, keepdim=True) + EPS).rsqrt() * s["gamma"]
    row = torch.cat((x, _turn(s, s["kv"][:, lat:])), dim=-1).bfloat16()
    s["pages"][s["page_table"][s["row_seq"], s["row_pos"] // page].long(), s["row_pos"] % page] = row
    return _turn(s, s["q"][..., s["head"]:]).to(s["dtype"]), s["pages"]


def _plain_product(s):
    w = s["w_v"].float().transpose(1, 2) if s["flag"] else s["w_k"].float()
    return torch.matmul(s["x"].float().transpose(0, 1), w).transpose(0, 1).to(s["dtype"])


def _context(s):
    """Rows of each sequence's tokens in 32 bits: [seqs, tokens, latent + rope]."""
    return s["pages"][s["page_table"].clamp_min(0).long()].flatten(1, 2)[:, :s["max_len"]].float()


def _by_sequence(s, x):
    """New rows [rows, heads, ...] -> [seqs, heads, most rows, ...] (zeros where a sequence has fewer), and their positions (-1)."""
    within = torch.arange(x.shape[0], device="cuda") - s["row_start"].long()[s["row_seq"]]
    out = torch.zeros(s["seqs"], s["max_rows"], *x.shape[1:], device="cuda")
    out[s["row_seq"], within] = x.float()
    pos = torch.full((s["seqs"], s["max_rows"]), -1, device="cuda", dtype=torch.long)
    pos[s["row_seq"], within] = s["row_pos"]
    return out.transpose(1, 2), pos, within


def _softmax(s, score, pos):
    """Scores [seqs, heads, rows, tokens], in place."""
    hidden = torch.arange(score.shape[-1], device="cuda") > pos[:, None, :, None]
    score.mul_(s["scale"]).masked_fill_(hidden, -math.inf)
    score.sub_(score.amax(-1, keepdim=True).clamp_min(-1e30)).exp_()
    return score, score.sum(-1, keepdim=True).clamp_min(1e-30)


def _plain_attend(s):
    rows = _context(s)
    q, pos, within = _by_sequence(s, s["q"])
    score = (q.flatten(1, 2) @ rows.transpose(1, 2)).unflatten(1, q.shape[1:3])
    p, total = _softmax(s, score, pos)
    o = (p.flatten(1, 2) @ rows[..., :s["latent"]]).unflatten(1, q.shape[1:3]) / total
    return o.transpose(1, 2)[s["row_seq"], within].to(s["dtype"])


def _plain_expanded(s):
    lat, rows = s["latent"], _context(s)
    q, pos, within = _by_sequence(s, s["q"])
    key = torch.einsum("stl,hdl->shtd", rows[..., :lat], s["w_k"].float())
    value = torch.einsum("stl,hdl->shtd", rows[..., :lat], s["w_v"].float())
    key = torch.cat((key, rows[:, None, :, lat:].expand(-1, key.shape[1], -1, -1)), dim=-1)
    p, total = _softmax(s, q @ key.transpose(-1, -2), pos)
    return (p @ value / total).transpose(1, 2)[s["row_seq"], within].to(s["dtype"])


# ---- the library's ----------------------------------------------------------
def _handles(s):
    """What a program that serves from such a cache keeps: the cache, the batch's layout, the rotation."""
    if "handles" not in s:
        from paper_2607_24787_b200 import kv_cache, latent_cache
        rope = cache = batch = None
        if "pages" in s:
            cache = latent_cache.LatentCache(s["pages"], s["latent"])
            batch = kv_cache.KVBatch(s["page_table"], s["lengths"], s["row_start"], n_rows=s["q"].shape[0], max_rows=s["max_rows"])
        if "inv_freq" in s:
            rope = kv_cache.Rope(s["inv_freq"], k_gamma=s["gamma"], eps=EPS, neighbours=s["flag"])
        s["handles"] = latent_cache, cache, batch, rope
    return s["handles"]


def _own(s):
    lib, cache, batch, rope = _handles(s)
    mode, lat = s["mode"], s["latent"]
    if mode == "write":
        q = cache.write(batch, s["kv"][:, :lat], s["kv"][:, lat:], q=s["q"][..., s["head"]:], positions=s["positions"], rope=rope)
        return q, s["pages"]
    if mode == "product":
        return lib.head_product(s["x"], s["w_v"], transposed=True) if s["flag"] else lib.head_product(s["x"], s["w_k"])
    if mode == "attend":
        return cache.attend(batch, s["q"], s["scale"])
    return cache.attend_expanded(batch, s["q"], s["w_k"], s["w_v"], s["scale"], n_tokens=s["n_tokens"])


def run(state):
    if own:
        return _own(state)
    return {"write": _plain_write, "product": _plain_product, "attend": _plain_attend, "expanded": _plain_expanded}[state["mode"]](state)


def work(case):
    lengths, rows = _sizes(case)
    h, lat, rope, head = (case[k] for k in ("heads", "latent", "rope", "head"))
    e = 2 if case["dtype"] == "bf16" else 4
    total, token = sum(rows), 2 * (lat + rope)
    if case["mode"] == "write":       # rows in, the cache's rows out, queries in and out
        return {"bytes": total * ((lat + rope) * e + token + 2 * h * rope * e + 4), "flops": total * (4 * lat + (h + 1) * rope * 3)}
    if case["mode"] == "product":
        return {"bytes": h * head * lat * 2 + total * h * (head + lat) * e, "flops": 2 * total * h * head * lat}
    pairs = sum(r * n - r * (r - 1) // 2 for n, r in zip(lengths, rows))
    if case["mode"] == "attend":
        return {"bytes": sum(lengths) * token + total * h * (2 * lat + rope) * e, "flops": 2 * pairs * h * (2 * lat + rope)}
    return {"bytes": sum(lengths) * token + 2 * h * head * lat * 2 + total * h * (2 * head + rope) * e,
            "flops": 2 * pairs * h * (2 * head + rope) + 2 * sum(lengths) * h * 2 * head * lat}


# ---- the definition, in 64 bits ----------------------------------------------
def _exact_turn(s, x):
    x = x.double()
    angle = s["positions"].double()[:, None] * s["inv_freq"].double()[None]
    z = torch.polar(torch.ones_like(angle), angle)
    half = x.shape[-1] // 2
    pairs = x.reshape(*x.shape[:-1], half, 2) if s["flag"] else torch.stack((x[..., :half], x[..., half:]), dim=-1)
    y = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * (z if x.dim() == 2 else z[:, None]))
    return y.flatten(-2) if s["flag"] else torch.cat((y[..., 0], y[..., 1]), dim=-1)


def exact(case, seed):
    s = prepare(case, seed)
    h, lat, head = s["heads"], s["latent"], s["head"]
    if s["mode"] == "write":
        x = s["kv"][:, :lat].double()
        x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / lat + EPS) * s["gamma"].double()
        row = torch.cat((x, _exact_turn(s, s["kv"][:, lat:])), dim=-1)
        pages = s["pages"].double()
        slot = s["page_table"].long()[s["row_seq"], torch.div(s["row_pos"], s["page"], rounding_mode="floor")]
        pages.view(-1, pages.shape[-1])[slot * s["page"] + s["row_pos"] % s["page"]] = row
        return _exact_turn(s, s["q"][..., head:]), pages
    if s["mode"] == "product":
        w = s["w_v"].double() if s["flag"] else s["w_k"].double().transpose(1, 2)             # [heads, out, in]
        return torch.stack([s["x"][:, i].double() @ w[i].T for i in range(h)], dim=1)
    lengths, rows = _sizes(case)
    outs, at = [], 0
    for i, (length, n) in enumerate(zip(lengths, rows)):
        c = s["pages"][s["page_table"][i, :(length + s["page"] - 1) // s["page"]].long()].flatten(0, 1)[:length].double()
        q = s["q"][at:at + n].double()
        at += n
        o = torch.empty(n, h, lat if s["mode"] == "attend" else head, dtype=torch.float64, device="cuda")
        if s["mode"] == "attend":      # all heads meet the same rows
            late = torch.arange(length, device="cuda")[None, None] > torch.arange(length - n, length, device="cuda")[:, None, None]
            z = (q.reshape(n * h, -1) @ c.T).reshape(n, h, length) * s["scale"]
            p = torch.softmax(z.masked_fill(late, -math.inf), dim=-1)
            outs.append((p.reshape(n * h, length) @ c[:, :lat]).reshape(n, h, lat))
            continue
        for j in range(h):
            key = torch.cat((c[:, :lat] @ s["w_k"][j].double().T, c[:, lat:]), dim=1)
            value = c[:, :lat] @ s["w_v"][j].double().T
            for r in range(0, n, 1024):
                m = min(n, r + 1024)
                late = torch.arange(length, device="cuda")[None] > torch.arange(length - n + r, length - n + m, device="cuda")[:, None]
                z = (q[r:m, j] @ key.T * s["scale"]).masked_fill(late, -math.inf)
                o[r:m, j] = torch.softmax(z, dim=-1) @ value
        outs.append(o)
    return torch.cat(outs)
