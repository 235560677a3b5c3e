"""Attention with keys and values from one latent vector a token, on torch tensors: a paged bf16 cache of latent rows, the products of
every head around it, attention over it.

Marshals to spm_latent_write, spm_head_product, spm_latent_attend and spm_latent_attend_expanded (include/spm.h says what they compute). Batches, rotations, streams,
graphs, outputs and workspaces are as in kv_cache.py. A decode step's attention, with w [heads, 2 * head, latent] the matrix that makes keys
and values from latent vectors, w_k = w[:, :head] and w_v = w[:, head:]:

    q = torch.empty(rows, heads, latent + rope)                       # the absorbed queries
    head_product(q_plain, w_k, out=q[..., :latent])
    cache.write(batch, latents, keys, q=q_turning, positions=positions, rope=rope, q_out=q[..., latent:])
    out = head_product(cache.attend(batch, q, scale), w_v, transposed=True)

A prompt's: cache.write, with q turned in place, then cache.attend_expanded(batch, q, w_k, w_v, scale, n_tokens).
"""
from __future__ import annotations

import torch

from . import binding as B
from .kv_cache import DTYPES, _dtype, _enqueue, _need, _rows, _vector


class LatentCache:
    """A pool of pages [n_pages, page_size, latent_dim + rope_dim] bf16. status: an int32 tensor of one element that SPM_KV_* bits are or-ed
    into (bad page numbers, lengths beyond the table, numbers that are not finite), or None."""

    def __init__(self, pages, latent_dim, status=None):
        _need(pages.is_cuda and pages.dtype is torch.bfloat16 and pages.dim() == 3 and pages.is_contiguous(),
              "pages: a contiguous bf16 CUDA tensor [n_pages, page_size, latent_dim + rope_dim]")
        self.device, self.pages, self.status = pages.device, pages, status
        self.page_size, self.latent_dim, self.rope_dim = pages.shape[1], latent_dim, pages.shape[2] - latent_dim
        self.c = B.LatentRows(pages.data_ptr(), None if status is None else _vector(status, torch.int32, self.device, "status", 1),
                              pages.shape[0], self.page_size, latent_dim, self.rope_dim)
        self._lib = B.load()
        self._workspace = {}        # bytes that a call of a batch's shape asks for
        self._check_shape()

    def _check_shape(self):
        """Raises for sizes that no call takes."""
        B.spm_latent_attend_workspace(self.c, B.KvBatch(), 1, B.DTYPE_BF16)

    @classmethod
    def empty(cls, n_pages, page_size, latent_dim, rope_dim, device="cuda", status=None):
        return cls(torch.zeros(n_pages, page_size, latent_dim + rope_dim, dtype=torch.bfloat16, device=device), latent_dim, status)

    def _on(self, thing, what):
        if thing.device != self.device:
            raise ValueError(f"the {what} is on another device than the cache")

    def _vectors(self, x, n, size, dtype, what):
        """spm_rows of a tensor [n, size] whose elements are contiguous."""
        if x.shape != (n, size):
            raise ValueError(f"{what}: shape [{n}, {size}], not {list(x.shape)}")
        if x.dtype is not dtype or x.device != self.device:
            raise ValueError(f"{what}: {dtype} on {self.device}, not {x.dtype} on {x.device}")
        row, one = x.stride()
        if one != 1:
            raise ValueError(f"{what}: the elements of a row must be contiguous")
        return B.Rows(x.data_ptr(), row, 0)

    def write(self, batch, latent, key, q=None, positions=None, rope=None, q_out=None):
        """latent [rows, latent_dim] and key [rows, rope_dim] of the batch's new rows go into the cache, normed by `rope`'s k_gamma and turned;
        returns q [rows, heads, rope_dim], the parts of the queries that turn, turned (None without q)."""
        self._on(batch, "batch")
        n, size, device, dtype = batch.n_rows, self.rope_dim, self.device, latent.dtype
        dt = DTYPES.get(dtype)
        if dt is None:
            raise ValueError(f"latent: fp32 or bf16, not {dtype}")
        cl, ck = self._vectors(latent, n, self.latent_dim, dtype, "latent"), self._vectors(key, n, size, dtype, "key")
        cq = co = cr = pos = None
        stride = heads = 0
        if rope is not None:
            self._on(rope, "rope")
            if rope.gamma_sizes[0] is not None:
                raise ValueError("rope: queries have no norm here, q_gamma is to be None")
            cr, pos, stride = rope._with(positions, n, self.latent_dim, False, True)
        if q is not None:
            if rope is None or q.dim() != 3:
                raise ValueError("q without rope: there is nothing to do to it" if rope is None else "q: [rows, heads, rope_dim]")
            heads = q.shape[1]
            cq = _rows(q, n, heads, size, dtype, device, "q")
            if q_out is None:
                q_out = q.new_empty(n, heads, size)
                co = B.Rows(q_out.data_ptr(), heads * size, size)
            else:
                co = _rows(q_out, n, heads, size, dtype, device, "q_out")
        _enqueue(device, self._lib.spm_latent_write, self.c, batch.c, cr, pos, stride, cq, co, heads, cl, ck, dt)
        return q_out

    def attend(self, batch, q, scale, out=None):
        """softmax(scale q . row) latent of absorbed queries q [rows, heads, latent_dim + rope_dim], each row over its sequence's tokens up to its
        own position: [rows, heads, latent_dim]. The scale is that of whole queries and keys, (head + rope_dim) ** -0.5."""
        self._on(batch, "batch")
        n, size = batch.n_rows, self.latent_dim
        dt, dtype, device = _dtype(q, "q"), q.dtype, self.device
        heads = q.shape[1]
        cq = _rows(q, n, heads, size + self.rope_dim, dtype, device, "q")
        if out is None:
            out = q.new_empty(n, heads, size)
            co = B.Rows(out.data_ptr(), heads * size, size)
        else:
            co = _rows(out, n, heads, size, dtype, device, "out")
        key = (batch.shape, heads, dt)
        work_size = self._workspace.get(key)
        if work_size is None:
            work_size = self._workspace[key] = B.spm_latent_attend_workspace(self.c, batch.c, heads, dt)
        work = torch.empty(work_size, dtype=torch.uint8, device=device)
        _enqueue(device, self._lib.spm_latent_attend, self.c, batch.c, cq, heads, co, scale, dt, work.data_ptr(), work_size)
        return out

    def attend_expanded(self, batch, q, w_k, w_v, scale, n_tokens, out=None):
        """The same attention for prompts, in bf16, of whole queries q [rows, heads, head + rope_dim]: keys and values are made from the cache by w_k and
        w_v [heads, head, latent_dim]; returns [rows, heads, head]. n_tokens: at least the tokens of all sequences together (the sum of
        their lengths, their new rows included), which the host knows: room for their keys and values."""
        self._on(batch, "batch")
        n, device = batch.n_rows, self.device
        dt, dtype = _dtype(q, "q"), q.dtype
        heads, size = q.shape[1], q.shape[2] - self.rope_dim
        cq = _rows(q, n, heads, size + self.rope_dim, dtype, device, "q")
        matrices = []
        for w, what in ((w_k, "w_k"), (w_v, "w_v")):
            if w.shape != (heads, size, self.latent_dim) or w.dtype is not torch.bfloat16 or w.device != device or w.stride(2) != 1:
                raise ValueError(f"{what}: bf16 [{heads}, {size}, {self.latent_dim}] on {device}, rows contiguous")
            matrices.append(B.Matrices(w.data_ptr(), w.stride(0), w.stride(1)))
        if out is None:
            out = q.new_empty(n, heads, size)
            co = B.Rows(out.data_ptr(), heads * size, size)
        else:
            co = _rows(out, n, heads, size, dtype, device, "out")
        work_size = B.spm_latent_attend_expanded_workspace(self.c, batch.c, heads, size, n_tokens, dt)
        work = torch.empty(work_size, dtype=torch.uint8, device=device)
        _enqueue(device, self._lib.spm_latent_attend_expanded, self.c, batch.c, cq, *matrices, heads, size, co, scale, n_tokens, dt,
                 work.data_ptr(), work_size)
        return out


def head_product(x, w, transposed=False, out=None):
    """x [rows, heads, in] times each head's matrix: w [heads, in, out], or transposed [heads, out, in], bf16. The rows of a matrix are contiguous,
    its heads and rows may be apart, as in a slice of a wider one."""
    dt = _dtype(x, "x")
    n, heads, size = x.shape
    device = x.device
    shape, strides = w.shape, w.stride()
    if (len(shape) != 3 or w.dtype is not torch.bfloat16 or w.device != device or shape[0] != heads or shape[2 if transposed else 1] != size
            or strides[2] != 1):
        raise ValueError(f"w: bf16 [{heads}, {'out, ' if transposed else ''}{size}{'' if transposed else ', out'}] on {device}, rows contiguous")
    to = shape[1 if transposed else 2]
    cx = _rows(x, n, heads, size, x.dtype, device, "x")
    if out is None:
        out = x.new_empty(n, heads, to)
        cy = B.Rows(out.data_ptr(), heads * to, to)
    else:
        cy = _rows(out, n, heads, to, x.dtype, device, "out")
    _enqueue(device, B.load().spm_head_product, cx, w.data_ptr(), strides[0], strides[1], int(transposed), cy, n, heads, size, to, dt)
    return out
