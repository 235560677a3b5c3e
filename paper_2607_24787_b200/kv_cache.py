"""The cache side of an attention block, on torch tensors: rotary positions, a key/value cache held in 4 bits, attention over it.

Marshals to spm_rotate_heads, spm_kv_write, spm_kv_read and spm_kv_attend (include/spm.h says what they compute and how a page is
laid out). Everything is enqueued on the current stream of the tensors' device and may be captured into a CUDA graph; lengths, row
starts, page numbers and positions are read on the device. Outputs and workspaces come from torch's allocator, a call's own each.
"""
from __future__ import annotations

import torch

from . import binding as B

DTYPES = {torch.float32: B.DTYPE_FP32, torch.bfloat16: B.DTYPE_BF16}
BLOCK = 16                      # tokens of a block


def _need(ok, message):
    if not ok:
        raise ValueError(message)


def _enqueue(device, call, *args):
    """call(*args, stream) on the current stream of the device, with the device current."""
    at = device.index
    stream = torch._C._cuda_getCurrentRawStream(at)       # (torch.cuda.current_stream builds an object, 2 us)
    if torch._C._cuda_getDevice() == at:
        rc = call(*args, stream)
    else:
        with torch.cuda.device(device):
            rc = call(*args, stream)
    if rc:
        B._check(rc)


def _vector(x, dtype, device, what, n=None):
    _need(x.dtype is dtype and x.dim() == 1 and x.is_contiguous() and x.device == device, f"{what}: a contiguous {dtype} vector on {device}")
    _need(n is None or x.numel() == n, f"{what}: {n} elements")
    return x.data_ptr()


def _rows(x, n, heads, hd, dtype, device, what):
    """spm_rows of a tensor [n, heads, hd] whose heads are contiguous."""
    if x.shape != (n, heads, hd):
        raise ValueError(f"{what}: shape [{n}, {heads}, {hd}], not {list(x.shape)}")
    if x.dtype is not dtype or x.device != device:
        raise ValueError(f"{what}: {dtype} on {device}, not {x.dtype} on {x.device}")
    row, head, one = x.stride()
    if one != 1:
        raise ValueError(f"{what}: the elements of a head must be contiguous")
    return B.Rows(x.data_ptr(), row, head)


def _dtype(x, what):
    if not x.is_cuda:
        raise ValueError(f"{what}: a CUDA tensor (there is no CPU implementation of this path)")
    dt = DTYPES.get(x.dtype)
    if dt is None or x.dim() != 3:
        raise ValueError(f"{what}: fp32 or bf16 [rows, heads, head_dim], not {x.dtype} {list(x.shape)}")
    return dt


class Rope:
    """How heads are normed and turned. inv_freq [rot_dim / 2] fp32; axis_of [rot_dim / 2] uint8: which of the position's axes turns a
    pair (None: the first); gammas [head_dim] fp32 or None (no norm); neighbours: pairs (2i, 2i + 1) instead of (i, i + rot_dim / 2)."""

    def __init__(self, inv_freq, axis_of=None, q_gamma=None, k_gamma=None, eps=1e-6, neighbours=False):
        _need(inv_freq.is_cuda, "inv_freq: a CUDA tensor")
        self.device = inv_freq.device
        self._keep = (inv_freq, axis_of, q_gamma, k_gamma)
        half = inv_freq.numel()
        self.gamma_sizes = tuple(None if g is None else g.numel() for g in (q_gamma, k_gamma))
        fields = (_vector(inv_freq, torch.float32, self.device, "inv_freq"),
                  None if axis_of is None else _vector(axis_of, torch.uint8, self.device, "axis_of", half),
                  None if q_gamma is None else _vector(q_gamma, torch.float32, self.device, "q_gamma"),
                  None if k_gamma is None else _vector(k_gamma, torch.float32, self.device, "k_gamma"))
        self._by_axes = {n: B.Rope(*fields, n, 2 * half, int(neighbours), eps) for n in range(1, 5)}

    def for_axes(self, n):
        """The spm_rope struct of positions with n axes."""
        return self._by_axes[n]

    def _with(self, positions, n_rows, hd, q, k):
        """(struct, positions' address, axis stride) of a call with positions [n_axes, rows] or [rows]; q, k: whose gammas it uses."""
        if positions is None:
            raise ValueError("positions are needed to turn heads")
        if positions.dtype is not torch.int32 or positions.device != self.device:
            raise ValueError(f"positions: int32 on {self.device}")
        if q and self.gamma_sizes[0] not in (None, hd) or k and self.gamma_sizes[1] not in (None, hd):
            raise ValueError(f"gammas: {hd} elements")
        shape, stride = positions.shape, positions.stride()
        axes = shape[0] if len(shape) == 2 else 1
        if not 1 <= len(shape) <= 2 or shape[-1] != n_rows or not 1 <= axes <= 4:
            raise ValueError(f"positions: [1..4 axes, {n_rows}], not {list(shape)}")
        if stride[-1] != 1 and n_rows > 1:
            raise ValueError("positions: the rows of an axis must be contiguous")
        return self._by_axes[axes], positions.data_ptr(), stride[0] if axes > 1 else n_rows


class KVBatch:
    """New rows of several sequences. page_table [n_seq, pages] int32; lengths [n_seq] int32: tokens each sequence holds, its new rows
    included; row_start [n_seq + 1] int32: where a sequence's rows begin (None: one row each); n_rows: rows of the row tensors (None:
    n_seq); max_rows: about how many rows a sequence has at most (0: not known), a hint."""

    def __init__(self, page_table, lengths, row_start=None, n_rows=None, max_rows=0):
        _need(page_table.is_cuda and page_table.dtype is torch.int32 and page_table.dim() == 2 and page_table.is_contiguous(),
              "page_table: a contiguous int32 CUDA tensor [n_seq, pages]")
        self.device = page_table.device
        n = page_table.shape[0]
        _need(row_start is not None or n_rows is None or n_rows >= n, "n_rows is less than the sequences, and there is no row_start")
        self.n_rows = n if n_rows is None else n_rows
        self._keep = (page_table, lengths, row_start)
        self.c = B.KvBatch(page_table.data_ptr(), _vector(lengths, torch.int32, self.device, "lengths", n),
                           None if row_start is None else _vector(row_start, torch.int32, self.device, "row_start", n + 1),
                           n, page_table.shape[1], self.n_rows, max_rows)
        self.shape = (n, page_table.shape[1], self.n_rows, max_rows, row_start is None)


class KVCache:
    """A pool of pages [n_pages, kv_heads, page_size / 16, 18 * head_dim] uint8. status: an int32 tensor of one element that SPM_KV_* bits are
    or-ed into (bad page numbers, lengths beyond the table, numbers that are not finite), or None."""

    def __init__(self, pages, status=None):
        _need(pages.is_cuda and pages.dtype is torch.uint8 and pages.dim() == 4 and pages.is_contiguous() and pages.shape[3] % 18 == 0,
              "pages: a contiguous uint8 CUDA tensor [n_pages, kv_heads, page_size / 16, 18 * head_dim]")
        self.device, self.pages, self.status = pages.device, pages, status
        self.kv_heads, self.page_size, self.head_dim = pages.shape[1], pages.shape[2] * BLOCK, pages.shape[3] // 18
        self.c = B.KvCache(pages.data_ptr(), None if status is None else _vector(status, torch.int32, self.device, "status", 1),
                           pages.shape[0], self.page_size, self.kv_heads, self.head_dim)
        self._lib = B.load()
        self._workspace = {}        # bytes that a call of a batch's shape asks for
        B.spm_kv_cache_bytes(self.c)

    @classmethod
    def empty(cls, n_pages, page_size, kv_heads, head_dim, device="cuda", status=None):
        _need(page_size % BLOCK == 0 and page_size > 0, "page_size: a multiple of 16")
        return cls(torch.zeros(n_pages, kv_heads, page_size // BLOCK, 18 * head_dim, dtype=torch.uint8, device=device), status)

    def _size(self, batch):
        if batch.device != self.device:
            raise ValueError("the batch is on another device than the cache")
        return batch.n_rows, self.kv_heads, self.head_dim

    def write(self, batch, k, v, q=None, positions=None, rope=None, q_out=None):
        """k, v [rows, kv_heads, head_dim] of the batch's new rows go into the cache, k normed and turned by `rope`; returns q [rows, q_heads,
        head_dim] normed and turned (None without q)."""
        n, heads, hd = self._size(batch)
        dt, dtype, device = _dtype(k, "k"), k.dtype, self.device
        ck, cv = _rows(k, n, heads, hd, dtype, device, "k"), _rows(v, n, heads, hd, dtype, device, "v")
        cq = co = cr = pos = None
        stride = q_heads = 0
        if rope is not None:
            if rope.device != device:
                raise ValueError("the rope is on another device than the cache")
            cr, pos, stride = rope._with(positions, n, hd, q is not None, True)
        if q is not None:
            if rope is None or q.dim() != 3:
                raise ValueError("q without rope: there is nothing to do to it" if rope is None else "q: [rows, heads, head_dim]")
            q_heads = q.shape[1]
            cq = _rows(q, n, q_heads, hd, dtype, device, "q")
            if q_out is None:
                q_out = torch.empty_like(q, memory_format=torch.contiguous_format)
                co = B.Rows(q_out.data_ptr(), q_heads * hd, hd)
            else:
                co = _rows(q_out, n, q_heads, hd, dtype, device, "q_out")
        _enqueue(device, self._lib.spm_kv_write, self.c, batch.c, cr, pos, stride, cq, co, q_heads, ck, cv, dt)
        return q_out

    def read(self, batch, dtype=torch.bfloat16, k_out=None, v_out=None):
        """The cache's keys and values at the positions of the batch's new rows: two tensors [rows, kv_heads, head_dim]."""
        n, heads, hd = size = self._size(batch)
        if k_out is None and v_out is None:
            k_out = self.pages.new_empty(size, dtype=dtype)
            v_out = torch.empty_like(k_out)
            dt = _dtype(k_out, "dtype")
            ck, cv = B.Rows(k_out.data_ptr(), heads * hd, hd), B.Rows(v_out.data_ptr(), heads * hd, hd)
        else:
            have = v_out if k_out is None else k_out
            k_out, v_out = (torch.empty_like(have, memory_format=torch.contiguous_format) if x is None else x for x in (k_out, v_out))
            dt, dtype = _dtype(have, "k_out, v_out"), have.dtype
            ck, cv = _rows(k_out, n, heads, hd, dtype, self.device, "k_out"), _rows(v_out, n, heads, hd, dtype, self.device, "v_out")
        _enqueue(self.device, self._lib.spm_kv_read, self.c, batch.c, ck, cv, dt)
        return k_out, v_out

    def attend(self, batch, q, scale=None, out=None):
        """softmax(scale q K^T) V of q [rows, q_heads, head_dim], each row over its sequence's tokens up to its own position. scale None:
        head_dim ** -0.5."""
        n, _, hd = self._size(batch)
        dt, dtype, device = _dtype(q, "q"), q.dtype, self.device
        heads = q.shape[1]
        cq = _rows(q, n, heads, hd, dtype, device, "q")
        if out is None:
            out = torch.empty_like(q, memory_format=torch.contiguous_format)
            co = B.Rows(out.data_ptr(), heads * hd, hd)
        else:
            co = _rows(out, n, heads, hd, dtype, device, "out")
        key = (batch.shape, heads, dt)
        size = self._workspace.get(key)
        if size is None:
            size = self._workspace[key] = B.spm_kv_attend_workspace(self.c, batch.c, heads, dt)
        work = self.pages.new_empty(size)
        _enqueue(device, self._lib.spm_kv_attend, self.c, batch.c, cq, heads, co, hd ** -0.5 if scale is None else scale, dt,
                 work.data_ptr(), size)
        return out


def rotate_heads(x, positions, rope, out=None):
    """Norm (rope's q_gamma) and rotation of x [rows, heads, head_dim] by positions [axes, rows]."""
    dt = _dtype(x, "x")
    n, heads, hd = x.shape
    device = rope.device
    c, pos, stride = rope._with(positions, n, hd, True, False)
    cx = _rows(x, n, heads, hd, x.dtype, device, "x")
    if out is None:
        out = torch.empty_like(x, memory_format=torch.contiguous_format)
        cy = B.Rows(out.data_ptr(), heads * hd, hd)
    else:
        cy = _rows(out, n, heads, hd, x.dtype, device, "out")
    _enqueue(device, B.load().spm_rotate_heads, c, pos, stride, cx, cy, n, heads, hd, dt)
    return out
