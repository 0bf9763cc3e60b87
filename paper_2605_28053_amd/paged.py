"""The owners' paged key-value cache on top of the C ABI, with torch as the allocator.

``PagedCache`` owns the pages of every layer, the block tables, the ring of free
pages and the library's workspace.  A step is

    cache.extend(want)            # lengths -> pages and slots of the new rows
    per layer:
        cache.append(l, k, v)     # the new rows
        cache.select(l, q, keep)  # long contexts: the pages each query attends to
        cache.attend(l, q)        # one new token's attention per owner
    cache.commit()                # or cache.rollback(): the old lengths again

Nothing here waits for the GPU: lengths and slots stay on the device, and
``result`` holds the step's status there for whoever wants to read it.  Host
code only marshals arguments; every number is computed by the library's
kernels.

``commit`` swaps the buffers of the committed lengths and of the open step's, so
a graph captures an even number of committed steps: replayed, it goes on from
where the last replay ended.  Calls go to the current stream, and a cache has
one workspace: its ``attend`` and ``select`` calls must not overlap in time, so
calls on several streams need to wait for each other.
"""

import torch

from . import _rwttt as R
from . import _rwttt_kv as KV

TORCH_DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn}
CODE = {"f32": R.RWTTT_F32, "bf16": R.RWTTT_BF16, "fp8": KV.RWTTT_FP8}


def _check(status, where):
    if status != R.RWTTT_OK:
        raise R.RwtttError(status, where)


class PagedCache:
    """Pages of n_layers caches for n_owners requests, and one step's slots.

    ``k_scale``, ``v_scale`` (8-bit caches) and ``bound_step`` (page selection)
    are numbers, or tensors [n_layers, n_kv_heads].  ``max_new`` is the most new
    rows that one step may add over all owners."""

    def __init__(self, n_owners, n_layers, n_heads, n_kv_heads, head_dim, n_pages, max_pages, page_rows=64,
                 io_dtype="bf16", cache_dtype="bf16", max_new=None, bound_step=None, k_scale=1.0, v_scale=1.0,
                 device="cuda"):
        self.n_owners, self.n_layers, self.n_heads, self.n_kv_heads = n_owners, n_layers, n_heads, n_kv_heads
        self.head_dim, self.io_dtype, self.device = head_dim, io_dtype, device
        self.max_new = n_owners if max_new is None else max_new
        shape = (n_pages, n_kv_heads, page_rows, head_dim)

        def i32(*size):
            return torch.zeros(size, dtype=torch.int32, device=device)

        def per_head(x):
            return torch.as_tensor(x, dtype=torch.float32, device=device).expand(n_layers, n_kv_heads).contiguous()

        self.k, self.v = ([torch.empty(shape, dtype=TORCH_DTYPE[cache_dtype], device=device) for _ in range(n_layers)]
                          for _ in range(2))
        self.table, self.ring = i32(n_owners, max_pages), torch.arange(n_pages, dtype=torch.int32, device=device)
        fp8 = cache_dtype == "fp8"
        self.k_scale, self.v_scale = (per_head(k_scale), per_head(v_scale)) if fp8 else (None, None)
        self.bounds = self.bound_step = None
        if bound_step is not None:
            self.bound_step = per_head(bound_step)
            self.bounds = [torch.zeros((n_pages, n_kv_heads, 2, head_dim), dtype=torch.int8, device=device)
                           for _ in range(n_layers)]
        # committed lengths and ring position, and the ones an open step leads to
        self.lengths, self.pos = i32(n_owners), i32(2)
        self.pos[1] = n_pages
        self.new_lengths, self.new_pos = i32(n_owners), i32(2)
        self.start, self.result = i32(n_owners + 1), i32(4)
        self.slots, self.owners, self.positions = (i32(max(1, self.max_new)) for _ in range(3))
        self.open = False

        def ptrs(tensors):
            return None if tensors is None else [t.data_ptr() for t in tensors]

        def ptr(t):
            return 0 if t is None else t.data_ptr()

        cfg = KV.make_kv_config(
            n_owners, n_layers, n_pages, page_rows, max_pages, n_heads, n_kv_heads, head_dim, CODE[io_dtype],
            CODE[cache_dtype], table=ptr(self.table), ring=ptr(self.ring), k=ptrs(self.k), v=ptrs(self.v),
            bounds=ptrs(self.bounds), k_scale=ptr(self.k_scale), v_scale=ptr(self.v_scale),
            bound_step=ptr(self.bound_step))
        self.workspace = torch.zeros(KV.rwttt_kv_workspace_bytes(cfg), dtype=torch.uint8, device=device)
        cfg.workspace, cfg.workspace_bytes = self.workspace.data_ptr(), self.workspace.numel()
        self.kv = KV.rwttt_kv_create(cfg)

    def close(self):
        if self.kv:
            KV.rwttt_kv_destroy(self.kv)
            self.kv = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ---- a step -------------------------------------------------------------
    def extend(self, want):
        """Open a step towards the lengths ``want`` (int32 device tensor [n_owners])."""
        want = self._index(want, self.n_owners)
        _check(KV.rwttt_kv_extend(
            self.kv, self.lengths.data_ptr(), want.data_ptr(), self.pos.data_ptr(), self.new_pos.data_ptr(),
            self.new_lengths.data_ptr(), self.start.data_ptr(), self.slots.data_ptr(), self.owners.data_ptr(),
            self.positions.data_ptr(), self.max_new, self.result.data_ptr(), _stream()), "rwttt_kv_extend")
        self.open = True

    def append(self, layer, k, v):
        """Store the open step's new rows: k, v [n, n_kv_heads, head_dim], n <= max_new, in slot order."""
        if not self.open:
            raise RuntimeError("append needs an open step: call extend first")
        self._counts(layer=layer)
        k_stride, v_stride = self._rows(k, self.n_kv_heads, "k"), self._rows(v, self.n_kv_heads, "v")
        if k.shape[0] != v.shape[0] or k.shape[0] > self.max_new:
            raise ValueError("k and v need the same number of rows, max_new at most")
        _check(KV.rwttt_kv_append(self.kv, layer, k.data_ptr(), k_stride, v.data_ptr(), v_stride,
                                  self.slots.data_ptr(), k.shape[0], _stream()), "rwttt_kv_append")

    def select(self, layer, q, keep, first=1, last=2, rows=None, out=None):
        """Pages [n_owners, n_kv_heads, keep] that each listed owner's query attends to; -1 for the others."""
        q_stride = self._rows(q, self.n_heads, "q", self.n_owners)
        self._counts(layer=layer, keep=keep, first=first, last=last)
        if out is None:
            shape = (self.n_owners, self.n_kv_heads, keep)
            out = torch.empty(shape, dtype=torch.int32, device=self.device) if rows is None else \
                torch.full(shape, -1, dtype=torch.int32, device=self.device)
        self._dense(out, torch.int32, (self.n_owners, self.n_kv_heads, keep), "out")
        listed, n = self._listed(rows)
        _check(KV.rwttt_kv_select(
            self.kv, layer, q.data_ptr(), q_stride, self.now().data_ptr(), listed, n, first, last, keep,
            out.data_ptr(), _stream()), "rwttt_kv_select")
        return out

    def attend(self, layer, q, scale=None, window=0, pages=None, rows=None, out=None, lse=None):
        """Attention [n_owners, n_heads, head_dim] of one token q (same shape) per listed owner; 0 for the others."""
        q_stride = self._rows(q, self.n_heads, "q", self.n_owners)
        self._counts(layer=layer, window=window)
        if out is None:
            out = (torch.empty if rows is None else torch.zeros)(q.shape, dtype=q.dtype, device=self.device)
        out_stride = self._rows(out, self.n_heads, "out", self.n_owners)
        if lse is not None:
            self._dense(lse, torch.float32, (self.n_owners, self.n_heads), "lse")
        if pages is not None:
            self._dense(pages, torch.int32, (self.n_owners, self.n_kv_heads, *pages.shape[-1:]), "pages")
        listed, n = self._listed(rows)
        _check(KV.rwttt_kv_attend(
            self.kv, layer, q.data_ptr(), q_stride, self.now().data_ptr(), listed, n,
            self.head_dim ** -0.5 if scale is None else scale, window, 0 if pages is None else pages.data_ptr(),
            0 if pages is None else pages.shape[2], out.data_ptr(), out_stride, 0 if lse is None else lse.data_ptr(),
            _stream()), "rwttt_kv_attend")
        return out

    def commit(self):
        """Adopt the open step's lengths and ring position."""
        if not self.open:
            raise RuntimeError("no open step")
        self.lengths, self.new_lengths = self.new_lengths, self.lengths
        self.pos, self.new_pos = self.new_pos, self.pos
        self.open = False

    def rollback(self):
        """Forget the open step: its rows lie behind the lengths, its pages are still in the ring."""
        if not self.open:
            raise RuntimeError("no open step")
        self.open = False

    def now(self):
        """The lengths that select and attend see: an open step's own rows are among them."""
        return self.new_lengths if self.open else self.lengths

    # ---- checks -------------------------------------------------------------
    @staticmethod
    def _counts(**numbers):
        for name, x in numbers.items():
            if not 0 <= x < 1 << 32:     # the binding would wrap it
                raise ValueError(f"{name} is {x}")

    def _here(self, t, name):
        if t.device != self.lengths.device:
            raise ValueError(f"{name} is on {t.device}, the cache on {self.lengths.device}")

    def _dense(self, t, dtype, shape, name):
        self._here(t, name)
        if t.dtype != dtype or tuple(t.shape) != shape or not t.is_contiguous():
            raise ValueError(f"{name}: contiguous {dtype} {list(shape)}")

    def _index(self, t, n=None):
        self._here(t, "an index array")
        if t.dtype != torch.int32 or t.dim() != 1 or not t.is_contiguous() or (n is not None and t.numel() != n):
            raise ValueError("index arrays are contiguous int32 vectors" + ("" if n is None else f" of {n}"))
        return t

    def _listed(self, rows):
        """Address and number of the listed owners; a null address means all of them."""
        if rows is None:
            return 0, self.n_owners
        n = self._index(rows).numel()
        return rows.data_ptr() if n else self.lengths.data_ptr(), n     # an empty tensor's address is null

    def _rows(self, t, heads, name, n=None):
        """Elements between the rows of t [n, heads, head_dim]; a dimension of one may have any stride."""
        self._here(t, name)
        n = t.shape[0] if n is None and t.dim() else n
        if t.dtype != TORCH_DTYPE[self.io_dtype] or tuple(t.shape) != (n, heads, self.head_dim) or t.stride(2) != 1 \
                or (heads > 1 and t.stride(1) != self.head_dim):
            raise ValueError(f"{name}: {self.io_dtype} [{n}, {heads}, {self.head_dim}] with dense rows")
        return t.stride(0) if n > 1 else heads * self.head_dim


def _stream():
    return torch.cuda.current_stream().cuda_stream
