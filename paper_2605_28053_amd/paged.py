"""The owners' paged key-value cache on top of the C ABI, with torch as the allocator.

``PagedCache`` owns the pages of every layer, the block tables, the ring of free
pages and the library's workspace.  A step is

    cache.extend(want)            # lengths -> pages and slots of the new rows
    per layer:
        cache.rotate(rotary, q, k)  # rotary positions, in place
        cache.append(l, k, v)     # the new rows
        cache.select(l, q, keep)  # long contexts: the pages each query attends to
        cache.attend(l, q)        # one new token's attention per owner
    cache.commit()                # or cache.rollback(): the old lengths again

and ``cache.gather(l, owners, positions)`` reads stored rows back.

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
CODE = {"f32": R.RWTTT_F32, "bf16": R.RWTTT_BF16, "fp8": KV.RWTTT_FP8, "fp4": KV.RWTTT_FP4}
LAYOUT = {"half": KV.RWTTT_ROTARY_HALF, "interleaved": KV.RWTTT_ROTARY_INTERLEAVED}
SCALING = {"plain": KV.RWTTT_ROTARY_PLAIN, "linear": KV.RWTTT_ROTARY_LINEAR, "base": KV.RWTTT_ROTARY_BASE,
           "parts": KV.RWTTT_ROTARY_PARTS}


def _check(status, where):
    if status != R.RWTTT_OK:
        raise R.RwtttError(status, where)


class Rotary:
    """Rotary positions: which channels turn, how, and how fast.

    ``turning`` channels of a head turn in pairs, i with i + turning / 2 (``layout``
    "half") or 2 i with 2 i + 1 ("interleaved"), by base^(-2 i / turning) a position.
    ``scaling`` stretches the context by ``factor``: "linear" slows all pairs, "base"
    the slow ones the most, "parts" those of fewer than ``low`` turns over ``context``
    positions and none of more than ``high``.  Turned channels are multiplied by ``gain``.
    ``inverse()`` turns back: the gradient of the inputs from that of the outputs."""

    def __init__(self, turning, base=10000.0, layout="half", scaling="plain", factor=1.0, low=1.0, high=32.0,
                 context=8192.0, gain=1.0, device="cuda"):
        if not 0 <= turning < 1 << 32:     # the binding would wrap it
            raise ValueError(f"turning is {turning}")
        if layout not in LAYOUT or scaling not in SCALING:
            raise ValueError(f"layout is one of {list(LAYOUT)}, scaling of {list(SCALING)}")
        units = KV.rwttt_kv_turns(turning, base, SCALING[scaling], factor, low, high, context)
        self.turns = torch.tensor(units, dtype=torch.uint64).to(device)
        self.turning, self.layout, self.gain = turning, layout, gain
        self.struct = KV.make_rotary(turning, LAYOUT[layout], self.turns.data_ptr(), gain)

    def inverse(self):
        other = object.__new__(Rotary)
        other.turns, other.turning, other.layout, other.gain = self.turns, self.turning, self.layout, self.gain
        other.struct = KV.make_rotary(self.turning, LAYOUT[self.layout], self.turns.data_ptr(), self.gain,
                                      not self.struct.inverse)
        return other


class PagedCache:
    """Pages of n_layers caches for n_owners requests, and one step's slots.

    ``cache_dtype`` is "bf16", "f32" (with fp32 io), "fp8" or "fp4": e2m1 codes in blocks of
    32 channels with a power of two each, whose pages are bytes.
    ``k_scale``, ``v_scale`` (8-bit caches) and ``bound_step`` (page selection)
    are numbers, or tensors [n_layers, n_kv_heads].  ``max_new`` is the most new
    rows that one step may add over all owners."""

    def __init__(self, n_owners, n_layers, n_heads, n_kv_heads, head_dim, n_pages, max_pages, page_rows=64,
                 io_dtype="bf16", cache_dtype="bf16", max_new=None, bound_step=None, k_scale=1.0, v_scale=1.0,
                 device="cuda"):
        self.n_owners, self.n_layers, self.n_heads, self.n_kv_heads = n_owners, n_layers, n_heads, n_kv_heads
        self.head_dim, self.io_dtype, self.device = head_dim, io_dtype, device
        self.max_new = n_owners if max_new is None else max_new
        fp4 = cache_dtype == "fp4"
        shape = (n_pages, n_kv_heads, page_rows * head_dim * 17 // 32) if fp4 else (n_pages, n_kv_heads, page_rows, head_dim)
        stored = torch.uint8 if fp4 else TORCH_DTYPE[cache_dtype]

        def i32(*size):
            return torch.zeros(size, dtype=torch.int32, device=device)

        def per_head(x):
            return torch.as_tensor(x, dtype=torch.float32, device=device).expand(n_layers, n_kv_heads).contiguous()

        self.k, self.v = ([torch.empty(shape, dtype=stored, device=device) for _ in range(n_layers)]
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

    def rotate(self, rotary, q=None, k=None, positions=None, q_out=None, k_out=None):
        """Turn queries and keys [n, heads, head_dim] to their positions; in place unless q_out or k_out is given.

        ``positions`` (int32 [n]) are the open step's, in slot order, if not given; tokens of
        negative ones are left as they are.  Returns (q_out, k_out), which autograd knows nothing
        of: ``rotary.inverse()`` turns their gradients to those of q and k."""
        if q is None and k is None:
            raise ValueError("queries or keys")
        if (q is None and q_out is not None) or (k is None and k_out is not None):
            raise ValueError("an output without its input")
        self._here(rotary.turns, "the rotary's table")
        q_out, k_out = q if q_out is None else q_out, k if k_out is None else k_out
        n = len(k if q is None else q)
        if positions is None:
            if not self.open:
                raise RuntimeError("no open step: give the positions")
            if n > self.max_new:
                raise ValueError("more rows than a step may add")
            positions = self.positions[:n]
        self._index(positions, n)
        self._written(q_out=q_out, k_out=k_out)
        args = []
        for t, heads, name in ((q, self.n_heads, "q"), (q_out, self.n_heads, "q_out"), (k, self.n_kv_heads, "k"),
                               (k_out, self.n_kv_heads, "k_out")):
            args += [0, 0] if t is None else [t.data_ptr(), self._rows(t, heads, name, n)]
        _check(KV.rwttt_kv_rotate(self.kv, rotary.struct, positions.data_ptr(), n, *args, _stream()), "rwttt_kv_rotate")
        return q_out, k_out

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

    def gather(self, layer, owners, positions, k=None, v=None):
        """The stored rows at ``positions`` of ``owners`` (int32 [n] each), as (k, v) [n, n_kv_heads, head_dim].

        Rows of pairs that name none -- an open step's own rows are held -- stay as they are in
        the given outputs, and are 0 in new ones."""
        n = self._index(owners).numel()
        self._index(positions, n)
        self._counts(layer=layer)
        shape, dtype = (n, self.n_kv_heads, self.head_dim), TORCH_DTYPE[self.io_dtype]
        k = torch.zeros(shape, dtype=dtype, device=self.device) if k is None else k
        v = torch.zeros(shape, dtype=dtype, device=self.device) if v is None else v
        k_stride, v_stride = self._rows(k, self.n_kv_heads, "k", n), self._rows(v, self.n_kv_heads, "v", n)
        self._written(k=k, v=v)
        _check(KV.rwttt_kv_gather(self.kv, layer, owners.data_ptr(), positions.data_ptr(), self.now().data_ptr(), n,
                                  k.data_ptr(), k_stride, v.data_ptr(), v_stride, _stream()), "rwttt_kv_gather")
        return k, v

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

    @staticmethod
    def _written(**tensors):
        """Autograd does not see a call's writes, so it must not hold gradients for what they replace."""
        for name, t in tensors.items():
            if t is not None and t.requires_grad and torch.is_grad_enabled():
                raise ValueError(f"{name} requires a gradient: give an output of its own, or call under torch.no_grad()")

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
