"""ctypes binding of ``include/rwttt_kv.h`` and ``include/rwttt_kv_rows.h`` (argument marshalling only).

Every function keeps its C name and returns the C status; device buffers and
streams are integers (``tensor.data_ptr()``, ``stream.cuda_stream``), 0 for
NULL.  The functions are in the library that ``_rwttt`` loads.
"""

import ctypes as C

from . import _rwttt as R

RWTTT_FP8 = 2
RWTTT_FP4 = 4
RWTTT_KV_BLOCK = 32
RWTTT_KV_MAX_OWNERS = 4096
RWTTT_KV_MAX_ROWS = 1 << 23
RWTTT_KV_MAX_SELECT = 32768
RWTTT_ROTARY_HALF, RWTTT_ROTARY_INTERLEAVED = 0, 1
RWTTT_ROTARY_PLAIN, RWTTT_ROTARY_LINEAR, RWTTT_ROTARY_BASE, RWTTT_ROTARY_PARTS = 0, 1, 2, 3


class rwttt_kv_config(C.Structure):
    _fields_ = [("n_owners", C.c_uint32), ("n_layers", C.c_uint32), ("n_pages", C.c_uint32),
                ("page_rows", C.c_uint32), ("max_pages", C.c_uint32), ("n_heads", C.c_uint32),
                ("n_kv_heads", C.c_uint32), ("head_dim", C.c_uint32),
                ("io_dtype", C.c_int32), ("cache_dtype", C.c_int32), ("reserved", C.c_uint32),
                ("table", C.c_void_p), ("ring", C.c_void_p),
                ("k", C.POINTER(C.c_void_p)), ("v", C.POINTER(C.c_void_p)), ("bounds", C.POINTER(C.c_void_p)),
                ("k_scale", C.c_void_p), ("v_scale", C.c_void_p), ("bound_step", C.c_void_p),
                ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t)]


class rwttt_kv_rotary(C.Structure):
    _fields_ = [("turning", C.c_uint32), ("layout", C.c_int32), ("gain", C.c_float), ("inverse", C.c_int32),
                ("turns", C.c_void_p)]


def _bind(lib):
    P, U32, U64, I32, VP, F64 = C.POINTER, C.c_uint32, C.c_uint64, C.c_int32, C.c_void_p, C.c_double
    sig = {
        "rwttt_kv_workspace_bytes": (I32, [P(rwttt_kv_config), P(C.c_size_t)]),
        "rwttt_kv_create": (I32, [P(rwttt_kv_config), P(VP)]),
        "rwttt_kv_destroy": (I32, [VP]),
        "rwttt_kv_extend": (I32, [VP] * 10 + [U32, VP, VP]),
        "rwttt_kv_append": (I32, [VP, U32, VP, U64, VP, U64, VP, U32, VP]),
        "rwttt_kv_gather": (I32, [VP, U32, VP, VP, VP, U32, VP, U64, VP, U64, VP]),
        "rwttt_kv_turns": (I32, [U32, F64, I32, F64, F64, F64, F64, P(U64)]),
        "rwttt_kv_rotate": (I32, [VP, P(rwttt_kv_rotary), VP, U32] + [VP, U64] * 4 + [VP]),
        "rwttt_kv_select": (I32, [VP, U32, VP, U64, VP, VP, U32, U32, U32, U32, VP, VP]),
        "rwttt_kv_attend": (I32, [VP, U32, VP, U64, VP, VP, U32, C.c_float, U32, VP, U32, VP, U64, VP, VP]),
        "rwttt_kv_last_hip_error": (I32, [VP]),
    }
    for name, (res, args) in sig.items():
        f = getattr(lib, name)
        f.restype = res
        f.argtypes = args
    return lib


_lib = _bind(R.lib())


def make_kv_config(n_owners, n_layers, n_pages, page_rows, max_pages, n_heads, n_kv_heads, head_dim, io_dtype,
                   cache_dtype, table=0, ring=0, k=None, v=None, bounds=None, k_scale=0, v_scale=0, bound_step=0,
                   workspace=0, workspace_bytes=0):
    """A ``rwttt_kv_config`` plus the pointer arrays it references (kept alive).

    ``k``, ``v`` and ``bounds`` are None or one pointer per layer."""
    def layers(ptrs):
        return None if ptrs is None else (C.c_void_p * len(ptrs))(*[int(p) for p in ptrs])

    kept = [layers(x) for x in (k, v, bounds)]
    for a in kept:
        if a is not None and len(a) != n_layers:
            raise ValueError("k, v and bounds hold one pointer per layer")
    ptr = [None if a is None else C.cast(a, C.POINTER(C.c_void_p)) for a in kept]
    cfg = rwttt_kv_config(n_owners, n_layers, n_pages, page_rows, max_pages, n_heads, n_kv_heads, head_dim,
                          io_dtype, cache_dtype, 0, int(table) or None, int(ring) or None, *ptr,
                          int(k_scale) or None, int(v_scale) or None, int(bound_step) or None,
                          int(workspace) or None, int(workspace_bytes))
    cfg._keep = kept
    return cfg


def rwttt_kv_workspace_bytes(cfg):
    out = C.c_size_t(0)
    st = _lib.rwttt_kv_workspace_bytes(C.byref(cfg), C.byref(out))
    if st != R.RWTTT_OK:
        raise R.RwtttError(st, "rwttt_kv_workspace_bytes")
    return out.value


def rwttt_kv_create(cfg):
    kv = C.c_void_p(0)
    st = _lib.rwttt_kv_create(C.byref(cfg), C.byref(kv))
    if st != R.RWTTT_OK:
        raise R.RwtttError(st, "rwttt_kv_create")
    return kv


def rwttt_kv_destroy(kv):
    return _lib.rwttt_kv_destroy(kv)


def rwttt_kv_extend(kv, have, want, pos, new_pos, lengths, start, slots, owners, positions, cap, result, stream=0):
    return _lib.rwttt_kv_extend(kv, have, want, pos, new_pos, lengths, start, slots, owners, positions, cap,
                                result, stream)


def rwttt_kv_append(kv, layer, k, k_stride, v, v_stride, slots, n, stream=0):
    return _lib.rwttt_kv_append(kv, layer, k, k_stride, v, v_stride, slots, n, stream)


def rwttt_kv_gather(kv, layer, owners, positions, lengths, n, k, k_stride, v, v_stride, stream=0):
    return _lib.rwttt_kv_gather(kv, layer, owners, positions, lengths, n, k, k_stride, v, v_stride, stream)


def rwttt_kv_turns(turning, base, scaling=RWTTT_ROTARY_PLAIN, factor=1.0, low=0.0, high=1.0, context=1.0):
    """The turning / 2 frequencies in units of 2^-64 turns a position."""
    out = (C.c_uint64 * max(1, turning // 2))()
    st = _lib.rwttt_kv_turns(turning, base, scaling, factor, low, high, context, out)
    if st != R.RWTTT_OK:
        raise R.RwtttError(st, "rwttt_kv_turns")
    return list(out)


def make_rotary(turning, layout, turns, gain=1.0, inverse=False):
    """``turns``: address of the frequencies on the device."""
    return rwttt_kv_rotary(turning, layout, gain, int(inverse), int(turns) or None)


def rwttt_kv_rotate(kv, rotary, positions, n, q, q_stride, q_out, q_out_stride, k, k_stride, k_out, k_out_stride,
                    stream=0):
    return _lib.rwttt_kv_rotate(kv, C.byref(rotary), positions, n, q, q_stride, q_out, q_out_stride, k, k_stride,
                                k_out, k_out_stride, stream)


def rwttt_kv_select(kv, layer, q, q_stride, lengths, rows, n, first, last, keep, pages, stream=0):
    """``rows``: 0, or the device array of the n owners to compute."""
    return _lib.rwttt_kv_select(kv, layer, q, q_stride, lengths, rows, n, first, last, keep, pages, stream)


def rwttt_kv_attend(kv, layer, q, q_stride, lengths, rows, n, scale, window, pages, keep, out, out_stride, lse=0,
                    stream=0):
    """``pages``/``keep``: 0, 0 or a selection; ``window``: 0 or the last rows to attend to."""
    return _lib.rwttt_kv_attend(kv, layer, q, q_stride, lengths, rows, n, scale, window, pages, keep, out,
                                out_stride, lse, stream)


def rwttt_kv_last_hip_error(kv):
    return _lib.rwttt_kv_last_hip_error(kv)
