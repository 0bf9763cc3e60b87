"""MI355X-native owner-scoped fast-weight READ/WRITE path of RW-TTT serving.

The compute lives in ``librwttt.so`` (HIP kernels for gfx950 plus the host
planner and owner table behind ``include/rwttt.h``).  ``_rwttt`` is its ctypes
binding and raises ImportError when the library has not been built;
``serving`` is the serving loop (Algorithm 1) that calls it.  ``_rwttt_kv``
binds ``include/rwttt_kv.h``, the owners' paged key-value cache, ``paged`` is the
cache over it and ``paged_decode`` a runnable example.  Importing the package
itself loads nothing, so ``build`` works before the first build.
"""
