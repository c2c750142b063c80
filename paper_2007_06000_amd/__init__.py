"""xl: cross-layer fused CNN blocks on MI355X (gfx950).

`binding` mirrors the C ABI of libxl.so (include/xl.h); `session` adds the
PyTorch plumbing (device buffers, streams) around it.  `seq` has the operators
of sequence models on torch tensors (libxl_seq.so, include/xl_seq.h).  All
arithmetic runs in the libraries' HIP kernels.
"""
from . import binding  # noqa: F401
from .binding import Plan, XlError  # noqa: F401
