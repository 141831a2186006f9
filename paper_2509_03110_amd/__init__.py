"""K-replica LSAM step engine for MI355X: HIP kernels behind a C boundary (include/lsam.h)
and its ctypes binding (paper_2509_03110_amd.lsam); operators of token models behind
include/lsam_ops.h and theirs (paper_2509_03110_amd.ops)."""
from . import lsam, ops  # noqa: F401
