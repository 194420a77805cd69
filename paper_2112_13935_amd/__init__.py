"""MI355X-native AET-SGD hot path: HIP kernels behind a C ABI (include/aet_sgd.h) and a
thin Python binding with the same names; operators for clients' models beside it
(include/aet_ops.h, ops)."""
from . import ops  # noqa: F401
from .binding import AetError, AetSgd, load_library  # noqa: F401
