"""libbuzz: the BUZZ sparse KV-cache hot path (prefill scoring, decode attention, eviction) as
hand-written CUDA for sm_100a behind a C ABI, with a thin ctypes binding. Beside it: the rotation of
queries and keys (norm_rope), and a paged cache for layers that keep their whole history (BuzzPaged: rows in and
out, attention of one new token, choice of pages)."""
from .binding import (BUZZ_BF16, BUZZ_E4M3, BUZZ_F32, BUZZ_FLAG_LOGN, BUZZ_I8, Buzz, BuzzError, BuzzPaged,  # noqa: F401
                      error_string, exported_symbols, load_library, norm_rope)
