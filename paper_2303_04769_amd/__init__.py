"""MI355X-native (gfx950) implementation of the SMaLL abstract-layer hot path.

`binding` is a thin ctypes layer over libsmall_hip.so (the C ABI of include/small.h):
argument marshalling only, every step of the path runs in the HIP kernels. PyTorch is
used for device memory and streams. There is no CPU fallback: loading fails loudly when
the library is missing. `attn` is the same for the attention block (include/small_attn.h of this package), `cache` for rotary positions and the paged cache
(include/small_cache.h).
"""
from . import attn, binding, cache  # noqa: F401
from .binding import *  # noqa: F401,F403
from .attn import *  # noqa: F401,F403
from .cache import *  # noqa: F401,F403
