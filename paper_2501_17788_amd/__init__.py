"""WARP multi-vector search engine for AMD Instinct MI355X (gfx950).

The search path (WARP_SELECT, implicit decompression, two-stage reduction,
top-k) runs in hand-written HIP kernels behind the C ABI of include/warp.h;
`warp` is its Python binding. `encoder` binds the operators of the token encoder's head
from the same library: layer norm, int8 products and the AdamW step.
"""
from .warp import (  # noqa: F401
    EINVAL, EDEVICE, ENOMEM, ENOTSUP, EXPORTS, FRAC_BITS, SCORING_EQ1_LITERAL, SCORING_PAPER, STAGES, T_PRIME_C,
    T_PRIME_MAX, Index, WarpError, build_index, initial_centroids, last_error, lib, sample_passages, t_prime_policy,
)

try:
    from .encoder import (  # noqa: F401
        AdamW, QuantizedRows, layer_norm, layer_norm_backward, layer_norm_int8, linear_int8, quantize_rows,
    )
except ImportError as e:  # search needs neither torch (for host arrays) nor the operators' binding
    _missing = e

    def __getattr__(name):
        if name in ("AdamW", "QuantizedRows", "layer_norm", "layer_norm_backward", "layer_norm_int8", "linear_int8",
                    "quantize_rows"):
            raise ImportError(f"{name} needs torch and _encoder.so: {_missing}") from _missing
        raise AttributeError(f"module {__name__!r} has no attribute {name!r}")
