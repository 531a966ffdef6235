"""B200-native chunked-prefill step with retaining-head eviction (Locret).

The package is a thin binding over ``liblocret.so`` (hand-written CUDA for sm_100a): ctypes, and the
compiled module ``_paged`` for the calls on pages, which a served batch makes many times a step.  Every step
of the path runs in the library's kernels; Python only marshals pointers.  There is no CPU fallback: importing
the binding without the built library raises, and so does asking for a call on pages without the module.
"""

from .binding import (  # noqa: F401
    K_NAMES,
    LAST_CHUNK,
    LayerStack,
    NO_EVICT,
    LocretBlock,
    LocretError,
    LocretLayer,
    LocretLayerTP,
    adamw_step,
    cis_labels,
    lib,
    lib_path,
    rh_loss_grad,
    shard_by_kv_head,
)
try:
    from .paged import (  # noqa: F401
        Pages,
        PagesStep,
        norm_rope,
        norm_rope_grad,
        paged_attention,
        pages_step,
        rope_turns,
    )
except ImportError as _error:
    # the rest of the package does not need the module: whoever asks for the calls on pages is told
    _why = str(_error)

    def __getattr__(name):
        if name in ("Pages", "PagesStep", "norm_rope", "norm_rope_grad", "paged_attention", "pages_step", "rope_turns"):
            raise ImportError(_why)
        raise AttributeError(f"module {__name__!r} has no attribute {name!r}")
