"""MI355X-native Variational Linear Attention forward, and the gated delta rule and the norm of queries and keys with the
position rotation, the selective state space scan with its short causal convolution, and the norms around a block next to it
(thin binding over libvla.so)."""
from .binding import (  # noqa: F401
    VLA_BF16,
    VLA_F32,
    MODE_AUTO,
    MODE_CHUNKED,
    MODE_SCAN,
    MODE_TIME_PARALLEL,
    MODE_TWO_PHASE,
    VlaError,
    lib_path,
    load_library,
    resolve_mode,
    status_string,
    version,
    vla_decode_step,
    vla_decode_step_raw,
    vla_forward,
    vla_forward_raw,
    vla_forward_static_raw,
    vla_forward_workspace_bytes,
)
from .causal_conv import causal_conv, causal_conv_backward, causal_conv_step  # noqa: F401
from .gated_delta import (  # noqa: F401
    gated_delta,
    gated_delta_backward,
    gated_delta_decode_step,
    gated_delta_forward,
)
from .qk_norm import qk_norm_rope, qk_norm_rope_backward  # noqa: F401
from .residual_norm import residual_norm, residual_norm_backward  # noqa: F401
from .selective_scan import (  # noqa: F401
    selective_scan,
    selective_scan_backward,
    selective_scan_forward,
    selective_scan_step,
)
