"""Few-Bit Backward hot path for NVIDIA B200: Python binding of the C ABI.

Every step of the path runs in the CUDA library ``libfewbit.so`` (built
in-tree by ``paper_2202_00441_b200.build``); this package only marshals
arguments.  PyTorch supplies device memory and streams.  There is no CPU
fallback: if the library is missing, every call raises.
"""
from .binding import (  # noqa: F401
    ACTS, FewbitError, Table, fewbit_table_create, fewbit_table_create_ex, fewbit_table_create_folded, fewbit_table_create_opt, fewbit_table_from_arrays,
    fewbit_packed_bytes, fewbit_fwd, fewbit_fwd_bias, fewbit_bwd, fewbit_fwd_host, fewbit_bwd_host,
    fewbit_host_workspace_bytes, fewbit_launch_count, library_path, load_library,
    fewbit_fwd_host_static, fewbit_static_max_elements, fewbit_f32_activation_scan,
    fewbit_set_option, fewbit_get_option, fewbit_tail_warp_count,
)
from .operators import (  # noqa: F401
    fewbit_adamw_create, fewbit_adamw_step, fewbit_add_rms_norm_bwd, fewbit_add_rms_norm_fwd, fewbit_attention_bwd, fewbit_attention_fwd,
    fewbit_attention_timeout_count, fewbit_dropout_bwd, fewbit_dropout_fwd, fewbit_qk_norm_rope_bwd, fewbit_qk_norm_rope_fwd,
    fewbit_relative_bias_bwd, fewbit_relative_bias_fwd,
)
from . import workloads  # noqa: F401
from .autograd import (  # noqa: F401
    FewBitActivation, fewbit_activation, fewbit_add_rms_norm, fewbit_attention, fewbit_dropout, fewbit_qk_norm_rope,
    fewbit_relative_bias,
)
from .optim import FewBitAdamW  # noqa: F401
