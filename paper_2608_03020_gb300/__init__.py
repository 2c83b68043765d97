"""LoCA forward-only adaptation hot path on one GB300 (sm_103a).

The CUDA library ``libloca.so`` (``csrc/``, C ABI in ``include/loca.h``) holds the kernels;
``paper_2608_03020_gb300.loca`` is its Python binding.  Build with ``_build.build()``.
"""

from . import loca  # noqa: F401
from .loca import (  # noqa: F401
    AdapterPlan,
    AdapterSet,
    GradClip,
    LOCA_BF16,
    LOCA_F32,
    LocaError,
    Pass,
    Q4Weight,
    loca_accumulate,
    loca_adapter_apply,
    loca_adapter_backward,
    loca_calib_fit,
    loca_device_status,
    loca_error,
    loca_gated,
    loca_gated_backward,
    loca_head_distill,
    loca_head_distill_backward,
    loca_head_loss,
    loca_head_loss_backward,
    loca_q4_apply,
    loca_ridge_solve,
    loca_targets,
    loca_version,
)
