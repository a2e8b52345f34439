"""GB300-native Curvature-Conditioned Query (arxiv 2606.01294) kernels.

The hot path -- CCQ-GLA / CCQ-Gated-DeltaNet chunkwise forward and the CCQ
decode step -- runs in libccq.so (hand-written sm_103a CUDA, C ABI in
include/ccq.h), and so do the operators around the mixer (:mod:`.ops`, C ABI in
include/ccq_ops.h).  This package is its thin binding; it needs a CUDA device.
"""
from . import ops  # noqa: F401
from .ccq import (  # noqa: F401
    CCQError,
    CCQState,
    GDN,
    GLA,
    decode_step,
    device_status,
    gdn_fwd,
    gla_fwd,
    load_library,
)
