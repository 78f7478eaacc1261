"""GB300 (sm_103a) Mutual Pair Merging: C-ABI CUDA library + thin binding.

The compute path lives in ``libmpm.so`` (CUDA kernels for sm_103a, built by
``paper_2604_05718_gb300.build.build()``); ``paper_2604_05718_gb300.mpm``
(the merge), ``paper_2604_05718_gb300.blocks`` (the encoder blocks around it:
fused norms, 4-bit linear layers) and ``paper_2604_05718_gb300.attention``
(attention between packed sequences, rotary positions) marshal torch tensors
into its C entry points.
"""

from .attention import (  # noqa: F401
    AttentionGrads,
    AttentionStats,
    cross_attention,
    cross_attention_backward,
    cross_attention_workspace,
    rotary,
    rotary_backward,
    rotary_frequencies,
)
from .blocks import (  # noqa: F401
    MXFP4,
    BlockNormGrads,
    block_norm,
    block_norm_backward,
    block_norm_workspace,
    dequantize_mxfp4,
    matmul_mxfp4,
    quantize_mxfp4,
)
from .mpm import (  # noqa: F401
    MPMError,
    compose_gather,
    compose_maps,
    device_status,
    library,
    merge,
    merge_no_alloc,
    nearest_neighbors,
    new_workspace,
    no_alloc_device_status,
    pad_batch,
    selftest_wait_timeout,
    trace_read,
    trace_reset,
    unmerge_gather,
    unpad_batch,
    workspace_size,
)
