"""BEVPoolv2 view-transform path for AMD Instinct MI355X (gfx950).

HIP kernels behind the C ABI of include/bevpool.h, include/bevpool_rows.h and
include/bevpool_logits.h, with thin ctypes bindings
(``paper_2211_17111_amd.bevpool`` for the pooling path,
``paper_2211_17111_amd.rows`` for the row operators,
``paper_2211_17111_amd.logits`` for the logits operators).
"""

from .bevpool import (  # noqa: F401
    BEVPOOL_F16,
    BEVPOOL_F32,
    BevpoolError,
    Plan,
    Schedule,
    backward,
    backward_scheduled,
    bev_pool,
    bevpool_backward,
    bevpool_backward_scheduled,
    bevpool_backward_workspace_size,
    bevpool_forward,
    bevpool_forward_scheduled,
    bevpool_forward_scheduled_workspace_size,
    bevpool_forward_workspace_size,
    bevpool_last_error,
    bevpool_prepare,
    bevpool_prepare_workspace_size,
    bevpool_schedule,
    bevpool_schedule_size,
    bevpool_strerror,
    bevpool_version,
    declared_symbols,
    forward,
    forward_scheduled,
    forward_scheduled_workspace,
    load_library,
    prepare,
    schedule,
)
from .logits import (  # noqa: F401
    Logprobs,
    distill,
    distill_backward,
    distill_forward,
    distill_step,
    logprobs,
    logprobs_backward,
    logprobs_forward,
)
from .rows import (  # noqa: F401
    BEVPOOL_BF16,
    KeyOrder,
    combine,
    combine_backward,
    combine_forward,
    dispatch,
    dispatch_backward,
    dispatch_forward,
    embed,
    embed_backward,
    embed_forward,
    expert_layer_forward,
    route,
    route_backward,
    route_forward,
    sort_keys,
)
