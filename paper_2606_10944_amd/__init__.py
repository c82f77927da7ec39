"""thin: MI355X-native thinned attention (kernel halving under kappa_att +
coreset attention), after "Express Language Modeling".

The compute path lives in the HIP library libthin.so (C ABI in include/thin.h);
this package only binds it.
"""
from ._lib import (THIN_BF16, THIN_EDTYPE, THIN_EHIP, THIN_EINVAL, THIN_EUNIFORMS,  # noqa: F401
                   THIN_EWORKSPACE, THIN_FP32, THIN_OK, ExpressCache, LaunchTimer, ThinError,
                   thin_attention, thin_compress, thin_express_plan, thin_express_prefill,
                   thin_express_prefill_plan, thin_plan,
                   thin_selftest_gram16, thin_status_str, workspace_status)
from .grad import coreset_attention, thin_attention_backward  # noqa: F401
from .q4 import (Q4Cache, thin_q4_attention, thin_q4_keep, thin_q4_load,  # noqa: F401
                 thin_q4_select, thin_q4_store, thin_q4_tree, thin_q4_tree_attention, thin_rotary,
                 thin_rotary_axes, thin_rotary_turns)
