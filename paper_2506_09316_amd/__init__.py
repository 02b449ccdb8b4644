"""MI355X-native dual-state linear attention (DSLA) layer forward.

The compute lives in a C-ABI shared library built from csrc/ (hand-written gfx950 HIP
kernels); `binding` is a thin ctypes layer with the same entry-point names.  Importing
the package does not load the library; the first call does, and fails loudly if the
library has not been built.
"""
from .binding import (dsla_project, dsla_attention_prefill, dsla_conversion_plan, dsla_kv_cache_bytes, dsla_max_conversion_rate, dsla_rank_layers,  # noqa: F401
                     )
from .binding import (DslaDesc, DslaError, DslaMulti, dsla_decode_multi, dsla_prefill_multi,  # noqa: F401
                      dsla_prefill_multi_workspace_bytes, make_multi,  # noqa: F401
                      dsla_attention_decode, dsla_attention_decode_workspace_bytes,  # noqa: F401
                      dsla_attention_entropy, dsla_attention_entropy_workspace_bytes,  # noqa: F401
                      dsla_decode, dsla_decode_slots, dsla_prefill, dsla_prefill_static_ws,  # noqa: F401
                      dsla_prefill_varlen, dsla_prefill_varlen_workspace_bytes, dsla_prefill_workspace_bytes,
                      dsla_state_init, library_path, load_library, make_desc, profile_collect, profile_enable)
from .binding import (DslaBatch, DslaCache, DslaRope, make_batch, make_cache, make_pools, make_rope,  # noqa: F401
                      dsla_attention_paged, dsla_attention_paged_workspace_bytes, dsla_cache_accept, dsla_cache_compact, dsla_cache_extend,
                      dsla_cache_fork, dsla_cache_init, dsla_cache_truncate, dsla_cache_workspace_bytes, dsla_qk_rope)
from .binding import (DSLA_ACT_NONE, DSLA_ACT_SIGMOID, DSLA_ACT_SILU, DSLA_BF16, DSLA_E4M3, DSLA_F32, DSLA_SCALE_E8M0, DSLA_SCALE_F32,  # noqa: F401
                      DslaHeads, DslaNorm, dsla_head_norm, dsla_project_fp8, dsla_quantize, dsla_residual_norm, make_head_norm, make_norm,
                      scale_pitch)
