"""MI355X-native hot path of entropy-routed stitched decoding.

The product is ``librstitch.so`` (HIP kernels for gfx950 behind a C ABI, see
``include/rstitch.h``); this package is its thin Python binding.  There is no
CPU fallback: importing the binding without the built library raises.
"""

from .binding import (  # noqa: F401
    RS_SLM, RS_LLM, FLAG_HI, FLAG_ACCEPT, FLAG_NEXT_LLM, FLAG_NONFINITE, FLAG_BADARG, FLAG_ABORTED, FLAG_ROUTER_STAY, FLAG_NO_PAGE,
    RsError, RsConfig, RouteOut, lib, library_path,
    rs_abi_version, rs_last_error, rs_workspace_bytes, rs_kv_bytes, rs_create_model, rs_destroy_model,
    rs_decode_step, rs_catchup_prefill, rs_route, rs_route_plus, RouterPlus, rs_route_static, rs_route_scratch_bytes, rs_set_phase_timer, rs_set_spin_limit, rs_set_sampling,
    rs_stitch_generate, STITCH_RUNNING, STITCH_DONE, STITCH_TRACE_FULL, STITCH_FLAGGED, STITCH_ABORTED,
    RS_F32, RS_BF16, RS_SCORES_F64, ROPE_PLAIN, ROPE_LINEAR, ROPE_BY_PARTS, PagedCache, Rope, rs_rope_frequencies, rs_rope_rows, rs_paged_append,
    rs_paged_attention, rs_paged_attention_scratch_bytes, rs_paged_workspace_bytes, rs_create_model_paged,
    rs_beam_select, rs_beam_select_scratch_bytes, PagePool, rs_pages_scratch_bytes, rs_pages_reserve, rs_pages_release, rs_pages_fork, rs_pages_copy, rs_pages_compact,
    Model, PagedModel,
)
from .beam import Beam, BeamSearch  # noqa: F401
