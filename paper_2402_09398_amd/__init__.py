"""lessdec: the LESS decode hot path (H2O-evicted KV cache + low-rank state) for MI355X.

`binding` is the ctypes front end of the HIP library, `pages` that of its paged 8-bit cache, `beams` that of the choice of beams, `workloads` the seeded synthetic
inputs, `build` the in-tree build of liblessdec.so.
"""
from . import beams, binding, pages, workloads  # noqa: F401
from .beams import BeamSearch, lessdec_beam_select, lessdec_beam_workspace_bytes  # noqa: F401
from .binding import (LessDec, LessdecError, lessdec_budget_tokens, lessdec_prefill, lessdec_probe_stream_read,  # noqa: F401
                      lessdec_state_reset, lessdec_state_select, lessdec_state_sync, lessdec_step, lessdec_step_attend,
                      lessdec_step_features, lessdec_step_static, lessdec_workspace_bytes, pack_weights)
from .pages import (PagedCache, lessdec_pages_append, lessdec_pages_attend, lessdec_pages_compact, lessdec_pages_copy,  # noqa: F401
                    lessdec_pages_attend_shared, lessdec_pages_read, lessdec_pages_reserve, lessdec_pages_reset, lessdec_pages_select,
                    lessdec_pages_share, lessdec_pages_share_ints, lessdec_pages_shared_workspace_bytes, lessdec_pages_workspace_bytes)
