"""CommitKV hot path on MI355X (gfx950): HIP kernels behind a C ABI.

The compute runs in ``libcommitkv.so`` (``python -m paper_2608_07855_amd.build``);
this package only marshals torch tensors into its calls.
"""
from .binding import (Agent, CKVError, Context, Pages, batch_view, cache_view,  # noqa: F401
                      ckv_attend_packed, ckv_attend_shared, ckv_attend_window, ckv_build_slots,
                      ckv_classify_pages, ckv_joint_test, ckv_measure_page_effects,
                      ckv_measure_page_effects_batch, ckv_measure_recorded, ckv_pack_tokens,
                      ckv_pool_scores, ckv_select_and_compact, ckv_unpack_tokens,
                      kv_view, lib, packed_row_bytes, packed_view, query_view, slot_step, version, window_view, PAPER_THRESHOLDS)
