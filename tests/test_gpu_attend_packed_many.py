"""The tests of ckv_attend_packed once more, with an estimate of rows so large that the many-rows kernel takes
every call: small batches would reach only the other one."""
import pytest

from tests import test_gpu_attend_packed as A
from tests import test_gpu_attend_packed_paths as B
from tests.packed_util import PackedBatch

pytestmark = pytest.mark.gpu

MANY = 1 << 28
OWN_CONTEXT = ("test_captured_step_serves_grown_caches", "test_two_contexts_on_two_streams", "test_workspace_limit")


@pytest.fixture(scope="module")
def ckv():
    import paper_2608_07855_amd as P
    ctx = P.Context(0)
    ctx.set_kernel_timing(True)
    yield P, ctx
    ctx.close()


@pytest.fixture(autouse=True)
def many_rows(monkeypatch, ckv, request):
    """Every batch's view says MANY rows; the join of the shares, which only that kernel has, was launched (where a test
    has a context of its own, nothing counts launches)."""
    device = PackedBatch.device
    monkeypatch.setattr(PackedBatch, "device", lambda self, P, fill=0xFF, max_rows=None: device(self, P, fill, MANY))
    ckv[1].reset_kernel_stats()
    yield
    stats = ckv[1].kernel_stats()
    if request.node.originalname not in OWN_CONTEXT:
        assert "attend" in stats and stats["attend_join"][1] == stats["attend"][1]


test_single_tokens = A.test_single_tokens
test_prompts = A.test_prompts
test_few_rows = A.test_few_rows
test_window_edges = A.test_window_edges
test_gapped_positions = A.test_gapped_positions
test_any_batch = A.test_any_batch
test_given_positions = A.test_given_positions
test_empty_sequences = A.test_empty_sequences
test_many_sequences = A.test_many_sequences
test_long_axis = A.test_long_axis
test_scale = A.test_scale
test_zero_queries = A.test_zero_queries
test_values_of_any_size = A.test_values_of_any_size
test_many_small_weights = A.test_many_small_weights
test_hidden_tokens_hold_anything = A.test_hidden_tokens_hold_anything
test_large_logits = A.test_large_logits
test_same_bits_again = A.test_same_bits_again
test_one_long_cache = B.test_one_long_cache
test_many_heads = B.test_many_heads
test_rows_that_differ_by_much = B.test_rows_that_differ_by_much
test_blocks_in_several_shares = B.test_blocks_in_several_shares
test_far_storage = B.test_far_storage
test_a_row_beside_larger_ones = B.test_a_row_beside_larger_ones
test_a_row_of_nan_stays_alone = B.test_a_row_of_nan_stays_alone
test_captured_step_serves_grown_caches = A.test_captured_step_serves_grown_caches
test_two_contexts_on_two_streams = A.test_two_contexts_on_two_streams
test_workspace_limit = A.test_workspace_limit
