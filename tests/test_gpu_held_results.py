"""The tests of attention over pools in 4 bits once more, compared so that NaN does not pass."""
import pytest

import test_gpu_held
import test_gpu_held_edges
from held_calls import Call
from test_gpu_held import (test_a_bound_below_the_rows, test_attention, test_attention_into_rows_with_gaps_and_without_logarithms,  # noqa: F401
                           test_pages_outside_the_pool_are_not_seen, test_queries_and_scales_of_all_sizes, test_rows_that_see_nothing,
                           test_what_is_not_seen_may_be_held_with_anything)
from test_gpu_held_edges import (test_a_prefix_row_that_is_too_short, test_heads_of_one_value, test_rows_far_from_zero,  # noqa: F401
                                 test_rows_that_end_inside_the_prefix, test_tokens_that_no_request_covers)

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def strictly(monkeypatch):
    for module in (test_gpu_held, test_gpu_held_edges):
        monkeypatch.setattr(module, "Attend", Call)
