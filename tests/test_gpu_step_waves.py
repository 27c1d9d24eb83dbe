"""The tests of decode behind shared prefixes once more with each of its kernels in ranges: workgroups of four wavefronts and of eight, whatever the estimates say."""
import pytest

from paper_2404_09526_amd import binding as esp
from test_gpu_step import (test_decode_behind_shared_prefixes, test_shared_bounds_larger_than_what_is_there, test_shared_long_prefixes_of_many_columns,  # noqa: F401
                           test_shared_nan_and_infinite_keys_show_where_they_are_seen, test_shared_requests_past_the_stated_group_are_left_without_the_prefix,
                           test_shared_rows_named_twice_count_twice, test_shared_rows_past_4_gb_of_the_pool, test_shared_scores_far_apart)
from test_gpu_step_layouts import (test_a_prefix_longer_than_stated_is_read_as_far_as_that, test_offsets_past_the_slots_read_none, test_one_workspace_for_all_steps,  # noqa: F401
                                   test_slots_past_the_offsets_belong_to_no_request, test_unequal_groups)
from test_gpu_step_values import test_infinite_values_show_as_themselves  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.fixture(params=[4, 8], ids=["four", "eight"], autouse=True)
def form(request, cuda):
    before = esp.esp_debug_set_decode_plan(request.param)
    assert esp.esp_debug_decode_shared_plan(4, 1, 300, 300, 4, 100, 60, 4, 4) == request.param
    yield request.param
    assert esp.esp_debug_set_decode_plan(before) == request.param
