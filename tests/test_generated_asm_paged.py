"""The static checks of hand-issued LDS reads (test_generated_asm) on the kernels for a cache in pages."""
import pytest

from tests import test_generated_asm as checks


@pytest.fixture(scope="module", params=["sta_paged.hip", "sta_paged_weights.hip"])
def asm(request):
    return request.param, checks._assembly(request.param)


test_inline_assembly_is_only_lds_access_and_waits = checks.test_inline_assembly_is_only_lds_access_and_waits
test_hand_issued_lds_reads_are_waited_for_before_use = checks.test_hand_issued_lds_reads_are_waited_for_before_use
test_hand_written_vector_instructions_keep_their_distance = checks.test_hand_written_vector_instructions_keep_their_distance_from_matrix_instructions
