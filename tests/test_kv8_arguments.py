"""More refusals of the 8-bit cache calls that need no device."""
import pytest


@pytest.fixture(scope="module")
def B():
    from paper_2405_14371_b200 import build
    build.build()
    from paper_2405_14371_b200 import binding
    return binding


A = 1 << 20            # stands for an aligned device address that a refused call never touches


@pytest.mark.parametrize("max_rows", [8, 5000])
def test_plan_takes_no_result_in_place_of_the_lengths_asked_for(B, max_rows):
    """In large calls a second kernel tells served requests from refused ones by comparing len_out with new_len."""
    new = 2 * A
    assert B.lib.es_op_kv_plan(A, new, A, A, A, 2, 4, 16, 8, max_rows, A, A, A, A, A, new, None) == 1
    assert "len_out" in B.es_last_error()
