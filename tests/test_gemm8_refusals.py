"""mcd_tc_gemm_e4m3 without a GPU: the error word lies in no other array (pointers are made up and never read)."""
import pytest

from test_rows_refusals import INVALID, P, Q, gemm_call, lib      # noqa: F401 (lib: the fixture)


@pytest.mark.parametrize("err", [P, P + 64 * 127 + 60, Q + 4, 2 * Q, 2 * Q + 4 * 128 * 16 - 4, 5 * Q + 8, 6 * Q + 60])
def test_the_error_word_overlaps_nothing(lib, err):                # noqa: F811
    assert gemm_call(lib, sa=5 * Q, sb=6 * Q, err=err) == INVALID
