"""Host-side refusals of the 8-bit cache's calls where operands overlap what a call writes, and scalars leave fp32's range."""
import pytest

from paper_2411_15785_b200 import binding as B

from test_qcache_abi_cpu import A, _attend, _c, lib  # noqa: F401  (lib: a fixture)


def test_the_account_of_weight_may_not_overlap_what_the_call_reads(lib):
    # it is written while CTAs still read the others: the result would hang on their order
    for other in (A[7], A[0], A[1], A[2], A[3], A[5], A[6]):
        assert _attend(lib, _c(weight=other)) == B.BCT_ERR_INVALID_ARG, other
        assert "weight" in B.last_error() and "overlaps" in B.last_error()
    assert _attend(lib, _c(), lens=A[4] + 16) == B.BCT_ERR_INVALID_ARG and "weight overlaps lens" in B.last_error()


@pytest.mark.parametrize("kw", [dict(scale=3e38), dict(scale=2.5e38), dict(scale=10.0, cap=3e38), dict(scale=100.0, cap=2.4e38)])
def test_scales_and_caps_that_overflow_in_powers_of_two_are_refused(lib, kw):
    # scores are formed in powers of two: 1.4427 times these is above the largest float
    assert _attend(lib, _c(), **kw) == B.BCT_ERR_INVALID_ARG
    assert "range" in B.last_error()
