"""Host-side refusals of the 8-bit cache's calls where operands overlap what a call writes."""
from paper_2411_15785_b200 import binding as B

from test_qcache_abi_cpu import A, _attend, _c, lib  # noqa: F401  (lib: a fixture)


def test_the_account_of_weight_may_not_overlap_what_the_call_reads(lib):
    # it is written while CTAs still read the others: the result would hang on their order
    for other in (A[7], A[0], A[1], A[2], A[3], A[5], A[6]):
        assert _attend(lib, _c(weight=other)) == B.BCT_ERR_INVALID_ARG, other
        assert "weight" in B.last_error() and "overlaps" in B.last_error()
    assert _attend(lib, _c(), lens=A[4] + 16) == B.BCT_ERR_INVALID_ARG and "weight overlaps lens" in B.last_error()
