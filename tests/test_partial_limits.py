"""Descriptors of kvshot_page_bounds without query heads, on the CPU."""
import pytest

from paper_2604_26412_gb300 import kvshot

from .test_partial_boundary import ALIGN, NULL, SHAPE, UNSUPPORTED, A, bounds, lib, scores, sparse, weights  # noqa: F401

ABSENT = dict(hq=0, n_nodes=0, n_query=0, n_max=0)


def test_bounds_without_query_heads():
    assert bounds({"k": None}, **ABSENT) == NULL  # (past the descriptor's checks)
    assert bounds({"out": A + 8}, **ABSENT) == ALIGN
    assert bounds({"k": None}, **(ABSENT | dict(hq=8))) == NULL


@pytest.mark.parametrize("kw,code", [(dict(hkv=0), SHAPE), (dict(hkv=-1), SHAPE), (dict(hq=-8), SHAPE), (dict(hq=30), SHAPE),
                                     (dict(head_dim=64), UNSUPPORTED), (dict(page_size=12), UNSUPPORTED), (dict(num_pages=0), SHAPE)])
def test_what_is_given_is_still_checked(kw, code):
    assert bounds(**(ABSENT | kw)) == code


@pytest.mark.parametrize("call", [scores, sparse, weights])
def test_the_calls_with_queries_need_their_heads(call):
    assert call(**ABSENT) == SHAPE
