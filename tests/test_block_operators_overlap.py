"""Outputs that are an input of the same call, or another output: refused before any launch."""
import pytest

from tests.test_block_operators_abi import (BACK, FFN, NORM, NORM_BACK, at, dm, ffn, ffn_backward, norm,  # noqa: F401
                                            norm_backward)

INVALID = 1


def pairs(outs, names, but=()):
    return [(o, n) for o in outs for n in names if n != o and (o, n) not in but]


@pytest.mark.parametrize("out,other", pairs(("pre", "h", "y"), FFN))
def test_expert_ffn(dm, out, other):  # noqa: F811
    assert ffn(dm, **{out: at(other, FFN)}) == INVALID


@pytest.mark.parametrize("out,other", pairs(("dpre", "dx", "dw_gate", "dw_up", "dw_down"), BACK))
def test_expert_ffn_backward(dm, out, other):  # noqa: F811
    assert ffn_backward(dm, **{out: at(other, BACK)}) == INVALID


# (r may be x and n may be y)
@pytest.mark.parametrize("out,other", pairs(("r", "n", "stats"), NORM, (("r", "x"), ("n", "y"))))
def test_norm_residual(dm, out, other):  # noqa: F811
    assert norm(dm, **{out: at(other, NORM)}) == INVALID


@pytest.mark.parametrize("out,other", pairs(("dx", "dy", "dgate", "dw_post", "dw_pre"), NORM_BACK))
def test_norm_residual_backward(dm, out, other):  # noqa: F811
    assert norm_backward(dm, **{out: at(other, NORM_BACK)}) == INVALID

