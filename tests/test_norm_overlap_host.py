"""Outputs of the norm over its operands: in their place or beside them, nothing between.  Refused before any HIP call."""
import pytest

from paper_2504_04673_amd import binding

P = 1 << 20          # an aligned address that is never used
EINVAL, ECAPACITY = -1, -2


def fwd(X, ldx, Y, ldy, m=100, C=24, dtype=0):
    # (no room in the workspace: what is not refused for its places ends there)
    return binding._calls().group_norm_act_fwd(dtype, X, ldx, P, 4, 0, m * 5000, C, 3, None, None, 1e-5, 1, Y, ldy, P, P, P, 0, None)


def bwd(X, ldx, G, ldg, Y, ldy, m=100, C=24, dtype=0):
    return binding._calls().group_norm_act_bwd(dtype, X, ldx, G, ldg, P, 4, 0, m * 5000, C, 3, None, None, 1, P, P, Y, ldy, P, P, P, 0, None)


FAR = P + (1 << 36)


@pytest.mark.parametrize("at,ldi,out,ldo", [
    (P, 24, P, 25), (P, 30, P, 24), (P, 24, P + 4, 24), (P, 64, P + 23 * 4, 64), (P + 40 * 4, 64, P + 17 * 4, 64), (P, 47, P + 24 * 4, 47), (P, 24, P + 24 * 4, 24),
    (P, 64, P + 64 * 4000 * 4 + 4, 64), (P + 64 * 4000 * 4, 64, P, 65)])
def test_overlaps_are_refused(at, ldi, out, ldo):
    assert fwd(at, ldi, out, ldo) == EINVAL
    assert bwd(at, ldi, FAR, 24, out, ldo) == EINVAL
    assert bwd(FAR, 24, at, ldi, out, ldo) == EINVAL


@pytest.mark.parametrize("at,ldi,out,ldo", [
    (P, 24, P, 24), (P, 30, P, 30), (P, 48, P + 24 * 4, 48), (P + 24 * 4, 48, P, 48), (P, 64, P + 40 * 4, 64), (P + 64 * 4000 * 4 + 30 * 4, 64, P, 64),
    (P, 24, P + 500000 * 24 * 4, 24), (P + 500000 * 24 * 4, 30, P, 24), (P, 24, FAR, 77)])
def test_places_that_are_taken(at, ldi, out, ldo):
    """(Nothing is launched: there is no workspace.)"""
    assert fwd(at, ldi, out, ldo) == ECAPACITY
    assert bwd(at, ldi, FAR * 2, 24, out, ldo) == ECAPACITY
    assert bwd(FAR * 2, 24, at, ldi, out, ldo) == ECAPACITY
