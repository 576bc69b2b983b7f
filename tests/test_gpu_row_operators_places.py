"""Results that take an operand's place."""
import pytest
import torch

import paper_2504_04673_amd as sagnn
from tests.test_gpu_row_operators import gen, normal

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("c", [5, 64, 602, 3001])
def test_norm_over_its_own_rows_has_no_sum_to_give(c, dtype):
    """Nothing is added or dropped, so that the sum is X, which the result has replaced: gradients of that would be wrong."""
    X, gamma = normal(gen(c), 40, c, dtype=dtype), normal(gen(1), c)
    Y, S, rstd = sagnn.rms_norm(X, gamma)
    assert S is X
    x = X.clone()
    y, s, r = sagnn.rms_norm(x, gamma, out=x)
    assert y is x and s is None and torch.equal(x, Y) and torch.equal(r, rstd)
    wide = torch.zeros(40, 2 * c + 3, dtype=dtype, device="cuda")
    wide[:, :c] = X
    y, s, r = sagnn.rms_norm(wide[:, :c], gamma, out=wide[:, :c])
    assert s is None and torch.equal(y, Y) and not wide[:, c:].any()
    # beside it, or where a sum is made, there is one
    wide[:, :c] = X
    y, s, r = sagnn.rms_norm(wide[:, :c], gamma, out=wide[:, c + 3:])
    assert torch.equal(s, X) and torch.equal(y, Y)
    x = X.clone()
    y, s, r = sagnn.rms_norm(x, gamma, p=0.5, seed=3, out=x)
    assert torch.equal(s, sagnn.dropout_add(X, 0.5, 3))
    x = X.clone()
    y, s, r = sagnn.rms_norm(x, gamma, residual=X, out_sum=x)
    assert s is x and torch.equal(x, X + X)


def test_norm_of_no_rows():
    x = torch.zeros(0, 8, device="cuda")
    assert sagnn.rms_norm(x)[1] is x
