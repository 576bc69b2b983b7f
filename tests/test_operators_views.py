"""Views that the binding takes and refuses: a row's elements have to be neighbours, however many rows there are.  No GPU: what is
asked of a tensor is asked of one that says it is on one, and every call here is refused before the library is called."""
import pytest
import torch

import paper_2504_04673_amd as sagnn
from paper_2504_04673_amd import binding


class OnGpu(torch.Tensor):
    """A tensor of the host that calls itself one of the GPU, its views too."""
    @property
    def is_cuda(self):
        return True


def gpu(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnGpu)


def one_row_views(f, dtype):
    """Rows whose elements are not neighbours: every other one, a column turned, one value repeated."""
    wide = gpu(f, 2 * f + 3, dtype=dtype)
    return {"every other": wide[1:2, :2 * f:2], "a column": wide[:, 3:4].t(), "repeated": gpu(1, dtype=dtype).expand(1, f)}


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind", ["every other", "a column", "repeated"])
def test_one_row_of_elements_apart_is_refused(kind, dtype):
    f = 8
    bad, good = one_row_views(f, dtype)[kind], gpu(1, f, dtype=dtype)
    assert bad.shape == (1, f)
    off, W, stats = gpu(2, dtype=torch.int32), gpu(1, f, f, dtype=dtype), gpu(1, 2)
    calls = [lambda: sagnn.grouped_gemm_act(bad, W, off), lambda: sagnn.grouped_gemm_act(good, W, off, mask=bad),
             lambda: sagnn.grouped_gemm_act(good, W, off, out=bad), lambda: sagnn.grouped_gemm_bwd(bad, W, off, good),
             lambda: sagnn.grouped_gemm_bwd(good, W, off, bad), lambda: sagnn.grouped_gemm_bwd(good, W, off, good, mask=bad),
             lambda: sagnn.group_norm_act(bad, 2), lambda: sagnn.group_norm_act(good, 2, out=bad),
             lambda: sagnn.group_norm_act_bwd(bad, good, stats, stats, 2), lambda: sagnn.group_norm_act_bwd(good, bad, stats, stats, 2),
             lambda: sagnn.group_norm_act_bwd(good, good, stats, stats, 2, out=bad)]
    if dtype is torch.float32:
        rows, csr = gpu(1, dtype=torch.int32), (gpu(2, dtype=torch.int32), gpu(0, dtype=torch.int32), gpu(0))
        calls += [lambda: sagnn.spmm_pack_rows(bad, rows), lambda: sagnn.spmm_pack_rows(good, rows, out=bad),
                  lambda: sagnn.spmm_csr_tallskinny(*csr, bad), lambda: sagnn.spmm_csr_tallskinny(*csr, good, C=bad),
                  lambda: sagnn.dense_gemm_act(bad, W[0]), lambda: sagnn.dense_gemm_act(good, bad, transW=True),
                  lambda: sagnn.gcn_layer_fwd(*csr, bad, W[0])]
    for call in calls:
        with pytest.raises(ValueError, match="rows must be contiguous"):
            call()


@pytest.mark.parametrize("check", [binding._mat, binding._typed])
def test_rows_of_neighbouring_elements_are_taken(check):
    wide = gpu(6, 20)
    for t in (wide, wide[:, 3:9], wide[2:3, 3:9], wide[:, 4:5], wide[::2, :7], wide[1:2, 1:2], wide[:, 3:4].t()[:, :1], gpu(0, 5), gpu(5, 0),
              wide[:, :0], wide[:0, ::2], wide[:, ::2][:, :1], gpu(4, 1, 3)[:, 0]):
        assert check(t, "t") is t
        assert binding._ld(t) >= t.shape[1]
    for t in (wide[:, ::2], wide.t(), gpu(20).expand(3, 20), gpu(1).expand(3, 1), wide[:, 3:4].t(), wide[2:3, ::3]):
        with pytest.raises(ValueError, match="rows must be contiguous"):
            check(t, "t")
