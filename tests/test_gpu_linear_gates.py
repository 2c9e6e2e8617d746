"""Tiles of 256 and 128 whose tokens lie under two rows of gates, in half
precision, with an activation and without, onto a residual and onto itself."""
import pytest
import torch

from test_gpu_linear_epilogue import epilogue_call

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act", ["none", "silu", "gelu"])
@pytest.mark.parametrize("M,N,K", [(4200, 4100, 256), (4200, 4128, 95), (2100, 2050, 128)])
@pytest.mark.parametrize("rows", [1, 300, 1000])
def test_rows_of_gates_that_meet_in_a_tile(act, M, N, K, rows):
    kw = dict(act=act, residual=True, rows=rows)
    assert torch.equal(epilogue_call(M, N, K, "i8", "f16", **kw), epilogue_call(M, N, K, "i8", "f16", in_place=True, **kw))
