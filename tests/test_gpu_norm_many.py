"""The norm and its gradients with eight rows and more a team of warps, so that the places of the rows on their way are used over and over: teams of one, three, five, eight and
sixteen warps, and blocks of columns. Bounds are test_gpu_norm's."""
import pytest
import torch

import paper_2605_26845_b200 as ms
from test_gpu_norm import check, inputs

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZES = [(20001, 256), (20001, 264), (20001, 40), (6001, 1032), (3601, 2056), (2501, 4096), (1201, 8192), (701, 8200), (701, 16392)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,D", SIZES)
def test_many_rows_a_team(rows, D, dtype):
    check(rows, D, TYPES[dtype], True, None, seed=rows + D)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,D", SIZES)
def test_every_row_counts_once(rows, D, dtype):
    """With one row alone of a gradient, dw is that row's and the other rows have none: a row that was passed over, taken twice or mixed with another shows."""
    x, _, w, dy, _ = inputs(rows, D, TYPES[dtype], 5)
    rstd = ms.rms_norm(x, w, save=True)["rstd"]
    each = ms.rms_norm_backward(dy, x, w, rstd)
    for row in (0, 1, rows // 2, rows - 149, rows - 1):
        one = torch.zeros_like(dy)
        one[row] = dy[row]
        got = ms.rms_norm_backward(one, x, w, rstd)
        want = (dy[row].float() * rstd[row]) * x[row].float()
        assert torch.equal(got["dweight"], want.to(x.dtype))
        assert torch.equal(got["dx"][row], each["dx"][row]) and torch.count_nonzero(got["dx"]) == torch.count_nonzero(got["dx"][row])
