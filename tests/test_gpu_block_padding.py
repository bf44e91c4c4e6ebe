"""What lies behind the d elements of rows in 8 bits is stored as zeros are, whatever the rows hold."""
import numpy as np
import pytest
import torch

from test_gpu_block import _normal

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [1, 5, 30, 100, 300, 999, 1030, 2049, 4100, 9001, 16390, 20001])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_padding_of_rows_with_nan_and_infinities(d, dtype):
    import paper_2403_08245_amd as smoe
    x = _normal((5, d), 1, dtype)
    x[0, 0], x[1, d - 1], x[2], x[3, d // 2] = float("nan"), float("inf"), float("nan"), float("-inf")
    w = torch.ones(d, dtype=dtype)
    for rows in (smoe.add_norm_fwd(x.cuda(), w.cuda(), packed=True).Y8, smoe.add_norm_fwd(x.cuda(), w.cuda(), x.cuda(), packed=True, plain=False).Y8, smoe.rows8_pack(x.cuda())):
        values, exps = rows.values.cpu().numpy(), rows.exps.cpu().numpy()
        assert ((values[:, d:] & 0x7F) == 0).all()
        assert (exps[:, -(-d // 32):] == 1).all()
