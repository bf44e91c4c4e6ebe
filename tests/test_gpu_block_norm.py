"""The norm at the ends of its types: rows whose squares leave fp32 at either end, with and without eps, and the padding of rows in 8 bits."""
import numpy as np
import pytest
import torch

import oracle
from test_gpu_block import HALF, NORM_UNITS, _f64, _log, _near, _near_packed, _normal

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def smoe():
    import paper_2403_08245_amd as m
    return m


WIDTHS = [1, 7, 128, 300, 1000, 2048, 4097, 20000]


@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("eps", [0.0, 1e-44, 1e-36, 1e-25, 1e-6, 1e30])
def test_rows_of_all_sizes(smoe, d, dtype, eps):
    """Values from 2^-149, the smallest fp32 has, to next to its end; mixed sizes in a row are not lost either."""
    _log(f"norm sizes {d} {dtype} {eps}")
    e = torch.tensor([-146.0, -140, -130, -126, -110, -90, -75, -70, -65, -50, -49, -40, -20, 0, 30, 60, 63, 64, 70, 100, 122])
    x = (_normal((len(e), d), 1, torch.float32).clamp(-4, 4).double() * 2.0 ** e.double()[:, None]).to(dtype)
    if d > 1:
        x[:, 0] *= 2.0 ** -20
    x[x == 0] = 2.0 ** -133                                   # bf16's smallest; what was rounded to nothing
    w = (1 + 0.3 * _normal((d,), 2, torch.float32)).to(dtype)
    n = smoe.add_norm_fwd(x.cuda(), w.cuda(), eps=eps, packed=True)
    eps = float(np.float32(eps))
    _, y, rstd = oracle.add_norm(_f64(x), None, _f64(w), eps)
    tol = (NORM_UNITS + 2.0 ** -23) * np.abs(y) + 2.0 ** -148                # under 2^-126 fp32 has fewer bits
    _near(n.Y, y, HALF[dtype] * np.abs(y) + 1.01 * tol + (2.0 ** -134 if dtype == torch.bfloat16 else 0), "Y")
    _near_packed(smoe, n.Y8, y, tol)
    held = rstd < 2.0 ** 127
    _near(n.rstd[torch.from_numpy(held).cuda()], rstd[held], NORM_UNITS * rstd[held], "rstd")
    assert torch.isinf(n.rstd[torch.from_numpy(rstd > 2.0 ** 128).cuda()]).all()


def test_zero_rows_without_eps(smoe):
    """0 / 0, as the definition has it."""
    x, w = torch.zeros(3, 100, device="cuda"), torch.ones(100, device="cuda")
    n = smoe.add_norm_fwd(x, w, eps=0.0)
    assert torch.isnan(n.Y).all() and torch.isinf(n.rstd).all()
    assert (smoe.add_norm_fwd(x, w, eps=1e-45).Y == 0).all()


@pytest.mark.parametrize("rows,d", [(1999, 999), (5000, 264), (700, 2048)])
def test_weight_gradient_in_fp32_in_the_root_mean_square(smoe, rows, d):
    """Roundings of 2^-24 / sqrt(3) = 3.4e-8 at most in the root mean square: the result's, u's, rstd's twice, and those of the sums of a thread's 2 to 16 rows, of which the last are as
    large as the sum: sqrt(3.4^2 + 3.4^2 + 2 * 3.4^2 + 2 * 3.4^2) = 8.3e-8.  The sum over the blocks is in 64 bits."""
    X, w, dY = _normal((rows, d), 1, torch.float32), 1 + 0.1 * _normal((d,), 2, torch.float32), _normal((rows, d), 3, torch.float32)
    n = smoe.add_norm_fwd(X.cuda(), w.cuda())
    dw = smoe.add_norm_bwd(dY.cuda(), n.S, w.cuda(), n.rstd)[1]
    x = _f64(X)
    want = (_f64(dY) * x / np.sqrt((x * x).mean(-1, keepdims=True) + float(np.float32(1e-6)))).sum(0)
    off = np.sqrt(np.mean((_f64(dw) - want) ** 2) / np.mean(want ** 2))
    _log(f"dweight {(rows, d)} {off:.2e}")
    assert off <= 1e-7


@pytest.mark.parametrize("d", [1, 2, 500])
def test_mean_square_and_eps_past_fp32_together(smoe, d):
    """Each of them within fp32's range (500 elements: the sum of the squares is not), their sum past it."""
    for dtype in (torch.bfloat16, torch.float32):
        x, w = (torch.linspace(1.0, 1.25, 4 * d).view(4, d) * 2.0 ** 63).to(dtype), torch.ones(d, dtype=dtype)
        n = smoe.add_norm_fwd(x.cuda(), w.cuda(), eps=3e38)
        _, y, rstd = oracle.add_norm(_f64(x), None, np.ones(d), float(np.float32(3e38)))
        _near(n.Y, y, (HALF[dtype] + 1.01 * NORM_UNITS + 2.0 ** -23) * np.abs(y), "Y")
        _near(n.rstd, rstd, NORM_UNITS * rstd, "rstd")
