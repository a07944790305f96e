"""The gradient of RMS norm at sizes that reach each form of its row kernel: units a
warp, rows a set, and with rows of 8193 to 16384 fp32 values one set at a time on the way.
The tolerances are those of test_gpu_rms.py."""

import pytest

from .gpu_common import lib_ready, torch_cuda
from .test_gpu_rms import U, chain, data, half_step

pytestmark = pytest.mark.gpu
# rows and columns: one to eight units a warp, few rows and many, the sizes at which the form changes and their neighbours
SIZES = [(1, 128), (2431, 128), (2432, 128), (2432, 250), (2433, 256), (1, 2176), (1216, 384), (2432, 384), (1216, 640), (2000, 640), (2000, 637),
         (500, 4224), (607, 4223), (700, 8192), (153, 8193), (40, 9000), (700, 9001), (153, 12000), (700, 12001), (31, 16383), (310, 16384)]


@pytest.mark.parametrize("joined", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("size", SIZES)
def test_gradients_of_every_form(size, dtype, joined):
    torch = torch_cuda()
    ff = lib_ready()
    rows, cols = size
    i = SIZES.index(size)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    gamma = torch.randn(cols, generator=torch.Generator().manual_seed(i)).cuda()
    for pad, lead in ((0, 0), (2, 2), (3, 1)):
        h, dy = (data(torch, rows, cols, dt, pad, lead, seed=100 * k + i) for k in range(2))
        dh = data(torch, rows, cols, dt, pad, lead, seed=200 + i) if joined else None
        _, _, rstd = ff.rms_norm(h, gamma)
        dx, dgamma = ff.rms_norm_backward(dy, h, rstd, gamma, dh=dh)
        r = rstd.double()[:, None]
        n, du = h.double() * r, dy.double() * gamma.double()
        mean, mean_abs = (du * n).mean(1, keepdim=True), (du * n).abs().mean(1, keepdim=True)
        want = r * (du - n * mean) + (dh.double() if joined else 0.0)
        tol = U * r * (8 * du.abs() + n.abs() * mean_abs * (chain(cols) + 16)) + want.abs() * (2 * U + half_step(torch, dt))
        assert bool(((dx.double() - want).abs() <= tol + 2.0 ** -130).all())
        terms = dy.double() * n
        depth = 128 + rows // 4096 + 32
        assert bool(((dgamma.double() - terms.sum(0)).abs() <= (depth + 3) * U * terms.abs().sum(0) + 2.0 ** -140).all())
        again = ff.rms_norm_backward(dy, h, rstd, gamma, dh=dh)
        assert torch.equal(dx, again[0]) and torch.equal(dgamma, again[1])
