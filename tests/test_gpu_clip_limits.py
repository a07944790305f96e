"""Gradient clipping at the ends of its range: limits and norms that are not
finite, and gradients whose squares fp32 cannot hold."""

import math

import pytest

from .gpu_common import lib_ready, torch_cuda

pytestmark = pytest.mark.gpu
COUNTS = {"cluster": [5000, 7], "two passes": [400000, 7], "several tables": [3000] * 130}


@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("path", list(COUNTS))
def test_an_infinite_limit_asks_for_the_norm_alone(path, dtype, value):
    torch = torch_cuda()
    ff = lib_ready()
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = [torch.randn(n, device="cuda").to(dt) for n in COUNTS[path]]
    g[0][g[0].numel() // 2] = value
    keep, out = [t.clone() for t in g], [torch.empty_like(t) for t in g]
    for into in (out, None):
        norm = float(ff.clip_grad_norm(g, math.inf, out=into))
        assert math.isnan(norm) if math.isnan(value) else norm == math.inf
        for t, k in zip(g if into is None else into, keep):
            assert torch.equal(t.nan_to_num(nan=-1.0), k.nan_to_num(nan=-1.0)) and torch.equal(t.isnan(), k.isnan())
            assert torch.equal(t.isinf(), k.isinf())
