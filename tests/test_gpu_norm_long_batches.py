"""dgamma and dbeta of long batches: sums whose terms all have one sign and
value, where every addition rounds the same way, on every path.

A thread adds at most 128 samples' terms in a row; that loses at most 64 units
of 2^-24 of the sum (the k-th addition half a unit of k terms).  The 32 positions
of a slab's thread, a block's threads (64 at most here) and eight partial sums at
a time add at most 16, 32 and 4 units, so 128 units are allowed.  Runs of
thousands of samples lose more (1.0001 added 1050 times: 167; 3618 times: 577)."""

import pytest

from .gpu_common import lib_ready, torch_cuda
from .test_gpu_norm import U

pytestmark = pytest.mark.gpu


# rows of a warp and of a block, slabs, column passes
@pytest.mark.parametrize("shape", [(1100000, 1, 2048, 16), (30000, 1, 65536, 16), (70000, 64, 512, 32), (40000, 500, 130, 2)])
def test_sums_of_equal_terms(shape):
    torch = torch_cuda()
    ff = lib_ready()
    n, S, C, G = shape
    sign = 1.0 - 2.0 * (torch.arange(C, device="cuda") % 2).float()
    sign[C // G - 1::C // G] *= 1 if (C // G) % 2 == 0 else 0  # odd groups: the sum of each is zero all the same
    x = torch.empty(n, S, C, device="cuda").copy_(sign)
    c = torch.tensor(1.0001, device="cuda")
    dy = torch.empty_like(x).copy_(c.expand(C))
    _, m, r = ff.group_norm_act(x, None, None, G, act="none")
    assert bool((m == 0).all()) and bool((r == r[0, 0]).all())
    _, dg, db = ff.group_norm_act_backward(dy, x, m, r, None, None, G, act="none", out=dy)
    want = n * S * c.double()
    assert float(((db.double() - want).abs() / want).max()) <= 128 * U
    want = want * (sign * r[0, 0]).double()
    assert bool(((dg.double() - want).abs() <= 128 * U * want.abs()).all())
