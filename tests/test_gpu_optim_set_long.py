"""Long runs of AdamW over a set with fp32 moments, betas close to 1: the moments against the same recursion in fp64.

A step rounds a moment by at most u = 2^-24 relative, to either side alike, a deviation of u / sqrt 3 at most; N steps of n elements
leave u sqrt(N / (3 n)) in the mean over the elements, and six of these are allowed.  A bias of the weights, which every step
has alike, is N times as large as one step's and shows there: b rounded to fp32 beside 1 - b, 1e-8 of the moment a step."""
import math

import pytest

torch = pytest.importorskip("torch")
import paper_2608_26430_amd as ff  # noqa: E402

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("betas", [(0.9999, 0.99999), (0.99, 0.9999), (0.9, 0.999)])
def test_moments_of_a_long_run_have_no_bias(betas):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    n, steps, scale = 4096, 2000, 0.3
    gen = torch.Generator(device="cuda").manual_seed(7)
    s = ff.AdamWSet([torch.zeros(n, device="cuda")], betas=betas)
    # about where the run has been going for long: mean 1 and mean square 1.01 of the gradients, scaled; their spread moves v by
    # many units in its last place, so that it rounds to either side alike
    s.m[0].fill_(scale)
    s.v[0].fill_(1.01 * scale * scale)
    m, v = s.m[0].double(), s.v[0].double()
    for t in range(1, steps + 1):
        g = 1.0 + 0.1 * torch.randn(n, generator=gen, device="cuda")
        s.step([g], 0.0, t, grad_scale=scale)
        x = g.double() * scale
        m = betas[0] * m + (1.0 - betas[0]) * x
        v = betas[1] * v + (1.0 - betas[1]) * x * x
    torch.cuda.synchronize()
    for got, want, b in ((s.m[0], m, betas[0]), (s.v[0], v, betas[1])):
        # what a step has left is still there after k more of them with the factor b^k
        lasting = min(steps, 1.0 / (1.0 - b))
        bound = 6 * U * math.sqrt(lasting / (3 * n))
        off = float(((got.double() - want) / want).mean())
        assert abs(off) <= bound, (betas, off, bound)
