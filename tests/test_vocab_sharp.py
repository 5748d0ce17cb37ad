"""The gradient of cross entropy without logits where the label's probability is near 1 (GPU)."""
import pytest
import torch

from tests.test_vocab_loss import backward
from tests.vocab_common import TYPES

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import paper_2608_07974_gb300 as pkg
    pkg.build()
    from paper_2608_07974_gb300 import binding
    return binding


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [64, 300, 1100])
def test_labels_with_a_probability_near_one(B, dtype, N):
    """Logits of 100 over 4096 columns, 1 - p of about 2e-4 at the label: its dz is p - 1, off by its logit's error. Products of one
    sign in accumulations of 512: each of 32 steps cuts the running sum by at most 2^-23 of it, (32 + 1) / 2 of the sum's in all, and
    8 (fp32 products, in accumulations of 128 or 256: fewer steps; up to 33, and 2^-21 of products left out) joins round it: 20.5 2^-23 of the
    logit, fp32 4.25 + 16.5 + 4 + 5 d / 2048 = 35. The exponential is good to 2^-22. Along the label's row of W the gradient is
    its dz and 0.9 of the others', each rounded to 2^-8 of at most 1 - p, as the result is (by elements, whose magnitudes sum up to four
    times the projection)."""
    d, V = 4096, 512
    g = torch.Generator(device="cuda").manual_seed(N)
    u = torch.where(torch.rand(d, generator=g, device="cuda") < 0.5, 9.2, -9.2) / d ** 0.5
    e = torch.randn(V, d, generator=g, device="cuda") * (4.0 / d ** 0.5)
    y = torch.randint(0, V, (N,), generator=torch.Generator().manual_seed(1), dtype=torch.int32).cuda()
    n, W = (u + e[y.long()] * (15.0 / 16.0)).to(TYPES[dtype]), (u + e).to(TYPES[dtype])
    n64, W64 = n.double(), W.double()
    z = n64 @ W64.T
    lse = torch.logsumexp(z, 1).float()
    dz = torch.exp(z - lse.double()[:, None])
    dz.scatter_add_(1, y.long()[:, None], torch.full((N, 1), -1.0, dtype=torch.float64, device="cuda"))
    dn = backward(B, dtype, n, W, y, lse, torch.tensor([float(N)], device="cuda"), "n")[0]
    at = W64[y.long()]
    off = ((dn.double() - dz @ W64) * at).sum(1) / (at * at).sum(1)
    left = dz.gather(1, y.long()[:, None])[:, 0].abs()
    zy = z.gather(1, y.long()[:, None])[:, 0]
    assert 90 < float(zy.min()) and float(zy.max()) < 110 and 1e-5 < float(left.min()) and float(left.max()) < 5e-3
    tol = (20.5 if dtype == "bf16" else 35.0) * 2.0 ** -23 * zy + 2.0 ** -21 + 8 * torch.finfo(TYPES[dtype]).eps / 2 * left
    assert bool((off.abs() <= tol).all()), (float(off.abs().max()), float(tol.min()))
