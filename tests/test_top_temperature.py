"""Records and the objective against them at low temperatures (GPU): softmaxes that are 0 and 1, logits over T of any finite size."""
import math

import pytest
import torch

from tests.vocab_common import TYPES, code, labels_of, lse_tolerance, ref_top, ref_top_loss, rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import paper_2608_07974_gb300 as pkg
    pkg.build()
    from paper_2608_07974_gb300 import binding
    return binding


def stream():
    return torch.cuda.current_stream().cuda_stream


def spread(N, V, step, seed):
    """Rows of V different logits, `step` apart, in any order."""
    g = torch.Generator().manual_seed(seed)
    return torch.stack([torch.randperm(V, generator=g).float() for _ in range(N)]) * step - 0.5 * step * V


@pytest.mark.parametrize("dtype,N,V,step", [("f32", 5, 203, 1.0), ("bf16", 5, 203, 1.0), ("f32", 2, 40003, 0.5)])
@pytest.mark.parametrize("T", [1e-2, 1e-4, 1e-6, 1e-10, 1e-20, 1e-30])
def test_rest_of_a_record(B, dtype, N, V, step, T):
    """The largest of the others over T, to its rounding; where a second one weighs as much, the sum."""
    z = spread(N, V, step, 1)
    z[1, z[1].argsort(descending=True)[6]] = z[1].sort(descending=True).values[5]     # two equal ones behind the record
    zd, k = rows(z, TYPES[dtype]), 5
    idx, val, rest = torch.empty(N, k, dtype=torch.int32, device="cuda"), torch.empty(N, k, device="cuda"), torch.empty(N, device="cuda")
    B.zl_op_top_logits(code(B, dtype), zd, N, V, V, k, T, idx, val, rest, stream())
    ri, rv, rr = ref_top(zd.double().cpu(), k, T)
    assert torch.equal(idx.cpu().long(), ri) and torch.equal(val.cpu().double(), rv)
    assert bool(((rest.cpu().double() - rr).abs() <= 2.0 ** -24 * (8 * rr.abs() + 64)).all())


@pytest.mark.parametrize("dtype,N,V,step", [("f32", 5, 203, 1.0), ("bf16", 5, 203, 1.0), ("f32", 2, 40003, 0.5)])
@pytest.mark.parametrize("T", [1e-2, 1e-4, 1e-6, 1e-10, 1e-20])
@pytest.mark.parametrize("alpha", [0.0, 0.5])
@pytest.mark.parametrize("kl_dir,with_rest", [(0, 1), (1, 1), (1, 0)])
def test_loss(B, dtype, N, V, step, T, alpha, kl_dir, with_rest):
    """Probabilities of 0 and 1 are that: they go by differences of logits, good to 2^-20 where e^(difference / T) is not 0. Log
    probabilities are differences of logits over T, rounded a few times; times T^2 (loss) or T (gradient) their error is 2^-20 of
    the logits' range, times T or 1. The teacher's rest is fp32 and may change places with nothing. The task term as elsewhere."""
    z, t, k = rows(spread(N, V, step, 2), TYPES[dtype]), rows(spread(N, V, step, 3), TYPES[dtype]), 5
    t[0] = z[0]                                                                   # a student that agrees
    y = labels_of(N, V)
    y[0] = int(z[0].argmax())
    y[1] = 0
    idx, val, rest = torch.empty(N, k, dtype=torch.int32, device="cuda"), torch.empty(N, k, device="cuda"), torch.empty(N, device="cuda")
    B.zl_op_top_logits(code(B, dtype), t, N, V, V, k, T, idx, val, rest, stream())
    dz, rl, loss = torch.full_like(z, math.nan), torch.empty(N, device="cuda"), torch.empty(2, device="cuda")
    B.zl_op_top_loss(code(B, dtype), z, idx, val, rest if with_rest else None, y.cuda(), N, V, V, k, alpha, T, kl_dir, dz, rl, loss, stream())
    z64 = z.double().cpu().requires_grad_(True)
    total, w = 0.0, 1.0 / float((y >= 0).sum())
    far = float(z.double().max() - z.double().min())
    for i in range(N):
        if int(y[i]) < 0:
            assert float(rl[i]) == 0 and not bool(dz[i].any())
            continue
        r = ref_top_loss(z64[i], idx[i].cpu(), val[i].double().cpu(), rest[i].double().cpu() if with_rest else None, int(y[i]), alpha, T, kl_dir)
        total = total + w * r
        e = lse_tolerance(z.abs().max())
        assert abs(float(rl[i]) - float(r.detach())) <= alpha * 4 * e + (1 - alpha) * 2.0 ** -20 * (T * far + T * T), i
    ref = torch.autograd.grad(total, z64)[0]
    p = torch.softmax(z64.detach(), 1)
    tol = w * (alpha * 4 * e + (1 - alpha) * 2.0 ** -20 * (far if kl_dir == 0 else T)) + torch.finfo(TYPES[dtype]).eps / 2 * ref.abs() + 1e-37
    assert bool(((dz.double().cpu() - ref).abs() <= tol).all()), float((dz.double().cpu() - ref).abs().max())
