"""Cross entropy without logits for fp32 above 1024 rows (GPU), where the operands' terms are cut before the products: heads and
hidden states of a wide range, several accumulations, all forms of the calls."""
import pytest
import torch

from tests.test_vocab_loss import backward, check, forward, inputs, reference, stream
from tests.vocab_common import lse_tolerance

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import paper_2608_07974_gb300 as pkg
    pkg.build()
    from paper_2608_07974_gb300 import binding
    return binding


@pytest.mark.parametrize("N", [1024, 1025])
def test_rows_of_the_head_with_small_values(B, N):
    """dW of a row does not go by how large the row is: rows down to the smallest numbers, and of zeros, have ordinary gradients,
    also scaled by a large factor (a loss scale)."""
    n, W, y = inputs("f32", N, 64, 1003)
    for i, e in enumerate((-60, -94, -100, -107, -113, -120, -126, -130)):
        W[7 * i + 1] *= 2.0 ** e
    W[64] = 0.0
    for i in range(9):
        y[4 * i + 1] = 7 * i + 1     # as labels too
    check(B, "f32", n, W, y)
    check(B, "f32", n, W, y, torch.tensor([65536.0], device="cuda"))


@pytest.mark.parametrize("N", [1024, 1025, 1300])
@pytest.mark.parametrize("factor", [30.0, 3000.0])
def test_columns_of_a_wide_range(B, N, factor):
    """A column of n `factor` times the others, the head small there: the other columns keep their bits."""
    n, W, y = inputs("f32", N, 64, 1003)
    n[:, 7] *= factor
    W[:, 7] /= factor
    check(B, "f32", n, W, y)


def test_large_values(B):
    """Up to 2^120 in a row of the head and 2^-110 in n at the same column."""
    n, W, y = inputs("f32", 1040, 64, 515)
    n[:, 5] *= 2.0 ** -110
    W[:, 5] *= 2.0 ** 110
    n, W = n.contiguous(), W.contiguous()
    check(B, "f32", n, W, y, want="n")


@pytest.mark.parametrize("N", [1024, 1100])
@pytest.mark.parametrize("d", [1024, 4096])
def test_logits_of_terms_of_one_sign(B, N, d):
    """All products positive, so that no error averages out: an accumulation of at most 256 cuts its running sum 16 times by at most
    2^-23 of it; the products of terms left out are below 2^-21 (leading bits: |m| < 2^-7 |x|, |l| < 2^-15 |x|, m l twice);
    the smaller pairs, below 2^-6 of the sum, are cut 5 d / 16 times; the accumulations are joined by d / 256 + 1 roundings (128
    each: twice). In units of 2^-23 of the logit: 16 + 4 + 5 d / 1024 + d / 256 + 1."""
    g = torch.Generator(device="cuda").manual_seed(d)
    n = 0.5 + torch.rand(N, d, generator=g, device="cuda")
    W = (0.5 + torch.rand(600, d, generator=g, device="cuda")) * (16.0 / d)
    y = torch.randint(0, 600, (N,), generator=torch.Generator().manual_seed(1), dtype=torch.int32).cuda()
    r = reference(n, W, y)
    rl, lse, loss = forward(B, "f32", n, W, y)
    ez = (21 + 5 * d / 1024 + d / 256) * 2.0 ** -23 * float(r["z"].max())
    el = ez + lse_tolerance(r["z"].max())
    assert float((lse.double() - r["lse"]).abs().max()) <= el
    assert float((rl.double() - r["row"]).abs().max()) <= ez + el
    check(B, "f32", n, W, y)


@pytest.mark.parametrize("N,d,V", [(1025, 8, 257), (1100, 2056, 1003), (1537, 4096, 513), (2049, 328, 5003)])
def test_shapes(B, N, d, V):
    check(B, "f32", *inputs("f32", N, d, V))


def test_frozen_head_frozen_input_and_scaled_loss(B):
    n, W, y = inputs("f32", 1030, 136, 1003)
    both = None
    for want in ("nw", "n", "w"):
        dn, dW = check(B, "f32", n, W, y, torch.tensor([-3.5], device="cuda"), want)[3:]
        both = both or (dn, dW)
        assert (dn is None or torch.equal(dn, both[0])) and (dW is None or torch.equal(dW, both[1]))


def test_rows_outside_the_loss_set(B):
    n, W, y = inputs("f32", 1030, 64, 777, holes=False)
    y[3], y[5], y[1029] = -1, 777, -2 ** 31
    want = check(B, "f32", n, W, y)
    bad = n.clone()
    bad[3], bad[5], bad[1029] = float("inf"), float("nan"), float("-inf")
    rl, lse, loss = forward(B, "f32", bad, W, y)
    assert torch.equal(rl, want[0]) and torch.equal(loss, want[2])
    dn, _ = backward(B, "f32", bad, W, y, lse, want="n")
    assert torch.equal(dn, want[3])


@pytest.mark.parametrize("dtype,N", [("bf16", 40), ("f32", 40), ("f32", 1030), ("bf16", 1030)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_broken_rows_of_the_loss_set(B, dtype, N, bad):
    """A NaN or an infinity in n of a row of the loss set: that row's loss and gradient are NaN, the others' as without it."""
    n, W, y = inputs(dtype, N, 64, 777, holes=False)
    rl0, lse0, loss0 = forward(B, dtype, n, W, y)
    dn0, _ = backward(B, dtype, n, W, y, lse0, want="n")
    n[9, 13] = bad
    rl, lse, loss = forward(B, dtype, n, W, y)
    dn, dW = backward(B, dtype, n, W, y, lse)
    keep = [i for i in range(N) if i != 9]
    assert bool(torch.isnan(rl[9])) and bool(torch.isnan(loss[0])) and float(loss[1]) == N and torch.equal(rl[keep], rl0[keep])
    assert bool(torch.isnan(dn[9]).all()) and torch.equal(dn[keep], dn0[keep]) and bool(torch.isnan(dW).all())


def test_a_step_captured_and_two_streams_at_once(B):
    N, d, V, e = 1030, 72, 1003, B.ZL_DTYPE_F32

    def spaces():
        return [torch.empty(f(e, N, d, V), dtype=torch.uint8, device="cuda") for f in (B.zl_op_vocab_loss_bytes, B.zl_op_vocab_loss_bwd_bytes)]

    def step(x, st, ws):
        rl, lse, loss = forward(B, "f32", *x, ws[0], st)
        return (rl, lse, loss, *backward(B, "f32", *x, lse, loss[:1], "nw", ws[1], st))

    x = [inputs("f32", N, d, V, s) for s in (1, 2)]
    alone = [step(a, stream(), spaces()) for a in x]
    torch.cuda.synchronize()
    streams, ws = [torch.cuda.Stream(), torch.cuda.Stream()], [spaces(), spaces()]
    torch.cuda.synchronize()
    for _ in range(3):
        got = []
        for a, st, w in zip(x, streams, ws):
            with torch.cuda.stream(st):
                got.append(step(a, st.cuda_stream, w))
    torch.cuda.synchronize()
    for a, b in zip(got, alone):
        assert all(torch.equal(p, q) for p, q in zip(a, b))
    own, held_in = spaces(), [t.clone() for t in x[0]]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        held = step(held_in, torch.cuda.current_stream().cuda_stream, own)
    for i in (1, 0):
        for a, b in zip(held_in, x[i]):
            a.copy_(b)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(held, alone[i]))


def test_outputs_and_workspace_stay_in_bounds(B):
    N, d, V, e, guard = 1031, 72, 1003, B.ZL_DTYPE_F32, 256
    n, W, y = inputs("f32", N, d, V)
    sizes = dict(rl=(N, torch.float32), lse=(N, torch.float32), loss=(2, torch.float32), dn=(N * d, torch.float32), dW=(V * d, torch.float32),
                 ws=(B.zl_op_vocab_loss_bytes(e, N, d, V), torch.uint8), wb=(B.zl_op_vocab_loss_bwd_bytes(e, N, d, V), torch.uint8))
    full = {k: torch.full((s + 2 * guard,), 55, dtype=t, device="cuda") for k, (s, t) in sizes.items()}
    i = {k: x[guard:-guard] for k, x in full.items()}
    B.zl_op_vocab_loss(e, n, W, y, N, d, V, i["rl"], i["lse"], i["loss"], i["ws"], stream())
    B.zl_op_vocab_loss_bwd(e, n, W, y, N, d, V, i["lse"], None, i["dn"], i["dW"], i["wb"], stream())
    torch.cuda.synchronize()
    for k, x in full.items():
        assert bool((x[:guard] == 55).all()) and bool((x[-guard:] == 55).all()), k
