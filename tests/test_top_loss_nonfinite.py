"""The objective against records with values that are no numbers in rows of the loss set (GPU): what the definition makes NaN
has to come out as NaN, not as a term that is left out."""
import math

import pytest
import torch

from tests.vocab_common import TYPES, code, labels_of, rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import paper_2608_07974_gb300 as pkg
    pkg.build()
    from paper_2608_07974_gb300 import binding
    return binding


def stream():
    return torch.cuda.current_stream().cuda_stream


def record(B, dtype, z, V, k, T):
    N = z.shape[0]
    idx, val, rest = torch.empty(N, k, dtype=torch.int32, device="cuda"), torch.empty(N, k, device="cuda"), torch.empty(N, device="cuda")
    B.zl_op_top_logits(code(B, dtype), z, N, V, z.shape[1], k, T, idx, val, rest, stream())
    return idx, val, rest


def loss_of(B, dtype, z, rec, y, V, alpha, T, kl_dir):
    N, ld = z.shape
    dz, rl, loss = torch.full_like(z, 77.0), torch.full((N,), 77.0, device="cuda"), torch.full((2,), 77.0, device="cuda")
    B.zl_op_top_loss(code(B, dtype), z, *rec, y, N, V, ld, rec[0].shape[1], alpha, T, kl_dir, dz, rl, loss, stream())
    return dz, rl, loss


def check_row_is_nan(got, want, r, V):
    """Row r all NaN but for its padding, the others as they were without it."""
    (dz, rl, loss), (dz0, rl0, loss0) = got, want
    keep = [i for i in range(dz.shape[0]) if i != r]
    assert bool(torch.isnan(rl[r])) and bool(torch.isnan(loss[0])) and float(loss[1]) == float(loss0[1])
    assert bool(torch.isnan(dz[r, :V]).all()) and bool((dz[r, V:] == 0).all())
    assert torch.equal(dz[keep], dz0[keep]) and torch.equal(rl[keep], rl0[keep]) and not bool(torch.isnan(rl0).any())


def case(dtype, N, V, ld, off, seed):
    g = torch.Generator().manual_seed(seed)
    z = 2 * torch.randn(N, V, generator=g)
    t = 0.8 * z + 0.5 * torch.randn(N, V, generator=g)
    y = labels_of(N, V, seed)
    return rows(z, TYPES[dtype], ld, off), rows(t, TYPES[dtype], ld, off), y.cuda()


# (the second shape: rows shared by several CTAs)
SHAPES = [(7, 1000, 1003, 1, 12), (3, 40000, 40001, 3, 40)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,V,ld,off,k", SHAPES)
@pytest.mark.parametrize("alpha", [0.0, 0.5, 1.0])
@pytest.mark.parametrize("kl_dir", [0, 1])
@pytest.mark.parametrize("T", [1.0, 2.0])
def test_a_broken_student_row(B, dtype, N, V, ld, off, k, alpha, kl_dir, T):
    """A NaN or +inf in the record, among the other columns, before the row's first 16-byte word or behind its last; a row of -inf."""
    z, t, y = case(dtype, N, V, ld, off, 11)
    rec, r = record(B, dtype, t, V, k, T), 1
    want = loss_of(B, dtype, z, rec, y, V, alpha, T, kl_dir)
    inside = set(rec[0][r].tolist())
    other = next(c for c in range(V // 2, V) if c not in inside and c != int(y[r]))
    clean = z.clone()
    for at in (int(rec[0][r, 3]), other, 0, V - 1, int(y[r])):
        for bad in (math.nan, math.inf):
            z.copy_(clean)
            z[r, at] = bad
            check_row_is_nan(loss_of(B, dtype, z, rec, y, V, alpha, T, kl_dir), want, r, V)
    z.copy_(clean)
    z[r, :V] = -math.inf
    check_row_is_nan(loss_of(B, dtype, z, rec, y, V, alpha, T, kl_dir), want, r, V)


@pytest.mark.parametrize("alpha", [0.0, 0.5])
@pytest.mark.parametrize("kl_dir", [0, 1])
def test_a_broken_student_row_against_an_empty_record(B, alpha, kl_dir):
    z, t, y = case("f32", 7, 1000, 1003, 1, 12)
    rec, r, V = record(B, "f32", t, 1000, 12, 1.0), 1, 1000
    c = int(rec[0][r, 3])
    for empty in ("columns", "mass"):
        if empty == "columns":
            rec[0][r] = -1
            rec[2][r] = -math.inf
        else:
            rec[0][r] = torch.arange(c, c + 12) % V
            rec[1][r] = -math.inf
        want = loss_of(B, "f32", z, rec, y, V, alpha, 1.0, kl_dir)
        clean = z[r].clone()
        for bad in (math.nan, math.inf):
            z[r, c] = bad
            check_row_is_nan(loss_of(B, "f32", z, rec, y, V, alpha, 1.0, kl_dir), want, r, V)
        z[r, :V] = -math.inf
        check_row_is_nan(loss_of(B, "f32", z, rec, y, V, alpha, 1.0, kl_dir), want, r, V)
        z[r] = clean


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,V,ld,off,k", SHAPES)
@pytest.mark.parametrize("alpha", [0.0, 0.5])
@pytest.mark.parametrize("kl_dir,with_rest", [(0, 1), (1, 1), (1, 0)])
@pytest.mark.parametrize("T", [1.0, 2.0])
def test_a_broken_teacher_row(B, dtype, N, V, ld, off, k, alpha, kl_dir, with_rest, T):
    """A NaN or +inf among the record's values or as its rest: no divergence is known. With an entry that is left out it goes too,
    and with alpha 1 nothing of the record is read."""
    z, t, y = case(dtype, N, V, ld, off, 13)
    idx, val, rest = record(B, dtype, t, V, k, T)
    r = 1

    def go(idx, val, rest, a=alpha):
        return loss_of(B, dtype, z, (idx, val, rest if with_rest else None), y, V, a, T, kl_dir)

    want = go(idx, val, rest)
    for bad in (math.nan, math.inf):
        for at in (0, k // 2, k - 1):
            v = val.clone()
            v[r, at] = bad
            check_row_is_nan(go(idx, v, rest), want, r, V)
        if with_rest:
            u = rest.clone()
            u[r] = bad
            check_row_is_nan(go(idx, val, u), want, r, V)
        i, v, v2 = idx.clone(), val.clone(), val.clone()
        i[r, 2], v[r, 2], v2[r, 2] = -1, bad, 0.0
        for a, b in zip(go(i, v, rest), go(i, v2, rest)):
            assert torch.equal(a, b) and not bool(torch.isnan(b).any())
        v[r] = bad
        for a, b in zip(go(idx, v, rest, 1.0), go(idx, val, rest, 1.0)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("kl_dir", [0, 1])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_a_teacher_that_diverged(B, kl_dir, bad):
    """Its logits to the record to the loss: NaN arrives."""
    z, t, y = case("bf16", 7, 1000, 1008, 0, 14)
    want = loss_of(B, "bf16", z, record(B, "bf16", t, 1000, 12, 1.0), y, 1000, 0.5, 1.0, kl_dir)
    t[1, 400] = bad
    check_row_is_nan(loss_of(B, "bf16", z, record(B, "bf16", t, 1000, 12, 1.0), y, 1000, 0.5, 1.0, kl_dir), want, 1, 1000)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,V,ld,off,k", SHAPES)
@pytest.mark.parametrize("alpha", [0.0, 0.5, 1.0])
@pytest.mark.parametrize("kl_dir,with_rest", [(0, 1), (1, 1), (1, 0)])
@pytest.mark.parametrize("T", [1.0, 2.0, 0.5])
def test_a_row_of_nothing_but_the_lowest_value(B, dtype, N, V, ld, off, k, alpha, kl_dir, with_rest, T):
    """A softmax does not change when a number is added to all logits: such a row has that of a row of zeros, to the rounding of its
    loss, log V and a divergence (2^-20 of up to 40), and of its gradient."""
    z, t, y = case(dtype, N, V, ld, off, 15)
    idx, val, rest = record(B, dtype, t, V, k, T)
    rec = (idx, val, rest if with_rest else None)
    z[1, :V] = 0.0
    dz0, rl0, loss0 = loss_of(B, dtype, z, rec, y, V, alpha, T, kl_dir)
    z[1, :V] = torch.finfo(TYPES[dtype]).min
    dz, rl, loss = loss_of(B, dtype, z, rec, y, V, alpha, T, kl_dir)
    tol = 2.0 ** -20 * 40 * max(1.0, T * T)
    assert float((rl - rl0).abs().max()) <= tol and float((loss - loss0).abs().max()) <= tol
    tol = (2.0 ** -18 + torch.finfo(TYPES[dtype]).eps) * dz0.float().abs() + (1 - alpha) * T * 2.0 ** -20 * 40 / V
    assert bool(((dz.float() - dz0.float()).abs() <= tol).all())
