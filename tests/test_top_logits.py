"""A teacher's record of top logits and the local objective against it (GPU), against 64-bit definitions."""
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


def top(B, dtype, z, V, k, T=1.0, st=None):
    N = z.shape[0]
    idx = torch.full((N, k), -7, dtype=torch.int32, device="cuda")
    val, rest = torch.full((N, k), 77.0, device="cuda"), torch.full((N,), 77.0, device="cuda")
    B.zl_op_top_logits(code(B, dtype), z, N, V, z.stride(0) if N > 1 else z.shape[1], k, T, idx, val, rest, stream() if st is None else st)
    return idx, val, rest


def check_top(B, dtype, z, V, k, T=1.0):
    idx, val, rest = top(B, dtype, z, V, k, T)
    z64 = z[:, :V].double().cpu()
    ri, rv, rr = ref_top(z64, k, T)
    assert torch.equal(idx.cpu().long(), ri)
    assert torch.equal(val.cpu().double().nan_to_num(nan=1e99), rv.nan_to_num(nan=1e99))
    fin = torch.isfinite(rr)
    got = rest.double().cpu()
    assert torch.equal(torch.isfinite(got), fin)
    assert torch.equal(got[~fin].nan_to_num(nan=1e9), rr[~fin].nan_to_num(nan=1e9))
    m = z64[torch.isfinite(z64)].abs().max() / T if torch.isfinite(z64).any() else 0.0
    assert float((got - rr)[fin].abs().max() if fin.any() else 0.0) <= lse_tolerance(m)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,V,ld,off,k,T", [
    (1, 2, 2, 0, 1, 1.0), (1, 2, 3, 1, 2, 1.0), (3, 7, 8, 0, 7, 2.0), (5, 33, 41, 3, 8, 0.5), (2, 500, 500, 1, 256, 1.0),
    (4, 1000, 1001, 0, 64, 1.0), (7, 5003, 5008, 0, 1, 1.0), (3, 32000, 32000, 0, 16, 1.0), (2, 50257, 50264, 0, 64, 1.0),
    (2, 50257, 50257, 5, 256, 2.0), (2, 32000, 32001, 0, 1024, 1.0), (1, 262144, 262144, 0, 100, 1.0), (3, 1025, 1025, 7, 1024, 0.7),
    (2, 4099, 4099, 0, 513, 1.0), (1, 1 << 20, 1 << 20, 0, 1024, 1.0)])
def test_record_of_random_logits(B, dtype, N, V, ld, off, k, T):
    torch.manual_seed(N + V + k)
    check_top(B, dtype, rows(3 * torch.randn(N, V), TYPES[dtype], ld, off, fill=1e30), V, k, T)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,k", [(5000, 64), (50257, 300), (32001, 1024), (40, 40)])
def test_record_of_rows_with_ties_masks_and_odd_values(B, dtype, V, k):
    g = torch.Generator().manual_seed(V + k)
    z = 3 * torch.randn(12, V, generator=g)
    z[0] = 0.0                                        # all equal: the first k columns
    z[1] = -math.inf                                  # nothing left of the row
    z[2] = -math.inf
    z[2, V // 2] = 1.5                                # one column left
    z[3] = torch.round(z[3])                          # few distinct values
    z[4, ::3] = -math.inf
    z[5] = torch.where(torch.arange(V) % 2 == 0, 0.0, -0.0)
    z[6] = torch.arange(V).float() / 64               # rising
    z[7] = -torch.arange(V).float() / 64              # falling
    z[8, V // 3] = math.inf
    z[9] = torch.finfo(torch.bfloat16).min            # a mask of the type's lowest value
    z[9, -1] = 2.0
    z[10, 5], z[10, V - 1] = math.nan, math.nan
    z[11] = 1.0
    z[11, :: max(1, V // 5)] = 9.0
    check_top(B, dtype, rows(z, TYPES[dtype]), V, k)


def test_the_same_bits_every_time(B):
    """Candidates are collected by atomics: neither the record nor the rest's sum goes by their order."""
    z = rows(torch.round(8 * torch.randn(16, 50257, generator=torch.Generator().manual_seed(3))) / 4, torch.bfloat16)
    first = top(B, "bf16", z, 50257, 200)
    for _ in range(20):
        for a, b in zip(first, top(B, "bf16", z, 50257, 200)):
            assert torch.equal(a, b)


def test_record_when_the_rest_lies_far_below(B):
    """The rest's sum goes by its own largest term: its logarithm holds where e^(rest - top) underflows."""
    z = torch.full((2, 9000), -400.0)
    z[:, :16] = 200.0 + torch.arange(16).float()
    check_top(B, "f32", rows(z, torch.float32), 9000, 16, 0.5)


def run_loss(B, dtype, z, idx, val, rest, y, V, k, alpha, T, kl_dir, inplace=False, st=None, dz=None):
    N, ld = z.shape
    if dz is None:
        dz = z if inplace else torch.full_like(z, math.nan)
    rl, loss = torch.full((N,), 77.0, device="cuda"), torch.full((2,), 77.0, device="cuda")
    B.zl_op_top_loss(code(B, dtype), z, idx, val, rest, y, N, V, ld, k, alpha, T, kl_dir, dz, rl, loss, stream() if st is None else st)
    return dz, rl, loss


def check_loss(B, dtype, z, idx, val, rest, y, V, alpha, T, kl_dir, inplace=False, dz_off=None):
    """Against the definition's value and gradient (autograd in 64 bits). The gradient's terms are w (alpha (p1 + [y]) + (1 -
    alpha) T (p |lp - lq - KL| or p + q)); each is off by a log-sum-exp's tolerance times a few, relative, and the whole by
    half a step of its type."""
    td, (N, ld), k = TYPES[dtype], z.shape, idx.shape[1]
    z64 = z[:, :V].double().cpu().requires_grad_(True)
    args = [t.cpu() for t in (idx, val)] + [None if rest is None else rest.cpu()]
    ok = [i for i in range(N) if 0 <= int(y[i]) < V]
    ref_rows = torch.zeros(N, dtype=torch.float64)
    total = torch.zeros((), dtype=torch.float64)
    for i in ok:
        r = ref_top_loss(z64[i], args[0][i], args[1][i], None if rest is None else args[2][i], int(y[i]), alpha, T, kl_dir)
        ref_rows[i] = r.detach()
        total = total + r / len(ok)
    ref = torch.zeros_like(z64) if not ok else torch.autograd.grad(total, z64)[0]
    out = None
    if dz_off is not None:
        out = torch.full((N * ld + dz_off,), math.nan, dtype=td, device="cuda")[dz_off:].view(N, ld)
    dz, rl, loss = run_loss(B, dtype, z, idx, val, rest, y.cuda(), V, k, alpha, T, kl_dir, inplace, dz=out)
    m = float(z64.detach()[torch.isfinite(z64)].abs().max()) / min(T, 1.0) if torch.isfinite(z64).any() else 0.0
    vv = args[1][torch.isfinite(args[1])]
    m = max(m, float(vv.abs().max()) / T if vv.numel() else 0.0)
    e = lse_tolerance(m)
    # KL is a sum of p |lp - lq| whose factors are off by 3 e: log-sum-exps of both sides and a logit
    tol_row = 4 * e * (1 + 2 * m + ((1 - alpha) * T * T + ref_rows.abs() if alpha < 1 else torch.zeros(N)))
    assert bool(((rl.double().cpu() - ref_rows).abs() <= tol_row).all())
    assert float(loss[1]) == len(ok)
    want = float(ref_rows.sum() / len(ok)) if ok else 0.0
    assert abs(float(loss[0]) - want) <= float(tol_row.max())
    got = dz.double().cpu()
    assert bool((got[:, V:] == 0).all())
    got = got[:, :V]
    p1, pt = torch.softmax(z64.detach(), 1), torch.softmax(z64.detach() / T, 1)
    size = alpha * p1
    for i in ok:
        size[i, int(y[i])] += alpha
    if alpha < 1:
        q = torch.zeros(N, V, dtype=torch.float64)
        lqn = torch.logsumexp(torch.cat([args[1].double() / T] + ([] if rest is None else [args[2].double()[:, None]]), 1), 1)
        for i in ok:
            for c, v in zip(args[0][i].tolist(), args[1][i].tolist()):
                if 0 <= c < V and math.isfinite(float(lqn[i])):
                    q[i, c] = max(float(q[i, c]), math.exp(v / T - float(lqn[i])))
        far = 2 * m + 20 if kl_dir == 0 else 1.0     # |lp - lq - KL|
        size += (1 - alpha) * T * (far * pt + q)
        if kl_dir == 1 and rest is not None:         # the others share q_r as they share p_r
            size += (1 - alpha) * T
    size /= max(1, len(ok))
    # (a share of the others' teacher mass: size above bounds it by 1; what is checked there is absolute)
    bad = (got - ref).abs() > 4 * e * size + torch.finfo(td).eps / 2 * ref.abs() + 1e-37
    assert not bool(bad.any()), float(((got - ref).abs() - torch.finfo(td).eps / 2 * ref.abs()).max())
    for i in range(N):
        if i not in ok:
            assert bool((got[i] == 0).all()) and float(rl[i]) == 0.0


def teacher_record(B, dtype, N, V, k, T, seed, noise=0.6):
    g = torch.Generator().manual_seed(seed)
    z = 2.5 * torch.randn(N, V, generator=g)
    t = rows(0.8 * z + noise * torch.randn(N, V, generator=g), TYPES[dtype])
    return z, top(B, dtype, t, V, k, T)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,V,ld,off,k,alpha,T,kl_dir,rest", [
    (1, 2, 2, 0, 1, 0.5, 1.0, 0, 1), (3, 9, 9, 1, 9, 0.5, 1.0, 1, 1), (3, 9, 16, 0, 9, 0.0, 2.0, 0, 1), (5, 33, 34, 0, 4, 0.3, 0.5, 1, 0),
    (6, 1000, 1000, 0, 20, 0.5, 1.0, 1, 0), (6, 1000, 1003, 5, 64, 0.3, 2.0, 0, 1), (4, 5003, 5003, 0, 100, 0.0, 1.0, 1, 1),
    (4, 5003, 5008, 0, 100, 1.0, 2.0, 0, 0), (3, 50257, 50264, 0, 64, 0.5, 1.0, 0, 1), (3, 32000, 32001, 0, 256, 0.5, 2.0, 1, 1),
    (2, 40000, 40000, 0, 1024, 0.5, 1.0, 0, 1)])
def test_loss_against_records(B, dtype, N, V, ld, off, k, alpha, T, kl_dir, rest):
    z, (idx, val, r) = teacher_record(B, dtype, N, V, k, T, N + V + k)
    y = labels_of(N, V, V)
    if N > 4:
        y[2] = int(idx[2, 0])     # a label inside the record
    zd = rows(z, TYPES[dtype], ld, off, fill=math.nan)
    check_loss(B, dtype, zd, idx, val, r if rest else None, y, V, alpha, T, kl_dir)
    check_loss(B, dtype, zd, idx, val, r if rest else None, y, V, alpha, T, kl_dir, dz_off=(off + 3) % 8)
    check_loss(B, dtype, zd, idx, val, r if rest else None, y, V, alpha, T, kl_dir, inplace=True)


@pytest.mark.parametrize("kl_dir,rest", [(0, 1), (1, 1), (1, 0)])
def test_records_with_fewer_entries_and_repeated_columns(B, kl_dir, rest):
    N, V, k = 6, 700, 12
    z, (idx, val, r) = teacher_record(B, "f32", N, V, k, 1.0, 5)
    idx[1, 4:] = -1                      # a short record
    idx[2, 3] = V                        # a column past the row
    idx[3, 5] = idx[3, 0]                # a column twice: the first entry counts
    idx[3, 7] = idx[3, 0]
    idx[4, 1:] = idx[4, 0].clone()
    val[5, 2] = -math.inf                # a class without teacher mass
    if kl_dir == 0:
        val[5, 2] = -60.0
    check_loss(B, "f32", rows(z, torch.float32), idx, val, r if rest else None, labels_of(N, V, holes=False), V, 0.5, 1.0, kl_dir)


def test_an_empty_record_adds_nothing(B):
    """All entries left out, or all without mass: the task term alone."""
    N, V, k = 4, 300, 5
    z, (idx, val, r) = teacher_record(B, "f32", N, V, k, 1.0, 6)
    idx[1] = -1
    r[1] = -math.inf
    val[2], r[2] = -math.inf, -math.inf
    check_loss(B, "f32", rows(z, torch.float32), idx, val, r, labels_of(N, V, holes=False), V, 0.5, 1.0, 1)
    check_loss(B, "f32", rows(z, torch.float32), idx, val, r, labels_of(N, V, holes=False), V, 0.5, 1.0, 0)


@pytest.mark.parametrize("kl_dir", [0, 1])
def test_student_columns_masked_out(B, kl_dir):
    """Columns of -inf in both, and rows outside the loss set that are all -inf or NaN."""
    N, V, k = 6, 900, 16
    g = torch.Generator().manual_seed(8)
    z = 2 * torch.randn(N, V, generator=g)
    z[:, 100:200] = -math.inf
    t = rows(0.8 * z, torch.float32)
    idx, val, r = top(B, "f32", t, V, k)
    z[0], z[4] = -math.inf, math.nan
    y = labels_of(N, V)
    y[4] = -1
    y[y.clamp(min=0).long().ge(100) & y.lt(200)] = 3
    zd = rows(z, torch.float32)
    dz, rl, loss = run_loss(B, "f32", zd, idx, val, r, y.cuda(), V, k, 0.5, 1.0, kl_dir)
    assert bool(torch.isfinite(dz).all()) and bool((dz[0] == 0).all()) and bool((dz[4] == 0).all()) and bool((dz[1:4, 100:200] == 0).all())
    keep = [i for i in range(N) if int(y[i]) >= 0]
    check_loss(B, "f32", zd[keep].contiguous(), idx[keep], val[keep], r[keep], y[keep], V, 0.5, 1.0, kl_dir)


def test_no_rows_of_the_loss_set_and_no_rows(B):
    z, (idx, val, r) = teacher_record(B, "f32", 3, 50, 4, 1.0, 1)
    check_loss(B, "f32", rows(z, torch.float32), idx, val, r, torch.full((3,), -1, dtype=torch.int32), 50, 0.5, 1.0, 0)
    e = torch.empty(0, 50, device="cuda")
    dz, rl, loss = run_loss(B, "f32", e, idx[:0], val[:0], r[:0], torch.empty(0, dtype=torch.int32, device="cuda"), 50, 4, 0.5, 1.0, 0)
    assert loss.tolist() == [0.0, 0.0]
    top(B, "f32", e, 50, 4)


@pytest.mark.parametrize("N", [1024, 1025, 5000])
def test_loss_set_of_many_rows(B, N):
    """|Omega| by the rows themselves and by a launch of its own."""
    V, k = 40, 4
    z, (idx, val, r) = teacher_record(B, "f32", N, V, k, 1.0, 2)
    check_loss(B, "f32", rows(z, torch.float32), idx, val, r, labels_of(N, V), V, 0.5, 1.0, 1)


def test_gradient_against_differences(B):
    """Central differences of the kernel's own loss in two directions; fp32 losses of about 3 are good to 2^-22, steps of 0.05
    leave a quotient good to 2e-5 and a third derivative's share of 0.05^2 / 6 of a gradient's norm."""
    N, V, k = 5, 200, 8
    z, (idx, val, r) = teacher_record(B, "f32", N, V, k, 2.0, 3)
    y = labels_of(N, V).cuda()
    zd = rows(z, torch.float32)
    for kl_dir in (0, 1):
        dz, _, _ = run_loss(B, "f32", zd, idx, val, r, y, V, k, 0.4, 2.0, kl_dir)
        for s in (0, 1):
            d = torch.randn(N, V, generator=torch.Generator().manual_seed(s)).cuda()
            h = 0.05
            up = run_loss(B, "f32", zd + h * d, idx, val, r, y, V, k, 0.4, 2.0, kl_dir)[2][0]
            dn = run_loss(B, "f32", zd - h * d, idx, val, r, y, V, k, 0.4, 2.0, kl_dir)[2][0]
            num, ana = (float(up) - float(dn)) / (2 * h), float((dz.double() * d.double()).sum())
            assert abs(num - ana) <= 2e-5 + h * h * float(dz.norm() * d.norm())


def test_record_then_loss_captured_and_on_another_stream(B):
    """Teacher to record to loss, as a step uses them: the eager pass, a pass on a side stream and a replayed graph (on new
    inputs in place) agree bit for bit."""
    N, V, ld, k = 130, 5003, 5008, 32
    y = labels_of(N, V).cuda()

    def step(z, t, st):
        rec = top(B, "bf16", t, V, k, 2.0, st)
        return (*rec, *run_loss(B, "bf16", z, *rec, y, V, k, 0.5, 2.0, 0, st=st))

    def fresh(seed):
        g = torch.Generator().manual_seed(seed)
        return [rows(2 * torch.randn(N, V, generator=g), torch.bfloat16, ld) for _ in range(2)]

    z, t = fresh(1)
    first = step(z, t, stream())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = step(z, t, side.cuda_stream)
    torch.cuda.synchronize()
    for a, b in zip(first, other):
        assert torch.equal(a, b)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        held = step(z, t, torch.cuda.current_stream().cuda_stream)
    for seed in (2, 3):
        z2, t2 = fresh(seed)
        z.copy_(z2)
        t.copy_(t2)
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(held, step(z2, t2, stream())):
            assert torch.equal(a, b)


def test_rows_past_2_to_the_31st_element(B):
    """2^31 and more logits: the last rows' offsets need 64 bits. The same rows in a call of their own are shared by more CTAs and
    sum in another order: both sides lie within a log-sum-exp's tolerance of the definition (twice that apart), relative in the
    gradient, whose values may then round to neighbouring steps of their type."""
    V, N, k = 50257, 42800, 8
    z = torch.zeros(N, V, dtype=torch.bfloat16, device="cuda")
    last = rows(3 * torch.randn(2, V, generator=torch.Generator().manual_seed(1)), torch.bfloat16)
    z[-2:] = last
    idx, val, rest = top(B, "bf16", z, V, k)
    i2, v2, r2 = top(B, "bf16", last, V, k)
    e = 2 * lse_tolerance(last.float().abs().max())
    assert torch.equal(idx[-2:], i2) and torch.equal(val[-2:], v2) and float((rest[-2:] - r2).abs().max()) <= e
    y = torch.full((N,), -1, dtype=torch.int32, device="cuda")
    y[-2:] = 5
    dz, rl, loss = run_loss(B, "bf16", z, idx, val, rest, y, V, k, 0.5, 1.0, 1, inplace=True)
    dz2, rl2, loss2 = run_loss(B, "bf16", last, i2, v2, r2, y[-2:], V, k, 0.5, 1.0, 1)
    near = (dz[-2:].double() - dz2.double()).abs() <= (4 * e + torch.finfo(torch.bfloat16).eps) * dz2.double().abs() + 1e-37
    assert bool(near.all()) and float((rl[-2:] - rl2).abs().max()) <= 4 * e and float((loss - loss2).abs().max()) <= 4 * e
    assert bool((dz[0] == 0).all()) and bool((dz[N // 2] == 0).all())


def test_outputs_stay_in_bounds(B):
    N, V, ld, k = 37, 1003, 1003, 9
    z, _ = teacher_record(B, "bf16", N, V, k, 1.0, 4)
    zd = rows(z, torch.bfloat16)
    guard = 64
    f = {n: torch.full((s + 2 * guard,), 55, dtype=t, device="cuda") for n, s, t in
         (("idx", N * k, torch.int32), ("val", N * k, torch.float32), ("rest", N, torch.float32), ("dz", N * ld, torch.bfloat16),
          ("rl", N, torch.float32), ("loss", 2, torch.float32))}
    i = {n: x[guard:-guard] for n, x in f.items()}
    B.zl_op_top_logits(B.ZL_DTYPE_BF16, zd, N, V, ld, k, 1.0, i["idx"], i["val"], i["rest"], stream())
    B.zl_op_top_loss(B.ZL_DTYPE_BF16, zd, i["idx"], i["val"], i["rest"], labels_of(N, V).cuda(), N, V, ld, k, 0.5, 1.0, 1,
                     i["dz"].view(N, ld), i["rl"], i["loss"], stream())
    torch.cuda.synchronize()
    for n, x in f.items():
        assert bool((x[:guard] == 55).all()) and bool((x[-guard:] == 55).all()), n


@pytest.mark.parametrize("N", [256, 257, 511, 512, 513])
def test_loss_set_counted_by_the_rows_or_by_a_launch(B, N):
    """Up to 512 rows every row counts |Omega| itself, one label a thread up to 256 and two above; more are counted by a launch. Holes
    lie on both sides of 256."""
    V, k = 40, 4
    z, (idx, val, r) = teacher_record(B, "f32", N, V, k, 1.0, 2)
    y = labels_of(N, V)
    y[N - 1], y[N - 2], y[255] = -1, 3, V
    check_loss(B, "f32", rows(z, torch.float32), idx, val, r, y, V, 0.5, 1.0, 1)
