"""Activations in 8 bits (zl_op_act8_*): codes, values, activations and weight gradients against a 64-bit restatement; refusals."""
import pytest
import torch

from tests import act8_common as R

gpu = pytest.mark.gpu
FMTS = [R.E4M3, R.INT8]


@pytest.fixture(scope="module")
def B():
    import paper_2608_07974_gb300 as pkg
    pkg.build()
    from paper_2608_07974_gb300 import binding
    return binding


def code(B, dtype):
    return B.ZL_DTYPE_F32 if dtype == "f32" else B.ZL_DTYPE_BF16


def rows(N, d, dtype, seed=0):
    """Rows whose groups differ in size by many powers of two, with zeros, ties and group borders among them."""
    g = torch.Generator().manual_seed(seed + 131 * N + d)
    x = torch.randn(N, d, generator=g, dtype=torch.float64) * torch.exp2(torch.randint(-30, 30, (N, d // 32 + 1), generator=g).double()).repeat_interleave(32, 1)[:, :d]
    x[torch.rand(N, d, generator=g) < 0.05] = 0
    tie = torch.rand(N, d, generator=g) < 0.1
    x[tie] = torch.randint(-300, 300, (int(tie.sum()),), generator=g).double() / 2      # halves of a step, and 448 and 127 themselves
    if N > 2:
        x[N // 2] = 0
    x[0, 0] = 448.0
    x[-1, -1] = -127.0
    return x.to(R.DT[dtype])


def empty_codes(N, d, device="cuda"):
    D = R.width(d)
    return torch.full((N, D), 0x55, dtype=torch.uint8, device=device), torch.full((N, D // 32), 0x55, dtype=torch.uint8, device=device)


# ---- the restatement itself ---------------------------------------------------------------------
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_reference_codes_are_the_nearest(fmt, dtype):
    """Every held value is a nearest one of its group's grid, exactly a bf16, and the group's power of two the smallest."""
    x = rows(9, 77, dtype)
    q, e = R.store(x, fmt)
    v = R.load(q, e, fmt, 77)
    assert torch.equal(v, v.to(torch.bfloat16).double())
    grid = R.load(torch.arange(256, dtype=torch.uint8).view(8, 32), torch.full((8, 1), 127, dtype=torch.uint8), fmt, 32).flatten()
    grid = grid[~torch.isnan(grid)]
    xd = x.double()
    s = R.two(e.long() - 127).repeat_interleave(32, 1)[:, :77]
    best = ((xd / s)[..., None] - grid).abs().amin(-1) * s
    assert torch.equal((v - xd).abs(), best)
    Q = 448.0 if fmt == R.E4M3 else 127.0
    big = torch.nn.functional.pad(xd, (0, 96 - 77)).abs().view(9, 3, 32).amax(2)
    sg = R.two(e.long() - 127)
    assert bool((big <= Q * sg).all()) and bool(((big > Q * sg / 2) | (e == 10)).all())
    if fmt == R.E4M3:
        y = (xd / s).float().to(torch.float8_e4m3fn)
        assert torch.equal(y.view(torch.uint8), q[:, :77])


def test_reference_special_values():
    big = torch.finfo(torch.float32).max
    x = torch.zeros(2, 40)
    x[0, 0], x[0, 1], x[0, 2], x[0, 3] = float("nan"), float("inf"), float("-inf"), 1.0
    x[1, 0], x[1, 33], x[1, 34] = big, 2.0 ** -140, -2.0 ** -126
    for fmt in FMTS:
        v = R.load(*R.store(x, fmt), fmt, 40)
        assert torch.isnan(v[0, :3]).all() and v[0, 3] == 1.0
        assert v[1, 0] == R.TOP and v[1, 33] == 0 and v[1, 34] in (-2.0 ** -126, 0)


# ---- refusals (no GPU needed: the arguments are checked on the host) -----------------------------
P = 1 << 20   # a 16-byte aligned address that no refused call touches


@pytest.mark.parametrize("bad", [dict(dtype=2), dict(fmt=2), dict(fmt=-1), dict(N=-1), dict(N=(1 << 24) + 1), dict(d=0), dict(d=(1 << 20) + 1),
                                 dict(ldx=63), dict(N=1 << 24, d=1024, ldx=1024), dict(x=None), dict(q=None), dict(e=None), dict(q=P + 8)])
def test_store_and_load_refuse(B, bad):
    a = dict(dtype=0, fmt=0, x=P, N=4, d=64, ldx=64, q=P, e=P) | bad
    for call in (lambda: B.zl_op_act8_store(a["dtype"], a["fmt"], a["x"], a["N"], a["d"], a["ldx"], a["q"], a["e"]),
                 lambda: B.zl_op_act8_load(a["dtype"], a["fmt"], a["q"], a["e"], a["N"], a["d"], a["ldx"], a["x"])):
        with pytest.raises(B.ZLError) as err:
            call()
        assert err.value.status == B.ZL_ERR_ARG


@pytest.mark.parametrize("bad", [dict(act=2), dict(act=-1), dict(dtype=7), dict(fmt=3), dict(f=0), dict(N=-2), dict(x=None), dict(y=None), dict(q=P + 4)])
def test_activations_refuse(B, bad):
    a = dict(dtype=1, act=0, fmt=0, x=P, N=4, f=64, y=P, q=P, e=P) | bad
    with pytest.raises(B.ZLError) as err:
        B.zl_op_act8_act(a["dtype"], a["act"], a["fmt"], a["x"], a["N"], a["f"], a["y"], a["q"], a["e"])
    assert err.value.status == B.ZL_ERR_ARG
    with pytest.raises(B.ZLError) as err:
        B.zl_op_act8_act_bwd(a["dtype"], a["act"], a["fmt"], a["q"], a["e"], a["x"], a["N"], a["f"], a["y"])
    assert err.value.status == B.ZL_ERR_ARG


@pytest.mark.parametrize("dtype,off", [(0, 1), (0, 2), (0, 3), (1, 1)])
def test_addresses_inside_an_element_are_refused(B, dtype, off):
    """Every tensor in turn off the alignment of its elements (4 bytes of fp32, 2 of bf16), which a kernel would fault on."""
    from paper_2608_07974_gb300.binding import _check, _lib
    Q = P + off
    calls = [lambda: B.zl_op_act8_store(dtype, 0, Q, 4, 64, 64, P, P), lambda: B.zl_op_act8_load(dtype, 0, P, P, 4, 64, 64, Q),
             lambda: B.zl_op_act8_act(dtype, 0, 0, Q, 4, 64, P, P, P), lambda: B.zl_op_act8_act(dtype, 1, 0, P, 4, 64, Q, P, P),
             lambda: B.zl_op_act8_act_bwd(dtype, 0, 0, P, P, Q, 4, 64, P), lambda: B.zl_op_act8_act_bwd(dtype, 1, 0, P, P, P, 4, 64, Q),
             lambda: B.zl_op_act8_act_bwd(dtype, 1, 0, P, P, P, 4, 64, P, Q),
             lambda: _check(_lib.zl_op_act8_dw(dtype, 0, 32, 64, 16, P, P, P, Q, 0, P, 1 << 24, None)),
             lambda: _check(_lib.zl_op_act8_dw(dtype, 0, 32, 64, 0, None, None, None, Q, 0, None, 0, None))]
    for k, call in enumerate(calls):
        with pytest.raises(B.ZLError) as err:
            call()
        assert err.value.status == B.ZL_ERR_ARG, k


@pytest.mark.parametrize("bad", [dict(dtype=-1), dict(fmt=2), dict(M=0), dict(N=0), dict(K=-1), dict(A=None), dict(q=None), dict(C=None),
                                 dict(acc=2), dict(ws=None), dict(ws="small"), dict(A=P + 8)])
def test_weight_gradient_refuses(B, bad):
    a = dict(dtype=1, fmt=0, M=32, N=64, K=16, A=P, q=P, e=P, C=P, acc=0, ws="ok") | bad
    n = B.zl_op_act8_dw_bytes(1, 32, 64, 16)
    ws = None if a["ws"] is None else torch.empty(n - 1 if a["ws"] == "small" else n, dtype=torch.uint8)
    from paper_2608_07974_gb300.binding import _check, _lib
    with pytest.raises(B.ZLError) as err:
        _check(_lib.zl_op_act8_dw(a["dtype"], a["fmt"], a["M"], a["N"], a["K"], a["A"], a["q"], a["e"], a["C"], a["acc"],
                                  None if ws is None else P, 0 if ws is None else ws.numel(), None))
    assert err.value.status == B.ZL_ERR_ARG


def test_no_rows_is_no_work(B):
    """N = 0 touches nothing, whatever the pointers."""
    B.zl_op_act8_store(0, 0, None, 0, 64, 64, None, None)
    B.zl_op_act8_load(0, 0, None, None, 0, 64, 64, None)
    B.zl_op_act8_act(1, 0, 0, None, 0, 64, None, None, None)
    B.zl_op_act8_act_bwd(1, 0, 0, None, None, None, 0, 64, None)


def test_binding_checks_tensors(B):
    x, q, e = torch.zeros(4, 64), torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(4, 2, dtype=torch.uint8)
    with pytest.raises(B.ZLError):          # on the CPU
        B.zl_op_act8_store(0, 0, x, 4, 64, 64, q, e)
    with pytest.raises(TypeError):
        B.zl_op_act8_store(1, 0, x, 4, 64, 64, q, e)
    with pytest.raises(TypeError):
        B.zl_op_act8_store(0, 0, P, 4, 64, 64, q.to(torch.int8), e)


def test_binding_takes_no_workspace_by_address(B):
    """An address says nothing of its size: refused by name (it ended in an AttributeError)."""
    p = B.zl_block_norm(dtype=0, post_norm=1, pre_norm=1, N=4, d=64, gate_rows=0, eps=1e-5, res_scale=1, branch_scale=1, fmt=0, accumulate=0)
    for call in (lambda: B.zl_op_act8_dw(1, 0, 32, 64, 16, P, P, P, P, 0, P),
                 lambda: B.zl_op_block_norm_bwd(p, P, P, None, None, P, None, None, P, P, P, P, P, P, None, None, None, None, None, P)):
        with pytest.raises(TypeError, match="ws"):
            call()


@gpu
def test_binding_checks_device_tensors(B):
    x = torch.zeros(4, 128, device="cuda")
    q, e = empty_codes(4, 64)
    for bad in (lambda: B.zl_op_act8_store(0, 0, x[:, ::2], 4, 64, 128, q, e),            # columns apart
                lambda: B.zl_op_act8_store(0, 0, x[:, :64], 4, 64, 64, q, e),              # another stride than given
                lambda: B.zl_op_act8_store(0, 0, x[:3, :64], 4, 64, 128, q, e),            # too few rows
                lambda: B.zl_op_act8_store(0, 0, x, 4, 128, 128, q, e),                    # codes too small
                lambda: B.zl_op_act8_store(0, 0, x[:, :64], 4, 64, 128, q.t(), e),
                lambda: B.zl_op_act8_store(0, 0, x[:, :64], 4, 64, 128, q.cpu(), e)):
        with pytest.raises(B.ZLError) as err:
            bad()
        assert err.value.status == B.ZL_ERR_ARG


# ---- codes and values ---------------------------------------------------------------------------
SHAPES = [(1, 1, 1), (1, 32, 32), (3, 31, 31), (2, 33, 40), (5, 100, 100), (128, 768, 768), (7, 1001, 1001), (33, 1100, 2200), (17, 4096, 4097),
          (1, 22016, 22016), (1025, 8, 8)]


@gpu
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,d,ld", SHAPES)
def test_store_and_load(B, dtype, fmt, N, d, ld):
    """Codes and group bytes bit for bit, values exactly, and columns behind the rows untouched."""
    x = rows(N, d, dtype)
    wide = torch.full((N, ld), 7.0, dtype=x.dtype, device="cuda")
    wide[:, :d] = x.cuda()
    q, e = empty_codes(N, d)
    B.zl_op_act8_store(code(B, dtype), fmt, wide[:, :d], N, d, ld, q, e)
    rq, re = R.store(x, fmt)
    assert torch.equal(e.cpu(), re)
    assert torch.equal(q.cpu(), rq)
    back = torch.full((N, ld), 7.0, dtype=x.dtype, device="cuda")
    B.zl_op_act8_load(code(B, dtype), fmt, q, e, N, d, ld, back[:, :d])
    assert torch.equal(back[:, :d].cpu().double(), R.load(rq, re, fmt, d))
    assert bool((back[:, d:] == 7.0).all())
    # from the other type's tensor the same values come back
    other = "bf16" if dtype == "f32" else "f32"
    b2 = torch.empty(N, d, dtype=R.DT[other], device="cuda")
    B.zl_op_act8_load(code(B, other), fmt, q, e, N, d, d, b2)
    assert torch.equal(b2.double().cpu(), back[:, :d].double().cpu())


@gpu
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_every_value_and_special_ones(B, dtype, fmt):
    """All bf16 bit patterns (and neighbours of them in fp32) in groups of their own size and mixed, NaN, infinities and the
    largest and smallest magnitudes among them."""
    bits = torch.arange(65536, dtype=torch.int32)
    x = (bits << 16).view(torch.float32)
    if dtype == "f32":
        x = torch.cat([x, ((bits << 16) + 0x7FFF).view(torch.float32), ((bits << 16) + 0x8001).view(torch.float32)])
    mixed = x[torch.randperm(len(x), generator=torch.Generator().manual_seed(3))]
    x = torch.cat([x, mixed]).view(-1, 256).to(R.DT[dtype])
    N = len(x)
    q, e = empty_codes(N, 256)
    B.zl_op_act8_store(code(B, dtype), fmt, x.cuda(), N, 256, 256, q, e)
    rq, re = R.store(x, fmt)
    assert torch.equal(e.cpu(), re)
    assert torch.equal(q.cpu(), rq)
    back = torch.empty(N, 256, dtype=x.dtype, device="cuda")
    B.zl_op_act8_load(code(B, dtype), fmt, q, e, N, 256, 256, back)
    v = R.load(rq, re, fmt, 256)
    assert torch.equal(torch.isnan(back).cpu(), torch.isnan(v))
    assert torch.equal(torch.nan_to_num(back.cpu().double()), torch.nan_to_num(v))


@gpu
@pytest.mark.parametrize("dtype,off", [("bf16", 1), ("bf16", 3), ("f32", 1), ("f32", 2)])
def test_tensors_off_16_bytes(B, dtype, off):
    """Rows that start anywhere an element may."""
    N, d = 5, 96
    x = rows(N, d, dtype)
    flat = torch.zeros(N * d + 8, dtype=x.dtype, device="cuda")
    view = flat[off:off + N * d].view(N, d)
    view.copy_(x)
    q, e = empty_codes(N, d)
    B.zl_op_act8_store(code(B, dtype), R.E4M3, view, N, d, d, q, e)
    rq, re = R.store(x, R.E4M3)
    assert torch.equal(q.cpu(), rq) and torch.equal(e.cpu(), re)
    out = torch.zeros_like(flat)
    B.zl_op_act8_load(code(B, dtype), R.E4M3, q, e, N, d, d, out[off:off + N * d].view(N, d))
    assert torch.equal(out[off:off + N * d].view(N, d).cpu().double(), R.load(rq, re, R.E4M3, d))
    assert bool((out[:off] == 0).all()) and bool((out[off + N * d:] == 0).all())


@gpu
def test_offsets_beyond_32_bits(B):
    """More than 2^32 values: the last rows of a tall tensor."""
    N, d = 65600, 65536
    x = torch.empty(N, d, dtype=torch.bfloat16, device="cuda")
    x[-70:] = rows(70, d, "bf16").cuda()
    x[:-70].zero_()
    q, e = torch.empty(N, d, dtype=torch.uint8, device="cuda"), torch.empty(N, d // 32, dtype=torch.uint8, device="cuda")
    B.zl_op_act8_store(B.ZL_DTYPE_BF16, R.INT8, x, N, d, d, q, e)
    rq, re = R.store(x[-70:].cpu(), R.INT8)
    assert torch.equal(q[-70:].cpu(), rq) and torch.equal(e[-70:].cpu(), re)
    assert int(q[:-70].count_nonzero()) == 0 and bool((e[:-70] == 10).all())
    x.fill_(7)
    B.zl_op_act8_load(B.ZL_DTYPE_BF16, R.INT8, q, e, N, d, d, x)
    assert torch.equal(x[-70:].cpu().double(), R.load(rq, re, R.INT8, d))
    assert int(x[:-70].count_nonzero()) == 0


# ---- activations --------------------------------------------------------------------------------
def act_bounds(x, kind, dtype, dy=None):
    """Error bounds of y and dx at x: half a step of the result, and 32 (1 + |exponent's argument|) roundings in 24 bits of
    the terms (e^z has |z| times its argument's relative error; its fast form adds 2 more), with the fast forms' flush of
    results below the normal range."""
    half, ulp, tiny = R.HALF[R.DT[dtype]], 2.0 ** -24, 2.0 ** -120
    y = R.act(x, kind)
    if kind == R.SWIGLU:
        g, u = x.chunk(2, 1)
        amp = 32 * ulp * (1 + g.abs())
        s = torch.sigmoid(g)
        by = (half + amp) * y.abs() + tiny
        if dy is None:
            return y, by
        dg, du = dy * u * s * (1 + g * (1 - s)), dy * g * s
        # 1 - s is formed by a subtraction: its error is that of s, absolute
        bg = half * dg.abs() + amp * (dy * u).abs() * s * (1 + g.abs()) + tiny
        return y, by, torch.cat([dg, du], 1), torch.cat([bg, (half + amp) * du.abs() + tiny], 1)
    k, c = (2 / torch.pi) ** 0.5, 0.044715
    z = 2 * k * (x + c * x ** 3)
    s = torch.sigmoid(z)
    amp = 32 * ulp * (1 + z.abs())
    by = (half + amp) * y.abs() + tiny
    if dy is None:
        return y, by
    t2 = 2 * x.abs() * s * k * (1 + 3 * c * x * x)
    dx = dy * (s + 2 * x * s * torch.sigmoid(-z) * k * (1 + 3 * c * x * x))
    return y, by, dx, half * dx.abs() + amp * dy.abs() * (s + t2) + tiny


ACTS = [(1, 8), (3, 5), (2, 33), (203, 344), (64, 1000), (9, 1001), (130, 2112), (5, 11008)]


@gpu
@pytest.mark.parametrize("kind", [R.SWIGLU, R.GELU])
@pytest.mark.parametrize("dtype,fmt", [("f32", R.E4M3), ("f32", R.INT8), ("bf16", R.E4M3), ("bf16", R.INT8)])
@pytest.mark.parametrize("N,f", ACTS)
def test_activation_and_its_backward(B, dtype, fmt, kind, N, f):
    g = torch.Generator().manual_seed(N + f)
    w = 2 if kind == R.SWIGLU else 1
    T = R.DT[dtype]
    x = 3 * torch.randn(N, w * f, generator=g)
    x[torch.rand(x.shape, generator=g) < 0.01] = -40.0          # a sigmoid that vanishes
    x, dy = x.to(T), torch.randn(N, f, generator=g).to(T)
    y, again = (torch.full((N, f), 7.0, dtype=T, device="cuda") for _ in range(2))
    dx = torch.full((N, w * f), 7.0, dtype=T, device="cuda")
    q, e = empty_codes(w * N, f)
    B.zl_op_act8_act(code(B, dtype), kind, fmt, x.cuda(), N, f, y, q, e)
    rq, re = R.store(x.view(-1, f), fmt)
    assert torch.equal(q.cpu(), rq) and torch.equal(e.cpu(), re)
    R.assert_close(y, *act_bounds(x.double(), kind, dtype), "y")
    B.zl_op_act8_act_bwd(code(B, dtype), kind, fmt, q, e, dy.cuda(), N, f, dx, again)
    x8 = R.load(rq, re, fmt, f).reshape(N, w * f)
    ry, by, rdx, bdx = act_bounds(x8, kind, dtype, dy.double())
    R.assert_close(again, ry, by, "y again")
    R.assert_close(dx, rdx, bdx, "dx")
    dx2 = torch.empty_like(dx)
    B.zl_op_act8_act_bwd(code(B, dtype), kind, fmt, q, e, dy.cuda(), N, f, dx2)
    assert torch.equal(dx, dx2)


@pytest.mark.parametrize("kind", [R.SWIGLU, R.GELU])
def test_activation_gradient_formula(kind):
    """The gradients of act_bounds against differences of the activation, in 64 bits: a step of 1e-4 leaves a third-order
    term of about 1e-8 and rounding of about 1e-12."""
    g = torch.Generator().manual_seed(1)
    x, dy = torch.randn(6, 20, generator=g, dtype=torch.float64), torch.randn(6, 10 if kind == R.SWIGLU else 20, generator=g, dtype=torch.float64)
    _, _, dx, _ = act_bounds(x, kind, "f32", dy)
    for _ in range(4):
        v = torch.randn(x.shape, generator=g, dtype=torch.float64)
        num = ((R.act(x + 1e-4 * v, kind) - R.act(x - 1e-4 * v, kind)) * dy).sum() / 2e-4
        assert abs(float(num - (dx * v).sum())) < 1e-6


def test_gelu_form():
    """The restated GELU is the tanh form (2^-53 |x| of absolute error in 1 + tanh)."""
    x = torch.linspace(-30, 30, 4001, dtype=torch.float64).view(1, -1)
    tanh = 0.5 * x * (1 + torch.tanh((2 / torch.pi) ** 0.5 * (x + 0.044715 * x ** 3)))
    assert float((R.act(x, R.GELU) - tanh).abs().max()) < 1e-14


@gpu
def test_activation_keeps_nan(B):
    x = torch.ones(2, 64, device="cuda")
    x[0, 3], x[0, 40], x[1, 5] = float("nan"), float("inf"), float("-inf")
    q, e = empty_codes(4, 32)
    y, dx = torch.empty(2, 32, device="cuda"), torch.empty(2, 64, device="cuda")
    B.zl_op_act8_act(B.ZL_DTYPE_F32, R.SWIGLU, R.INT8, x, 2, 32, y, q, e)
    B.zl_op_act8_act_bwd(B.ZL_DTYPE_F32, R.SWIGLU, R.INT8, q, e, torch.ones(2, 32, device="cuda"), 2, 32, dx)
    bad = torch.isnan(dx)
    # a NaN gate spoils its dg and du (du = dy g s), a NaN up its dg alone: 2 + 1 + 2
    assert bad[0, 3] and bad[0, 35] and bad[0, 8] and bad[1, 5] and bad[1, 37]
    assert int(bad.sum()) == 5


@gpu
@pytest.mark.parametrize("dtype,fmt", [("f32", R.E4M3), ("bf16", R.INT8)])
@pytest.mark.parametrize("kind", [R.SWIGLU, R.GELU])
def test_activation_of_large_values(B, dtype, fmt, kind):
    """Values whose square and cube overflow, a group of 32 columns for each: an activation is 0 or its input (times up) and
    its derivative 0 or 1 (times up). Sigmoids above are 1 in fp32; below, that of -64 is e^-64 = 1.6e-28 (SwiGLU; GELU's
    argument is the cube), times at most 64 below 1.1e-26, and the others are 0."""
    T = R.DT[dtype]
    mags = torch.tensor([2.0 ** k for k in (6, 20, 43, 64, 90, 127)])
    v = torch.cat([mags, -mags])
    x = v.repeat_interleave(32).view(1, -1).to(T)
    f, w = x.shape[1], 2 if kind == R.SWIGLU else 1
    full = torch.cat([x, torch.full_like(x, 0.5)], 1) if w == 2 else x
    y, dx, again = (torch.full((1, n), 7.0, dtype=T, device="cuda") for n in (f, w * f, f))
    q, e = empty_codes(w, f)
    B.zl_op_act8_act(code(B, dtype), kind, fmt, full.cuda(), 1, f, y, q, e)
    B.zl_op_act8_act_bwd(code(B, dtype), kind, fmt, q, e, torch.full((1, f), 0.25, dtype=T, device="cuda"), 1, f, dx, again)
    up = 0.5 if w == 2 else 1.0
    want = torch.where(x > 0, x * up, torch.zeros_like(x))

    def same(got, want):
        return bool(((got.cpu().double() - want.double()).abs() <= 1.1e-26).all())

    assert same(y, want) and same(again, want)
    assert same(dx[:, :f], torch.where(x > 0, 0.25 * up, 0.0))
    if w == 2:
        assert same(dx[:, f:], 0.25 * torch.where(x > 0, x, torch.zeros_like(x)))


@gpu
@pytest.mark.parametrize("dtype,fmt", [("f32", R.E4M3), ("f32", R.INT8), ("bf16", R.E4M3), ("bf16", R.INT8)])
def test_swiglu_gradient_of_large_factors(B, dtype, fmt):
    """Large dy and up beside gates of every size: no gradient is NaN, and where the result fits into the type (below half its
    largest value) it keeps the bounds of ordinary values. Powers of two, a group of 32 columns for each, so that the
    checkpoint holds them exactly."""
    T = R.DT[dtype]
    gates = torch.tensor([-(2.0 ** 100), -256.0, -128.0, -64.0, -16.0, -2.0, 0.0, 2.0, 2.5, 16.0, 128.0])
    ups, dys = torch.tensor([2.0 ** -100, 1.0, -(2.0 ** 64), 2.0 ** 127]), torch.tensor([2.0 ** -64, 4.0, -(2.0 ** 90), 1.9375 * 2.0 ** 127])
    gate, up, dy = (v.flatten().repeat_interleave(32).view(1, -1).to(T) for v in torch.meshgrid(gates, ups, dys, indexing="ij"))
    x, f = torch.cat([gate, up], 1), gate.shape[1]
    q, e = R.store(x.view(2, f), fmt)
    assert torch.equal(R.load(q, e, fmt, f).view(1, -1), x.double())
    dx = torch.full((1, 2 * f), 7.0, dtype=T, device="cuda")
    B.zl_op_act8_act_bwd(code(B, dtype), R.SWIGLU, fmt, q.cuda(), e.cuda(), dy.cuda(), 1, f, dx)
    assert not bool(torch.isnan(dx).any())
    _, _, ref, bound = act_bounds(x.double(), R.SWIGLU, dtype, dy.double())
    # a factor s below 2^-120 is flushed or loses digits on the way, its share of the product with it; silu' up / 2 below 2^-126
    # is off by half of 2^-149, twice dy times which is an error of dg
    lost = 2.0 ** -120 * (dy.double().abs() * torch.cat([up, gate], 0).double().abs().clamp(min=1)).reshape(1, -1)
    lost[:, :f] += 2.0 ** -149 * dy.double().abs()
    fits = ref.abs() <= torch.finfo(T).max / 2
    R.assert_close(dx.cpu()[fits], ref[fits], (bound + lost)[fits], "dx")
    assert bool((torch.sign(dx.cpu().double()) == torch.sign(ref))[~fits].all())


# ---- weight gradient ----------------------------------------------------------------------------
DWS = [(1, 1, 1), (16, 16, 16), (24, 40, 1), (8, 32, 5), (130, 72, 50), (256, 128, 203), (33, 65, 77), (384, 1000, 129), (257, 96, 1021), (768, 768, 4096),
       (130, 770, 300)]


@gpu
@pytest.mark.parametrize("dtype,fmt", [("f32", R.E4M3), ("f32", R.INT8), ("bf16", R.E4M3), ("bf16", R.INT8)])
@pytest.mark.parametrize("M,N,K", DWS)
def test_weight_gradient(B, dtype, fmt, M, N, K):
    """C = A^T X and C += A^T X: |error| <= (K + 64) 2^-23 sum |A| |X| (every product and sum in 24 bits, each off by a step at
    most, whatever the order), and one rounding more of the sum that it is added to."""
    g = torch.Generator().manual_seed(M + N + K)
    A = (torch.randn(K, M, generator=g)).to(R.DT[dtype])
    x = (torch.randn(K, N, generator=g) * torch.exp(torch.randn(N, generator=g))).to(R.DT[dtype])
    q, e = R.store(x, fmt)
    X = R.load(q, e, fmt, N)
    ref, scale = A.double().T @ X, A.double().abs().T @ X.abs()
    ws = torch.empty(B.zl_op_act8_dw_bytes(code(B, dtype), M, N, K), dtype=torch.uint8, device="cuda")
    ws.fill_(0xFF)
    C = torch.full((M, N), float("nan"), device="cuda")
    B.zl_op_act8_dw(code(B, dtype), fmt, M, N, K, A.cuda(), q.cuda(), e.cuda(), C, 0, ws)
    bound = (K + 64) * 2.0 ** -23 * scale
    R.assert_close(C, ref, bound, "C")
    C0 = torch.randn(M, N, generator=g)
    C = C0.cuda()
    B.zl_op_act8_dw(code(B, dtype), fmt, M, N, K, A.cuda(), q.cuda(), e.cuda(), C, 1, ws)
    R.assert_close(C, C0.double() + ref, bound + (K + 64) * 2.0 ** -23 * C0.double().abs(), "C +=")
    again = C0.cuda()
    B.zl_op_act8_dw(code(B, dtype), fmt, M, N, K, A.cuda(), q.cuda(), e.cuda(), again, 1, ws)
    assert torch.equal(C, again)


@gpu
@pytest.mark.parametrize("plan", ["", "256:1:1", "256:1:0", "128:1:1", "128:1:0", "64:1", "256:2:1", "64:3"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("K", [4096, 4500, 6145])
def test_weight_gradient_over_many_tokens(B, monkeypatch, dtype, plan, K):
    """Sums cut into segments of at most 2048 tokens (fp32: of 2048 rows of its three terms), under every kind of plan: the
    truncation of one accumulation, at most a step for each of 2048 products and sums of |A| |X|, and a rounding for each
    of the segments (at most 12) and splits; the products of 512 x 520 in blocks that the tiles do not divide."""
    if plan:
        monkeypatch.setenv("ZL_GEMM_TILE", plan)
    M, N = 520, 328
    g = torch.Generator(device="cuda").manual_seed(K)
    A = (torch.randn(K, M, generator=g, device="cuda") + 0.5).to(R.DT[dtype])
    x = (torch.randn(K, N, generator=g, device="cuda") + 0.5).to(R.DT[dtype])
    q, e = empty_codes(K, N)
    B.zl_op_act8_store(code(B, dtype), R.INT8, x, K, N, N, q, e)
    X = torch.empty(K, N, device="cuda")
    B.zl_op_act8_load(B.ZL_DTYPE_F32, R.INT8, q, e, K, N, N, X)
    ref, scale = (A.double().T @ X.double()).cpu(), (A.double().abs().T @ X.double().abs()).cpu()
    ws = torch.empty(B.zl_op_act8_dw_bytes(code(B, dtype), M, N, K), dtype=torch.uint8, device="cuda")
    C = torch.full((M, N), float("nan"), device="cuda")
    B.zl_op_act8_dw(code(B, dtype), R.INT8, M, N, K, A, q, e, C, 0, ws)
    bound = (2048 + 64 + 16) * 2.0 ** -23 * scale
    R.assert_close(C, ref, bound, "C")
    C0 = torch.randn(M, N, generator=g, device="cuda")
    outs = []
    for _ in range(2):
        outs.append(C0.clone())
        B.zl_op_act8_dw(code(B, dtype), R.INT8, M, N, K, A, q, e, outs[-1], 1, ws)
    R.assert_close(outs[0], ref + C0.cpu().double(), bound + 16 * 2.0 ** -23 * C0.cpu().double().abs(), "C +=")
    assert torch.equal(*outs)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("M,N,K", [(128, 64, 4096), (520, 333, 1000), (8, 8, 64)])
def test_workspace_follows_the_plan(B, monkeypatch, dtype, M, N, K):
    """The workspace is sized by the plan that the call runs: each of its splits has room for its sums."""
    size, blocks = {}, -(-K // 64) * (3 if dtype == 0 else 1)     # blocks of 64 tokens, three terms of an fp32 gradient
    for splits in (1, 2, 3):
        monkeypatch.setenv("ZL_GEMM_TILE", f"64:{splits}")
        size[splits] = B.zl_op_act8_dw_bytes(dtype, M, N, K)
    for splits in (2, 3):
        n = -(-blocks // -(-blocks // min(splits, blocks)))
        part = n * M * (-(-N // 8) * 8) * 4 if n > 1 else 0
        assert size[splits] - size[1] == -(-part // 256) * 256


FIRST_CALLS = """
import sys, threading, torch
sys.path.insert(0, %r)
from paper_2608_07974_gb300 import binding as B
n, M, N, K = 8, 256, 256, 128
A = torch.randn(K, M, device="cuda").to(torch.bfloat16)
x = torch.randn(K, N, device="cuda").to(torch.bfloat16)
q, e = torch.empty(K, N, dtype=torch.uint8, device="cuda"), torch.empty(K, N // 32, dtype=torch.uint8, device="cuda")
B.zl_op_act8_store(1, 0, x, K, N, N, q, e)
C, ws = torch.zeros(n, M, N, device="cuda"), torch.empty(n, 16 << 20, dtype=torch.uint8, device="cuda")
streams = [torch.cuda.Stream() for _ in range(n)]
torch.cuda.synchronize()
start, errors = threading.Barrier(n), []
def call(i):
    torch.cuda.set_device(0)
    start.wait()
    try:
        B.zl_op_act8_dw(1, 0, M, N, K, A, q, e, C[i], 0, ws[i], streams[i].cuda_stream)
    except Exception as err:
        errors.append(str(err))
threads = [threading.Thread(target=call, args=(i,)) for i in range(n)]
[t.start() for t in threads]
[t.join() for t in threads]
torch.cuda.synchronize()
assert not errors, errors
assert all(torch.equal(C[i], C[0]) for i in range(n)) and bool(C[0].any())
print("all")
"""


@gpu
def test_first_calls_of_several_threads(B):
    """A process whose first weight gradients come from eight threads at once."""
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST_CALLS % root], capture_output=True, text=True, timeout=300, cwd=root)
    assert r.returncode == 0 and "all" in r.stdout, r.stderr[-2000:]


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_weight_gradient_of_no_tokens(B, dtype):
    C = torch.ones(8, 16, device="cuda")
    B.zl_op_act8_dw(code(B, dtype), 0, 8, 16, 0, None, None, None, C, 1, None)
    assert bool((C == 1).all())
    B.zl_op_act8_dw(code(B, dtype), 0, 8, 16, 0, None, None, None, C, 0, None)
    assert bool((C == 0).all())


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_weight_gradient_keeps_nan_to_its_column(B, dtype):
    """A NaN in column j of X reaches column j of C and no other, wherever in K it stands."""
    M, N, K = 64, 96, 70
    x = torch.ones(K, N)
    x[69, 50] = float("nan")
    q, e = R.store(x.to(R.DT[dtype]), R.INT8)
    ws = torch.empty(B.zl_op_act8_dw_bytes(code(B, dtype), M, N, K), dtype=torch.uint8, device="cuda")
    C = torch.zeros(M, N, device="cuda")
    B.zl_op_act8_dw(code(B, dtype), R.INT8, M, N, K, torch.ones(K, M, dtype=R.DT[dtype], device="cuda"), q.cuda(), e.cuda(), C, 0, ws)
    bad = torch.isnan(C)
    assert bool(bad[:, 50].all()) and int(bad.sum()) == M and float(C[0, 0]) == K


# ---- streams, graphs ----------------------------------------------------------------------------
@gpu
def test_on_another_stream_and_in_a_graph(B):
    """Store, activation, backward and weight gradient captured once and replayed on new inputs, on a stream of their own."""
    N, f, M = 96, 256, 128
    T = torch.bfloat16
    x, dy, A = (torch.randn(*s, device="cuda").to(T) for s in ((N, 2 * f), (N, f), (N, M)))
    y, again, dx = torch.empty(N, f, dtype=T, device="cuda"), torch.empty(N, f, dtype=T, device="cuda"), torch.empty(N, 2 * f, dtype=T, device="cuda")
    q, e = empty_codes(2 * N, f)
    yq, ye = empty_codes(N, f)
    C = torch.empty(M, f, device="cuda")
    ws = torch.empty(B.zl_op_act8_dw_bytes(1, M, f, N), dtype=torch.uint8, device="cuda")

    def step(s):
        B.zl_op_act8_act(1, R.SWIGLU, R.E4M3, x, N, f, y, q, e, s)
        B.zl_op_act8_act_bwd(1, R.SWIGLU, R.E4M3, q, e, dy, N, f, dx, again, s)
        B.zl_op_act8_store(1, R.E4M3, again, N, f, f, yq, ye, s)
        B.zl_op_act8_dw(1, R.E4M3, M, f, N, A, yq, ye, C, 0, ws, s)

    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        step(st.cuda_stream)
    st.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        step(st.cuda_stream)
    for _ in range(3):
        x.copy_(torch.randn(N, 2 * f, device="cuda"))
        A.copy_(torch.randn(N, M, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (y, dx, again, C)]
        step(0)
        torch.cuda.synchronize()
        for a, b in zip(got, (y, dx, again, C)):
            assert torch.equal(a, b)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,d", [(1, 1), (5, 31), (37, 1001), (130, 264), (3, 5000)])
def test_outputs_stay_in_bounds(B, dtype, N, d):
    """Every output between two bands of a bit pattern, which stay as they are."""
    T, dt, bufs = R.DT[dtype], code(B, dtype), {}

    def out(name, n, t):
        size = torch.empty(0, dtype=t).element_size()
        bufs[name] = (torch.full((n * size + 8192,), 0xA5, dtype=torch.uint8, device="cuda"), n * size)
        return bufs[name][0][4096:4096 + n * size].view(t)

    D = R.width(d)
    x, dy, A = (torch.randn(*s, device="cuda").to(T) for s in ((N, 2 * d), (N, d), (N, 24)))
    q, e = out("q", 2 * N * D, torch.uint8), out("e", 2 * N * D // 32, torch.uint8)
    y, again, dx, back = out("y", N * d, T), out("again", N * d, T), out("dx", 2 * N * d, T), out("back", 2 * N * d, T)
    B.zl_op_act8_act(dt, R.SWIGLU, R.INT8, x, N, d, y, q, e)
    B.zl_op_act8_act_bwd(dt, R.SWIGLU, R.INT8, q, e, dy, N, d, dx, again)
    B.zl_op_act8_load(dt, R.INT8, q, e, 2 * N, d, d, back.view(2 * N, d))
    q2, e2 = out("q2", N * D, torch.uint8), out("e2", N * D // 32, torch.uint8)
    B.zl_op_act8_store(dt, R.E4M3, y.view(N, d), N, d, d, q2, e2)
    C = out("C", 24 * d, torch.float32)
    nws = B.zl_op_act8_dw_bytes(dt, 24, d, N)
    ws = torch.full((nws + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
    B.zl_op_act8_dw(dt, R.E4M3, 24, d, N, A, q2, e2, C, 0, ws[:nws])
    torch.cuda.synchronize()
    for name, (b, m) in bufs.items():
        assert bool((b[:4096] == 0xA5).all()) and bool((b[4096 + m:] == 0xA5).all()), name
    assert bool((ws[nws:] == 0xA5).all())
