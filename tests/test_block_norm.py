"""The fused step between two blocks (zl_op_block_norm) and its backward, against a 64-bit restatement; refusals; a whole
feed-forward block with 8-bit checkpoints."""
import pytest
import torch

from tests import act8_common as R

gpu = pytest.mark.gpu
ULP = 2.0 ** -24


@pytest.fixture(scope="module")
def B():
    import paper_2608_07974_gb300 as pkg
    pkg.build()
    from paper_2608_07974_gb300 import binding
    return binding


def code(B, dtype):
    return B.ZL_DTYPE_F32 if dtype == "f32" else B.ZL_DTYPE_BF16


def dims(B, dtype, c, N, d, fmt=R.E4M3, accumulate=0):
    return B.zl_block_norm(dtype=code(B, dtype), post_norm=c["post"], pre_norm=c["pre"], N=N, d=d, gate_rows=c["rows"], eps=c["eps"],
                           res_scale=c["alpha"], branch_scale=c["beta"], fmt=fmt, accumulate=accumulate)


def setting(post, pre, rows=0, eps=1e-5, alpha=1.25, beta=-0.75):
    eps, alpha, beta = (float(torch.tensor(v, dtype=torch.float32)) for v in (eps, alpha, beta))   # as the call holds them
    return dict(post=post, pre=pre, rows=rows, eps=eps, alpha=alpha, beta=beta)


def params(c, N, d, g, gated=True, weighted=True):
    def w(on, b):
        return (b + 0.2 * torch.randn(d, generator=g)) if on and weighted else None

    G = -(-N // c["rows"]) if c["rows"] else 1
    return dict(post_w=w(c["post"], 1), post_b=w(c["post"] == R.LAYER, 0), gate=0.5 + 0.5 * torch.randn(G, d, generator=g) if gated else None,
                pre_w=w(c["pre"], 1), pre_b=w(c["pre"] == R.LAYER, 0))


def acts(N, d, dtype, g):
    return (torch.randn(N, d, generator=g) * torch.exp(0.5 * torch.randn(d, generator=g)) + 0.3).to(R.DT[dtype])


def cuda(p):
    return {k: None if v is None else v.cuda() for k, v in p.items()}


def dbl(p):
    return {k: None if v is None else v.double() for k, v in p.items()}


def codes(N, d):
    D = R.width(d)
    return torch.full((N, D), 0x55, dtype=torch.uint8, device="cuda"), torch.full((N, D // 32), 0x55, dtype=torch.uint8, device="cuda")


# ---- refusals ------------------------------------------------------------------------------------
P = 1 << 20


def call_forward(B, **bad):
    a = dict(dtype=0, post=1, pre=1, N=4, d=64, rows=0, eps=1e-5, fmt=0, accumulate=0, h=P, f=P, post_w=P, post_b=None, gate=P, pre_w=P, pre_b=None,
             h_out=P, n_out=P, stats=P, f_q=None, f_e=None, n_q=None, n_e=None) | bad
    p = B.zl_block_norm(dtype=a["dtype"], post_norm=a["post"], pre_norm=a["pre"], N=a["N"], d=a["d"], gate_rows=a["rows"], eps=a["eps"], res_scale=1,
                        branch_scale=1, fmt=a["fmt"], accumulate=a["accumulate"])
    B.zl_op_block_norm(p, *(a[k] for k in ("h", "f", "post_w", "post_b", "gate", "pre_w", "pre_b", "h_out", "n_out", "stats", "f_q", "f_e", "n_q", "n_e")))


DIMS_BAD = [dict(dtype=2), dict(post=3), dict(pre=-1), dict(N=-1), dict(N=(1 << 24) + 1), dict(d=0), dict(d=(1 << 20) + 1), dict(N=1 << 24, d=2048),
            dict(rows=-1), dict(eps=0.0), dict(eps=float("nan")), dict(fmt=2), dict(accumulate=2)]


@pytest.mark.parametrize("bad", DIMS_BAD + [dict(post_b=P), dict(pre_b=P), dict(post=0), dict(pre=0), dict(pre=0, pre_w=None), dict(n_out=None), dict(h=None),
                                            dict(f=None), dict(h_out=None), dict(stats=None), dict(f_q=P), dict(n_e=P), dict(f_q=P + 8, f_e=P),
                                            dict(n_q=P + 4, n_e=P), dict(pre=0, pre_w=None, n_out=None, n_q=P, n_e=P)])
def test_forward_refuses(B, bad):
    with pytest.raises(B.ZLError) as err:
        call_forward(B, **bad)
    assert err.value.status == B.ZL_ERR_ARG


def call_backward(B, **bad):
    a = dict(dtype=0, post=1, pre=1, N=4, d=64, rows=0, eps=1e-5, fmt=0, accumulate=0, h_out=P, f=None, f_q=P, f_e=P, post_w=P, post_b=None, gate=P,
             pre_w=P, stats=P, dn=P, dh_out=P, dh=P, df=P, dpost_w=P, dpost_b=None, dgate=P, dpre_w=P, dpre_b=None, ws=P, ws_bytes=None) | bad
    from ctypes import byref
    from paper_2608_07974_gb300.binding import _check, _lib
    p = B.zl_block_norm(dtype=a["dtype"], post_norm=a["post"], pre_norm=a["pre"], N=a["N"], d=a["d"], gate_rows=a["rows"], eps=a["eps"], res_scale=1,
                        branch_scale=1, fmt=a["fmt"], accumulate=a["accumulate"])
    n = a["ws_bytes"] if a["ws_bytes"] is not None else 1 << 20
    _check(_lib.zl_op_block_norm_bwd(byref(p), *(a[k] for k in ("h_out", "f", "f_q", "f_e", "post_w", "post_b", "gate", "pre_w", "stats", "dn", "dh_out", "dh",
                                                               "df", "dpost_w", "dpost_b", "dgate", "dpre_w", "dpre_b", "ws")), n, None))


@pytest.mark.parametrize("bad", DIMS_BAD + [dict(post_b=P), dict(dpost_b=P), dict(dpre_b=P), dict(post=0), dict(pre=0), dict(gate=None), dict(h_out=None),
                                            dict(stats=None), dict(df=None), dict(dn=None), dict(f=P), dict(f_q=None, f_e=None), dict(f_e=None),
                                            dict(f_q=P + 8), dict(ws=None), dict(ws=P + 16), dict(ws_bytes=0), dict(ws_bytes=255),
                                            dict(pre=0, pre_w=None, dpre_w=None, dn=None, dh_out=None)])
def test_backward_refuses(B, bad):
    with pytest.raises(B.ZLError) as err:
        call_backward(B, **bad)
    assert err.value.status == B.ZL_ERR_ARG


@pytest.mark.parametrize("dtype,off", [(0, 1), (0, 2), (0, 3), (1, 1)])
def test_addresses_inside_an_element_are_refused(B, dtype, off):
    """Every tensor in turn off the alignment of its elements (4 bytes of fp32, 2 of bf16), which a kernel would fault on."""
    Q = P + off
    for name in ("h", "f", "h_out", "n_out", "post_w", "post_b", "gate", "pre_w", "pre_b", "stats"):
        with pytest.raises(B.ZLError) as err:
            call_forward(B, dtype=dtype, post=2, pre=2, **{name: Q})
        assert err.value.status == B.ZL_ERR_ARG, name
    for name in ("h_out", "f", "dn", "dh_out", "dh", "df", "post_w", "post_b", "gate", "pre_w", "stats", "dpost_w", "dpost_b", "dgate", "dpre_w", "dpre_b"):
        with pytest.raises(B.ZLError) as err:
            call_backward(B, dtype=dtype, post=2, pre=2, **({"f_q": None, "f_e": None} if name == "f" else {}), **{name: Q})
        assert err.value.status == B.ZL_ERR_ARG, name


def test_struct_matches_the_header(B):
    import ctypes
    from tests.test_abi import _header_struct_fields
    kinds = {"int": ctypes.c_int, "float": ctypes.c_float}
    assert [(n, kinds[t]) for n, t in _header_struct_fields("zl_block_norm")] == list(B.zl_block_norm._fields_)


# ---- the restatement's gradients ------------------------------------------------------------------
@pytest.mark.parametrize("post", [R.NONE, R.RMS, R.LAYER])
@pytest.mark.parametrize("pre", [R.NONE, R.RMS, R.LAYER])
def test_reference_gradients(post, pre):
    """The restated backward against autograd of the restated forward (1e-9: some thousand roundings of 2^-53) and against
    differences along random directions (step 1e-4: third-order term about 1e-8)."""
    c, g = setting(post, pre, rows=3), torch.Generator().manual_seed(post * 3 + pre)
    N, d = 7, 20
    t = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)  # noqa: E731
    p = dbl(params(c, N, d, g))
    x = dict(h=t(N, d), f=t(N, d), **p)
    dn, dho = t(N, d) if pre else None, t(N, d)

    def loss(v):
        ho, n, _ = R.block_norm(c, **v)
        return (ho * dho).sum() + ((n * dn).sum() if pre else 0)

    ho, n, stats = R.block_norm(c, **x)
    got = R.block_norm_bwd(c, ho, x["f"], p["post_w"], p["post_b"], p["gate"], p["pre_w"], stats, dn, dho)
    leaves = {k: v.clone().requires_grad_(True) for k, v in x.items() if v is not None}
    auto = dict(zip(leaves, torch.autograd.grad(loss({**x, **leaves}), list(leaves.values()))))
    for k, v in auto.items():
        assert float((got["d" + k][0] - v).abs().max()) < 1e-9, k
        for _ in range(2):
            v1 = t(*v.shape)
            num = (loss({**x, k: x[k] + 1e-4 * v1}) - loss({**x, k: x[k] - 1e-4 * v1})) / 2e-4
            assert abs(float(num - (v * v1).sum())) < 1e-5, k


# ---- forward ---------------------------------------------------------------------------------------
def spread(x, kind, eps):
    """How much larger than themselves the rounding errors of the values under a norm weigh in its deviation."""
    xc = x - x.mean(1, keepdim=True) if kind == R.LAYER else x
    return 1 + ((x.abs() + x.abs().mean(1, keepdim=True)) * xc.abs()).mean(1, keepdim=True) / (xc.square().mean(1, keepdim=True) + eps)


def check_forward(B, dtype, c, N, d, fmt, keep, seed=0, gated=True, weighted=True, inplace=False):
    g = torch.Generator().manual_seed(seed + N + d)
    T = R.DT[dtype]
    h, f, p = acts(N, d, dtype, g), acts(N, d, dtype, g), params(c, N, d, g, gated, weighted)
    q = cuda(p)
    hc = h.cuda()
    ho = hc if inplace else torch.full((N, d), 7.0, dtype=T, device="cuda")
    n = torch.full((N, d), 7.0, dtype=T, device="cuda") if c["pre"] else None
    stats = torch.full((4, N), 7.0, device="cuda")
    fq, fe = codes(N, d) if keep else (None, None)
    nq, ne = codes(N, d) if keep and c["pre"] else (None, None)
    B.zl_op_block_norm(dims(B, dtype, c, N, d, fmt), hc, f.cuda(), q["post_w"], q["post_b"], q["gate"], q["pre_w"], q["pre_b"], ho, n, stats, fq, fe, nq, ne)
    torch.cuda.synchronize()
    hd, fd, pd = h.double(), f.double(), dbl(p)
    rho, rn, rst = R.block_norm(c, hd, fd, **pd)
    # 64 roundings: of a tree over at most 512 threads of 32 values (9 + 32), and a dozen of the arithmetic around it
    e64 = 64 * ULP
    one = torch.ones(d, dtype=torch.float64)
    aw, ab = (one if pd["post_w"] is None else pd["post_w"].abs()), (0 * one if pd["post_b"] is None else pd["post_b"].abs())
    gt = 1.0 if pd["gate"] is None else pd["gate"][R.gate_index(N, c["rows"])].abs()
    rp = rst[1][:, None]
    sp = fd.abs()
    if c["post"]:
        k = spread(fd, c["post"], c["eps"])
        sp = (fd.abs() + fd.abs().mean(1, keepdim=True)) * rp * k * aw + ab
        R.assert_close(stats[0], rst[0], e64 * fd.abs().mean(1), "post mean")
        R.assert_close(stats[1], rst[1], e64 * rst[1] * k[:, 0], "post rstd")
    sh = (c["alpha"] * hd).abs() + abs(c["beta"]) * gt * sp
    R.assert_close(ho, rho, R.HALF[T] * rho.abs() + e64 * sh, "h'")
    if c["pre"]:
        var = rst[3][:, None] ** -2
        hc_ = rho - rst[2][:, None]
        k = 1 + ((sh + sh.mean(1, keepdim=True)) * hc_.abs()).mean(1, keepdim=True) / var
        R.assert_close(stats[2], rst[2], e64 * sh.mean(1), "pre mean")
        R.assert_close(stats[3], rst[3], e64 * rst[3] * k[:, 0], "pre rstd")
        w = one if pd["pre_w"] is None else pd["pre_w"].abs()
        b = 0 * one if pd["pre_b"] is None else pd["pre_b"].abs()
        bound = R.HALF[T] * rn.abs() + e64 * ((sh + sh.mean(1, keepdim=True)) * rst[3][:, None] * w + k * (hc_ * rst[3][:, None]).abs() * w + b)
        R.assert_close(n, rn, bound * (1 + R.HALF[T]), "n")
    if keep:   # the checkpoints are those of what was given and of what was written, bit for bit
        rq, re = R.store(f, fmt)
        assert torch.equal(fq.cpu(), rq) and torch.equal(fe.cpu(), re)
        if c["pre"]:
            rq, re = R.store(n.cpu(), fmt)
            assert torch.equal(nq.cpu(), rq) and torch.equal(ne.cpu(), re)
    if not c["post"]:
        assert bool((stats[0] == 0).all()) and bool((stats[1] == 1).all())
    if not c["pre"]:
        assert bool((stats[2] == 0).all()) and bool((stats[3] == 1).all())


SHAPES = [(1, 1), (3, 8), (2, 31), (5, 100), (9, 256), (130, 300), (7, 768), (65, 1001), (3, 1024), (4, 1032), (33, 2048), (6, 3200), (5, 4097), (3, 8192),
          (2, 16384), (2, 16390), (3, 20000)]


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,d", SHAPES)
def test_forward(B, dtype, N, d):
    check_forward(B, dtype, setting(R.RMS, R.RMS), N, d, R.E4M3, True)
    check_forward(B, dtype, setting(R.LAYER, R.LAYER, rows=2), N, d, R.INT8, True, seed=5)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("post", [R.NONE, R.RMS, R.LAYER])
@pytest.mark.parametrize("pre", [R.NONE, R.RMS, R.LAYER])
@pytest.mark.parametrize("N,d", [(13, 264), (6, 2056), (2, 16400)])
def test_forward_variants(B, dtype, post, pre, N, d):
    check_forward(B, dtype, setting(post, pre, rows=4), N, d, R.INT8, False)
    check_forward(B, dtype, setting(post, pre), N, d, R.E4M3, True, gated=False, weighted=False, inplace=True)
    check_forward(B, dtype, setting(post, pre, rows=1), N, d, R.E4M3, True)
    check_forward(B, dtype, setting(post, pre, rows=100), N, d, R.E4M3, False)


# ---- backward --------------------------------------------------------------------------------------
NAMES = ("dpost_w", "dpost_b", "dgate", "dpre_w", "dpre_b")


def check_backward(B, dtype, c, N, d, fmt, seed=0, gated=True, weighted=True, inplace=False, residual=True, accumulate=0, subset=None):
    """fmt None: f in the compute dtype."""
    g = torch.Generator().manual_seed(seed + N + d)
    T = R.DT[dtype]
    f, p = acts(N, d, dtype, g), params(c, N, d, g, gated, weighted)
    ho = acts(N, d, dtype, g)
    st = torch.stack([*R.norm(f.double(), c["post"], None, None, c["eps"])[2:], *R.norm(ho.double(), c["pre"], None, None, c["eps"])[2:]]).float()
    dn = torch.randn(N, d, generator=g).to(T) if c["pre"] else None
    dho = torch.randn(N, d, generator=g).to(T) if residual or not c["pre"] else None
    rq, re = R.store(f, fmt or 0)
    fv = f.double() if fmt is None else R.load(rq, re, fmt, d)
    pd = dbl(p)
    ref = R.block_norm_bwd(c, ho.double(), fv, pd["post_w"], pd["post_b"], pd["gate"], pd["pre_w"], st.double(), None if dn is None else dn.double(),
                           None if dho is None else dho.double())
    q = cuda(p)
    grads, before = {}, {}
    for k in NAMES:
        has = k in ref and (k != "dpost_b" or c["post"] == R.LAYER) and (k != "dpre_b" or c["pre"] == R.LAYER)
        if has and (subset is None or k in subset):
            before[k] = torch.randn(ref[k][0].shape, generator=g) if accumulate else None
            grads[k] = before[k].cuda() if accumulate else torch.full(ref[k][0].shape, float("nan"), device="cuda")
    dhoc = None if dho is None else dho.cuda()
    dh = dhoc if inplace and dhoc is not None else torch.full((N, d), 7.0, dtype=T, device="cuda")
    df = torch.full((N, d), 7.0, dtype=T, device="cuda")
    pr = dims(B, dtype, c, N, d, fmt or 0, accumulate)
    ws = torch.full((B.zl_op_block_norm_bwd_bytes(pr),), 0xFF, dtype=torch.uint8, device="cuda")
    src = (f.cuda(), None, None) if fmt is None else (None, rq.cuda(), re.cuda())
    B.zl_op_block_norm_bwd(pr, ho.cuda(), *src, q["post_w"], q["post_b"], q["gate"], q["pre_w"], st.cuda(), None if dn is None else dn.cuda(), dhoc, dh, df,
                           *(grads.get(k) for k in NAMES), ws)
    torch.cuda.synchronize()
    # rows: 64 roundings as in the forward, twice over for df, which follows from G; columns: as many more as there are rows
    for k, dt in (("dh", T), ("df", T)):
        v, s = ref[k]
        R.assert_close({"dh": dh, "df": df}[k], v, R.HALF[dt] * v.abs() + 256 * ULP * s, k)
    for k, t in grads.items():
        v, s = ref[k]
        b = (256 + N) * ULP * s
        if accumulate:
            v, b = v + before[k].double(), b + 4 * ULP * (before[k].double().abs() + v.abs())
        R.assert_close(t, v, b, k)
    return dh, df, grads


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,d", SHAPES + [(300, 520), (517, 96), (2100, 40), (129, 4096)])
def test_backward(B, dtype, N, d):
    check_backward(B, dtype, setting(R.RMS, R.RMS), N, d, R.E4M3)
    check_backward(B, dtype, setting(R.LAYER, R.LAYER, rows=2), N, d, R.INT8, seed=3, accumulate=1)
    check_backward(B, dtype, setting(R.RMS, R.LAYER, rows=max(1, N // 3)), N, d, None, inplace=True)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("post", [R.NONE, R.RMS, R.LAYER])
@pytest.mark.parametrize("pre", [R.NONE, R.RMS, R.LAYER])
@pytest.mark.parametrize("N,d", [(13, 264), (70, 2056), (2, 16400)])
def test_backward_variants(B, dtype, post, pre, N, d):
    check_backward(B, dtype, setting(post, pre, rows=4), N, d, R.INT8)
    check_backward(B, dtype, setting(post, pre), N, d, R.E4M3, gated=False, weighted=False, inplace=True)
    check_backward(B, dtype, setting(post, pre, rows=1), N, d, None, accumulate=1)
    check_backward(B, dtype, setting(post, pre, rows=1000), N, d, R.E4M3, residual=False, subset=("dgate", "dpre_w"))
    check_backward(B, dtype, setting(post, pre, rows=3), N, d, R.INT8, subset=())


@gpu
@pytest.mark.parametrize("rows", [0, 1, 5, 63, 64, 65, 128, 200, 640, 1000])
def test_gate_groups(B, rows):
    """Gate groups around every border of the row chunks, the last one cut short."""
    check_backward(B, "f32", setting(R.RMS, R.RMS, rows=rows), 643, 72, R.E4M3)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("post,pre", [(R.RMS, R.RMS), (R.LAYER, R.RMS), (R.NONE, R.LAYER)])
@pytest.mark.parametrize("N,d,rows", [(1300, 520, 26), (1300, 1001, 9), (700, 2056, 31), (2500, 33, 300), (5000, 16400, 129)])
def test_many_gate_groups(B, dtype, post, pre, N, d, rows):
    """More than a few groups, each cut into chunks of rows, the last one short; the last shape beyond the ring kernels' width."""
    if d == 16400 and (dtype == "f32" or post != R.RMS):
        N = 1500
    check_backward(B, dtype, setting(post, pre, rows=rows), N, d, R.E4M3, accumulate=1)
    check_backward(B, dtype, setting(post, pre, rows=rows), N, d, R.INT8, subset=("dgate",))
    check_backward(B, dtype, setting(post, pre, rows=rows), N, d, R.INT8, subset=("dpost_w",))


@gpu
def test_backward_repeats_bit_for_bit(B):
    a = check_backward(B, "bf16", setting(R.LAYER, R.RMS, rows=100), 517, 1032, R.INT8)
    b = check_backward(B, "bf16", setting(R.LAYER, R.RMS, rows=100), 517, 1032, R.INT8)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    for k in a[2]:
        assert torch.equal(a[2][k], b[2][k]), k


@gpu
def test_no_rows(B):
    """No rows: nothing is touched but the gradients, which become zero unless they accumulate."""
    c = setting(R.LAYER, R.LAYER)
    for acc in (0, 1):
        p = dims(B, "f32", c, 0, 64, accumulate=acc)
        assert B.zl_op_block_norm_bwd_bytes(p) == 0
        B.zl_op_block_norm(p, None, None, None, None, None, None, None, None, None, None)
        gr = [torch.ones(64, device="cuda") for _ in range(4)]
        dg = torch.ones(1, 64, device="cuda")
        gate = torch.ones(1, 64, device="cuda")
        B.zl_op_block_norm_bwd(p, None, None, None, None, None, None, gate, None, None, None, None, None, None, gr[0], gr[1], dg, gr[2], gr[3], None)
        for t in (*gr, dg):
            assert bool((t == acc).all())


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_of_zeros_and_nan(B, dtype):
    """A row of zeros stays finite, a row with a NaN spoils no other row."""
    c, N, d, T = setting(R.RMS, R.LAYER), 5, 320, R.DT[dtype]
    g = torch.Generator().manual_seed(9)
    h, f = acts(N, d, dtype, g).cuda(), acts(N, d, dtype, g).cuda()
    f[1].zero_(), h[1].zero_()
    f[3, 7] = float("nan")
    ho, n, st = torch.empty(N, d, dtype=T, device="cuda"), torch.empty(N, d, dtype=T, device="cuda"), torch.empty(4, N, device="cuda")
    fq, fe = codes(N, d)
    p = dims(B, dtype, c, N, d)
    B.zl_op_block_norm(p, h, f, None, None, None, None, None, ho, n, st, fq, fe)
    ok = torch.tensor([True, True, True, False, True], device="cuda")
    assert torch.equal(torch.isfinite(n).all(1), ok) and bool((n[1] == 0).all())
    dn = torch.ones(N, d, dtype=T, device="cuda")
    dh, df = torch.empty_like(dn), torch.empty_like(dn)
    ws = torch.empty(B.zl_op_block_norm_bwd_bytes(p), dtype=torch.uint8, device="cuda")
    B.zl_op_block_norm_bwd(p, ho, None, fq, fe, None, None, None, None, st, dn, dn, dh, df, None, None, None, None, None, ws)
    assert torch.equal(torch.isfinite(df).all(1), ok)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("post,pre", [(R.RMS, R.RMS), (R.LAYER, R.LAYER), (R.NONE, R.RMS)])
@pytest.mark.parametrize("d", [35, 38, 40, 64])
def test_nan_rows_among_many(B, dtype, post, pre, d):
    """Rows with a NaN or an infinity among many (a block takes several): every other row keeps its bits, in shapes whose rows
    end inside a vector, a word or a group of the codes; columns past d of the codes stay 0."""
    c, N, T = setting(post, pre), 20000, R.DT[dtype]
    g = torch.Generator().manual_seed(d)
    h, f, dn, dho = (acts(N, d, dtype, g).cuda() for _ in range(4))
    bad = torch.zeros(N, dtype=torch.bool, device="cuda")
    bad[3::7] = True
    p = dims(B, dtype, c, N, d)
    D = (d + 31) // 32 * 32
    ws = torch.empty(B.zl_op_block_norm_bwd_bytes(p), dtype=torch.uint8, device="cuda")

    def run(f, h):
        ho, n, dh, df = (torch.empty(N, d, dtype=T, device="cuda") for _ in range(4))
        st, (fq, fe), (nq, ne) = torch.empty(4, N, device="cuda"), codes(N, d), codes(N, d)
        B.zl_op_block_norm(p, h, f, None, None, None, None, None, ho, n, st, fq, fe, nq, ne)
        B.zl_op_block_norm_bwd(p, ho, f, None, None, None, None, None, None, st, dn, dho, dh, df, None, None, None, None, None, ws)
        torch.cuda.synchronize()
        return ho, n, dh, df, fq, fe, nq, ne, st.t().contiguous()

    clean = run(f, h)
    f2, h2 = f.clone(), h.clone()
    f2[3::14, d // 2] = float("nan")
    h2[10::14, d - 1] = float("inf")
    spoilt = run(f2, h2)
    for a, b in zip(clean, spoilt):
        a, b = a.view(N, -1), b.view(N, -1)
        assert torch.equal(a[~bad], b[~bad])
    for k in (4, 6):
        assert not bool(spoilt[k].view(N, D)[:, d:].any())
    assert not bool(torch.isfinite(spoilt[1][bad]).all(1).any()) and not bool(torch.isfinite(spoilt[3][3::14]).all(1).any())


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kept", [None, R.E4M3, R.INT8])
@pytest.mark.parametrize("d", [35, 64, 1000, 4096, 8200])
def test_branch_gradient_without_norms_holds_no_branch(B, dtype, kept, d):
    """Neither norm: dh = alpha dh', df = beta gate dh', whatever stands in f (a NaN or an infinity reaches dgate alone, in its
    own column). One product more than beta gate: three roundings in 24 bits, then the one to the type."""
    c, N, T = setting(R.NONE, R.NONE), 9, R.DT[dtype]
    g = torch.Generator().manual_seed(d)
    f, dho = acts(N, d, dtype, g), torch.randn(N, d, generator=g).to(T)
    f[1, d // 2], f[4, 3], f[5, d - 1] = float("nan"), float("inf"), float("-inf")
    gate = 0.5 + torch.rand(1, d, generator=g)
    dh, df = (torch.full((N, d), 7.0, dtype=T, device="cuda") for _ in range(2))
    dgate, st = torch.empty(1, d, device="cuda"), torch.tensor([0.0, 1.0, 0.0, 1.0], device="cuda").repeat_interleave(N).view(4, N)
    p = dims(B, dtype, c, N, d, kept or 0)
    ws = torch.empty(B.zl_op_block_norm_bwd_bytes(p), dtype=torch.uint8, device="cuda")
    src = (f.cuda(), None, None) if kept is None else (None, *(t.cuda() for t in R.store(f, kept)))
    B.zl_op_block_norm_bwd(p, None, *src, None, None, gate.cuda(), None, st, None, dho.cuda(), dh, df, None, None, dgate, None, None, ws)
    G = dho.double()
    for got, ref in ((dh, c["alpha"] * G), (df, c["beta"] * gate.double() * G)):
        R.assert_close(got, ref, (R.HALF[T] + 3 * ULP) * (1 + R.HALF[T]) * ref.abs(), d)
    bad = torch.zeros(d, dtype=torch.bool)
    bad[[d // 2, 3, d - 1]] = True
    assert torch.equal(torch.isfinite(dgate[0]).cpu(), ~bad)


# ---- together --------------------------------------------------------------------------------------
@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("fmt", [R.E4M3, R.INT8])
def test_feed_forward_block_with_checkpoints(B, dtype, fmt):
    """n -> SwiGLU feed-forward -> fused norm step, forward and local backward, nothing kept but h', the statistics and 8-bit
    tensors; every gradient against 64-bit arithmetic on the values that the checkpoints stand for. The chain rounds its
    intermediates to the compute dtype five times; relative to their norms the gradients stay within 5 x 2 half steps
    (fp32: within 2^-24 x 4096, the products' length)."""
    N, d, f, T, dt = 203, 256, 344, R.DT[dtype], code(B, dtype)
    g = torch.Generator().manual_seed(4)
    c = setting(R.RMS, R.RMS, rows=100)
    n0 = torch.randn(N, d, generator=g).to(T)
    h0 = acts(N, d, dtype, g)
    w1, w2 = (torch.randn(2 * f, d, generator=g) / d ** 0.5).to(T), (torch.randn(d, f, generator=g) / f ** 0.5).to(T)
    p = params(c, N, d, g)
    dn, dho = torch.randn(N, d, generator=g).to(T), torch.randn(N, d, generator=g).to(T)
    dev = lambda *s: torch.empty(*s, dtype=T, device="cuda")  # noqa: E731
    W1, W2, q = w1.cuda(), w2.cuda(), cuda(p)
    # forward
    x, y, fo, ho, n = dev(N, 2 * f), dev(N, f), dev(N, d), dev(N, d), dev(N, d)
    n8, x8, f8 = codes(N, d), codes(2 * N, f), codes(N, d)
    B.zl_op_act8_store(dt, fmt, n0.cuda(), N, d, d, *n8)
    B.zl_op_gemm(dt, 0, N, 2 * f, d, n0.cuda(), W1, x)
    B.zl_op_act8_act(dt, R.SWIGLU, fmt, x, N, f, y, *x8)
    B.zl_op_gemm(dt, 0, N, d, f, y, W2, fo)
    st = torch.empty(4, N, device="cuda")
    pr = dims(B, dtype, c, N, d, fmt)
    B.zl_op_block_norm(pr, h0.cuda(), fo, q["post_w"], None, q["gate"], q["pre_w"], None, ho, n, st, *f8)
    kept_x, kept_f = x.clone(), fo.clone()
    del x, y, fo
    # backward
    dh, df, dy, dx, again, dn0 = dev(N, d), dev(N, d), dev(N, f), dev(N, 2 * f), dev(N, f), dev(N, d)
    gr = {k: torch.empty_like(q[k[1:]]) for k in ("dpost_w", "dgate", "dpre_w")}
    ws = torch.empty(max(B.zl_op_block_norm_bwd_bytes(pr), B.zl_op_act8_dw_bytes(dt, 2 * f, d, N), B.zl_op_act8_dw_bytes(dt, d, f, N)), dtype=torch.uint8, device="cuda")
    B.zl_op_block_norm_bwd(pr, ho, None, *f8, q["post_w"], None, q["gate"], q["pre_w"], st, dn.cuda(), dho.cuda(), dh, df, gr["dpost_w"], None, gr["dgate"],
                           gr["dpre_w"], None, ws)
    B.zl_op_gemm(dt, 1, N, f, d, df, W2, dy)
    B.zl_op_act8_act_bwd(dt, R.SWIGLU, fmt, *x8, dy, N, f, dx, again)
    y8 = codes(N, f)
    B.zl_op_act8_store(dt, fmt, again, N, f, f, *y8)
    dW1, dW2 = torch.empty(2 * f, d, device="cuda"), torch.empty(d, f, device="cuda")
    B.zl_op_act8_dw(dt, fmt, d, f, N, df, *y8, dW2, 0, ws)
    B.zl_op_act8_dw(dt, fmt, 2 * f, d, N, dx, *n8, dW1, 0, ws)
    B.zl_op_gemm(dt, 1, N, d, 2 * f, dx, W1, dn0)
    torch.cuda.synchronize()
    # 64 bits, from what the checkpoints of the same tensors stand for
    v = lambda t, w: R.load(*R.store(t.cpu().view(-1, w), fmt), fmt, w).reshape(t.shape)  # noqa: E731
    pd = dbl(p)
    ref = R.block_norm_bwd(c, ho.cpu().double(), v(kept_f, d), pd["post_w"], None, pd["gate"], pd["pre_w"], st.cpu().double(), dn.double(), dho.double())
    xr = v(kept_x, f).requires_grad_(True)
    yr = R.act(xr, R.SWIGLU)
    dfr = ref["df"][0]
    (dxr,) = torch.autograd.grad(yr, xr, dfr @ w2.double())
    want = dict(dh=(dh, ref["dh"][0]), df=(df, dfr), dx=(dx, dxr), dn0=(dn0, dxr @ w1.double()), dW2=(dW2, dfr.T @ v(again, f)),
                dW1=(dW1, dxr.T @ v(n0, d)), **{k: (t, ref[k][0]) for k, t in gr.items()})
    tol = 5 * 2 * 2.0 ** -8 if dtype == "bf16" else 4096 * 2.0 ** -24
    for k, (a, b) in want.items():
        a = a.cpu().double()
        assert float((a - b).norm() / b.norm()) <= tol, (k, float((a - b).norm() / b.norm()))


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,d,rows", [(37, 1000, 5), (130, 72, 0), (9, 4097, 2), (3, 8192, 0), (2, 9000, 1), (301, 264, 100)])
def test_outputs_stay_in_bounds(B, dtype, N, d, rows):
    """Every output between two bands of a bit pattern, which stay as they are; and nothing but the outputs is written."""
    T, c = R.DT[dtype], setting(R.LAYER, R.LAYER, rows=rows)
    g = torch.Generator().manual_seed(N)
    p = cuda(params(c, N, d, g))
    D, G = R.width(d), p["gate"].shape[0]
    bufs = {}

    def out(name, n, dt):
        size = torch.empty(0, dtype=dt).element_size()
        bufs[name] = (torch.full((n * size + 8192,), 0xA5, dtype=torch.uint8, device="cuda"), n * size)
        return bufs[name][0][4096:4096 + n * size].view(dt)

    h, f = acts(N, d, dtype, g).cuda(), acts(N, d, dtype, g).cuda()
    pr = dims(B, dtype, c, N, d, R.INT8)
    keep = [t.clone() for t in (h, f)]
    ho, n, st = out("ho", N * d, T), out("n", N * d, T), out("stats", 4 * N, torch.float32)
    fq, fe, nq, ne = out("fq", N * D, torch.uint8), out("fe", N * D // 32, torch.uint8), out("nq", N * D, torch.uint8), out("ne", N * D // 32, torch.uint8)
    B.zl_op_block_norm(pr, h, f, p["post_w"], p["post_b"], p["gate"], p["pre_w"], p["pre_b"], ho, n, st, fq, fe, nq, ne)
    nws = B.zl_op_block_norm_bwd_bytes(pr)
    ws = torch.full((nws + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
    dh, df = out("dh", N * d, T), out("df", N * d, T)
    gr = [out(k, m, torch.float32) for k, m in (("dpost_w", d), ("dpost_b", d), ("dgate", G * d), ("dpre_w", d), ("dpre_b", d))]
    dn, dho = acts(N, d, dtype, g).cuda(), acts(N, d, dtype, g).cuda()
    B.zl_op_block_norm_bwd(pr, ho, None, fq, fe, p["post_w"], p["post_b"], p["gate"], p["pre_w"], st, dn, dho, dh, df, *gr, ws[:nws])
    torch.cuda.synchronize()
    for name, (b, m) in bufs.items():
        assert bool((b[:4096] == 0xA5).all()) and bool((b[4096 + m:] == 0xA5).all()), name
    assert bool((ws[nws:] == 0xA5).all())
    assert torch.equal(h, keep[0]) and torch.equal(f, keep[1])


@gpu
def test_calls_on_two_streams_at_once(B):
    """The same work on two streams, each with its own workspace, gives what it gives alone."""
    N, d, T = 517, 2048, torch.bfloat16
    c, g = setting(R.RMS, R.RMS), torch.Generator().manual_seed(2)
    p = cuda(params(c, N, d, g))
    pr = dims(B, "bf16", c, N, d)
    nws = B.zl_op_block_norm_bwd_bytes(pr)
    ins = [[acts(N, d, "bf16", g).cuda() for _ in range(4)] for _ in range(2)]

    def work(k, s):
        h, f, dn, dho = ins[k]
        e = lambda *a, dt=T: torch.empty(*a, dtype=dt, device="cuda")  # noqa: E731
        o = [e(N, d), e(N, d), e(4, N, dt=torch.float32), *codes(N, d), e(N, d), e(N, d), e(d, dt=torch.float32), e(1, d, dt=torch.float32), e(d, dt=torch.float32),
             e(nws, dt=torch.uint8)]
        torch.cuda.synchronize()

        def go():
            for _ in range(10):
                B.zl_op_block_norm(pr, h, f, p["post_w"], None, p["gate"], p["pre_w"], None, *o[:3], o[3], o[4], None, None, s)
                B.zl_op_block_norm_bwd(pr, o[0], None, o[3], o[4], p["post_w"], None, p["gate"], p["pre_w"], o[2], dn, dho, o[5], o[6], o[7], None, o[8], o[9], None,
                                       o[10], s)
        return o[:-1], go

    alone = []
    for k in range(2):
        o, go = work(k, 0)
        go()
        torch.cuda.synchronize()
        alone.append(o)
    st = [torch.cuda.Stream(), torch.cuda.Stream()]
    both = [work(k, st[k].cuda_stream) for k in range(2)]
    for _, go in both:
        go()
    torch.cuda.synchronize()
    for k in range(2):
        for a, b in zip(alone[k], both[k][0]):
            assert torch.equal(a, b)


FIRST_CALL = """
import sys, torch
sys.path.insert(0, %r)
from paper_2608_07974_gb300 import binding as B
T, N, d = torch.bfloat16, 64, 512
x = torch.randn(N, d, device="cuda").to(T)
e = lambda *a, dt=T: torch.empty(*a, dtype=dt, device="cuda")
q, s = e(N, d, dt=torch.uint8), e(N, d // 32, dt=torch.uint8)
p = B.zl_block_norm(dtype=1, post_norm=1, pre_norm=1, N=N, d=d, gate_rows=0, eps=1e-5, res_scale=1, branch_scale=1, fmt=0, accumulate=0)
w, C = e(d, dt=torch.float32).fill_(1), e(d, d, dt=torch.float32)
ho, n, st, dh, df = e(N, d), e(N, d), e(4, N, dt=torch.float32), e(N, d), e(N, d)
gr, ws, ws2 = e(d, dt=torch.float32), e(B.zl_op_block_norm_bwd_bytes(p), dt=torch.uint8), e(B.zl_op_act8_dw_bytes(1, d, d, N), dt=torch.uint8)
torch.cuda.synchronize()
def step(s_):
    B.zl_op_block_norm(p, x, x, w, None, None, w, None, ho, n, st, q, s, None, None, s_)
    B.zl_op_block_norm_bwd(p, ho, None, q, s, w, None, None, w, st, n, x, dh, df, gr, None, None, None, None, ws, s_)
    B.zl_op_act8_dw(1, 0, d, d, N, df, q, s, C, 0, ws2, s_)
g, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
with torch.cuda.graph(g, stream=side):
    step(side.cuda_stream)
g.replay()
torch.cuda.synchronize()
got = [t.clone() for t in (ho, n, st, dh, df, gr, C)]
step(0)
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(got, (ho, n, st, dh, df, gr, C)))
print("captured")
"""


@gpu
def test_first_call_may_be_captured(B):
    """A process whose first calls are those of a capture: nothing has to run before it."""
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST_CALL % root], capture_output=True, text=True, timeout=300, cwd=root)
    assert r.returncode == 0 and "captured" in r.stdout, r.stderr[-2000:]
