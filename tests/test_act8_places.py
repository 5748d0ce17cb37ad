"""The 8-bit operators and the block norm with every tensor somewhere else than on 16 bytes, each at an offset of its own; weight
gradients of many tokens, whose sums are cut into segments, into rows of C wherever they start."""
import pytest
import torch

from tests import act8_common as R
from tests import test_act8, test_block_norm

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import paper_2608_07974_gb300 as pkg
    pkg.build()
    from paper_2608_07974_gb300 import binding
    return binding


def shifted(t, k):
    """t on the GPU, k elements behind a 16-byte boundary."""
    buf = torch.empty(t.numel() + 16, dtype=t.dtype, device="cuda")
    v = buf[k:k + t.numel()].view(t.shape)
    v.copy_(t)
    assert v.data_ptr() % 16 == k * t.element_size() % 16
    return v


def place(monkeypatch, which):
    """Moves what a test sends to the GPU or fills there: 1, 2, 3 .. elements off in turn (codes and workspaces stay: bytes)."""
    n, to_gpu, full = [0], torch.Tensor.cuda, torch.full

    def move(t):
        if not which(t):
            return t
        n[0] += 1
        return shifted(t, 1 + n[0] % 7)

    monkeypatch.setattr(torch.Tensor, "cuda", lambda t, *a: move(to_gpu(t, *a)))
    monkeypatch.setattr(torch, "full", lambda *a, **k: move(full(*a, **k)) if k.get("device") == "cuda" else full(*a, **k))


def any_float(t):
    return t.dtype != torch.uint8


def parameters(t):
    return t.dtype == torch.float32


WIDTHS = [(13, 264), (9, 36), (5, 1001), (6, 2056), (3, 8192), (2, 8200)]


@pytest.mark.parametrize("dtype,which", [("f32", any_float), ("bf16", any_float), ("bf16", parameters)])
@pytest.mark.parametrize("N,d", WIDTHS)
def test_block_norm_forward(B, monkeypatch, dtype, which, N, d):
    place(monkeypatch, which)
    for seed in (0, 1):          # other offsets too
        test_block_norm.check_forward(B, dtype, test_block_norm.setting(R.RMS, R.RMS), N, d, R.E4M3, True, seed=seed)
        test_block_norm.check_forward(B, dtype, test_block_norm.setting(R.LAYER, R.LAYER, rows=2), N, d, R.INT8, True, seed=seed)
        test_block_norm.check_forward(B, dtype, test_block_norm.setting(R.NONE, R.LAYER), N, d, R.INT8, False, seed=seed, inplace=True)


@pytest.mark.parametrize("dtype,which", [("f32", any_float), ("bf16", any_float), ("bf16", parameters)])
@pytest.mark.parametrize("N,d", WIDTHS + [(300, 520)])
def test_block_norm_backward(B, monkeypatch, dtype, which, N, d):
    place(monkeypatch, which)
    for seed in (0, 1):
        test_block_norm.check_backward(B, dtype, test_block_norm.setting(R.RMS, R.RMS), N, d, R.E4M3, seed=seed)
        test_block_norm.check_backward(B, dtype, test_block_norm.setting(R.LAYER, R.LAYER, rows=2), N, d, R.INT8, seed=seed, accumulate=1)
        test_block_norm.check_backward(B, dtype, test_block_norm.setting(R.NONE, R.LAYER, rows=max(1, N // 3)), N, d, None, seed=seed, inplace=True)


@pytest.mark.parametrize("dtype,fmt", [("f32", R.E4M3), ("bf16", R.INT8)])
@pytest.mark.parametrize("kind", [R.SWIGLU, R.GELU])
@pytest.mark.parametrize("N,f", [(1, 8), (2, 33), (9, 1001), (64, 1000)])
def test_activations(B, monkeypatch, dtype, fmt, kind, N, f):
    place(monkeypatch, any_float)
    for _ in range(3):
        test_act8.test_activation_and_its_backward(B, dtype, fmt, kind, N, f)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("off", [0, 1, 2])
@pytest.mark.parametrize("plan", ["", "256:1:1", "256:1:0", "128:1:1", "128:1:0", "64:1", "64:3"])
@pytest.mark.parametrize("N,K", [(328, 300), (333, 4500), (328, 6145), (301, 4500)])
def test_weight_gradient(B, monkeypatch, dtype, off, plan, N, K):
    """C off 16 bytes or with rows off them, one segment and several, written and added to, under every kind of plan; the bounds
    are those of sums of at most 2048 products and as many roundings, 12 segments and a few splits, and of what C held."""
    if plan:
        monkeypatch.setenv("ZL_GEMM_TILE", plan)
    M, dt = 264, test_act8.code(B, dtype)
    g = torch.Generator(device="cuda").manual_seed(K + N)
    A = (torch.randn(K, M, generator=g, device="cuda") + 0.5).to(R.DT[dtype])
    x = (torch.randn(K, N, generator=g, device="cuda") + 0.5).to(R.DT[dtype])
    q, e = test_act8.empty_codes(K, N)
    B.zl_op_act8_store(dt, R.INT8, x, K, N, N, q, e)
    X = torch.empty(K, N, device="cuda")
    B.zl_op_act8_load(B.ZL_DTYPE_F32, R.INT8, q, e, K, N, N, X)
    ref, scale = (A.double().T @ X.double()).cpu(), (A.double().abs().T @ X.double().abs()).cpu()
    ws = torch.empty(B.zl_op_act8_dw_bytes(dt, M, N, K), dtype=torch.uint8, device="cuda")
    band = torch.full((M * N + 64,), 7.0, device="cuda")
    C = band[off:off + M * N].view(M, N)
    bound = (2048 + 64 + 16) * 2.0 ** -23 * scale
    for _ in range(2):
        B.zl_op_act8_dw(dt, R.INT8, M, N, K, A, q, e, C, 0, ws)
        R.assert_close(C, ref, bound, "C")
    C0 = torch.randn(M, N, generator=g, device="cuda")
    outs = []
    for _ in range(2):
        C.copy_(C0)
        B.zl_op_act8_dw(dt, R.INT8, M, N, K, A, q, e, C, 1, ws)
        outs.append(C.clone())
    R.assert_close(outs[0], ref + C0.cpu().double(), bound + 16 * 2.0 ** -23 * C0.cpu().double().abs(), "C +=")
    assert torch.equal(*outs)
    assert bool((band[:off] == 7.0).all()) and bool((band[off + M * N:] == 7.0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("plan", ["128:1:0", "256:1:1"])
@pytest.mark.parametrize("N,off", [(264, 0), (264, 1), (261, 0)])
def test_segments_bound_the_truncation(B, monkeypatch, dtype, plan, N, off):
    """Sums of 65536 products of one sign in one split. The tensor cores shorten an accumulator by up to a step (2^-23 of it) each
    time that 16 products are added, always towards zero. Over a segment of 2048 tokens, 128 additions to an accumulator that
    grows evenly, that is up to 64.5 steps of the segment's sum; 32 segments are then added with one rounding (2^-24) each of a
    sum that grows evenly, 16.5 in all, an fp32 gradient's smaller terms among them at half as much again. In one accumulation
    it would be 4096 additions, half a step and more of each for data of one sign."""
    monkeypatch.setenv("ZL_GEMM_TILE", plan)
    M, K, dt = 264, 65536, test_act8.code(B, dtype)
    g = torch.Generator(device="cuda").manual_seed(N + off)
    # sizes of many powers of two, so that the products have no last place in common
    A, x = (torch.exp(1.5 * torch.randn(K, w, generator=g, device="cuda")).to(R.DT[dtype]) for w in (M, N))
    q, e = test_act8.empty_codes(K, N)
    B.zl_op_act8_store(dt, R.E4M3, x, K, N, N, q, e)
    X = torch.empty(K, N, device="cuda")
    B.zl_op_act8_load(B.ZL_DTYPE_F32, R.E4M3, q, e, K, N, N, X)
    ref = A.double().T @ X.double()
    ws = torch.empty(B.zl_op_act8_dw_bytes(dt, M, N, K), dtype=torch.uint8, device="cuda")
    C = torch.empty(M * N + 8, device="cuda")[off:off + M * N].view(M, N)
    B.zl_op_act8_dw(dt, R.E4M3, M, N, K, A, q, e, C, 0, ws)
    err = float((C.double() - ref).norm() / ref.norm())
    print(f"relative error {err:.2e}")
    assert err <= 64.5 * 2.0 ** -23 + 1.5 * 16.5 * 2.0 ** -24, err


def big(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype, device="cuda")


@pytest.fixture
def room():
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


TAIL = 70


def test_activation_beyond_32_bits(B, room):
    """More than 2^32 values of x: the last rows as in a call of their own."""
    f, dt = 11008, B.ZL_DTYPE_BF16
    N = (1 << 32) // (2 * f) + 2 * TAIL
    x, y, again, dx, dy = big(N, 2 * f), big(N, f), big(N, f), big(N, 2 * f), big(N, f)
    q, e = big(2 * N, f, dtype=torch.uint8), big(2 * N, f // 32, dtype=torch.uint8)
    x[-TAIL:].normal_()
    dy[-TAIL:].normal_()
    B.zl_op_act8_act(dt, R.SWIGLU, R.INT8, x, N, f, y, q, e)
    B.zl_op_act8_act_bwd(dt, R.SWIGLU, R.INT8, q, e, dy, N, f, dx, again)
    y2, again2, dx2 = big(TAIL, f), big(TAIL, f), big(TAIL, 2 * f)
    q2, e2 = big(2 * TAIL, f, dtype=torch.uint8), big(2 * TAIL, f // 32, dtype=torch.uint8)
    B.zl_op_act8_act(dt, R.SWIGLU, R.INT8, x[-TAIL:], TAIL, f, y2, q2, e2)
    B.zl_op_act8_act_bwd(dt, R.SWIGLU, R.INT8, q2, e2, dy[-TAIL:], TAIL, f, dx2, again2)
    for a, b in ((y, y2), (again, again2), (dx, dx2), (q, q2), (e, e2)):
        assert torch.equal(a[-len(b):], b)
        assert bool((a[:-len(b)] == (10 if a is e else 0)).all())


@pytest.mark.parametrize("d", [4096, 4095, 9000])
def test_block_norm_beyond_32_bits(B, room, d):
    """More than 2^32 values a tensor: the last rows as in a call of their own (each kernel's rows do not depend on their number)."""
    N, D, dt = (1 << 32) // d + 2 * TAIL, R.width(d), B.ZL_DTYPE_BF16
    h, f, ho, n = big(N, d), big(N, d), big(N, d), big(N, d)
    st, (fq, fe) = big(4, N, dtype=torch.float32), (big(N, D, dtype=torch.uint8), big(N, D // 32, dtype=torch.uint8))
    h[-TAIL:].normal_()
    f[-TAIL:].normal_()
    w = torch.rand(d, device="cuda") + 0.5

    def call(rows, *t):
        p = B.zl_block_norm(dtype=dt, post_norm=R.RMS, pre_norm=R.RMS, N=rows, d=d, gate_rows=0, eps=1e-5, res_scale=1, branch_scale=0.5, fmt=0, accumulate=0)
        h_, f_, ho_, n_, st_, fq_, fe_ = t
        B.zl_op_block_norm(p, h_, f_, w, None, None, w, None, ho_, n_, st_, fq_, fe_)
        ws = torch.empty(B.zl_op_block_norm_bwd_bytes(p), dtype=torch.uint8, device="cuda")
        dn, dh, df = n_, h_, f_          # n as its own gradient; the inputs are not needed any more
        B.zl_op_block_norm_bwd(p, ho_, None, fq_, fe_, w, None, None, w, st_, dn, None, dh, df, None, None, None, None, None, ws)

    small = [h[-TAIL:].clone(), f[-TAIL:].clone(), big(TAIL, d), big(TAIL, d), big(4, TAIL, dtype=torch.float32), big(TAIL, D, dtype=torch.uint8),
             big(TAIL, D // 32, dtype=torch.uint8)]
    call(TAIL, *small)
    call(N, h, f, ho, n, st, fq, fe)
    for a, b in zip((h, f, ho, n, st.t(), fq, fe), [t.t() if t.shape[0] == 4 and t.dtype == torch.float32 else t for t in small]):
        assert torch.equal(a[-TAIL:], b)
    for t in (h, f, ho, n, fq):
        assert not bool(t[:-TAIL].any())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_weight_gradient_beyond_32_bits(B, room, dtype):
    """More than 2^32 values of X, nothing in the first rows but zeros: the gradient of the last ones."""
    M, N, K, dt, T = 64, 8200, 525000, test_act8.code(B, dtype), R.DT[dtype]
    A, x = big(K, M, dtype=T), torch.randn(TAIL, N, device="cuda").to(T)
    q, e = big(K, R.width(N), dtype=torch.uint8), torch.full((K, R.width(N) // 32), 10, dtype=torch.uint8, device="cuda")
    A[-TAIL:].normal_()
    A[:-TAIL] = 1
    B.zl_op_act8_store(dt, R.E4M3, x, TAIL, N, N, q[-TAIL:], e[-TAIL:])
    ws = torch.empty(B.zl_op_act8_dw_bytes(dt, M, N, K), dtype=torch.uint8, device="cuda")
    C = torch.full((M, N), float("nan"), device="cuda")
    B.zl_op_act8_dw(dt, R.E4M3, M, N, K, A, q, e, C, 0, ws)
    X = R.load(q[-TAIL:].cpu(), e[-TAIL:].cpu(), R.E4M3, N)
    a = A[-TAIL:].double().cpu()
    R.assert_close(C, a.T @ X, (TAIL + 64) * 2.0 ** -23 * (a.abs().T @ X.abs()), "C")
