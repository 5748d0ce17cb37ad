"""What the calls on losses over a vocabulary refuse, on the host (no GPU: placeholder pointers never reach a kernel)."""
import pytest
import torch

P = 256   # placeholder device address


@pytest.fixture(scope="module")
def B():
    import paper_2608_07974_gb300 as pkg
    pkg.build()
    from paper_2608_07974_gb300 import binding
    return binding


host_only = pytest.mark.skipif(torch.cuda.is_available(), reason="placeholder pointers: host-only check")

TOP = dict(dtype=1, z=P, N=4, V=100, ld=100, k=8, T=1.0, idx=P, val=P, rest=P, stream=None)
LOSS = dict(dtype=1, z=P, idx=P, val=P, rest=P, labels=P, N=4, V=100, ld=100, k=8, alpha=0.5, T=1.0, kl_dir=0, dz=P, row_loss=P,
            loss=P, stream=None)
SIZES = [dict(dtype=2), dict(N=-1), dict(N=(1 << 24) + 1), dict(V=1, k=1), dict(V=(1 << 20) + 1, ld=1 << 21), dict(ld=99), dict(k=0),
         dict(k=101), dict(V=5000, ld=5000, k=1025), dict(T=0.0), dict(T=-1.0), dict(T=float("inf")), dict(T=float("nan")),
         dict(T=1e-45)]


@host_only
@pytest.mark.parametrize("bad", SIZES + [dict(z=None), dict(idx=None), dict(val=None), dict(rest=None), dict(z=P + 1), dict(idx=P + 2),
                                         dict(val=P + 1), dict(rest=P + 3)])
def test_top_logits_refuses(B, bad):
    assert B._lib.zl_op_top_logits(*{**TOP, **bad}.values()) == B.ZL_ERR_ARG
    assert B.last_error()


@host_only
@pytest.mark.parametrize("bad", SIZES + [dict(z=None), dict(dz=None), dict(labels=None), dict(row_loss=None), dict(loss=None),
                                         dict(idx=None), dict(val=None), dict(rest=None), dict(alpha=-0.1), dict(alpha=1.1),
                                         dict(alpha=float("nan")), dict(kl_dir=2), dict(z=P + 1), dict(dz=P + 1), dict(labels=P + 1),
                                         dict(idx=P + 1), dict(val=P + 2), dict(rest=P + 1), dict(row_loss=P + 2), dict(loss=P + 1)])
def test_top_loss_refuses(B, bad):
    assert B._lib.zl_op_top_loss(*{**LOSS, **bad}.values()) == B.ZL_ERR_ARG
    assert B.last_error()


@pytest.mark.parametrize("name,bad,error", [
    ("z", torch.zeros(4, 100), TypeError), ("idx", torch.zeros(32, dtype=torch.int64), TypeError), ("val", torch.zeros(32, dtype=torch.float64), TypeError)])
def test_binding_refuses_types(B, name, bad, error):
    args = dict(z=P, idx=P, val=P, rest=P)
    args[name] = bad
    with pytest.raises(error):
        B.zl_op_top_logits(B.ZL_DTYPE_BF16, args["z"], 4, 100, 100, 8, 1.0, args["idx"], args["val"], args["rest"])


FWD = dict(dtype=1, n=P, W=P, labels=P, N=4, d=64, V=100, row_loss=P, lse=P, loss=P, ws=P, ws_bytes=1 << 40, stream=None)
BWD = dict(dtype=1, n=P, W=P, labels=P, N=4, d=64, V=100, lse=P, dloss=None, dn=P, dW=P, ws=P, ws_bytes=1 << 40, stream=None)
VOCAB = [dict(dtype=2), dict(N=-1), dict(N=(1 << 24) + 1), dict(V=1), dict(V=(1 << 20) + 1), dict(d=0), dict(d=12), dict(d=(1 << 16) + 8),
         dict(n=None), dict(W=None), dict(labels=None), dict(lse=None), dict(ws=None), dict(n=P + 8), dict(W=P + 4), dict(labels=P + 2),
         dict(lse=P + 1), dict(ws=P + 128), dict(ws_bytes=64)]


@host_only
@pytest.mark.parametrize("bad", VOCAB + [dict(row_loss=None), dict(loss=None), dict(row_loss=P + 1), dict(loss=P + 2)])
def test_vocab_loss_refuses(B, bad):
    assert B._lib.zl_op_vocab_loss(*{**FWD, **bad}.values()) == B.ZL_ERR_ARG
    assert B.last_error()


@host_only
@pytest.mark.parametrize("bad", VOCAB + [dict(dn=None, dW=None), dict(dn=P + 8), dict(dW=P + 2), dict(dloss=P + 1)])
def test_vocab_loss_bwd_refuses(B, bad):
    assert B._lib.zl_op_vocab_loss_bwd(*{**BWD, **bad}.values()) == B.ZL_ERR_ARG
    assert B.last_error()


def test_workspace_sizes(B):
    """They hold what they are for, go with the sizes, and refuse what the calls refuse."""
    for f in (B.zl_op_vocab_loss_bytes, B.zl_op_vocab_loss_bwd_bytes):
        for dtype in (B.ZL_DTYPE_F32, B.ZL_DTYPE_BF16):
            assert f(dtype, 0, 64, 100) == 0 and f(dtype, 1, 8, 2) > 0
            for bad in ((2, 4, 64, 100), (dtype, -1, 64, 100), (dtype, 4, 60, 100), (dtype, 4, 64, 1)):
                with pytest.raises(B.ZLError):
                    f(*bad)
    assert B.zl_op_vocab_loss_bytes(B.ZL_DTYPE_F32, 2000, 64, 1000) >= 6 * 64 * 3000   # the terms of n and, for many rows, of W
    assert B.zl_op_vocab_loss_bytes(B.ZL_DTYPE_BF16, 4096, 768, 50257) < 64 << 20      # no logits
    assert B.zl_op_vocab_loss_bwd_bytes(B.ZL_DTYPE_BF16, 4096, 768, 50257) < 4096 * 50257


def test_binding_refuses_types_and_addresses_of_workspaces(B):
    with pytest.raises(TypeError):
        B.zl_op_vocab_loss(B.ZL_DTYPE_BF16, torch.zeros(4, 64), P, P, 4, 64, 100, P, P, P, None)
    with pytest.raises(TypeError):
        B.zl_op_vocab_loss(B.ZL_DTYPE_BF16, P, P, torch.zeros(4, dtype=torch.int64), 4, 64, 100, P, P, P, None)
    with pytest.raises(TypeError):
        B.zl_op_vocab_loss_bwd(B.ZL_DTYPE_BF16, P, P, P, 4, 64, 100, P, None, P, P, P)


@host_only
@pytest.mark.parametrize("T", [3e-39, 4.1e-39])
def test_temperatures_whose_scale_overflows_are_refused(B, T):
    """1 / T is finite there, log2(e) / T, by which exponents are scaled, is not."""
    assert B._lib.zl_op_top_logits(*{**TOP, "T": T}.values()) == B.ZL_ERR_ARG
    assert B._lib.zl_op_top_loss(*{**LOSS, "T": T}.values()) == B.ZL_ERR_ARG
