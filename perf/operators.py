"""The operators of the 8-bit activation checkpoints, measured: plain forms beside the library's calls.

What a chunk holds between its forward and its local backward are the inputs of its linears, activations
and norms. These operators hold them in 8 bits (groups of 32 columns share a power of two; codes are
e4m3 or integers) and read them there in the backward. Each case is one pass through one operator:

    kind "ckpt"      rows written to 8 bits and read back (zl_op_act8_store, zl_op_act8_load)
    kind "act"       an activation's forward, which writes the checkpoint of its input in the same pass, and
                     its backward from that checkpoint, which gives the activation again for the next
                     linear's weight gradient (zl_op_act8_act, zl_op_act8_act_bwd)
    kind "dw"        a linear's weight gradient from the 8-bit checkpoint of its input (zl_op_act8_dw)
    kind "norm"      residual + gate * norm of a block's output, then the next block's norm (zl_op_block_norm);
                     with `keep` the checkpoints of the block's output and of the next block's input too,
                     read back as bf16, which holds them exactly
    kind "norm_bwd"  its backward, the block's output read from its checkpoint (zl_op_block_norm_bwd)

Sizes are those of the model configurations of this repository (GPT-2-small, Llama 1.1B, 3B and 7B
shapes), and `draw` gives others of the same ranges, odd ones among them.
"""
import math

import torch

own = False

E4M3, INT8 = 0, 1                 # code formats
SWIGLU, GELU = 0, 1               # activations
NONE, RMS, LAYER = 0, 1, 2        # norms
EPS = 1e-5
RES, BRANCH = 1.25, 0.75          # residual and branch scales of the block norm
TOP = 1.875 * 2.0 ** 127          # larger magnitudes are kept as this one


# ------------------------------------------------------------------------------------------------
# The cases
# ------------------------------------------------------------------------------------------------
def listed():
    return [
        # the smallest call: one micro-batch of 128 tokens at the GPT-2 width, where latency counts
        dict(name="ckpt-small", kind="ckpt", dtype="bf16", fmt=E4M3, N=128, d=768, ld=768),
        # a ragged fp32 batch, a slice of columns out of wider rows
        dict(name="ckpt-f32-slice", kind="ckpt", dtype="f32", fmt=INT8, N=1023, d=1100, ld=2200),
        # gate and up of the 7B shape, 2 x 1024 tokens: the widest tensor that a layer holds
        dict(name="ckpt-7b-gate-up", kind="ckpt", dtype="bf16", fmt=INT8, N=2048, d=22016, ld=22016),
        # GPT-2-style MLP in fp32 on a ragged micro-batch
        dict(name="act-gelu-f32", kind="act", dtype="f32", act=GELU, fmt=INT8, N=203, f=2112),
        # the 7B feed-forward's SwiGLU, 2 x 1024 tokens
        dict(name="act-swiglu-7b", kind="act", dtype="bf16", act=SWIGLU, fmt=E4M3, N=2048, f=11008),
        # a ragged micro-batch through one GPT-2 projection
        dict(name="dw-small", kind="dw", dtype="bf16", fmt=INT8, M=2304, N=768, K=203),
        # fp32 training of the 1.1B attention output projection, odd token count
        dict(name="dw-f32-1b", kind="dw", dtype="f32", fmt=E4M3, M=2048, N=2048, K=1021),
        # gate and up projection of the 7B shape, 2 x 1024 tokens: the largest product
        dict(name="dw-7b-gate-up", kind="dw", dtype="bf16", fmt=E4M3, M=22016, N=4096, K=2048),
        # GPT-2-style sandwich of LayerNorms, a gate row for every sequence of 128 tokens
        dict(name="norm-layer-f32", kind="norm", dtype="f32", fmt=INT8, post=LAYER, pre=LAYER, N=512, d=768, rows=128, keep=0),
        # the 7B shape with RMSNorms, one gate for all rows, both checkpoints written as the values are formed
        dict(name="norm-rms-7b-keep", kind="norm", dtype="bf16", fmt=E4M3, post=RMS, pre=RMS, N=2048, d=4096, rows=0, keep=1),
        # ragged batch at the 3B width, LayerNorm before and none after, a gate row for every 130 tokens
        dict(name="norm-bwd-3b-ragged", kind="norm_bwd", dtype="f32", fmt=INT8, post=NONE, pre=LAYER, N=517, d=3200, rows=130),
        # the 7B shape, backward from the e4m3 checkpoint
        dict(name="norm-bwd-rms-7b", kind="norm_bwd", dtype="bf16", fmt=E4M3, post=RMS, pre=RMS, N=2048, d=4096, rows=0),
    ]


def _log(rng, lo, hi, multiple=1):
    """A whole number spread over the logarithm of [lo, hi], a multiple of `multiple`."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(multiple, int(round(v / multiple)) * multiple)


def draw(rng):
    kind = rng.choice(["ckpt", "act", "dw", "norm", "norm_bwd"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    fmt = rng.choice([E4M3, INT8])
    step = rng.choice([8, 8, 1])      # odd widths among them
    if kind == "ckpt":
        N, d = _log(rng, 1, 4096), _log(rng, 100, 22016, step)
        return dict(kind=kind, dtype=dtype, fmt=fmt, N=N, d=d, ld=d if rng.random() < 0.7 else d + _log(rng, 8, 1024, step))
    if kind == "act":
        return dict(kind=kind, dtype=dtype, act=rng.choice([SWIGLU, GELU]), fmt=fmt, N=_log(rng, 1, 4096), f=_log(rng, 344, 11008, step))
    if kind == "dw":
        K = _log(rng, 1, 8192)
        M, N = _log(rng, 128, 11008, 8 if step == 8 else 2), _log(rng, 128, 8192, step)
        if dtype == "f32":            # no larger than the largest listed product
            K = min(K, 2048)
        return dict(kind=kind, dtype=dtype, fmt=fmt, M=M, N=N, K=min(K, int(22016 * 4096 * 2048 / (M * N))))
    N = _log(rng, 1, 4096)
    c = dict(kind=kind, dtype=dtype, fmt=fmt, post=rng.choice([NONE, RMS, RMS, LAYER]), pre=rng.choice([RMS, RMS, LAYER]), N=N,
             d=_log(rng, 128, 8192, step), rows=rng.choice([0, 0, 1, max(1, N // 4), _log(rng, 1, 1024)]))
    if kind == "norm":
        c["keep"] = rng.choice([0, 1])
    return c


def _pad(d):
    return (d + 31) // 32 * 32


def work(case):
    c, b = case, 2 if case["dtype"] == "bf16" else 4
    code = 33 / 32                     # bytes of a checkpointed value, its share of the group's scale with it
    if c["kind"] == "ckpt":
        n = c["N"] * c["d"]
        return {"bytes": n * 2 * (b + code), "flops": 4 * n}
    if c["kind"] == "act":
        n, w = c["N"] * c["f"], 2 if c["act"] == SWIGLU else 1
        return {"bytes": n * (w * (b + code) + b + w * code + b + w * b + b), "flops": 40 * n}
    if c["kind"] == "dw":
        M, N, K = c["M"], c["N"], c["K"]
        return {"bytes": b * K * M + code * K * N + 4 * M * N, "flops": 2 * M * N * K}
    n = c["N"] * c["d"]
    if c["kind"] == "norm":
        return {"bytes": n * (4 * b + (2 * (code + code + 2) if c["keep"] else 0)), "flops": 14 * n}
    return {"bytes": n * (5 * b + code), "flops": 30 * n}


# ------------------------------------------------------------------------------------------------
# Inputs
# ------------------------------------------------------------------------------------------------
def _dt(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _rows(g, N, d, T):
    """Activations as layers give them: channels of different size and offset, a few of them large."""
    size = torch.exp(0.5 * torch.randn(d, generator=g, device="cuda"))
    size[torch.randint(0, d, (max(1, d // 256),), generator=g, device="cuda")] *= 20.0
    off = 0.3 + 0.3 * torch.randn(d, generator=g, device="cuda")
    return (torch.randn(N, d, generator=g, device="cuda") * size + off).to(T)


def prepare(case, seed):
    c, T = case, _dt(case)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def rand(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    s = dict(case)
    if c["kind"] == "ckpt":
        s["x"] = _rows(g, c["N"], c["ld"], T)[:, :c["d"]]
    elif c["kind"] == "act":
        w = 2 if c["act"] == SWIGLU else 1
        s["x"] = _rows(g, c["N"], w * c["f"], T)
        s["dy"] = (1e-2 * rand(c["N"], c["f"])).to(T)
    elif c["kind"] == "dw":
        s["dy"] = (1e-2 * rand(c["K"], c["M"])).to(T)
        s["q"], s["e"] = plain_store(_rows(g, c["K"], c["N"], T), c["fmt"])
    else:
        N, d = c["N"], c["d"]
        G = -(-N // c["rows"]) if c["rows"] else 1
        s["gate"] = 0.5 + 0.2 * rand(G, d)
        s["post_w"] = 1 + 0.1 * rand(d) if c["post"] else None
        s["post_b"] = 0.1 * rand(d) if c["post"] == LAYER else None
        s["pre_w"] = 1 + 0.1 * rand(d)
        s["pre_b"] = 0.1 * rand(d) if c["pre"] == LAYER else None
        f = _rows(g, N, d, T)
        if c["kind"] == "norm":
            s["h"], s["f"] = _rows(g, N, d, T), f
        else:                          # what the forward left: h', the checkpoint of f, the statistics
            s["h_out"] = _rows(g, N, d, T)
            s["f_q"], s["f_e"] = plain_store(f, c["fmt"])
            s["stats"] = torch.cat([plain_stats(f.double(), c["post"]), plain_stats(s["h_out"].double(), c["pre"])], 1).T.float().contiguous()
            s["dn"], s["dh_out"] = (1e-2 * rand(N, d)).to(T), (1e-2 * rand(N, d)).to(T)
    return s


# ------------------------------------------------------------------------------------------------
# Plain forms
# ------------------------------------------------------------------------------------------------
def _pow2(e):
    """2^e for whole numbers -126 <= e <= 127."""
    return ((e + 127).to(torch.int32) << 23).view(torch.float32)


def plain_store(x, fmt):
    """(codes [N, D], exponent bytes [N, D / 32]), D the width in whole groups."""
    N, d = x.shape
    v = torch.nn.functional.pad(x.float(), (0, _pad(d) - d)).view(N, -1, 32)
    fin = torch.isfinite(v)
    v = v.clamp(-TOP, TOP)
    m, ex = torch.frexp(torch.where(fin, v, torch.zeros_like(v)).abs().amax(2))
    top, at = (0.875, 9) if fmt == E4M3 else (0.9921875, 7)      # 448 = 0.875 2^9, 127 = 0.9921875 2^7
    E = torch.where(m > 0, ex - at + (m > top).int(), torch.full_like(ex, -117)).clamp(min=-117)
    v = v * _pow2(-E).unsqueeze(2)
    if fmt == E4M3:
        q = v.to(torch.float8_e4m3fn).view(torch.uint8)
        q = torch.where(fin, q, torch.full_like(q, 0x7F))
    else:
        q = torch.where(fin, torch.round(v), torch.full_like(v, -128.0)).to(torch.int8).view(torch.uint8)
    return q.view(N, -1), (E + 127).to(torch.uint8)


def plain_load(q, e, fmt, d):
    """The values [N, d] in fp32."""
    N = q.shape[0]
    if fmt == E4M3:
        v = q.view(torch.float8_e4m3fn).float()
    else:
        v = q.view(torch.int8).float()
        v = torch.where(v == -128, torch.full_like(v, float("nan")), v)
    return (v.view(N, -1, 32) * _pow2(e.int() - 127).unsqueeze(2)).view(N, -1)[:, :d]


def plain_stats(x, norm):
    """[N, 2]: mean (0 but for LayerNorm) and 1 / deviation (1 where there is no norm)."""
    mean = x.mean(1) if norm == LAYER else torch.zeros_like(x[:, 0])
    var = (x - mean[:, None]).square().mean(1)
    return torch.stack([mean, torch.rsqrt(var + EPS) if norm else torch.ones_like(mean)], 1)


def _gate_rows(s):
    """The gate row of every row."""
    n = torch.arange(s["N"], device="cuda")
    return n // s["rows"] if s["rows"] else torch.zeros_like(n)


def _plain(s):
    T, fmt = _dt(s), s["fmt"]
    if s["kind"] == "ckpt":
        q, e = plain_store(s["x"], fmt)
        return plain_load(q, e, fmt, s["d"]).to(T)
    if s["kind"] == "act":
        f = s["f"]
        w = s["x"].shape[1]

        def act(x, dy):
            if s["act"] == SWIGLU:
                g, u = x[:, :f], x[:, f:]
                sg = 1 / (1 + torch.exp(-g))
                return g * sg * u, None if dy is None else torch.cat([dy * u * sg * (1 + g * (1 - sg)), dy * g * sg], 1)
            k, c = 0.7978845608028654, 0.044715
            t = torch.tanh(k * (x + c * x * x * x))
            return 0.5 * x * (1 + t), None if dy is None else dy * (0.5 * (1 + t) + 0.5 * x * (1 - t * t) * k * (1 + 3 * c * x * x))

        y, _ = act(s["x"].float(), None)
        q, e = plain_store(s["x"].view(-1, f), fmt)          # rows of f values: gate and up apart
        again, dx = act(plain_load(q, e, fmt, f).reshape(-1, w), s["dy"].float())
        return {"y": y.to(T), "dx": dx.to(T), "again": again.to(T)}
    if s["kind"] == "dw":
        return s["dy"].float().T @ plain_load(s["q"], s["e"], fmt, s["N"])
    gate = s["gate"][_gate_rows(s)]
    if s["kind"] == "norm":
        f = s["f"].float()
        st = plain_stats(f, s["post"])
        p = (f - st[:, :1]) * st[:, 1:]
        p = p * s["post_w"] if s["post"] else p
        p = p + s["post_b"] if s["post"] == LAYER else p
        h = RES * s["h"].float() + BRANCH * gate * p
        st2 = plain_stats(h, s["pre"])
        n = (h - st2[:, :1]) * st2[:, 1:] * s["pre_w"]
        n = n + s["pre_b"] if s["pre"] == LAYER else n
        out = {"h_out": h.to(T), "n_out": n.to(T), "stats": torch.cat([st, st2], 1).T.contiguous()}
        if s["keep"]:
            for name, x in (("f8", s["f"]), ("n8", out["n_out"])):
                q, e = plain_store(x, fmt)
                out[name] = plain_load(q, e, fmt, s["d"]).to(torch.bfloat16)
        return out
    mp, rp, m, r = s["stats"][:, :, None]
    fh = (plain_load(s["f_q"], s["f_e"], fmt, s["d"]) - mp) * rp
    xh = (s["h_out"].float() - m) * r
    dn = s["dn"].float()
    u = s["pre_w"] * dn
    G = u - xh * (u * xh).mean(1, keepdim=True)
    G = G - u.mean(1, keepdim=True) if s["pre"] == LAYER else G
    G = s["dh_out"].float() + r * G
    p = fh * s["post_w"] if s["post"] else fh
    p = p + s["post_b"] if s["post"] == LAYER else p
    dp = BRANCH * gate * G
    rows = s["rows"] or s["N"]
    per = torch.nn.functional.pad(BRANCH * G * p, (0, 0, 0, s["gate"].shape[0] * rows - s["N"]))
    out = {"dh": (RES * G).to(T), "dgate": per.view(-1, rows, s["d"]).sum(1), "dpre_w": (dn * xh).sum(0)}
    if s["pre"] == LAYER:
        out["dpre_b"] = dn.sum(0)
    if s["post"]:
        v = s["post_w"] * dp
        df = v - fh * (v * fh).mean(1, keepdim=True)
        df = rp * (df - v.mean(1, keepdim=True) if s["post"] == LAYER else df)
        out["dpost_w"] = (dp * fh).sum(0)
        if s["post"] == LAYER:
            out["dpost_b"] = dp.sum(0)
    else:
        df = dp
    out["df"] = df.to(T)
    return out


# ------------------------------------------------------------------------------------------------
# The library's calls
# ------------------------------------------------------------------------------------------------
def _own(s):
    from paper_2608_07974_gb300 import binding as zl
    T, fmt = _dt(s), s["fmt"]
    dt = zl.ZL_DTYPE_BF16 if T == torch.bfloat16 else zl.ZL_DTYPE_F32
    stream = torch.cuda.current_stream().cuda_stream

    def codes(N, d):
        D = _pad(d)
        return torch.empty(N, D, dtype=torch.uint8, device="cuda"), torch.empty(N, D // 32, dtype=torch.uint8, device="cuda")

    def load(q, e, d, T, dt):
        x = torch.empty(q.shape[0], d, dtype=T, device="cuda")
        zl.zl_op_act8_load(dt, fmt, q, e, q.shape[0], d, d, x, stream)
        return x

    if s["kind"] == "ckpt":
        q, e = codes(s["N"], s["d"])
        zl.zl_op_act8_store(dt, fmt, s["x"], s["N"], s["d"], s["ld"], q, e, stream)
        return load(q, e, s["d"], T, dt)
    if s["kind"] == "act":
        N, f, x = s["N"], s["f"], s["x"]
        y, again, dx = (torch.empty(N, w, dtype=T, device="cuda") for w in (f, f, x.shape[1]))
        q, e = codes(x.numel() // f, f)
        zl.zl_op_act8_act(dt, s["act"], fmt, x, N, f, y, q, e, stream)
        zl.zl_op_act8_act_bwd(dt, s["act"], fmt, q, e, s["dy"], N, f, dx, again, stream)
        return {"y": y, "dx": dx, "again": again}
    if s["kind"] == "dw":
        M, N, K = s["M"], s["N"], s["K"]
        ws = torch.empty(zl.zl_op_act8_dw_bytes(dt, M, N, K), dtype=torch.uint8, device="cuda")
        C = torch.empty(M, N, device="cuda")
        zl.zl_op_act8_dw(dt, fmt, M, N, K, s["dy"], s["q"], s["e"], C, 0, ws, stream)
        return C
    N, d = s["N"], s["d"]
    p = zl.zl_block_norm(dtype=dt, post_norm=s["post"], pre_norm=s["pre"], N=N, d=d, gate_rows=s["rows"], eps=EPS, res_scale=RES,
                         branch_scale=BRANCH, fmt=fmt, accumulate=0)
    a, b = (torch.empty(N, d, dtype=T, device="cuda") for _ in range(2))
    if s["kind"] == "norm":
        stats = torch.empty(4, N, device="cuda")
        f8, n8 = (codes(N, d), codes(N, d)) if s["keep"] else ((None, None), (None, None))
        zl.zl_op_block_norm(p, s["h"], s["f"], s["post_w"], s["post_b"], s["gate"], s["pre_w"], s["pre_b"], a, b, stats, *f8, *n8, stream)
        out = {"h_out": a, "n_out": b, "stats": stats}
        if s["keep"]:
            out["f8"], out["n8"] = load(*f8, d, torch.bfloat16, zl.ZL_DTYPE_BF16), load(*n8, d, torch.bfloat16, zl.ZL_DTYPE_BF16)
        return out
    grads = {"dpre_w": torch.empty(d, device="cuda"), "dgate": torch.empty_like(s["gate"])}
    if s["post"]:
        grads["dpost_w"] = torch.empty(d, device="cuda")
    for name in ("pre", "post"):
        if s[name] == LAYER:
            grads["d%s_b" % name] = torch.empty(d, device="cuda")
    ws = torch.empty(zl.zl_op_block_norm_bwd_bytes(p), dtype=torch.uint8, device="cuda")
    zl.zl_op_block_norm_bwd(p, s["h_out"], None, s["f_q"], s["f_e"], s["post_w"], s["post_b"], s["gate"], s["pre_w"], s["stats"], s["dn"],
                            s["dh_out"], a, b, grads.get("dpost_w"), grads.get("dpost_b"), grads["dgate"], grads["dpre_w"],
                            grads.get("dpre_b"), ws, stream)
    return {"dh": a, "df": b, **grads}


def run(state):
    if own:
        return _own(state)
    else:
        return _plain(state)


# ------------------------------------------------------------------------------------------------
# The same in 64 bits, from the definitions
# ------------------------------------------------------------------------------------------------
def _two(e):
    """2^e in 64 bits, exactly, for whole numbers e."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _exact_codes(x, fmt):
    """The values that the 8-bit form of x [N, d] stands for: every value rounded, ties to even, to the grid of its group."""
    N, d = x.shape
    D = _pad(d)
    v = torch.zeros(N, D, dtype=torch.float64, device="cuda")
    v[:, :d] = x
    v = v.reshape(N * D // 32, 32)
    top = 448.0 if fmt == E4M3 else 127.0
    big = v.abs().max(1, keepdim=True).values
    E = torch.ceil(torch.log2(big.clamp(min=2.0 ** -140) / top)).clamp(min=-117)
    E = torch.where(big > top * _two(E), E + 1, E)                               # the logarithm's rounding
    E = torch.where((big <= top * _two(E - 1)) & (E > -117), E - 1, E)
    y = v / _two(E)
    if fmt == E4M3:                                                              # steps of 1/8 of the power of two, from 2^-9 up
        a = y.abs().clamp(min=2.0 ** -6)
        ex = torch.floor(torch.log2(a))
        ex = torch.where(a < _two(ex), ex - 1, torch.where(a >= _two(ex + 1), ex + 1, ex))
        step = _two(ex - 3)
    else:
        step = torch.ones_like(y)
    return (torch.round(y / step) * step * _two(E)).reshape(N, D)[:, :d]


def _exact_values(q, e, fmt, d):
    """What codes stand for, by the bits of each."""
    b = q.to(torch.int64)
    if fmt == E4M3:
        ex, man = (b >> 3) & 15, (b & 7).double()
        v = torch.where(ex == 0, man * 2.0 ** -9, (8 + man) * _two(ex - 10)) * (1.0 - 2.0 * (b >> 7).double())
    else:
        v = torch.where(b > 127, b - 256, b).double()
    return (v * _two(e.to(torch.int64) - 127).repeat_interleave(32, 1))[:, :d]


def _exact_norm(x, kind, w, b):
    """Normalised rows (before gain and bias), the rows after them, mean, 1 / deviation."""
    N = x.shape[0]
    mean, rstd = x.new_zeros(N, 1), x.new_ones(N, 1)
    if kind == LAYER:
        mean = x.sum(1, keepdim=True) / x.shape[1]
    if kind != NONE:
        rstd = 1 / torch.sqrt(((x - mean) ** 2).sum(1, keepdim=True) / x.shape[1] + EPS)
    xh = (x - mean) * rstd
    y = xh if w is None else xh * w.double()
    return xh, y if b is None else y + b.double(), mean[:, 0], rstd[:, 0]


def exact(case, seed):
    s, fmt = prepare(case, seed), case["fmt"]
    if s["kind"] == "ckpt":
        return _exact_codes(s["x"].double(), fmt)
    if s["kind"] == "act":
        def act(x):
            if s["act"] == SWIGLU:
                g, u = x.chunk(2, 1)
                return torch.sigmoid(g) * g * u
            return 0.5 * x * (1 + torch.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3)))

        x8 = _exact_codes(s["x"].double().view(-1, s["f"]), fmt).reshape(s["x"].shape).requires_grad_(True)
        again = act(x8)
        (dx,) = torch.autograd.grad(again, x8, s["dy"].double())
        return {"y": act(s["x"].double()), "dx": dx, "again": again.detach()}
    if s["kind"] == "dw":
        return torch.mm(s["dy"].double().t(), _exact_values(s["q"], s["e"], fmt, s["N"]))
    rows = s["rows"] or s["N"]
    gate = s["gate"].double().repeat_interleave(rows, 0)[:s["N"]]
    if s["kind"] == "norm":
        _, p, mp, rp = _exact_norm(s["f"].double(), s["post"], s["post_w"], s["post_b"])
        h = RES * s["h"].double() + BRANCH * gate * p
        _, n, m, r = _exact_norm(h, s["pre"], s["pre_w"], s["pre_b"])
        out = {"h_out": h, "n_out": n, "stats": torch.stack([mp, rp, m, r])}
        if s["keep"]:
            out["f8"], out["n8"] = _exact_codes(s["f"].double(), fmt), _exact_codes(n.to(_dt(s)).double(), fmt)
        return out
    # the vector-Jacobian product, the statistics of the forward taken as they were given
    mp, rp, m, r = (t.double()[:, None] for t in s["stats"])
    d, dn = s["d"], s["dn"].double()
    fh, xh = (_exact_values(s["f_q"], s["f_e"], fmt, d) - mp) * rp, (s["h_out"].double() - m) * r

    def back(dy, w, hat, rstd, kind):
        if kind == NONE:
            return dy
        t = dy if w is None else dy * w.double()
        t = t - hat * ((t * hat).sum(1, keepdim=True) / d) - ((t.sum(1, keepdim=True) / d) if kind == LAYER else 0)
        return rstd * t

    G = s["dh_out"].double() + back(dn, s["pre_w"], xh, r, s["pre"])
    p = fh if s["post_w"] is None else fh * s["post_w"].double()
    p = p if s["post_b"] is None else p + s["post_b"].double()
    dp = BRANCH * gate * G
    per = BRANCH * G * p
    full = torch.zeros(s["gate"].shape[0] * rows, d, dtype=torch.float64, device="cuda")
    full[:s["N"]] = per
    out = {"dh": RES * G, "df": back(dp, s["post_w"], fh, rp, s["post"]), "dgate": full.view(-1, rows, d).sum(1), "dpre_w": (dn * xh).sum(0)}
    if s["pre"] == LAYER:
        out["dpre_b"] = dn.sum(0)
    if s["post"]:
        out["dpost_w"] = (dp * fh).sum(0)
    if s["post"] == LAYER:
        out["dpost_b"] = dp.sum(0)
    return out
