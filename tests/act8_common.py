"""64-bit restatement of the 8-bit checkpoint operators (CPU, plain loops over nothing: tensor arithmetic), for their tests."""
import torch

E4M3, INT8 = 0, 1
SWIGLU, GELU = 0, 1
NONE, RMS, LAYER = 0, 1, 2
TOP = 1.875 * 2.0 ** 127
# half a step of a value's last place, relative
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def two(e):
    """2^e in 64 bits for whole numbers."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def width(d):
    return (d + 31) // 32 * 32


def store(x, fmt):
    """Codes (uint8 [N, D]) and group bytes (uint8 [N, D / 32]) of x [N, d], by rounding to the grid in 64 bits."""
    N, d = x.shape
    v = torch.zeros(N, width(d), dtype=torch.float64)
    v[:, :d] = x.double()
    v = v.view(N, -1, 32)
    fin = torch.isfinite(v)
    v = torch.where(fin, v.clamp(-TOP, TOP), torch.zeros_like(v))
    big = v.abs().amax(2)
    Q = 448.0 if fmt == E4M3 else 127.0
    E = torch.full_like(big, -117).to(torch.int64)
    guess = torch.floor(torch.log2((big / Q).clamp(min=2.0 ** -200))).to(torch.int64)
    for k in (-1, 0, 1, 2):                        # the smallest of the neighbours that holds the group
        c = (guess + k).clamp(min=-117)
        if k == -1:
            E = c
        else:
            E = torch.where(big > Q * two(E), torch.maximum(c, E), E)
    y = v / two(E)[..., None]
    if fmt == INT8:
        q = torch.round(y).to(torch.int64) & 255
        q = torch.where(fin, q, torch.full_like(q, 128))
    else:
        a = y.abs()
        ex = torch.floor(torch.log2(a.clamp(min=2.0 ** -6))).to(torch.int64)
        ex = torch.where(a >= two(ex + 1), ex + 1, torch.where((a < two(ex)) & (ex > -6), ex - 1, ex))
        n = torch.round(a / two(ex - 3)).to(torch.int64)          # 8 .. 16 steps, or fewer below 2^-6
        ex, n = torch.where(n == 16, ex + 1, ex), torch.where(n == 16, torch.full_like(n, 8), n)
        code = torch.where(n < 8, n, ((ex + 7) << 3) + n - 8)
        neg = torch.signbit(y).to(torch.int64)
        q = torch.where(fin, code + (neg << 7), torch.full_like(code, 0x7F))
    return q.to(torch.uint8).view(N, -1), (E + 127).to(torch.uint8)


def load(q, e, fmt, d):
    """What the codes stand for, in 64 bits."""
    N = q.shape[0]
    b = q.to(torch.int64)
    if fmt == E4M3:
        ex, man = (b >> 3) & 15, (b & 7).double()
        v = torch.where(ex == 0, man * 2.0 ** -9, (8 + man) * two(ex - 10)) * torch.where(b > 127, -1.0, 1.0).double()
        v = torch.where((b & 127) == 127, torch.full_like(v, float("nan")), v)
    else:
        v = torch.where(b > 127, b - 256, b).double()
        v = torch.where(b == 128, torch.full_like(v, float("nan")), v)
    return (v.view(N, -1, 32) * two(e.to(torch.int64) - 127)[..., None]).view(N, -1)[:, :d]


def act(x, kind):
    """y of x [N, 2 f] or [N, f]."""
    if kind == SWIGLU:
        g, u = x.chunk(2, 1)
        return g * torch.sigmoid(g) * u
    # 0.5 (1 + tanh a) = 1 / (1 + e^-2a), which keeps its digits where tanh a is near -1
    return x * torch.sigmoid(2 * (2 / torch.pi) ** 0.5 * (x + 0.044715 * x ** 3))


def norm(x, kind, w, b, eps):
    """(normalised rows, rows after gain and bias, mean, 1 / deviation)."""
    mean, rstd = torch.zeros_like(x[:, :1]), torch.ones_like(x[:, :1])
    if kind == LAYER:
        mean = x.mean(1, keepdim=True)
    if kind != NONE:
        rstd = ((x - mean).square().mean(1, keepdim=True) + eps) ** -0.5
    xh = (x - mean) * rstd
    y = xh if w is None else xh * w
    return xh, y if b is None else y + b, mean[:, 0], rstd[:, 0]


def gate_index(N, gate_rows):
    n = torch.arange(N)
    return n // gate_rows if gate_rows else torch.zeros_like(n)


def block_norm(c, h, f, post_w, post_b, gate, pre_w, pre_b):
    """(h', n, stats [4, N]); c: dict(post, pre, rows, eps, alpha, beta)."""
    _, p, mp, rp = norm(f, c["post"], post_w, post_b, c["eps"])
    g = 1.0 if gate is None else gate[gate_index(len(h), c["rows"])]
    ho = c["alpha"] * h + c["beta"] * g * p
    _, n, m, r = norm(ho, c["pre"], pre_w, pre_b, c["eps"])
    return ho, n, torch.stack([mp, rp, m, r])


def block_norm_bwd(c, ho, f, post_w, post_b, gate, pre_w, stats, dn, dho):
    """Gradients, and per output the sum of magnitudes that its rounding errors are relative to: name -> (value, scale)."""
    N, d = f.shape
    mp, rp, m, r = stats[:, :, None]
    one = torch.ones(d, dtype=f.dtype)
    G, sG = (torch.zeros_like(f), torch.zeros_like(f)) if dho is None else (dho, dho.abs())
    out = {}
    if c["pre"]:
        xh, sxh = (ho - m) * r, (ho.abs() + m.abs()) * r
        u = dn * (one if pre_w is None else pre_w)
        s1 = u.mean(1, keepdim=True) if c["pre"] == LAYER else 0.0
        G = G + r * (u - s1 - xh * (u * xh).mean(1, keepdim=True))
        sG = sG + r * (u.abs() + (u.abs().mean(1, keepdim=True) if c["pre"] == LAYER else 0) + sxh * (u.abs() * sxh).mean(1, keepdim=True))
        out["dpre_w"], out["dpre_b"] = ((dn * xh).sum(0), (dn.abs() * sxh).sum(0)), (dn.sum(0), dn.abs().sum(0))
    fh, sfh = ((f - mp) * rp, (f.abs() + mp.abs()) * rp) if c["post"] else (f, f.abs())
    w, b = (one if post_w is None else post_w), (0 * one if post_b is None else post_b)
    at = gate_index(N, c["rows"])
    g = torch.ones_like(f) if gate is None else gate[at]
    p, sp = fh * w + b, sfh * w.abs() + b.abs()
    dp, sdp = c["beta"] * g * G, abs(c["beta"]) * g.abs() * sG
    if gate is not None:
        z = torch.zeros_like(gate)
        out["dgate"] = (z.index_add(0, at, c["beta"] * G * p), z.index_add(0, at, abs(c["beta"]) * sG * sp))
    out["dh"] = (c["alpha"] * G, abs(c["alpha"]) * sG)
    if c["post"]:
        v, sv = dp * w, sdp * w.abs()
        t1 = v.mean(1, keepdim=True) if c["post"] == LAYER else 0.0
        df = rp * (v - t1 - fh * (v * fh).mean(1, keepdim=True))
        sdf = rp * (sv + (sv.mean(1, keepdim=True) if c["post"] == LAYER else 0) + sfh * (sv * sfh).mean(1, keepdim=True))
        out["df"] = (df, sdf)
        out["dpost_w"], out["dpost_b"] = ((dp * fh).sum(0), (sdp * sfh).sum(0)), (dp.sum(0), sdp.sum(0))
    else:
        out["df"] = (dp, sdp)
    return out


def assert_close(got, ref, bound, what):
    """|got - ref| <= bound element by element, NaN where ref is NaN."""
    got, ref = got.detach().cpu().double(), ref.double()
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    nan = torch.isnan(ref)
    assert torch.equal(torch.isnan(got), nan), what
    over = ((got - ref).abs() - bound)[~nan]
    assert over.numel() == 0 or float(over.max()) <= 0, (what, float(over.max()), float((got - ref).abs()[~nan].max()))
