"""Plain 64-bit forms of the operators of a model's end and the bounds their kernels are held to (no GPU code, no library calls)."""
import torch

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float8_e4m3fn: 2.0 ** -4}   # half a step, relative to the value
U = 2.0 ** -24

M0, M1, W0, W1, LOW = 0xD2511F53, 0xCD9E8D57, 0x9E3779B9, 0xBB67AE85, 0xFFFFFFFF


def philox(counter, key):
    """Philox4x32-10 of one counter, in Python integers."""
    c, k = list(counter), list(key)
    for _ in range(10):
        a, b = M0 * c[0], M1 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & LOW, (a >> 32) ^ c[3] ^ k[1], a & LOW]
        k = [(k[0] + W0) & LOW, (k[1] + W1) & LOW]
    return c


def threshold(p):
    return min(65535, int(65536 * float(torch.tensor(p, dtype=torch.float32)) + 0.5))


def factors(rows, cols, p, seed, offset, first=0):
    """What dropout multiplies every element by, 0 or 65536 / (65536 - threshold), as float64 on the CPU: rows first .. first + rows."""
    thr = threshold(p)
    out = torch.empty(rows, cols, dtype=torch.float64)
    key = (seed & LOW, seed >> 32 & LOW)
    offset &= (1 << 64) - 1
    for r in range(rows):
        bits = []
        for g in range((cols + 7) // 8):
            for w in philox((g, (first + r) & LOW, offset & LOW, offset >> 32), key):
                bits += [w & 0xFFFF, w >> 16]
        out[r] = torch.tensor([65536.0 / (65536 - thr) if b >= thr else 0.0 for b in bits[:cols]], dtype=torch.float64)
    return out


def norm(h, weight, eps):
    h, w = h.double(), weight.double()
    rstd = (h.square().mean(-1, keepdim=True) + eps) ** -0.5
    return h * rstd * w, rstd[..., 0]


def norm_backward(dy, h, weight, rstd, dh=None):
    """dh', dweight, and a bound of what fp32 sums and products are off for each."""
    dy, n, g = dy.double(), h.double() * rstd.double()[..., None], weight.double()
    dn, r = dy * g, rstd.double()[..., None]
    out = r * (dn - n * (dn * n).mean(-1, keepdim=True))
    size = r * (dn.abs() + n.abs() * (dn * n).abs().mean(-1, keepdim=True))
    if dh is not None:
        out, size = out + dh.double(), size + dh.double().abs()
    flat = lambda t: t.reshape(-1, t.shape[-1])     # noqa: E731
    return out, size, flat(dy * n).sum(0), flat((dy * n).abs()).sum(0)


def head(x, weight, targets, row_weight=None, reduction="mean", scale=1.0, upstream=1.0, dtype=torch.bfloat16):
    """Loss, row losses, lse, dx, dweight in float64 and elementwise bounds of the kernels' errors, from the roundings that the
    operator makes: products and sums in fp32, exponentials to 2^-21, P rounded to dtype, the gradients rounded to dtype."""
    x64, w64 = x.double().reshape(-1, x.shape[-1]), weight.double()
    t = targets.reshape(-1)
    live = torch.nonzero((t >= 0) & (t < w64.shape[0]))[:, 0]
    n, k, v = len(live), x64.shape[1], w64.shape[0]
    xl, tl = x64[live], t[live]
    s = xl @ w64.t()
    s_off = (k + 2) * U * (xl.abs() @ w64.abs().t())         # a sum of k products, in whatever order
    lse = torch.logsumexp(s, 1)
    at = torch.arange(n, device=t.device)
    row = lse - s[at, tl]
    # the lse moves as much as its logits at most; its own sum of v exponentials and the logarithm are below 2^-19
    lse_off = s_off.amax(1) if n else lse
    lse_off = lse_off + 2.0 ** -19 + 4 * U * lse.abs()
    row_off = 2 * lse_off
    w = torch.ones(n, dtype=torch.float64, device=t.device) if row_weight is None else row_weight.reshape(-1)[live].double()
    f = scale / (max(1, n) if reduction == "mean" else 1)
    out = {"loss": (w * row).sum() * f, "loss_off": (w.abs() * row_off).sum() * abs(f) + 2 * U * ((w * row).sum() * f).abs()}
    full = lambda z: torch.zeros(len(t), dtype=torch.float64, device=t.device).index_copy_(0, live, z)      # noqa: E731
    out.update(row=full(row), row_off=full(row_off), lse=full(lse), lse_off=full(lse_off))
    f = f * upstream
    p = (s - lse[:, None]).exp()
    p_off = p * (s_off + lse_off[:, None] + 2.0 ** -21 * (1 + (s - lse[:, None]).abs()))
    p[at, tl] -= 1.0
    p, p_off = p * w[:, None], p_off * w.abs()[:, None]
    half = HALF[dtype]
    p_off = p_off + (half + 2 * U) * p.abs() + 1e-37
    dx = f * (p @ w64)
    dx_off = abs(f) * ((p_off + (v + 4) * U * p.abs()) @ w64.abs())
    dw = f * (p.t() @ xl)
    dw_off = abs(f) * ((p_off + (n + 4) * U * p.abs()).t() @ xl.abs())
    wide = lambda z: torch.zeros_like(x64).index_copy_(0, live, z)      # noqa: E731
    out.update(dx=wide(dx), dx_off=wide(dx_off) * (1 + half), dw=dw, dw_off=dw_off * (1 + half))
    return out


def within(name, got, want, off, dtype=torch.float32):
    """|got - want| at most the bound and half a step of the type, everywhere."""
    got, want = got.double().reshape(want.shape), want.double()
    assert bool(torch.isfinite(got).all()), f"{name}: not finite"
    far = (got - want).abs() - (off + HALF[dtype] * want.abs() * (1 + 2 ** -8) + 1e-37)
    worst = float(far.max()) if far.numel() else -1.0
    assert worst <= 0, f"{name}: {worst:.3g} outside its bound at {int(far.argmax())} of {far.numel()}"
