"""What the updates' arithmetic may be off by, entry by entry: the steps on the CPU with operands of two float16 parts and
float32 sums, against float64.

An error that a step makes passes the steps behind it as the matrix itself does, and bounds of that by the largest slopes
are some thousand times what comes out.  So the bound is taken from the same arithmetic on the CPU: operands split alike,
X, P and B held in float32, sums of float32.  What differs from the kernels' is the order of the sums: either way no more
than a rounding of the running sum for each value that is added.  The operands' roundings are as large in both, but other
draws: the Frobenius norm of 256 and more independent errors, and the largest of them, differ between two draws by less
than 2, and where a few weak directions hold most of the error by 4.  FACTOR = 8 leaves another 2 for the order of the
sums.  Without a low part the error is 20 to 300 times the emulation's (test_update_precision.py)."""
import torch

import training_reference as ref

FACTOR = 8.0
F32 = torch.float32


def matrix(r, c, seed, kind):
    g = torch.Generator().manual_seed(seed)
    if kind == "plain":
        return torch.randn(r, c, generator=g)
    # a few strong directions ("strong": two, whose singular values are near one) and noise
    few = 2 if kind == "strong" else max(1, min(r, c) // 8)
    return torch.randn(r, few, generator=g) @ torch.randn(few, c, generator=g) * few ** -0.5 + 0.1 * torch.randn(r, c, generator=g)


def single(x):
    """As the C interface takes it."""
    return ref.float32(x)


def split(x):
    """float32 -> two parts of 11 bits each, scaled to float16's range and back."""
    most = float(x.abs().max())
    if not most > 0:
        return x, torch.zeros_like(x)
    up = 2.0 ** (14 - torch.frexp(torch.tensor(most)).exponent.item())
    hi = (x * up).half().float()
    lo = (x * up - hi).half().float()
    return hi / up, lo / up


def product(a, b, drop=()):
    """a b^T; drop: "left", "right": that operand's low part is lost."""
    ah, al = split(a)
    bh, bl = split(b)
    s = torch.zeros(a.shape[0], b.shape[0])
    if "left" not in drop:
        s = s + al @ bh.t()
    if "right" not in drop:
        s = s + ah @ bl.t()
    return s + ah @ bh.t()


def start(g, moment=None, momentum=0.95, nesterov=True, eps=1e-7, dtype=torch.float64):
    """X before the steps, its shorter side as rows."""
    mu = single(momentum)
    u = g.to(dtype)
    if moment is not None:
        m = mu * moment.to(dtype) + u
        u = u + mu * m if nesterov else m
    x = (u.double() * (1.0 / (float(u.double().norm()) + single(eps)))).to(dtype)
    return x.t().contiguous() if x.shape[0] >= x.shape[1] else x


def exact(x, coefs):
    for a, b, c in coefs:
        a, b, c = map(single, (a, b, c))
        p = x @ x.t()
        x = a * x + (b * p + c * p @ p) @ x
    return x


def emulated(x, coefs, gram=(), poly=(), apply=()):
    for a, b, c in coefs:
        a, b, c = map(single, (a, b, c))
        p = product(x, x, gram)
        q = b * p + c * product(p, p, poly)
        x = a * x + product(q, x.t().contiguous(), apply)
    return x


def expected(g, moment=None, weight=None, momentum=0.95, nesterov=True, coefs=(ref.MUON,) * 5, scale=1.0, decay=0.0, eps=1e-7,
             dtype=F32):
    """(out, entries' room, norm's room) of one matrix in float64."""
    turned = g.shape[0] >= g.shape[1]
    kw = dict(momentum=momentum, nesterov=nesterov, eps=eps)
    x = exact(start(g, moment, **kw), coefs)
    off = emulated(start(g, moment, dtype=F32, **kw), coefs).double() - x
    x, off = (x.t(), off.t()) if turned else (x, off)
    scale, decay = single(scale), single(decay)
    out, size = scale * x, abs(scale) * x.abs()
    if weight is not None:
        out, size = out + decay * weight.double(), size + abs(decay) * weight.double().abs()
    # the scaling and the sum, and the output's type; without steps X is two roundings
    ends = 3 * ref.U * size + (0.0 if dtype == F32 else ref.half_step(dtype) * 1.01 * out.abs())
    most, norm = float(off.abs().max()), float(off.norm())
    return out, abs(scale) * FACTOR * most + ends, abs(scale) * FACTOR * norm + float(ends.norm())


def check(got, want, name=""):
    out, entries, norm = want
    off = (got.detach().cpu().double() - out).abs()
    assert bool((off <= entries + 1e-37).all()), (name, float((off / (entries + 1e-37)).max()))
    assert float(off.norm()) <= norm + 1e-37, (name, float(off.norm()) / norm)
