"""Normalisations, AdamW steps and 8-bit states from their definitions, with plain torch operations on the CPU (nothing of the
library), and the inputs that their tests share."""
import torch

EPS_HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}     # half a step of a type, relative: what one rounding takes


# ------------------------------------------------------------- normalisation, in 64 bits
def norm(x, w=None, b=None, eps=1e-6, layer=True):
    """(y, h, mean, rstd) of rows of x float64."""
    mean = x.mean(dim=1, keepdim=True) if layer else torch.zeros((x.shape[0], 1), dtype=torch.float64)
    d = x - mean
    rstd = ((d * d).mean(dim=1, keepdim=True) + eps) ** -0.5
    h = d * rstd
    y = h if w is None else h * w
    return (y if b is None else y + b), h, mean[:, 0], rstd[:, 0]


def norm_grad(h, rstd, dy, w=None, layer=True):
    """(dx, d_weight, d_bias, the size of what dx is a difference of)."""
    g = dy if w is None else dy * w
    mgh = (g * h).mean(dim=1, keepdim=True)
    mg = g.mean(dim=1, keepdim=True) if layer else torch.zeros_like(mgh)
    r = rstd[:, None]
    size = r * (g.abs() + g.abs().mean(dim=1, keepdim=True) + h.abs() * (g * h).abs().mean(dim=1, keepdim=True))
    return r * (g - mg - h * mgh), (dy * h).sum(dim=0), dy.sum(dim=0), size


# ------------------------------------------------------------- 8-bit states
BLOCK = 64
FIRST, ROOT, WEIGHT = 0, 1 << 31, 1 << 30


def blocks(x):
    """[n] -> [ceil(n / 64), 64], zeros behind the end."""
    return torch.nn.functional.pad(x, (0, -x.numel() % BLOCK)).view(-1, BLOCK)


def turns(step, start):
    place = torch.arange(BLOCK, dtype=torch.int64)
    return ((step % (1 << 32)) * 0x9E3779B9 + start + place * 0xC13FA9A9) % (1 << 32)


def root(v):
    """The rounded root of fp32 numbers: rounded once from 64 bits, since torch's own on the CPU is off by a place for one number in six."""
    return v.double().sqrt().float()


def encode(x, mantissa, step):
    """x fp32 [n]: (codes, scales), by the places of values between codes; mantissa 3: with a sign, 4: a root."""
    size = blocks(x).double().abs()
    top = size.amax(dim=1, keepdim=True)
    ok = torch.isfinite(top)
    part, power = torch.frexp(torch.where(ok, top, torch.ones_like(top)))         # top = part 2^power, part in [1/2, 1)
    power = power + (part > 1 - 2.0 ** -(mantissa + 1)).int() - 1                  # of the largest binade that is used
    power = torch.where(top > 0, power, torch.full_like(power, -127)).clamp(min=15 - 127)
    ok = ok & (power <= 127)
    low = (power - 14).double()                                                    # of the lowest binade; below it codes go down to zero
    _, binade = torch.frexp(size)
    gap = torch.exp2(torch.maximum(binade.double() - 1, low) - mantissa)
    threshold = torch.div(turns(step, FIRST if mantissa == 3 else ROOT), 1 << (9 + mantissa), rounding_mode="floor").double() / 2.0 ** (23 - mantissa)
    held = torch.floor(size / gap + threshold) * gap
    if mantissa == 4:
        held = torch.where(size > 0, torch.maximum(held, torch.exp2(low - 4)), held)
    # a value's code: (exponent, mantissa), counted from the lowest binade's zero
    y = held / torch.exp2(low)                                                     # 1 at the lowest binade's begin
    part, power_y = torch.frexp(y)
    code = torch.where(y < 1, y * 2 ** mantissa, power_y.double() * 2 ** mantissa + (part * 2 - 1) * 2 ** mantissa)
    code = code.to(torch.int64)
    if mantissa == 3:
        code = code | (torch.signbit(blocks(x)).to(torch.int64) << 7)
    n = x.numel()
    scale = torch.where(ok, power + 127, torch.full_like(power, 255))[:, 0]
    return code.view(-1)[:n].to(torch.uint8), scale.to(torch.uint8)


def decode(code, scale, mantissa):
    """[n] fp32."""
    c = blocks(code).long()
    sign = torch.ones_like(c)
    if mantissa == 3:
        sign, c = 1 - 2 * (c >> 7), c & 127
    exponent, m = c >> mantissa, (c & ((1 << mantissa) - 1)).double() / 2 ** mantissa
    y = torch.where(exponent > 0, (1 + m) * torch.exp2(exponent.double() - 1), m)
    value = sign * y * torch.exp2(scale[:, None].double() - 127 - 14)
    value[scale == 255] = float("nan")
    return value.view(-1)[:code.numel()].float()


# ------------------------------------------------------------- one step of one tensor
def moments(g, m, v_or_root, beta1, beta2, root=False):
    """(m, v) in fp32, each operation rounded once: what the state is made of."""
    v = v_or_root * v_or_root if root else v_or_root
    return m * beta1 + g * (1 - beta1), v * beta2 + g * g * (1 - beta2)


def adamw(p, g, m, v, step, lr, beta1, beta2, eps, decay):
    """In 64 bits: (new p, m, v, the size of the change)."""
    # m is a sum of two terms, each rounded relative to itself: where their signs differ, m is off by 2^-24 of their sizes' sum,
    # which may be any multiple of |m|, and so the change by as much of what that sum would make
    m, size = beta1 * m + (1 - beta1) * g, beta1 * m.abs() + (1 - beta1) * g.abs()
    v = beta2 * v + (1 - beta2) * g * g
    rate = lr / (1 - beta1 ** step) / (torch.sqrt(v) / (1 - beta2 ** step) ** 0.5 + eps)
    return p - (rate * m + lr * decay * p), m, v, rate * size + (lr * decay * p).abs()


def off(got, want, bound, what=""):
    """got, want: nowhere further apart than bound (an array of its shape)."""
    got, want, bound = got.double().cpu(), want.double().cpu(), bound.double().cpu()
    bad = ~((got - want).abs() <= bound)
    assert not bool(bad.any()), (what, int(bad.sum()), float(((got - want).abs() / bound)[bad].max()), bad.nonzero()[:4].tolist())
