"""Plain 64-bit forms of the 8-bit layers and of the optimizer's step, on the CPU."""
import numpy as np
import torch

FP8 = torch.float8_e4m3fn


def f32(x):
    return x.float().double()


def e4m3(x):
    """Nearest e4m3 value, ties to even, by the spacing of the format: 2^-9 below 2^-6, an eighth of the power of two above."""
    step = torch.ldexp(torch.ones_like(x), torch.frexp(x)[1].clamp(min=-5) - 4)
    return torch.round(x / step) * step


def scale_of(amax):
    """fp32 arithmetic: a quotient of two fp32 numbers in fp64, rounded, is the rounded quotient."""
    s = f32(amax / 448).clamp(min=2.0 ** -126)
    return torch.where(torch.isfinite(amax), s, torch.full_like(s, float("nan")))


def quantize(x, tiles=False):
    """-> (code values, scales), fp64, of an fp32 or bf16 matrix on the CPU."""
    m, d = x.shape
    rows = 128 if tiles else 1
    b = torch.zeros(-(-m // rows) * rows, -(-d // 128) * 128, dtype=torch.float64)
    b[:m, :d] = x.double()
    b = b.view(-1, rows, b.shape[1] // 128, 128)
    s = scale_of(b.abs().amax((1, 3)))
    q = e4m3(f32(b * f32(1 / s)[:, None, :, None]))
    return q.reshape(-1, b.shape[2] * 128)[:m, :d], s


def values(q, s):
    m, d = q.shape
    s = s.double()
    if s.shape[0] != m:
        s = s.repeat_interleave(128, 0)[:m]
    return q.double() * s.repeat_interleave(128, 1)[:, :d]


def draws(n, step, index, seed):
    """The 16 random bits of each of n elements."""
    u64, low = np.uint64, np.uint64(0xFFFFFFFF)
    g = np.arange((n + 7) // 8, dtype=u64)
    c = [g & low, g >> u64(32), np.full_like(g, step & 0xFFFFFFFF), np.full_like(g, index)]
    k = np.array([seed & 0xFFFFFFFF, seed >> 32], u64)
    for _ in range(7):
        a, b = c[0] * u64(0xD2511F53), c[2] * u64(0xCD9E8D57)
        c = [(b >> u64(32)) ^ c[1] ^ k[0], b & low, (a >> u64(32)) ^ c[3] ^ k[1], a & low]
        k = (k + np.array([0x9E3779B9, 0xBB67AE85], u64)) & low
    return torch.from_numpy(np.stack(c, 1).astype("<u4").view("<u2").reshape(-1)[:n].astype(np.int64))


def _over_blocks(x, f):
    out = torch.zeros(-(-x.numel() // 256) * 256, dtype=torch.float64)
    out[:x.numel()] = x
    return f(out.view(-1, 256))


def state_values(codes, scale, n):
    """fl(code scale) of a state."""
    return f32(codes.double().cpu() * scale.double().cpu().repeat_interleave(256)[:n])


def adamw(p, g, m, v, step, lr, betas, eps, decay, coef=None):
    """One step in the fp32 arithmetic that the header fixes, carried out in fp64 with every operation rounded (products and sums of
    two fp32 numbers, quotients and roots are rounded rightly this way): -> (p, m, v, root of v), fp64 holding fp32 values."""
    c = lambda x: float(np.float32(x))  # noqa: E731
    (b1, b2), g = betas, g.double()
    if coef is not None:
        g = f32(g * coef)
    m = f32(f32(m * c(b1)) + f32(g * c(1 - b1)))
    v = f32(f32(v * c(b2)) + f32(f32(g * c(1 - b2)) * g))
    r = f32(v.sqrt())
    size = f32(f32(r * c((1 - b2 ** step) ** -0.5)) + c(eps))
    p = f32(f32(p.double() * c(1 - lr * decay)) - f32(f32(m / size) * c(lr / (1 - b1 ** step))))
    return p, m, v, r


def state_codes(m, r, step, index, seed):
    """Codes' values and scales of the two states in 8 bits."""
    n = m.numel()
    ms, rs = (_over_blocks(x, lambda b: scale_of(b.abs().amax(1))) for x in (m, r))
    each = lambda s: s.repeat_interleave(256)[:n]  # noqa: E731
    mq = e4m3(f32(m * f32(1 / each(ms))))
    x = f32(r * f32(1 / each(rs))).clamp(max=448.0)
    gap = torch.ldexp(torch.ones_like(x), torch.frexp(x)[1].clamp(min=-5) - 4)
    lo = torch.floor(x / gap) * gap
    share = f32(f32(f32(x - lo) * f32(x + lo)) * 65536)
    y = torch.where(share > draws(n, step, index, seed).double() * gap * (2 * lo + gap), lo + gap, lo)
    return mq, ms, torch.where((x > 0) & (y == 0), torch.full_like(y, 2.0 ** -9), y), rs
