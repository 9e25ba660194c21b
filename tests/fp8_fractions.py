"""Blocks whose codes tell whether the quantizer multiplies by the rounded reciprocal of their scale: for the fractions of amax, values next to
where the product with it lies half way between two codes."""
import torch

FP8 = torch.float8_e4m3fn
# half way between codes: of normal ones from 1.4 on, and of the small ones, which lie 2^-9 apart
MIDDLES = [23 / 16, 25 / 16, 27 / 16, 29 / 16, 31 / 16] + [(2 * k + 1) / 1024 for k in range(4, 8)]


def next_float(x, steps):
    return (x.view(torch.int32) + steps).view(torch.float32)


def scales(fractions):
    """fractions (int32, 0 .. 2^23 - 1) -> (amax = 1 + fraction / 2^23, scale, reciprocal).  Quotients of two fp32 numbers in fp64, rounded to
    fp32, are the rounded quotients."""
    amax = (fractions + 0x3F800000).view(torch.float32)
    scale = (amax.double() / 448).float()
    return amax, scale, (1 / scale.double()).float()


def blocks(fractions):
    """-> (x, scale, reciprocal): a row of 28 values for each fraction, amax first."""
    amax, scale, reciprocal = scales(fractions)
    x = [amax]
    for c in MIDDLES:
        x += [next_float((c * scale.double()).float(), steps) for steps in (-1, 0, 1)]
    return torch.stack(x, 1), scale, reciprocal


def codes(x, reciprocal):
    return (x * reciprocal[:, None]).to(FP8).view(torch.uint8)


def delicate():
    """Fractions whose scales' reciprocals come out wrong by a Newton step from an estimate one unit in the last place too high or too low."""
    fractions = torch.arange(1 << 23, dtype=torch.int32)
    _, scale, right = scales(fractions)
    wrong = torch.zeros(1 << 23, dtype=torch.bool)
    for steps in (1, -1):
        y = next_float(right, steps).double()
        rest = (1 - scale.double() * y).float().double()
        wrong |= (rest * y + y).float() != right
    return fractions[wrong]
