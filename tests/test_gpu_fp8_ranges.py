"""8-bit layers at the ends of what the header allows: many rows, scales of every size, long sums, every fraction of a scale."""
import pytest
import torch

import fp8_fractions as F
import fp8_reference as R
from paper_2311_12023_amd import lq

pytestmark = pytest.mark.gpu

HALF = torch.finfo(torch.bfloat16).eps / 2


def _randn(m, d, seed):
    return torch.randn(m, d, generator=torch.Generator().manual_seed(seed))


def _close(got, a, b):
    """bf16's half step of the result, the matrix unit's 2^-12 of the sum of the terms' magnitudes, and bf16's least numbers."""
    want, size = a @ b.t(), a.abs() @ b.abs().t()
    assert ((got.double().cpu() - want).abs() <= HALF * want.abs() + (1 + HALF) * 2.0 ** -12 * size + 1e-38).all()


def test_gradients_of_more_rows_than_a_sum_may_have():
    """dX of 2^22 and some rows, dW of as many outputs: what neither sums over.  Rows that repeat every 1024 give the result of 1024, which is
    made by the same kernel."""
    many, n, k = (1 << 22) + 3, 48, 32
    w, s, wt, ts = lq.fp8_quantize(_randn(n, k, 1).cuda(), tiles=True, both=True)
    few = _randn(1024, n, 2).bfloat16()
    want, _ = lq.fp8_backward(few.cuda(), None, wt, ts, want_dw=False)
    _close(want, R.values(*R.quantize(few)), R.values(wt.cpu(), ts.cpu()))
    got, _ = lq.fp8_backward(few.cuda().repeat(many // 1024 + 1, 1)[:many], None, wt, ts, want_dw=False)
    assert torch.equal(got[:-3].view(-1, 1024, k), want.expand(many // 1024, -1, -1)) and torch.equal(got[-3:], want[:3])

    x, few = _randn(20, k, 3), _randn(20, 1024, 4).bfloat16()
    _, want = lq.fp8_backward(few.cuda(), x.cuda(), want_dx=False)
    _close(want, R.values(*R.quantize(few.t().contiguous())), R.values(*R.quantize(x.t().contiguous())))
    _, got = lq.fp8_backward(few.cuda().repeat(1, many // 1024 + 1)[:, :many], x.cuda(), want_dx=False)
    assert torch.equal(got[:-3].view(-1, 1024, k), want.expand(many // 1024, -1, -1)) and torch.equal(got[-3:], want[:3])


def test_every_fraction_of_a_scale():
    """amax of all 2^23 fractions, with values that show a reciprocal one unit off: the scale is the rounded quotient by 448 and the codes are
    those of its rounded reciprocal."""
    for first in range(0, 1 << 23, 1 << 20):
        x, scale, reciprocal = F.blocks(torch.arange(first, first + (1 << 20), dtype=torch.int32, device="cuda"))
        q, s = lq.fp8_quantize(x)
        assert torch.equal(s[:, 0], scale) and torch.equal(q.view(torch.uint8), F.codes(x, reciprocal))
