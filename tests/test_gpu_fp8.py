"""Matrices in 8 bits: the quantizer bit for bit, products and gradients against 64 bits."""
import pytest
import torch

import fp8_reference as R
from paper_2311_12023_amd import lq

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16]


def _matrix(m, d, dtype, seed, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(m, d, generator=g) * torch.exp(spread * torch.randn(m, 1, generator=g))
    return x.to(dtype)


def _same(got, want):
    assert torch.equal(torch.nan_to_num(got.double().cpu(), nan=1e300), torch.nan_to_num(want.double(), nan=1e300))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tiles", [False, True])
@pytest.mark.parametrize("m,d", [(1, 1), (1, 4096), (7, 127), (128, 128), (129, 257), (300, 1000), (1001, 1027), (64, 8)])
def test_codes_and_scales_bit_for_bit(dtype, tiles, m, d):
    x = _matrix(m, d, dtype, m + d)
    q, s, qt, st = lq.fp8_quantize(x.cuda(), tiles=tiles, both=True)
    want, scale = R.quantize(x, tiles)
    _same(q, want)
    _same(s, scale)
    want, scale = R.quantize(x.t().contiguous(), tiles)
    _same(qt, want)
    _same(st, scale)
    alone, alone_s = lq.fp8_quantize(x.cuda(), tiles=tiles)
    assert torch.equal(alone.view(torch.uint8), q.view(torch.uint8)) and torch.equal(alone_s, s)


def test_values_at_borders():
    """Ties, subnormal codes, blocks of zeros, of the smallest and the largest numbers."""
    codes = torch.arange(0, 127, dtype=torch.uint8).view(R.FP8).float()
    mids = (codes[1:] + codes[:-1]) / 2
    near = [torch.nextafter(mids, torch.zeros_like(mids)), mids, torch.nextafter(mids, torch.full_like(mids, 500.0)), codes[1:]]
    x = torch.zeros(12, 128)
    for i, v in enumerate(near):
        x[i, :126], x[i, 126] = v * (-1.0) ** i, 448.0
    x[5] = 1e-45
    x[6] = torch.linspace(-3.4e38, 3.4e38, 128)
    x[7, 3] = 2.0 ** -126
    x[8] = torch.linspace(0, 1e-36, 128)
    x[9, :] = -0.0
    q, s = lq.fp8_quantize(x.cuda())
    want, scale = R.quantize(x)
    _same(q, want)
    _same(s, scale)


@pytest.mark.parametrize("tiles", [False, True])
def test_blocks_that_are_not_finite(tiles):
    x = _matrix(300, 400, torch.float32, 5)
    x[3, 130], x[200, 399], x[299, 0] = float("inf"), float("nan"), float("-inf")
    _, s, _, st = lq.fp8_quantize(x.cuda(), tiles=tiles, both=True)
    _same(s, R.quantize(x, tiles)[1])
    _same(st, R.quantize(x.t().contiguous(), tiles)[1])
    assert torch.isnan(s).sum() == 3
    w, ws = lq.fp8_quantize(_matrix(16, 400, torch.float32, 6).cuda(), tiles=True)
    y = lq.fp8_matmul(*lq.fp8_quantize(x.cuda()), w, ws)
    rows = torch.isnan(y).any(1).nonzero()[:, 0].tolist()
    assert rows == [3, 200, 299] and torch.isnan(y[rows]).all()


def test_strided_rows_and_odd_addresses():
    base = _matrix(70, 523, torch.bfloat16, 9).cuda()
    for view in (base[:, 1:300], base[5:60:2, 8:264], base[:1, 3:200]):
        q, s, qt, st = lq.fp8_quantize(view, both=True)
        for got, want in zip((q, s, qt, st), (*R.quantize(view.cpu()), *R.quantize(view.cpu().t().contiguous()))):
            _same(got, want)


# A product's error: the matrix unit keeps a block's sums to 2^-16 of its largest term (measured 2^-13.6 of the sum of magnitudes at worst
# over 128 terms of full range); fp32 sums over the blocks add 2^-24 each; the result is rounded to bf16,
# half a step of eight significant bits: eps / 2 = 2^-8 of it.
HALF = torch.finfo(torch.bfloat16).eps / 2


def _close(got, a, b):
    want, size = a @ b.t(), a.abs() @ b.abs().t()
    err = (got.double().cpu() - want).abs()
    assert (err <= HALF * want.abs() + (1 + HALF) * 2.0 ** -12 * size + 1e-38).all()


SIZES = [(1, 1, 1), (1, 1000, 4096), (3, 17, 5), (16, 16, 128), (17, 100, 129), (50, 4096, 1024), (37, 768, 768), (129, 257, 300),
         (300, 520, 1111), (1000, 700, 2055), (513, 1025, 640), (3, 8200, 1500), (9, 16500, 700), (60, 8195, 260), (100, 9000, 384),
         (2, 40, 20000), (50, 33, 9999), (129, 130, 5000)]


@pytest.mark.parametrize("a_tiles,b_tiles", [(False, True), (False, False), (True, False), (True, True)])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_product(m, n, k, a_tiles, b_tiles):
    a, a_s = lq.fp8_quantize(_matrix(m, k, torch.float32, 1).cuda(), tiles=a_tiles)
    b, b_s = lq.fp8_quantize(_matrix(n, k, torch.bfloat16, 2).cuda(), tiles=b_tiles)
    y = lq.fp8_matmul(a, a_s, b, b_s)
    assert y.dtype == torch.bfloat16
    _close(y, R.values(a.cpu(), a_s.cpu()), R.values(b.cpu(), b_s.cpu()))
    assert torch.equal(y, lq.fp8_matmul(a, a_s, b, b_s))


@pytest.mark.parametrize("m", [1, 2, 16, 40, 200, 600])
def test_bytes_past_a_row_do_not_count(m):
    """Operands that are parts of larger arrays full of NaN, with scales strided as they come."""
    n, k = 200, 333
    wide = {}
    for name, rows in (("a", m), ("b", n)):
        codes, scale = lq.fp8_quantize(_matrix(rows, k, torch.float32, rows).cuda())
        held = torch.full((rows + 2, 512), 0x7F, dtype=torch.uint8, device="cuda").view(R.FP8)
        held[1:rows + 1, 16:16 + k] = codes
        scales = torch.full((rows, 7), float("nan"), device="cuda")
        scales[:, 1:7:2] = scale
        wide[name] = held[1:rows + 1, 16:16 + k], scales[:, 1:7:2], codes, scale
    a, b = wide["a"], wide["b"]
    held = torch.full((m, n + 9), 7.0, dtype=torch.bfloat16, device="cuda")
    out = lq.fp8_matmul(a[0], a[1], b[0], b[1], out=held[:, 4:4 + n])
    assert torch.equal(out, lq.fp8_matmul(*a[2:], *b[2:]))
    assert (held[:, :4] == 7).all() and (held[:, 4 + n:] == 7).all()
    _close(out, R.values(a[2].cpu(), a[3].cpu()), R.values(b[2].cpu(), b[3].cpu()))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", [(1, 300, 1000), (5, 17, 130), (8, 16400, 900), (4, 9000, 1999), (8, 70, 9000), (2, 33000, 300), (12, 8200, 700), (16, 17000, 1000), (30, 9000, 1024), (64, 500, 130),
                                   (33, 8193, 900), (13, 300, 3000), (16, 8200, 4096), (16, 1024, 512), (37, 768, 768), (130, 515, 259), (700, 900, 1030)])
def test_layer_and_gradients(dtype, m, n, k):
    x, dy = _matrix(m, k, dtype, 3), _matrix(m, n, dtype, 4) * 1e-3
    w, s, wt, ts = lq.fp8_quantize(_matrix(n, k, torch.float32, 5, 0.0).cuda() * 0.02, tiles=True, both=True)
    ws = lq.fp8_workspace(m, n, k)
    y = lq.fp8_forward(x.cuda(), w, s, workspace=ws)
    wv = R.values(w.cpu(), s.cpu())
    _close(y, R.values(*R.quantize(x)), wv)
    assert torch.equal(y, lq.fp8_matmul(*lq.fp8_quantize(x.cuda()), w, s))
    ws = lq.fp8_workspace(m, n, k, backward=True)
    ws.fill_(255)
    dx, dw = lq.fp8_backward(dy.cuda(), x.cuda(), wt, ts, workspace=ws)
    _close(dx, R.values(*R.quantize(dy)), wv.t())
    _close(dw, R.values(*R.quantize(dy.t().contiguous())), R.values(*R.quantize(x.t().contiguous())))
    only, none = lq.fp8_backward(dy.cuda(), None, wt, ts, want_dw=False)
    assert none is None and torch.equal(only, dx)
    none, only = lq.fp8_backward(dy.cuda(), x.cuda(), want_dx=False)
    assert none is None and torch.equal(only, dw)


def test_gradients_against_differences():
    """The layer of values that are e4m3 multiples: nothing is rounded on the way in, so the product is linear and differences are exact
    up to the result's rounding."""
    g = torch.Generator().manual_seed(1)
    m, n, k = 24, 40, 48
    whole = lambda *s: torch.randint(-7, 8, s, generator=g).float()  # noqa: E731
    x, w, dy = whole(m, k), whole(n, k), whole(m, n)
    x[:, 0], w[:, 0], dy[:, 0] = 7.0, 7.0, 7.0                       # every block's scale is 7 / 448 = 2^-6
    x[0], dy[0], w[0] = 7.0, 7.0, 7.0
    wq, ws, wt, wts = lq.fp8_quantize(w.cuda(), tiles=True, both=True)
    f = lambda v: lq.fp8_forward(v.cuda(), wq, ws).double().cpu()  # noqa: E731
    assert torch.equal(f(x), (x @ w.t()).bfloat16().double())
    dx, dw = lq.fp8_backward(dy.cuda(), x.cuda(), wt, wts)
    step = torch.zeros_like(x)
    step[3, 5] = 1.0 if x[3, 5] < 7 else -1.0
    change = ((x + step) @ w.t() - x @ w.t()).double() * dy.double()
    assert abs(change.sum() * step[3, 5] - dx[3, 5].double().cpu()) <= HALF * abs(change.sum())
    assert torch.equal(dx.cpu(), (dy @ w).bfloat16()) and torch.equal(dw.cpu(), (dy.t() @ x).bfloat16())


def test_far_rows():
    """Codes whose offsets pass 2^32 bytes."""
    n, ld = 1100, 1 << 22
    held = torch.empty((n, ld), dtype=torch.uint8, device="cuda").view(R.FP8)
    w, s = lq.fp8_quantize(_matrix(n, 256, torch.float32, 1).cuda(), tiles=True)
    held[:, :256] = w
    for m in (1, 30, 600):
        a = lq.fp8_quantize(_matrix(m, 256, torch.float32, 2).cuda())
        assert torch.equal(lq.fp8_matmul(*a, held[:, :256], s), lq.fp8_matmul(*a, w, s))
        big = torch.empty((m, ld), dtype=torch.uint8, device="cuda").view(R.FP8)
        big[:, :256] = a[0]
        assert torch.equal(lq.fp8_matmul(big[:, :256], a[1], w, s), lq.fp8_matmul(*a, w, s))


def test_graph_and_streams():
    m, n, k = 70, 300, 520
    x, dy = _matrix(m, k, torch.bfloat16, 1).cuda(), _matrix(m, n, torch.bfloat16, 2).cuda()
    w, s, wt, ts = lq.fp8_quantize(_matrix(n, k, torch.float32, 3).cuda(), tiles=True, both=True)
    spaces = lq.fp8_workspace(m, n, k), lq.fp8_workspace(m, n, k, backward=True)

    def both():
        return (lq.fp8_forward(x, w, s, workspace=spaces[0]), *lq.fp8_backward(dy, x, wt, ts, workspace=spaces[1]))

    both()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both()
    for seed in range(4, 7):
        x.copy_(_matrix(m, k, torch.bfloat16, seed))
        dy.copy_(_matrix(m, n, torch.bfloat16, seed + 9))
        graph.replay()
        torch.cuda.synchronize()
        want = both()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = both()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(other, want))


def test_scales_that_are_expanded_and_mixed_types():
    """One scale for a whole matrix is a tensor expanded to the blocks; X and dY of different types."""
    m, n, k = 70, 150, 260
    a = _matrix(m, k, torch.float32, 1, 0.0)
    one = (a.abs().max() / 448).reshape(1, 1).cuda()
    codes = torch.zeros(m, 272, device="cuda").to(R.FP8)[:, :k]
    codes.copy_((a.cuda() / one).to(R.FP8))
    w, s, wt, ts = lq.fp8_quantize(_matrix(n, k, torch.float32, 2).cuda(), tiles=True, both=True)
    for rows in (m, 3):
        y = lq.fp8_matmul(codes[:rows], one.expand(rows, 3), w, s)
        _close(y, R.values(codes[:rows].cpu(), one.expand(rows, 3).cpu()), R.values(w.cpu(), s.cpu()))
    x, dy = _matrix(m, k, torch.float32, 3), _matrix(m, n, torch.bfloat16, 4)
    dx, dw = lq.fp8_backward(dy.cuda(), x.cuda(), wt, ts)
    _close(dx, R.values(*R.quantize(dy)), R.values(wt.cpu(), ts.cpu()))
    _close(dw, R.values(*R.quantize(dy.t().contiguous())), R.values(*R.quantize(x.t().contiguous())))


@pytest.mark.parametrize("m", [1, 12, 300])
@pytest.mark.parametrize("x_size,w_size", [(1e-34, 1.0), (1e-20, 1e-13), (1e25, 1e-25), (3e30, 1e-8)])
def test_sizes_far_from_one(m, x_size, w_size):
    x, w = _matrix(m, 300, torch.float32, 1, 0.0) * x_size, _matrix(270, 300, torch.float32, 2, 0.0) * w_size
    wq, s = lq.fp8_quantize(w.cuda(), tiles=True)
    _close(lq.fp8_forward(x.cuda(), wq, s), R.values(*R.quantize(x)), R.values(wq.cpu(), s.cpu()))


def test_more_values_than_32_bits_count():
    """A matrix of over 2^31 values: its last rows and columns, both ways."""
    m, d = 66000, 33000
    x = torch.zeros((m, d), dtype=torch.bfloat16, device="cuda")
    x[-40:, -300:] = _matrix(40, 300, torch.bfloat16, 1).cuda()
    q, s, qt, st = lq.fp8_quantize(x, both=True)
    corner = torch.zeros(m % 128 + 128, d % 128 + 384)
    corner[-40:, -300:] = x[-40:, -300:].cpu().float()
    rows, cols = corner.shape
    for got, scale, part in ((q, s, corner), (qt, st, corner.t().contiguous())):
        want, want_s = R.quantize(part)
        _same(got[-part.shape[0]:, -part.shape[1]:], want)
        _same(scale[-part.shape[0]:, -want_s.shape[1]:], want_s)


def test_refusals_on_the_gpu():
    w, s = lq.fp8_quantize(torch.ones(64, 100, device="cuda"), tiles=True)
    x = torch.ones(4, 100, device="cuda")
    for call in (lambda: lq.fp8_forward(x[:, :90], w, s), lambda: lq.fp8_forward(x, w, s[:, :0]), lambda: lq.fp8_matmul(w, s, w[:, 1:], s),
                 lambda: lq.fp8_matmul(w, s, w.t(), s), lambda: lq.fp8_backward(x, None), lambda: lq.fp8_backward(x, x, want_dx=False, want_dw=False),
                 lambda: lq.fp8_backward(x, x[:2], want_dx=False), lambda: lq.fp8_matmul(w, s, w, s, out=torch.empty(64, 65, dtype=torch.bfloat16, device="cuda"))):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: lq.fp8_quantize(x.half()), lambda: lq.fp8_quantize(x[0]), lambda: lq.fp8_quantize(x[:1].expand(4, 100)),
                 lambda: lq.fp8_forward(x, w.view(torch.uint8), s), lambda: lq.fp8_forward(x, w, s.half()),
                 lambda: lq.fp8_backward(x, x.half(), want_dx=False), lambda: lq.fp8_forward(x, w, s, workspace=torch.empty(10, device="cuda"))):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(lq.LqError):
        lq.fp8_quantize(x[:0])
