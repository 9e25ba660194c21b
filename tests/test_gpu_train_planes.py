"""Every 16-bit plane of every fp32 operand of the training operators counts: products with one-hot operands return the other operand, so
that a plane left out, or one of the products between planes, shows.

Tolerances (derived before any run).  Three bf16 planes hold the 24 bits of a float, and the sum of a value's planes in fp32 is exact,
smallest first: 2^-22 leaves room for a rounding or two.  Two fp16 planes after a power of two hold 22 bits, and 2^-38 of the largest
value that shares the power: 2^-21 with the other operand's, and 2^-37.  A logit that is a class's alone comes back as the row's
log-sum-exp, of a size around one: one rounding each of the product with log2 e, the exponential, the sum, its logarithm, the way back:
2^-20 of one.  The gradients of a loss take the quotient of two such: 2^-19.  Each test also makes sure that its inputs would show a
missing plane: the operand without its last one, split on the host, is past the tolerance."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    assert torch.cuda.is_available()
    from paper_2311_12023_amd import lq
    return torch, lq


def _without_last(torch, v, planes):
    """v from its first planes alone: two of three in bf16, one of two in fp16."""
    if planes == 3:
        high = v.bfloat16().float()
        return high + (v - high).bfloat16().float()
    return v.half().float()


def _same(torch, got, want, planes, largest=1.0, rel=None):
    rel = rel or (2.0 ** -22 if planes == 3 else 2.0 ** -21)
    bound = rel * want.abs().double() + (0.0 if planes == 3 else 2.0 ** -37 * largest)
    assert torch.all((got.double() - want.double()).abs() <= bound), float(((got.double() - want.double()).abs() - bound).max())
    assert torch.any((_without_last(torch, want, planes).double() - want.double()).abs() > 2 * bound)


def _values(torch, *shape, seed=0):
    """Floats between 1/2 and 1 of either sign with all their bits."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    v = 0.5 + 0.5 * torch.rand(*shape, generator=gen, device="cuda", dtype=torch.float64).float()
    return torch.where(torch.rand(*shape, generator=gen, device="cuda") < 0.5, v, -v)


def _one_hot(torch, rows, cols, at):
    out = torch.zeros(rows, cols, device="cuda")
    out[torch.arange(rows, device="cuda"), at] = 1.0
    return out


CFG = (4, 16, 16)


@pytest.fixture(scope="module")
def sizes():
    return 160, 96, 192, 40                    # m, d, k, rank


def _empty(torch, lq, d, k):
    c = lq.config(*CFG)
    return c, lq.nf_quantize(torch.zeros(d * k, device="cuda"), c)


def test_thin_project(env, sizes):
    """T = X L1 (planes of X, of L1)."""
    torch, lq = env
    m, d, k, r = sizes
    c, stored = _empty(torch, lq, d, k)
    l2 = torch.zeros(r, k, device="cuda")
    at = torch.randperm(d, device="cuda")[:r]
    x = _values(torch, m, d)
    _, t = lq.adapter_forward(x, *stored, c, _one_hot(torch, r, d, at).t().contiguous(), l2)
    _same(torch, t, x[:, at], 3)
    rows = torch.arange(m, device="cuda") % d
    l1 = _values(torch, d, r, seed=1)
    _, t = lq.adapter_forward(_one_hot(torch, m, d, rows), *stored, c, l1, l2)
    _same(torch, t, l1[rows], 3)


def test_low_rank_part_of_the_large_product(env, sizes):
    """Y = T L2 and dX = U L1^T without stored weights (planes of T, L2, U, L1)."""
    torch, lq = env
    m, d, k, r = sizes
    c, stored = _empty(torch, lq, d, k)
    rows = torch.arange(m, device="cuda") % d
    hot = _one_hot(torch, m, d, rows)
    l1, at = _values(torch, d, r, seed=2), torch.randperm(k, device="cuda")[:r]
    y, _ = lq.adapter_forward(hot, *stored, c, l1, _one_hot(torch, r, k, at))
    _same(torch, y[:, at], l1[rows], 3)
    cols = torch.arange(d, device="cuda") % r
    l2 = _values(torch, r, k, seed=3)
    y, _ = lq.adapter_forward(hot, *stored, c, _one_hot(torch, d, r, cols), l2)
    _same(torch, y, l2[cols[rows]], 3)
    t = torch.zeros(m, r, device="cuda")
    picks = torch.arange(m, device="cuda") % k
    turned = _one_hot(torch, k, r, torch.arange(k, device="cuda") % r).t().contiguous()
    l1 = _values(torch, d, r, seed=4)
    dx, _, _ = lq.adapter_backward(_one_hot(torch, m, k, picks), torch.zeros(m, d, device="cuda"), *stored, c, l1, turned, t)
    _same(torch, dx, l1.t()[picks % r], 3)
    l2 = _values(torch, r, k, seed=5)
    at = torch.randperm(d, device="cuda")[:r]
    dx, _, _ = lq.adapter_backward(_one_hot(torch, m, k, picks), torch.zeros(m, d, device="cuda"), *stored, c,
                                   _one_hot(torch, r, d, at).t().contiguous(), l2, t)
    _same(torch, dx[:, at], l2.t()[picks], 3)


def test_stored_weights_and_activations(env, sizes):
    """Y = X Q and dX = dY Q^T without a low-rank part (planes of X, dY, Q)."""
    torch, lq = env
    m, d, k, r = sizes
    l1, l2 = torch.zeros(d, r, device="cuda"), torch.zeros(r, k, device="cuda")
    c = lq.config(*CFG)
    stored = lq.nf_quantize(_values(torch, d, k, seed=6).reshape(-1), c)
    q = lq.nf_dequantize(*stored, d * k, c).reshape(d, k)
    rows, picks = torch.arange(m, device="cuda") % d, torch.arange(m, device="cuda") % k
    y, t = lq.adapter_forward(_one_hot(torch, m, d, rows), *stored, c, l1, l2)
    _same(torch, y, q[rows], 2)
    dx, _, _ = lq.adapter_backward(_one_hot(torch, m, k, picks), torch.zeros(m, d, device="cuda"), *stored, c, l1, l2, t)
    _same(torch, dx, q.t()[picks], 2)
    # one stored weight a row: the others of its blocks are codes of zero
    cols = torch.arange(d, device="cuda") % k
    stored = lq.nf_quantize(_one_hot(torch, d, k, cols).reshape(-1), c)
    q = lq.nf_dequantize(*stored, d * k, c).reshape(d, k)
    assert torch.all((q != 0).sum(1) == 1)
    x, dy = _values(torch, m, d, seed=7), _values(torch, m, k, seed=8)
    y, t = lq.adapter_forward(x, *stored, c, l1, l2)
    rel = 2.0 ** -21
    want = (x.double() * q[torch.arange(d, device="cuda"), cols].double()).float()
    _same(torch, y[:, cols], want, 2, rel=rel)
    dx, _, _ = lq.adapter_backward(dy, x, *stored, c, l1, l2, t)
    _same(torch, dx, (dy[:, cols].double() * q[torch.arange(d, device="cuda"), cols].double()).float(), 2, rel=rel)


@pytest.mark.parametrize("m", [40, 1100])        # one range of rows, several
def test_gradients_of_the_factors(env, sizes, m):
    """dL1 = X^T U, dL2 = T^T dY (planes of X, U, T, dY, L2)."""
    torch, lq = env
    _, d, k, r = sizes
    c, stored = _empty(torch, lq, d, k)
    at = torch.randperm(m, device="cuda")[:r]    # row at[j] alone has a one in column j
    hot = _one_hot(torch, r, m, at).t().contiguous()
    x, dy, l1 = _values(torch, m, d, seed=9), _values(torch, m, k, seed=10), torch.zeros(d, r, device="cuda")
    cols = torch.randperm(k, device="cuda")[:r]
    picks = _one_hot(torch, r, k, cols)
    _, dl1, dl2 = lq.adapter_backward(hot @ picks, x, *stored, c, l1, picks, hot)
    _same(torch, dl1.t(), x[at], 3)
    _, _, dl2 = lq.adapter_backward(dy, x, *stored, c, l1, picks, hot)
    _same(torch, dl2, dy[at], 3)
    t = _values(torch, m, r, seed=11)
    rows = torch.randperm(m, device="cuda")[:d]
    chosen = rows[:k][: min(m, d)]
    ones = torch.zeros(m, k, device="cuda")
    ones[chosen, torch.arange(chosen.numel(), device="cuda")] = 1.0
    _, _, dl2 = lq.adapter_backward(ones, x, *stored, c, l1, picks, t)
    _same(torch, dl2[:, :chosen.numel()], t[chosen].t(), 3)
    # U = dY L2^T: columns of dY, rows of L2
    xs = torch.zeros(m, d, device="cuda")
    xs[chosen, torch.arange(chosen.numel(), device="cuda")] = 1.0
    _, dl1, _ = lq.adapter_backward(dy, xs, *stored, c, l1, picks, t)
    _same(torch, dl1[:chosen.numel()], dy[chosen][:, cols], 3)
    l2 = _values(torch, r, k, seed=12)
    _, dl1, _ = lq.adapter_backward(ones, xs, *stored, c, l1, l2, t)
    _same(torch, dl1[:chosen.numel()], l2[:, :chosen.numel()].t(), 3)


# ---------------------------------------------------------------- cross entropy: few rows (three planes), many rows (two)

VOCAB, WIDTH = 64, 128
ROWS = [(100, False, 3), (140, False, 2), (100, True, 2), (140, True, 2)]


def _far(torch, width=WIDTH):
    """Weights of classes that count for nothing: a logit of -100 for rows whose last feature is one."""
    w = torch.zeros(VOCAB, width, device="cuda")
    w[:, -1] = -100.0
    return w


@pytest.mark.parametrize("n,want_dw,planes", ROWS)
def test_logits(env, n, want_dw, planes):
    """The log-sum-exp of a row with one class that counts is that class's logit (planes of X, of W)."""
    torch, lq = env
    none = torch.full((n,), -100, device="cuda")
    x = _values(torch, n, WIDTH, seed=13)
    x[:, -1] = 1.0
    w = _far(torch)
    w[5] = 0
    w[5, 17] = 1.0
    o = lq.cross_entropy(x, w, none, want_dw=want_dw)
    bound = 2.0 ** -20
    assert torch.all((o["lse"].double() - x[:, 17].double()).abs() <= bound)
    assert torch.any((_without_last(torch, x[:, 17], planes) - x[:, 17]).abs() > 2 * bound)
    rows = torch.arange(n, device="cuda") % (WIDTH - 1)
    x = _one_hot(torch, n, WIDTH, rows)
    x[:, -1] = 1.0
    w[5] = _values(torch, WIDTH, seed=14)
    w[5, -1] = 0
    o = lq.cross_entropy(x, w, none, want_dw=want_dw)
    assert torch.all((o["lse"].double() - w[5, rows].double()).abs() <= bound + (0 if planes == 3 else 100 * 2.0 ** -37))
    assert torch.any((_without_last(torch, w[5, rows], planes) - w[5, rows]).abs() > 2 * bound)


@pytest.mark.parametrize("n,want_dw,planes", ROWS)
def test_gradient_of_the_features(env, n, want_dw, planes):
    """dX of a row whose target is improbable: the weights of the one class that counts (planes of W), or the probabilities of two classes
    in features that only one of them has (planes of E)."""
    torch, lq = env
    t = torch.full((n,), 9, device="cuda")
    x = torch.zeros(n, WIDTH, device="cuda")
    x[:, -1] = 1.0
    w = _far(torch)
    w[5] = _values(torch, WIDTH, seed=15)
    w[5, -1] = 1.0
    rel = 2.0 ** -19
    o = lq.cross_entropy(x, w, t, mean=False, want_dw=want_dw)
    want = (w[5] - w[9]).expand(n, WIDTH)[:, :-1]
    assert torch.all((o["dx"][:, :-1].double() - want.double()).abs() <= rel * want.abs().double())
    assert torch.any((_without_last(torch, w[5, :-1], planes) - w[5, :-1]).abs() > 2 * rel * w[5, :-1].abs())
    w[5], w[6] = 0, 0
    w[5, 3], w[6, 4] = 1.0, 1.0
    x[:, 3], x[:, 4] = 2 * _values(torch, n, seed=16), 2 * _values(torch, n, seed=17)
    o = lq.cross_entropy(x, w, t, mean=False, want_dw=want_dw)
    p = torch.softmax(x[:, 3:5].double(), 1)
    assert torch.all((o["dx"][:, 3:5].double() - p).abs() <= rel * p)
    # E is the exponential at a power of two: its bits are those of the probabilities times the row's sum
    e = torch.exp2((x[:, 3].double() * 1.4426950408889634)).float()
    assert torch.any((_without_last(torch, e, planes) - e).abs() > 2 * rel * e)


@pytest.mark.parametrize("n", [100, 140])
def test_gradient_of_the_weights(env, n):
    """dW of a class that one row has (planes of X), and in features that one row has (planes of the probabilities)."""
    torch, lq = env
    rel = 2.0 ** -19
    t = torch.full((n,), -100, device="cuda")
    t[7] = 9
    w = _far(torch)
    w[5] = 0
    x = _values(torch, n, WIDTH, seed=18)
    x[:, -1] = 1.0
    o = lq.cross_entropy(x, w, t, mean=False, want_dw=True)
    assert torch.all((o["dw"][5].double() - x[7].double()).abs() <= rel * x[7].abs().double())
    assert torch.any((_without_last(torch, x[7], 2) - x[7]).abs() > 2 * rel * x[7].abs())
    t = torch.full((n,), 9, device="cuda")
    rows = torch.arange(n, device="cuda")
    width = 256
    w = _far(torch, width)
    w[5], w[6] = 0, 0
    w[5, -2], w[6, -3] = 1.0, 1.0
    x = _one_hot(torch, n, width, rows)
    x[:, -1] = 1.0
    x[:, -2], x[:, -3] = 2 * _values(torch, n, seed=19), 2 * _values(torch, n, seed=20)
    o = lq.cross_entropy(x, w, t, mean=False, want_dw=True)
    p = torch.softmax(x[:, [-2, -3]].double(), 1)
    assert torch.all((o["dw"][5, :n].double() - p[:, 0]).abs() <= rel * p[:, 0])
    assert torch.all((o["dw"][6, :n].double() - p[:, 1]).abs() <= rel * p[:, 1])
    q = p[:, 0].float()
    assert torch.any((_without_last(torch, q, 2) - q).abs() > 2 * rel * q)


# ---------------------------------------------------------------- the generator

KNOWN = (0x5f6fb709, 0x0d893f64, 0x4f121f81, 0x4f730a48)      # Philox4x32 with seven rounds for a counter and a key of zeros


def test_known_answer_of_the_generator(env):
    """The published words for a counter and a key of zeros, 16 bits an element: each decides at its own value and not one past it."""
    torch, lq = env
    bits = [w >> s & 0xffff for w in KNOWN for s in (0, 16)]
    ones = torch.ones(8, device="cuda")
    for e, u in enumerate(bits):
        assert float(lq.dropout(ones, u / 65536, 0, 0)[e]) != 0, e
        assert float(lq.dropout(ones, (u + 1) / 65536, 0, 0)[e]) == 0, e
