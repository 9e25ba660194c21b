"""The cross entropy of few rows (up to 128 without dW take kernels of their own): rows with strides, rows that lie far
apart, rows that do not count, certain rows, workspaces, graphs.

Tolerances (derived before any run).  fp32 operands are three bf16 planes, 24 bits, six products per 32 reduction indices, each of which
rounds by at most 2^-23 of the terms: a logit is off by 2^-24 and that of |x||w|, one of bf16 operands (whose products are exact) by one
product per 32 indices; 2^-22 |s| for the conversion to the base of the exponential.  A log-sum-exp and a row loss are off by twice
that and 4e-7, a probability by 1 +- twice that.  E goes into its product with 24 (fp32) or 8 bits (bf16, 2^-8 with room for a
neighbour), over the classes with one rounding per 32 and plane product; results are rounded by 2^-23 or 2^-8."""
import pytest

pytestmark = pytest.mark.gpu

OUT = {"fp32": 2.0 ** -23, "bf16": 2.0 ** -8}
MID = {"fp32": 2.0 ** -22, "bf16": 2.0 ** -8}


@pytest.fixture(scope="module")
def env():
    import torch
    assert torch.cuda.is_available()
    from paper_2311_12023_amd import lq
    return torch, lq


def _type(torch, name):
    return {"fp32": torch.float32, "bf16": torch.bfloat16}[name]


def _eps(dtype, depth):
    return 2.0 ** -24 + (6 if dtype == "fp32" else 1) * (depth // 32 + 2) * 2.0 ** -23


def _check_loss(torch, got, x, w, t, dtype):
    """got: outputs of the mean loss without dW."""
    x, w = x.double(), w.double().contiguous()
    n, vocab = x.shape[0], w.shape[0]
    counts = (t >= 0) & (t < vocab)
    x = torch.where(counts[:, None], x, torch.zeros_like(x))
    s = x @ w.t().contiguous()
    delta = _eps(dtype, x.shape[1]) * (x.abs() @ w.abs().t().contiguous()).max(1).values + 2.0 ** -22 * s.abs().max(1).values
    lse = torch.logsumexp(s, 1)
    rows = torch.nonzero(counts)[:, 0]
    row_loss = torch.zeros_like(lse)
    row_loss[rows] = lse[rows] - s[rows, t[rows]]
    g = torch.exp(s - lse[:, None])
    g[rows, t[rows]] = 0
    g[rows, t[rows]] = -g[rows].sum(1)
    g[~counts] = 0
    f = 1.0 / max(1, rows.numel())
    for name, want in (("row_loss", row_loss), ("lse", lse)):
        gap = (got[name].double() - want).abs()[counts]
        assert torch.all(gap <= 2 * delta[counts] + 4e-7 * (1 + want[counts].abs())), (name, float(gap.max()))
    assert torch.all(got["row_loss"][~counts] == 0)
    total = row_loss.sum() * f
    assert abs(got["loss"].double() - total) <= 2 * f * delta.sum() + 1e-6 * (1 + abs(total))
    if got["dx"] is not None:
        want, terms = g @ w * f, g.abs() @ w.abs() * f
        bound = terms * (6 * delta[:, None] + MID[dtype] + _eps(dtype, vocab)) + OUT[dtype] * want.abs() + 1e-30
        worst = ((got["dx"].double() - want).abs() / bound).max()
        assert worst <= 1, float(worst)


def _inputs(torch, n, d, vocab, dtype, seed, ignored=0.1):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(n, d, generator=gen, device="cuda")
    w = torch.randn(vocab, d, generator=gen, device="cuda") * (2 / d ** 0.5)
    t = torch.randint(0, vocab, (n,), generator=gen, device="cuda")
    t[torch.rand(n, generator=gen, device="cuda") < ignored] = -100
    return x.to(_type(torch, dtype)), w.to(_type(torch, dtype)), t


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n,d,vocab", [(1, 96, 64), (5, 72, 70), (16, 1096, 900), (17, 33, 511), (50, 96, 900), (128, 520, 777)])
def test_rows_with_strides(env, n, d, vocab, dtype):
    """Slices of wider matrices, on and off the 16-byte addresses, bit for bit what contiguous copies give."""
    torch, lq = env
    x, w, t = _inputs(torch, n, d, vocab, dtype, n + d)
    want = lq.cross_entropy(x, w, t)
    _check_loss(torch, want, x, w, t, dtype)
    for pad, at in ((16, 8), (5, 1), (24, 0)):
        wide_x, wide_w = (torch.full((rows, d + pad), float("nan"), device="cuda").to(x.dtype) for rows in (n, vocab))
        wide_x[:, at:at + d], wide_w[:, at:at + d] = x, w
        for a, b in ((wide_x[:, at:at + d], wide_w[:, at:at + d]), (x, wide_w[:, at:at + d]), (wide_x[:, at:at + d], w)):
            o = lq.cross_entropy(a, b, t)
            assert all(torch.equal(o[k], want[k]) for k in o if o[k] is not None), (pad, at)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("gap", [68_174_088, 90_000_001])
def test_rows_of_weights_far_apart(env, gap, dtype):
    """A few columns of a very wide matrix: within a step of 64 classes offsets pass 2^32 elements (rows on and off 16-byte addresses).
    What lies between is not a number."""
    torch, lq = env
    n, d, vocab = 5, 72, 70
    x, w, t = _inputs(torch, n, d, vocab, dtype, gap % 97)
    buffer = torch.empty(vocab * gap, dtype=x.dtype, device="cuda")
    for lo in range(0, buffer.numel(), 1 << 30):
        buffer[lo:lo + (1 << 30)] = float("nan")
    wide = buffer.view(vocab, gap)[:, 8:8 + d]
    wide.copy_(w)
    for want_dw in (False, True):
        far, near = lq.cross_entropy(x, wide, t, want_dw=want_dw), lq.cross_entropy(x, w, t, want_dw=want_dw)
        assert all(torch.equal(far[k], near[k]) for k in near if near[k] is not None)
        if not want_dw:
            _check_loss(torch, far, x, w, t, dtype)


SIZES = [(1, 64, 300), (16, 96, 1000), (17, 33, 511), (50, 72, 1500), (128, 520, 777)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n,d,vocab", SIZES)
def test_rows_that_do_not_count(env, n, d, vocab, dtype):
    """Whatever they hold (NaN, infinities, the type's lowest value), they change nothing else and get zeros; with none left the loss is
    zero."""
    torch, lq = env
    x, w, t = _inputs(torch, n, d, vocab, dtype, n, ignored=0.0)
    t[1::3] = torch.tensor([-1, -100, vocab, 1 << 40, -(1 << 62)] * 10, device="cuda")[:t[1::3].numel()]
    clean = lq.cross_entropy(x, w, t)
    _check_loss(torch, clean, x, w, t, dtype)
    dirty = x.clone()
    dirty[1::9], dirty[4::9], dirty[7::9] = float("nan"), float("inf"), torch.finfo(x.dtype).min
    o = lq.cross_entropy(dirty, w, t)
    assert all(torch.equal(o[k], clean[k]) for k in ("loss", "row_loss", "dx"))
    assert torch.all(o["dx"][1::3] == 0) and torch.all(o["row_loss"][1::3] == 0)
    t[:] = -100
    o = lq.cross_entropy(dirty, w, t)
    assert float(o["loss"]) == 0 and torch.all(o["row_loss"] == 0) and torch.all(o["dx"] == 0)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n,d,vocab", SIZES)
def test_workspace_contents_and_other_outputs(env, n, d, vocab, dtype):
    """Neither what the workspace held before nor whether dX is wanted changes a bit."""
    torch, lq = env
    x, w, t = _inputs(torch, n, d, vocab, dtype, n)
    ws = lq.cross_entropy_workspace(n, d, vocab, x.dtype)
    outs = [lq.cross_entropy(x, w, t, workspace=ws.fill_(fill)) for fill in (0, 0xff, 0x7f)]
    assert all(torch.equal(o[k], outs[0][k]) for o in outs[1:] for k in ("loss", "row_loss", "lse", "dx"))
    ws = lq.cross_entropy_workspace(n, d, vocab, x.dtype, want_dx=False).fill_(0xff)
    o = lq.cross_entropy(x, w, t, want_dx=False, workspace=ws)
    assert o["dx"] is None and all(torch.equal(o[k], outs[0][k]) for k in ("loss", "row_loss", "lse"))
    full, only = (lq.cross_entropy(x, w, t, want_dx=dx, want_dw=True) for dx in (True, False))       # dW: the kernels of many rows
    assert only["dx"] is None and all(torch.equal(only[k], full[k]) for k in ("loss", "row_loss", "lse", "dw"))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n", [8, 24, 128, 140])         # 140: the kernels of many rows
def test_certain_rows(env, n, dtype):
    """Rows that are certain of their target (1 - p down to 1e-26) and of another class: loss and gradient keep their relative accuracy.
    The row loss is log(1 + e^-z), so its relative error is what z is off by, 2 delta, and a few units of fp32."""
    torch, lq = env
    d, vocab = 64, 5000
    x, w, t = _inputs(torch, n, d, vocab, dtype, n, ignored=0.0)
    wt = w[t].float()
    gain = torch.tensor([10.0, 20.0, 30.0, 40.0, 60.0, -30.0, -60.0, 0.0], device="cuda")[torch.arange(n, device="cuda") % 8][:, None]
    x = (x.float() * 0.1 + gain * wt / (wt * wt).sum(1, keepdim=True)).to(x.dtype)
    got = lq.cross_entropy(x, w, t)
    eps = 2.0 ** -20 if dtype == "fp32" and n > 128 else 0.0          # two fp16 planes an operand there
    X, W = x.double(), w.double()
    s = X @ W.t().contiguous()
    delta = (eps + _eps(dtype, d)) * (X.abs() @ W.abs().t().contiguous()).max(1).values + 2.0 ** -22 * s.abs().max(1).values
    rows = torch.arange(n, device="cuda")
    others = torch.exp(s - s[rows, t][:, None])
    others[rows, t] = 0
    total = others.sum(1, keepdim=True)
    want = torch.log1p(total[:, 0])
    assert torch.all((got["row_loss"].double() - want).abs() <= want * (2 * delta + 2e-6) + 1e-37)
    g = others / (1 + total) / n
    terms = g @ W.abs() + g.sum(1, keepdim=True) * W[t].abs()
    want = g @ W - g.sum(1, keepdim=True) * W[t]
    bound = terms * (6 * delta[:, None] + max(MID[dtype], eps) + _eps(dtype, vocab)) + OUT[dtype] * want.abs() + 1e-37
    worst = ((got["dx"].double() - want).abs() / bound).max()
    assert worst <= 1, float(worst)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n", [3, 40])
def test_in_a_hip_graph(env, n, dtype):
    """Replays with new inputs, eager work between them, give the eager results."""
    torch, lq = env
    x, w, t = _inputs(torch, n, 128, 900, dtype, n)
    ws = lq.cross_entropy_workspace(n, 128, 900, x.dtype)
    step = lambda: lq.cross_entropy(x, w, t, workspace=ws)
    step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for i in range(4):
        x.copy_(torch.randn(n, 128, device="cuda"))
        t.copy_(torch.randint(0, 900, (n,), device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        got = {k: v.clone() for k, v in outs.items() if v is not None}
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(got[k], want[k]) for k in got), i
