"""The adapter product for activations and weights of extreme magnitudes: rows of dY and X from 1e-25 to 1e-37 beside ordinary ones (the
gradient of a token that is certain of its target is such a row), stored weights from 1e-30 to 1e30.

Tolerances (derived before any run).  fp32, large product: two fp16 planes hold 22 bits and lo times lo is left out, together 2^-21 of
|a||b|; its sum takes three products per 32 reduction indices and the low-rank part's six, each of which rounds by at most 2^-23 of
the terms.  Thin products: three bf16 planes hold 24 bits, 2^-24 with what is left out, and six products per 32 indices.  bf16: weights
and results are rounded by 2^-9 (2^-8 with room for a neighbour).  An operand below 2^-126 in a plane may be lost: 2^-126 of whatever it
meets, and so may the part of a sum below that in each product.  Weights are multiplied by at most 2^80, and fp16 ends at 2^-25: 2^-104 of an activation with some room."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    assert torch.cuda.is_available()
    from paper_2311_12023_amd import lq
    return torch, lq


TINY, SMALLEST = 2.0 ** -125, 2.0 ** -104


def _inputs(torch, lq, m, d, k, cfg, rank, dtype, seed, weights=1.0, adapter=True):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    kind = {"fp32": torch.float32, "bf16": torch.bfloat16}[dtype]
    c = lq.config(*cfg)
    codes, index, v = lq.nf_quantize((normal(d, k) * 0.05).reshape(-1), c)
    powers = torch.tensor([0, -25, 0, -28, -30, -31, 0, -33, -36, -37], device="cuda")[torch.arange(m, device="cuda") % 10]
    rows = (10.0 ** powers.double())[:, None].float()
    x, dy = (normal(m, d) * rows).to(kind), (normal(m, k) * rows).to(kind)
    x[m // 2] = 0
    dy[m // 2] = 0
    l1, l2 = normal(d, rank) * 0.1, normal(rank, k) * (0.1 if adapter else 0.0)
    return c, (codes, index, v * weights), x, dy, l1, l2


def _check(torch, lq, dtype, p, inputs, m, d, k, rank):
    c, stored, x, dy, l1, l2 = inputs
    y, t = lq.adapter_forward(x, *stored, c, l1, l2, p, 5, 1)
    dx, dl1, dl2 = lq.adapter_backward(dy, x, *stored, c, l1, l2, t, p, 5, 1)
    q = lq.nf_dequantize(*stored, d * k, c).double().reshape(d, k)
    mask = (lq.dropout(torch.ones(m, d, device="cuda"), p, 5, 1)).double()
    X, DY, L1, L2, T = x.double(), dy.double(), l1.double(), l2.double(), t.double()
    xd, A = X * mask, torch.abs
    turned = lambda a: a.t().contiguous()
    fp32 = dtype == "fp32"
    rounds = lambda depth: 6 * (depth // 32 + 2) * 2.0 ** -23
    thin = lambda depth: 2.0 ** -24 + rounds(depth)
    main = lambda depth: 2.0 ** -21 + rounds(depth) + rounds(rank) if fp32 else 2.0 ** -8
    result = 2.0 ** -23 if fp32 else 2.0 ** -8
    flush = lambda depth: 6 * (depth // 32 + 2) * TINY

    def close(name, got, want, scale, eps, rounded, floor):
        assert got.shape == want.shape and torch.isfinite(got).all(), name
        worst = (A(got.double() - want) / (eps * scale + rounded * A(want) + floor)).max()
        assert worst <= 1, (name, float(worst))

    lost = lambda a: A(a).sum(0, keepdim=True) * TINY
    close("T", t, xd @ L1, A(xd) @ A(L1), thin(d), 2.0 ** -23, 2 * lost(L1) + flush(d))
    close("Y", y, X @ q + T @ L2, A(X) @ A(q) + A(T) @ A(L2), main(d), result, 2 * lost(L2) + SMALLEST * A(X).sum(1, keepdim=True) + flush(d + rank))
    u, au = DY @ turned(L2), A(DY) @ turned(A(L2))
    u_lost = lost(turned(L2)) + flush(k)
    close("dX", dx, DY @ turned(q) + mask * (u @ turned(L1)), A(DY) @ turned(A(q)) + mask * (au @ turned(A(L1))), main(d) + main(k), result,
          2 * mask * (u_lost @ turned(A(L1)) + lost(turned(L1))) + SMALLEST * A(DY).sum(1, keepdim=True) + flush(k + rank))
    close("dL1", dl1, turned(xd) @ u, turned(A(xd)) @ au, thin(m) + thin(k), 2.0 ** -23,
          turned(A(xd)).sum(1, keepdim=True) * 2 * u_lost + TINY * au.sum(0, keepdim=True) + flush(m))
    close("dL2", dl2, turned(T) @ DY, turned(A(T)) @ A(DY), thin(m), 2.0 ** -23,
          TINY * (A(T).sum(0)[:, None] + A(DY).sum(0, keepdim=True)) + flush(m))


SHAPES = [
    (37, 96, 128, (4, 64, 256), 8),          # one tile in stretches
    (300, 2080, 1024, (4, 64, 64), 20),      # eight and sixteen tiles in stretches
    (2000, 4096, 1024, (3, 64, 64), 64),     # backwards a workgroup a tile
    (2000, 1024, 4096, (3, 64, 64), 64),     # forwards
]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("p", [0.0, 0.3])
@pytest.mark.parametrize("m,d,k,cfg,rank", SHAPES)
def test_rows_of_tiny_magnitude(env, m, d, k, cfg, rank, p, dtype):
    torch, lq = env
    for adapter in (True, False):
        _check(torch, lq, dtype, p, _inputs(torch, lq, m, d, k, cfg, rank, dtype, m + d, adapter=adapter), m, d, k, rank)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("p", [0.0, 0.3])
@pytest.mark.parametrize("weights", [1e-30, 1e-22, 1e-10, 1e10, 1e30])
def test_weights_of_extreme_magnitude(env, weights, p, dtype):
    torch, lq = env
    m, d, k, cfg, rank = SHAPES[1]
    _check(torch, lq, dtype, p, _inputs(torch, lq, m, d, k, cfg, rank, dtype, 7, weights=weights), m, d, k, rank)
