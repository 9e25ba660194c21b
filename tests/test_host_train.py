"""What the training operators refuse, and the sizes of their workspaces.  Needs no GPU: nothing gets past the checks."""
import ctypes as C

import pytest
import torch

from paper_2311_12023_amd import lq

L = lq._lib
P = 4096                                     # never dereferenced: the calls end before a launch
BIG = 1 << 60


def _dropout(x=P, n=64, dtype=0, p=0.5, y=P):
    return L.lq_dropout(x, n, dtype, p, 1, 0, y, None)


@pytest.mark.parametrize("change,status", [
    (dict(x=None), -1), (dict(y=None), -1), (dict(n=0), -2), (dict(n=-1), -2), (dict(n=1 << 60), -2), (dict(dtype=2), -8),
    (dict(dtype=-1), -8), (dict(p=-1e-9), -8), (dict(p=1.0000001), -8), (dict(p=float("nan")), -8), (dict(x=P + 2), -8),
    (dict(y=P + 1, dtype=1), -8)])
def test_dropout_refusals(change, status):
    assert _dropout(**change) == status


def _loss(X=P, ldx=64, W=P, ldw=64, t=P, n=10, d=64, vocab=100, dtype=0, mean=1, loss=P, row=P, lse=P, dX=P, dW=P, ws=P, size=BIG):
    return L.lq_cross_entropy(X, ldx, W, ldw, t, n, d, vocab, dtype, mean, loss, row, lse, dX, dW, ws, size, None)


@pytest.mark.parametrize("change,status", [
    (dict(X=None), -1), (dict(W=None), -1), (dict(t=None), -1), (dict(loss=None), -1), (dict(row=None), -1), (dict(n=0), -2),
    (dict(d=0), -2), (dict(vocab=0), -2), (dict(n=1 << 31), -2), (dict(vocab=1 << 31), -2), (dict(d=1 << 21, ldx=1 << 21, ldw=1 << 21), -2),
    (dict(ldx=63), -2), (dict(ldw=63), -2), (dict(dtype=2), -8), (dict(mean=2), -8), (dict(X=P + 2), -8), (dict(t=P + 4), -8),
    (dict(dX=P + 1, dtype=1), -8), (dict(ws=None), -6), (dict(ws=P + 128), -6), (dict(size=1000), -6)])
def test_cross_entropy_refusals(change, status):
    assert _loss(**change) == status


CFG = (4, 64, 256)


def _adapter(backward, X=P, m=8, d=64, k=128, codes=P, s=P, v=P, cfg=CFG, L1=P, L2=P, rank=8, dtype=0, p=0.1, out=P, t=P, g1=P, g2=P,
             ws=P, size=BIG):
    c = lq.config(*cfg)
    if backward:
        return L.lq_adapter_backward(P, X, m, d, k, codes, s, v, c, L1, L2, rank, dtype, t, p, 1, 0, out, g1, g2, ws, size, None)
    return L.lq_adapter_forward(X, m, d, k, codes, s, v, c, L1, L2, rank, dtype, p, 1, 0, out, t, ws, size, None)


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("change,status", [
    (dict(X=None), -1), (dict(codes=None), -1), (dict(s=None), -1), (dict(v=None), -1), (dict(L1=None), -1), (dict(L2=None), -1),
    (dict(t=None), -1), (dict(rank=0), -4), (dict(rank=129), -4), (dict(m=0), -2), (dict(d=48), -2), (dict(k=96), -2), (dict(k=0), -2),
    (dict(m=1 << 31), -2), (dict(m=1 << 26), -2), (dict(d=1 << 20, k=1 << 12), -2), (dict(cfg=(5, 64, 256)), -3),
    (dict(cfg=(4, 48, 256)), -3), (dict(dtype=2), -8), (dict(p=-0.1), -8), (dict(p=float("nan")), -8), (dict(X=P + 8), -8),
    (dict(out=P + 4), -8), (dict(ws=None), -6), (dict(ws=P + 16), -6), (dict(size=100), -6)])
def test_adapter_refusals(backward, change, status):
    assert _adapter(backward, **change) == status


def test_adapter_backward_needs_its_outputs():
    assert _adapter(True, g1=None) == -1 and _adapter(True, g2=None) == -1


def test_workspace_sizes():
    assert L.lq_cross_entropy_workspace_bytes(0, 64, 100, 0, 1, 1) == 0 and L.lq_cross_entropy_workspace_bytes(4, 64, 100, 3, 1, 1) == 0
    assert L.lq_adapter_workspace_bytes(8, 48, 64, 8, 0, 0) == 0 and L.lq_adapter_workspace_bytes(8, 64, 64, 129, 0, 1) == 0
    sizes = [L.lq_cross_entropy_workspace_bytes(4096, 4096, 128000, 1, a, b) for a, b in ((0, 0), (1, 0), (1, 1))]
    assert 0 < sizes[0] < sizes[1] < sizes[2]
    logits = 4096 * 128000 * 2
    assert sizes[1] < logits                     # no array of all logits hides in it
    # for the largest call one byte less is refused, at odd sizes too
    for n, d, vocab, dtype in ((1, 1, 1, 0), (777, 1000, 50265, 1), (4096, 4096, 128000, 1)):
        need = L.lq_cross_entropy_workspace_bytes(n, d, vocab, dtype, 1, 1)
        assert _loss(n=n, d=d, ldx=d, ldw=d, vocab=vocab, dtype=dtype, size=need - 1) == -6


def test_binding_checks_tensors():
    x = torch.zeros(4, 64)
    with pytest.raises(TypeError):
        lq.dropout(x, 0.5, 1)                    # not on the GPU
    with pytest.raises(TypeError):
        lq.dropout(x.double(), 0.5, 1)
    with pytest.raises(TypeError):
        lq.cross_entropy(x, torch.zeros(10, 64), torch.zeros(4, dtype=torch.int64))
    with pytest.raises(TypeError):
        lq.cross_entropy(x.half(), torch.zeros(10, 64).half(), torch.zeros(4, dtype=torch.int64))
    with pytest.raises(ValueError):
        lq.adapter_forward(x, *(torch.zeros(1, dtype=torch.uint8),) * 2, torch.zeros(1), lq.config(*CFG), torch.zeros(64, 8),
                           torch.zeros(8, 128))   # buffers too small for 64 x 128 weights
