"""Workspaces that the binding of the training operators refuses: memory of the host, other types, pieces with gaps, too little."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    assert torch.cuda.is_available()
    from paper_2311_12023_amd import lq
    return torch, lq


def test_workspaces(env):
    torch, lq = env
    c = lq.config(4, 64, 256)
    stored = lq.nf_quantize(torch.randn(64 * 128, device="cuda"), c)
    x, dy = torch.randn(8, 64, device="cuda"), torch.randn(8, 128, device="cuda")
    l1, l2 = torch.randn(64, 8, device="cuda"), torch.randn(8, 128, device="cuda")
    w, t = torch.randn(100, 64, device="cuda"), torch.zeros(8, dtype=torch.int64, device="cuda")
    _, low = lq.adapter_forward(x, *stored, c, l1, l2)
    calls = [lambda ws: lq.cross_entropy(x, w, t, workspace=ws), lambda ws: lq.adapter_forward(x, *stored, c, l1, l2, workspace=ws),
             lambda ws: lq.adapter_backward(dy, x, *stored, c, l1, l2, low, workspace=ws)]
    size = 1 << 24
    for call in calls:
        call(torch.empty(size, dtype=torch.uint8, device="cuda"))
        call(torch.empty(size, dtype=torch.uint8, device="cuda")[3:])
        for bad in (torch.empty(size, dtype=torch.uint8), torch.empty(size, dtype=torch.float32, device="cuda"),
                    torch.empty(2 * size, dtype=torch.uint8, device="cuda")[::2], size):
            with pytest.raises(TypeError):
                call(bad)
        for few in (0, 1, 300):
            with pytest.raises(lq.LqError):
                call(torch.empty(few, dtype=torch.uint8, device="cuda"))
        with pytest.raises(lq.LqError):
            call(torch.empty(100, dtype=torch.uint8, device="cuda")[3:])         # ends before its first aligned byte


def test_workspaces_of_the_other_calls(env):
    torch, lq = env
    c = lq.config(4, 64, 256)
    a = torch.randn(128, 256, device="cuda")
    calls = [lambda ws: lq.factorize(a, 8, workspace=ws), lambda ws: lq.decompose(a, 8, c, 2, workspace=ws),
             lambda ws: lq.error_table(a, 8, [c], 2, workspace=ws)]
    for call in calls:
        with pytest.raises(lq.LqError):
            call(torch.empty(100, dtype=torch.uint8, device="cuda")[3:])
        with pytest.raises(TypeError):
            call(torch.empty(1 << 24, dtype=torch.uint8))
        call(None)
