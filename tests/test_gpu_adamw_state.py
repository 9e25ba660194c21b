"""AdamW's public state on the GPU: restored by replacing it, step numbers on the host and on the device, and graphs that have saved what a
step writes."""
import pytest
import torch

from paper_2311_12023_amd import lq

pytestmark = pytest.mark.gpu

SIZES = (3000, 77, 256)


def _values(seed, dtype=torch.float32):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(n, generator=g).to(dtype).cuda() for n in SIZES]


def _bytes(tensors):
    return [t.detach().contiguous().view(torch.uint8) for t in tensors]


def _same(a, b):
    return all(torch.equal(x, y) for x, y in zip(_bytes(a), _bytes(b)))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("device_step", [False, True])
def test_a_checkpoint_replaces_the_state(bits, device_step):
    """Two steps, then two more: by the same object, and by another whose buffers and t are the first's by assignment.  The other's own first
    buffers stay as they were."""
    params = _values(1)
    opt = lq.AdamW(params, bits=bits, seed=8, device_step=device_step)
    for t in range(2):
        opt.step(_values(10 + t), 0.01)
    again = [p.clone() for p in params]
    other = lq.AdamW(again, bits=bits, seed=8, device_step=device_step)
    other.step(_values(50), 0.0, weight_decay=0.0)               # steps of rate 0 leave the parameters
    own, kept = other.buffers, [b.clone() for b in other.buffers.values()]
    other.buffers = {name: b.clone() for name, b in opt.buffers.items()}
    other.t = opt.t.clone() if device_step else opt.t
    for t in range(2, 4):
        opt.step(_values(10 + t), 0.01)
        other.step(_values(10 + t), 0.01)
    assert _same(params, again) and _same(opt.buffers.values(), other.buffers.values()) and _same(own.values(), kept)
    assert int(opt.t) == int(other.t) == 4


@pytest.mark.parametrize("bits", [32, 8])
def test_numbers_of_both_kinds_in_turn(bits):
    """t as a tensor, as a number and as another tensor: every step is that of the number it is given."""
    params, again = _values(1), _values(1)
    opt, ref = (lq.AdamW(p, bits=bits, seed=3) for p in (params, again))
    for t, given in ((5, torch.tensor(5).cuda()), (9, 9), (2, torch.tensor([2]).cuda()), (30, 30)):
        opt.t, ref.t = given, t
        opt.step(_values(20 + t), 0.01)
        ref.step(_values(20 + t), 0.01)
        assert int(opt.t) == t + 1
    # the factors of step and rate come from the device's fp64 powers there and from the host's here: a unit in the last place of each
    for p, q in zip(params, again):
        assert (p - q).abs().max() <= 4 * (2.0 ** -22 * 0.1 + 2.0 ** -23 * q.abs().max())


def test_states_and_numbers_that_are_refused():
    p, g = _values(1), _values(2)
    opt = lq.AdamW(p, device_step=True)
    before = [x.clone() for x in p]
    good_t, good = opt.t, dict(opt.buffers)
    for t, error in ((torch.zeros((), dtype=torch.int64), TypeError), (good_t.int(), TypeError), (good_t.float(), TypeError),
                     (torch.zeros(2, dtype=torch.int64, device="cuda"), ValueError)):
        opt.t = t
        with pytest.raises(error):
            opt.step(g, 0.1)
    opt.t = good_t
    for m, error in ((good["m"].cpu(), TypeError), (good["m"].bfloat16(), TypeError), (good["m"][:-1], ValueError), (None, TypeError),
                     (good["v"], lq.LqError)):
        opt.buffers["m"] = m
        with pytest.raises(error):
            opt.step(g, 0.1)
    assert _same(p, before) and good_t.item() == 0
    opt.buffers["m"] = good["m"]
    opt.step(g, 0.1)
    assert good_t.item() == 1 and not _same(p, before)


@pytest.mark.parametrize("kind", ["copy", "plain bf16", "plain fp32", "parameter"])
def test_a_graph_that_has_saved_what_a_step_writes_fails(kind):
    """Activations that require a gradient times a weight that does not: the product's graph holds the weight."""
    g = torch.Generator().manual_seed(1)
    w = torch.randn(6, 16, generator=g).to(torch.bfloat16 if kind == "plain bf16" else torch.float32).cuda()
    w = torch.nn.Parameter(w) if kind == "parameter" else w
    held = w.bfloat16() if kind == "copy" else None
    used = held if kind == "copy" else w
    opt = lq.AdamW([w], copies=[held])
    x = torch.randn(3, 16, generator=g).to(used.dtype).cuda().requires_grad_()
    grad = torch.ones_like(w)
    (x @ used.t()).sum().backward()                              # nothing was written yet
    y = (x @ used.t()).sum()
    opt.step([grad], 0.1)
    with pytest.raises(RuntimeError):
        y.backward()
    (x @ used.t()).sum().backward()                              # one made after the step does not


@pytest.mark.parametrize("bits", [32, 8])
def test_addresses_on_16_bytes(bits):
    """Tensors and states on addresses that are multiples of 16 and not of 32 give what others give."""
    def at(start, values):
        held = torch.empty(values.numel() + 64, dtype=values.dtype, device="cuda")
        while (held[start:].data_ptr() // 16) % 2 != 1 or held[start:].data_ptr() % 16:
            start += 1
        held[start:start + values.numel()] = values
        return held[start:start + values.numel()]

    params, grads = _values(1), _values(2)
    moved, moved_grads = [at(1, p) for p in params], [at(1, g) for g in grads]
    opt, other = lq.AdamW(params, bits=bits, seed=5), lq.AdamW(moved, bits=bits, seed=5)
    if bits == 32:
        other.buffers = {name: at(1, b) for name, b in other.buffers.items()}
    for _ in range(2):
        norm, again = lq.grad_norm(grads, 1.0), lq.grad_norm(moved_grads, 1.0)
        assert torch.equal(norm[0], again[0])
        opt.step(grads, 0.01, coef=norm[1])
        other.step(moved_grads, 0.01, coef=again[1])
    assert _same(params, moved) and _same(opt.buffers.values(), other.buffers.values())
