"""What AdamW.step hands to the library when its public state (t, buffers) changes between steps.  Needs no GPU: tensors of the CPU
stand for the GPU's, and the call is recorded instead of made."""
import ctypes as C

import pytest
import torch

from paper_2311_12023_amd import lq


@pytest.fixture
def calls(monkeypatch):
    """-> the calls' numbers, addresses and tables, one dict each."""
    made = []

    def dev(t, dtype, name):
        if t is None:
            return None
        if not (isinstance(t, torch.Tensor) and t.device.type == "cpu" and t.dtype == dtype and t.is_contiguous()):
            raise TypeError(name)
        return t.data_ptr()

    def adamw(table, count, bits, params, coef, stream):
        h = params._obj
        entries = (lq.AdamWTensor * count).from_address(table)
        made.append(dict(step=h.step, step_device=h.step_device, lr_device=h.lr_device,
                         table=[{n: getattr(e, n) for n, _ in lq.AdamWTensor._fields_} for e in entries]))
        return 0

    monkeypatch.setattr(lq, "_dev", dev)
    monkeypatch.setattr(lq, "_stream", lambda: None)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: -1)                  # a CPU tensor's get_device()
    monkeypatch.setattr(torch._C, "_cuda_isCurrentStreamCapturing", lambda: False)
    monkeypatch.setattr(lq._lib, "lq_adamw", adamw)
    return made


def _made(bits=32, sizes=(300, 5), **more):
    params = [torch.zeros(n) for n in sizes]
    return lq.AdamW(params, bits=bits, **more), [torch.ones(n) for n in sizes]


def test_a_number_in_place_of_a_device_number(calls):
    """t as a checkpoint's number after steps that were counted on the device: the number counts, the tensor is not read any more."""
    opt, grads = _made(device_step=True)
    opt.step(grads, 0.1)
    assert calls[-1]["step_device"] == opt.t.data_ptr() and opt.t.item() == 1
    opt.t = 40
    opt.step(grads, 0.1)
    assert calls[-1]["step_device"] is None and calls[-1]["step"] == 41 and opt.t == 41
    opt.t = torch.tensor(6)
    opt.step(grads, 0.1)
    assert calls[-1]["step_device"] == opt.t.data_ptr() and opt.t.item() == 7


@pytest.mark.parametrize("t,error", [(torch.zeros((), dtype=torch.int32), TypeError), (torch.zeros(()), TypeError),
                                     (torch.zeros((), dtype=torch.int64, device="meta"), TypeError), (torch.zeros(2, dtype=torch.int64), ValueError),
                                     (torch.zeros(0, dtype=torch.int64), ValueError), (1.5, TypeError), (None, TypeError)])
def test_a_step_number_that_cannot_be_read(calls, t, error):
    """Of another type, in other memory (here: not the CPU's), of no or several elements: refused before anything is called or counted."""
    opt, grads = _made()
    opt.t = t
    with pytest.raises(error):
        opt.step(grads, 0.1)
    assert not calls and opt.t is t and (not isinstance(t, torch.Tensor) or t.is_meta or not t.any())


def _expected(opt, buffers):
    """The states' addresses of every tensor: its blocks of 256 behind those of the tensors before it."""
    at, want = 0, []
    for p in opt.params:
        want.append({name: b.data_ptr() + (at // 256 * 4 if name.endswith("scale") else at * b.element_size()) for name, b in buffers.items()})
        at += -(-p.numel() // 256) * 256
    return want


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("sizes", [(300, 5), (7,) * 20 + (0, 513)])
def test_states_that_are_replaced(calls, bits, sizes):
    """A checkpoint's tensors in place of the states, one by one or all at once: the step goes on in them."""
    opt, grads = _made(bits, sizes)
    opt.step(grads, 0.1)
    first = opt.buffers
    changed = [dict(first), {k: b.clone() for k, b in first.items()}]
    changed[0]["m"] = first["m"].clone()
    for buffers in (first, *changed, first):
        opt.buffers = buffers
        opt.step(grads, 0.1)
        for have, want in zip(calls[-1]["table"], _expected(opt, buffers)):
            assert all(have[name] == place for name, place in want.items())
    opt.buffers["v"] = first["v"].clone()
    opt.step(grads, 0.1)
    for have, want in zip(calls[-1]["table"], _expected(opt, opt.buffers)):
        assert all(have[name] == place for name, place in want.items())


@pytest.mark.parametrize("change,error", [
    (dict(m=None), TypeError), (dict(v=torch.zeros(1024)), ValueError), (dict(m=torch.zeros(767)), ValueError), (dict(m=torch.zeros(768).half()), TypeError),
    (dict(v=torch.zeros(768, device="meta")), TypeError), (dict(v=torch.zeros(1536)[::2]), TypeError), (dict(m=[0.0] * 768), TypeError)])
def test_states_that_do_not_fit(calls, change, error):
    opt, grads = _made()                                       # 300 and 5 values: three blocks of 256
    opt.buffers.update(change)
    with pytest.raises(error):
        opt.step(grads, 0.1)
    assert not calls and opt.t == 0


def test_old_states_after_new_ones_were_refused(calls):
    """One of two that were replaced does not fit: the step is refused, and the old ones put back are used again."""
    opt, grads = _made()
    opt.step(grads, 0.1)
    first = opt.buffers
    opt.buffers = dict(m=first["m"].clone(), v=torch.zeros(5))
    with pytest.raises(ValueError):
        opt.step(grads, 0.1)
    opt.buffers = first
    opt.step(grads, 0.1)
    for have, want in zip(calls[-1]["table"], _expected(opt, first)):
        assert all(have[name] == place for name, place in want.items())


@pytest.mark.parametrize("change", [dict(m_scale=torch.zeros(2)), dict(v_scale=torch.zeros(4))])
def test_scales_that_do_not_fit(calls, change):
    opt, grads = _made(8, device_step=True)
    opt.buffers.update(change)
    with pytest.raises(ValueError):
        opt.step(grads, 0.1)
    del opt.buffers["m"]
    with pytest.raises(TypeError):
        opt.step(grads, 0.1)
    assert not calls and opt.t.item() == 0


def test_everything_that_a_step_writes_gets_a_new_version(calls):
    """Parameters and copies, whether they require gradients or not: a graph that has saved their old values fails instead of using the new."""
    params = [torch.zeros(4, 3), torch.nn.Parameter(torch.zeros(2)), torch.zeros(5)]
    copies = [torch.zeros(4, 3, dtype=torch.bfloat16), None, None]
    with torch.inference_mode():
        params.append(torch.zeros(2))
    opt = lq.AdamW(params, copies=copies + [None])
    written = [*params[:3], copies[0]]
    before = [x._version for x in written]
    x = torch.ones(2, 3, dtype=torch.bfloat16, requires_grad=True)
    y = x @ copies[0].t()
    opt.step([torch.ones(p.shape) for p in params], 0.1)
    assert all(x._version > old for x, old in zip(written, before))
    with pytest.raises(RuntimeError):
        y.sum().backward()


def test_old_parameters_after_moved_ones_were_refused(calls):
    """One that moved is taken up, the next does not fit: the step is refused, and the old ones put back are used again."""
    opt, grads = _made()
    opt.step(grads, 0.1)
    old = [p.data for p in opt.params]
    opt.params[0].data = old[0].clone()
    opt.params[1].data = torch.zeros(10)[::2]
    with pytest.raises(TypeError):
        opt.step(grads, 0.1)
    for p, data in zip(opt.params, old):
        p.data = data
    opt.step(grads, 0.1)
    assert [entry["p"] for entry in calls[-1]["table"]] == [p.data_ptr() for p in old]


def test_states_that_were_replaced_are_let_go(calls):
    """States moved elsewhere between steps, to free their memory: the optimizer does not hold on to them."""
    import weakref
    opt, grads = _made(8)
    opt.step(grads, 0.1)
    away = {name: b.clone() for name, b in opt.buffers.items()}
    refs = [weakref.ref(b) for b in opt.buffers.values()]
    opt.buffers = {}
    assert all(ref() is None for ref in refs)
    opt.buffers = away
    opt.step(grads, 0.1)
    for have, want in zip(calls[-1]["table"], _expected(opt, away)):
        assert all(have[name] == place for name, place in want.items())
