"""What the handles of the server's update keep and look at on the host (CPU): streams, the device's state and the launches are
stand-ins that write down what they are asked for; sizes, plans and refusals are the library's own."""
import contextlib
import gc
import weakref

import pytest
import torch

LAUNCHES = ("co3_grad_sumsq", "co3_grad_norm", "co3_step_begin", "co3_adamw", "co3_adamw8", "co3_adamw_clipped", "co3_adamw8_clipped")


class Host:
    """The machine as the handles see it: the current stream, whether it is being captured, what was launched and recorded."""

    def __init__(self, lib):
        self.stream, self.capturing, self.launched, self.recorded, self.lib = 1, False, [], [], lib

    def synchronize(self):
        pass

    def __getattr__(self, name):                         # the library: launches are written down, the host side is its own
        if name in LAUNCHES:
            return lambda *a: self.launched.append(name) or 0
        return getattr(self.lib, name)

    def known_to(self, t):
        return {s for kept, s in self.recorded if kept is t}


@pytest.fixture
def host(monkeypatch):
    from paper_2203_09044_amd import binding, optim
    h = Host(binding._lib)
    monkeypatch.setattr(binding, "_lib", h)
    monkeypatch.setattr(optim, "_raw_stream", lambda index: h.stream)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: h.capturing)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: h)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: None)
    monkeypatch.setattr(torch.cuda, "device", lambda device: contextlib.nullcontext())
    monkeypatch.setattr(torch.Tensor, "is_cuda", property(lambda t: True))
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: h.recorded.append((t, h.stream)))
    return h


def make(kind, sizes=(300, 5), **kw):
    """A handle, and the list of what its launches use beside the plan."""
    from paper_2203_09044_amd import AdamW, GradNorm, MixedAdamW
    if kind == "norm":
        opt = GradNorm([torch.zeros(n) for n in sizes])
        return opt, opt.compute, opt._table.also
    params = [torch.zeros(n) for n in sizes]
    if kind == "mixed":
        params[1] = params[1].half()
        opt = MixedAdamW(params, [torch.zeros_like(p) for p in params], max_norm=1.0, **kw)
        return opt, opt.step, [t for part in opt.parts for t in part._table.also]
    opt = AdamW(params, [torch.zeros_like(p) for p in params], state_bits=8, max_norm=1.0, **kw)
    return opt, opt.step, opt._table.also


def new_gradients(opt):
    tables = [part._table for part in getattr(opt, "parts", [])] or [opt._table]
    places = getattr(opt, "places", [list(range(len(tables[0].grads)))])
    by_place = {k: torch.zeros_like(g) for ks, t in zip(places, tables) for k, g in zip(ks, t.grads)}
    return [by_place[k] for k in sorted(by_place)]


@pytest.mark.parametrize("kind", ["norm", "step", "mixed"])
def test_memory_is_known_to_a_stream_that_makes_a_new_plan(host, kind):
    """The handle's memory belongs to the stream it was made on.  A call on another stream makes it known there, also where that
    call makes a new plan (whose own memory belongs to the stream of that call); else it could be given away under the call."""
    opt, call, memory = make(kind)
    call()
    assert not host.recorded
    for stream in (2, 3):
        host.stream = stream
        call(new_gradients(opt))
        assert all(stream in host.known_to(t) for t in memory)
        call(new_gradients(opt))
        call()
    host.stream = 1                                       # back: the last plan belongs to stream 3
    call()
    tables = [part._table for part in getattr(opt, "parts", [])] or [opt._table]
    assert all(1 in host.known_to(t.plan) for t in tables)


def gone(refs):
    gc.collect()
    return [r() is None for r in refs]


@pytest.mark.parametrize("kind", ["step", "mixed"])
def test_a_captured_step_keeps_the_learning_rate_that_it_reads(host, kind):
    """A graph reads the device float that was the learning rate at its capture, at every replay: the handle keeps it when it gets
    another one.  One that no graph reads is not kept, and is known to the streams that it was used on."""
    opt, call, _ = make(kind, lr=torch.tensor([1e-3]))
    host.capturing = True
    call()
    host.capturing = False
    refs = [weakref.ref(opt.lr)]
    opt.lr = torch.tensor([2e-3])
    refs.append(weakref.ref(opt.lr))
    host.stream = 2
    call()
    assert 2 in host.known_to(opt.lr)
    host.recorded.clear()
    opt.lr = torch.tensor([3e-3])
    call()
    assert 2 in host.known_to(opt.lr)
    host.recorded.clear()
    opt.lr = 1e-3
    call()
    assert not host.recorded and gone(refs) == [False, True]


def test_a_plan_and_a_rate_that_were_captured_are_kept_once(host):
    opt, call, _ = make("step", lr=torch.tensor([1e-3]))
    host.capturing = True
    for _ in range(5):
        call()
    assert len(opt._table._captured) == 1


def two_types():
    """Parameters of two types, 32 bytes each, with their gradients as a handle of two parts."""
    from paper_2203_09044_amd import MixedAdamW
    x, y = torch.nn.Parameter(torch.ones(8)), torch.nn.Parameter(torch.ones(16).half())
    return x, y, MixedAdamW([x, y], [torch.ones(8), torch.ones(16).half()])


def test_a_gradient_on_another_parts_parameter_is_refused(host):
    """A part that is stepped first would change the other's gradient before that is read."""
    x, y, opt = two_types()
    opt.step()
    before, launched = [part._table.grads[0] for part in opt.parts], len(host.launched)
    for bad in ([y.detach().view(torch.float32), torch.ones(16).half()], [torch.ones(8), x.detach().view(torch.float16)],
                [y.detach()[4:12].view(torch.float32).repeat(2), x.detach().view(torch.float16)]):
        for _ in range(2):
            with pytest.raises(ValueError):
                opt.step(bad)
            assert len(host.launched) == launched and all(part._table.grads[0] is g for part, g in zip(opt.parts, before))
    host.capturing = True                                       # what was refused changed nothing: a capture needs no call before it
    opt.step()
    host.capturing = False
    fine = [torch.ones(8), torch.ones(16).half()]
    opt.step(fine)
    assert len(host.launched) == launched + 6 and all(part._table.grads[0] is g for part, g in zip(opt.parts, fine))


def test_a_parameter_moved_onto_another_parts_memory_is_refused(host):
    x, y, opt = two_types()
    opt.step()
    own, launched = x.data, len(host.launched)
    x.data = y.detach().view(torch.float32)
    for _ in range(2):
        with pytest.raises(ValueError):
            opt.step()
    x.data = opt.parts[1]._table.grads[0].view(torch.float32)   # a parameter on another part's gradient
    with pytest.raises(ValueError):
        opt.step()
    assert len(host.launched) == launched
    x.data = own
    opt.step()
    assert len(host.launched) == launched + 3


def one_type(dtype=torch.float32, **kw):
    from paper_2203_09044_amd import AdamW
    p, g = torch.nn.Parameter(torch.ones(6, 6, dtype=dtype)), torch.ones(6, 6, dtype=dtype)
    return p, g, AdamW([p], [g], **kw)


CHANGES = {"shorter": lambda x: x[:3], "transposed": lambda x: x.t(), "strided": lambda x: x[:, ::2], "longer": lambda x: x.as_strided((6, 7), (7, 1)),
           "of a type that has no step": lambda x: x.view(torch.int32)}


@pytest.mark.parametrize("which,change", [(w, c) for w in ("parameter", "gradient") for c in CHANGES if w == "gradient" or "type" not in c])
def test_a_tensor_that_is_another_one_at_the_same_address_is_refused(host, which, change):
    """What the tensor is goes with where it lies: the plan would go on with the elements, their order or their type from before."""
    p, g, opt = one_type()
    room = torch.ones(50)
    p.data, g.data = room[:36].view(6, 6), room.clone()[:36].view(6, 6)
    opt.step()
    x = p if which == "parameter" else g
    was = x.data
    x.data = CHANGES[change](was)
    assert x.data_ptr() == was.data_ptr()
    for _ in range(2):
        with pytest.raises(ValueError):
            opt.step()
    host.capturing = True
    with pytest.raises((RuntimeError, ValueError)):
        opt.step()
    host.capturing = False
    assert host.launched == ["co3_adamw"] and opt.t == 1
    x.data = was
    opt.step()
    assert host.launched == ["co3_adamw"] * 2


def test_a_norms_gradient_that_became_shorter_is_refused(host):
    from paper_2203_09044_amd import GradNorm
    g = torch.ones(10)
    norm = GradNorm([g])
    norm.compute()
    g.data = g.data[:4]
    with pytest.raises(ValueError):
        norm.compute()
    assert host.launched == ["co3_grad_norm"]


def test_a_parameter_of_another_type_at_the_same_address_has_a_plan_of_its_type(host):
    """16-bit types may change: the next step is that of the new one, as where a tensor moves."""
    p, g, opt = one_type(torch.bfloat16)
    opt.step()
    assert (opt._table.layout.param_type, opt._table.layout.grad_type) == (1, 1)
    p.data = p.data.view(torch.float16)
    opt.step()
    assert (opt._table.layout.param_type, opt._table.layout.grad_type) == (2, 1)
    p.data = p.data.view(torch.bfloat16)
    opt.step([g])                                             # with gradients given, too
    assert (opt._table.layout.param_type, opt._table.layout.grad_type) == (1, 1)
    g.data = g.data.view(torch.float16)
    opt.step()
    assert (opt._table.layout.param_type, opt._table.layout.grad_type) == (1, 2)


def test_parameters_that_became_their_own_masters_are_refused(host):
    p, g, opt = one_type(torch.bfloat16, master=True)
    opt.step()
    p.data = p.data.float()
    for grads in (None, [g]):
        with pytest.raises(ValueError):
            opt.step(grads)
    assert host.launched == ["co3_adamw"]


@pytest.mark.parametrize("kind", ["step", "mixed"])
def test_a_learning_rate_that_moved_is_read_where_it_lies(host, kind):
    lr = torch.tensor([1e-3])
    opt, call, _ = make(kind, lr=lr)
    parts = getattr(opt, "parts", [opt])
    host.capturing = True
    call()
    host.capturing = False
    storage = weakref.ref(lr.untyped_storage())
    lr.data = torch.tensor([2e-3])
    call()
    assert all(part._lr_ptr.value == lr.data_ptr() for part in parts) and gone([storage]) == [False]
    for bad in (torch.ones(2), torch.ones(1).half()):
        lr.data = bad
        with pytest.raises(ValueError):
            call()


def contents(opt):
    parts = getattr(opt, "parts", [opt])
    return [x.view(torch.uint8).clone() for part in parts for x in list(part._named().values()) + [part._dev]] + [
        torch.tensor([part._args.seed, part._t]) for part in parts]


@pytest.mark.parametrize("kind", ["step", "mixed"])
@pytest.mark.parametrize("fault", ["array missing", "array short", "array of another type", "no seed", "no count", "count below zero", "no skipped", "no state"])
def test_a_state_that_is_refused_changes_nothing(host, kind, fault):
    """The last array of the last part is the one that does not fit, or a number is missing: nothing of the others is loaded."""
    opt, _, _ = make(kind, seed=3)
    other, _, _ = make(kind, seed=4)
    for part in getattr(other, "parts", [other]):
        for x in part._named().values():
            x.view(torch.uint8).fill_(17)
        part.t = 5
    saved = other.state_dict()
    last = saved["parts"][-1] if kind == "mixed" else saved
    name = list((getattr(other, "parts", [other])[-1])._named())[-1]
    if fault == "array missing":
        del last[name]
    elif fault == "array short":
        last[name] = last[name][1:]
    elif fault == "array of another type":
        last[name] = last[name].float().double()
    elif fault == "count below zero":
        last["t"] = -1
    elif fault == "no state":
        saved = {"parts": saved["parts"][:-1] + [None]} if kind == "mixed" else {}
    else:
        del last[{"no seed": "seed", "no count": "t", "no skipped": "skipped"}[fault]]
    before = contents(opt)
    with pytest.raises(ValueError):
        opt.load_state_dict(saved)
    assert all(torch.equal(a, b) for a, b in zip(before, contents(opt)))
    opt.load_state_dict(other.state_dict())
    assert all(torch.equal(a, b) for a, b in zip(contents(other), contents(opt))) and opt.t == 5


def test_a_state_of_parts_goes_to_parts(host):
    step, _, _ = make("step")
    mixed, _, _ = make("mixed")
    for opt, saved in ((mixed, step.state_dict()), (mixed, {"parts": [step.state_dict()]}), (step, mixed.state_dict())):
        with pytest.raises(ValueError):
            opt.load_state_dict(saved)


def test_masters_of_every_part_are_taken_anew(host):
    """A program loads other weights into a model of several types: the masters follow where it says so, the 32-bit part has none."""
    from paper_2203_09044_amd import MixedAdamW
    params = [torch.zeros(5), torch.zeros(3, 2).half(), torch.zeros(4).bfloat16(), torch.zeros(2).half()]
    opt = MixedAdamW(params, [torch.zeros_like(p) for p in params], master=True)
    for k, p in enumerate(params):
        p.fill_(k + 1.5)
    opt.take_masters()
    by_place = {k: part._views(part.master)[i] for places, part in zip(opt.places, opt.parts) if part.master is not None
                for i, k in enumerate(places)}
    assert sorted(by_place) == [1, 2, 3] and all(torch.equal(x, params[k].float()) for k, x in by_place.items())
    make("mixed")[0].take_masters()                             # without masters there is nothing to take


def test_the_device_does_not_begin_to_count_inside_a_capture(host):
    """The count that the device starts from would be part of the graph, and every replay the same step."""
    _, _, opt = one_type()
    opt.step()
    host.capturing = True
    with pytest.raises(RuntimeError):
        opt.lr = torch.tensor([1e-3])
    host.capturing = False
    assert opt.lr == 1e-3 and not opt._device_steps and opt._lr_ptr is None
    opt.step()
    assert opt.t == 2
    opt.lr = torch.tensor([1e-3])
    host.capturing = True
    opt.lr = torch.tensor([2e-3])                               # the device counts already
    opt.step()
    assert int(opt._dev[0]) == 2
