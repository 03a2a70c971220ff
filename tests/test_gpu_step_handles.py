"""The handles of the server's update on the GPU: memory that another stream still uses, what a captured step goes on reading,
tensors that are no longer what a plan is for, several tables under one workspace, checkpoints of parts."""
import math

import numpy as np
import pytest

from oracle import step as O

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
U = 2.0 ** -24                                      # a float32 rounding, relative


@pytest.fixture(scope="module")
def co3():
    import paper_2203_09044_amd as pkg
    return pkg


def occupied(stream, gigabytes=8):
    """Work that a stream has before it: some milliseconds."""
    x = torch.zeros(1 << 28, device="cuda")
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        for _ in range(gigabytes):
            x.add_(1.0)
    x.record_stream(stream)


@pytest.mark.parametrize("kind", ["32", "8", "mixed"])
def test_a_handle_dropped_behind_a_step_with_a_new_plan_on_another_stream(co3, kind):
    """The first call on another stream brings gradients of its own and the handle is dropped while the call waits there: what
    is allocated then on the first stream is not the handle's memory."""
    def make():
        torch.manual_seed(31)
        params = [torch.randn(1_000_003, device="cuda"), torch.randn(77, device="cuda")]
        if kind == "mixed":
            params[1] = params[1].to(BF16)
        grads = [torch.randn_like(p) for p in params]
        if kind == "mixed":
            return params, grads, co3.MixedAdamW(params, [torch.zeros_like(p) for p in params], max_norm=1.0, state_bits=8, lr=0.1)
        return params, grads, co3.AdamW(params, [torch.zeros_like(p) for p in params], state_bits=int(kind), max_norm=1.0, lr=0.1)
    want, grads, opt = make()
    opt.step(grads)
    opt.step()
    torch.cuda.synchronize()
    del opt
    got, grads, opt = make()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    occupied(side)
    with torch.cuda.stream(side):
        opt.step(grads)
        opt.step()
    del opt
    junk = [torch.full((n,), math.nan, device="cuda") for n in (1_000_080, 2_000_000, 250_020, 7_816, 64, 16) for _ in range(8)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got)) and junk


def test_replays_read_the_learning_rate_of_their_capture(co3):
    p, g = torch.randn(5000, device="cuda"), torch.randn(5000, device="cuda")
    want = p.clone()
    opt = co3.AdamW([p], [g], lr=torch.tensor([1e-2], device="cuda"), max_norm=1.0)
    ref = co3.AdamW([want], [g], lr=torch.tensor([1e-2], device="cuda"), max_norm=1.0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        opt.step()
    for t in range(3):
        opt.lr = torch.tensor([1e-3 * (t + 1)], device="cuda") if t < 2 else 5e-3     # the captured one has no other owner
        junk = [torch.full((1,), math.nan, device="cuda") for _ in range(256)]
        graph.replay()
        ref.lr = torch.tensor([1e-2], device="cuda")
        ref.step()
        opt.step()
        ref.lr = opt.lr
        ref.step()
        torch.cuda.synchronize()
        assert torch.equal(p, want) and opt.t == ref.t == 2 * t + 2 and junk


def norms(co3, sizes, dtype=F32):
    """Tables for the C calls: gradients, layout, plan and the norm in float64 of every one."""
    out = []
    for k, n in enumerate(sizes):
        g = torch.from_numpy(np.random.default_rng(k).standard_normal(n).astype(np.float32) * (k + 1)).cuda().to(dtype)
        t = co3.GradNorm([g])._table
        out.append((g, t.layout, t.plan, O.norm([g.double().cpu().numpy()])[0]))
    return out


def test_tables_of_different_sizes_take_turns_on_one_workspace(co3):
    """A workspace zeroed once serves one table after another, with as many partial sums as each of them has, whole norms and
    sums that a step is begun with."""
    B = co3.binding
    tables = norms(co3, [3_000_000, 40_000, 700, 9_000_000, 1, 250_000])
    assert len({L.partials for _, L, _, _ in tables}) >= 4
    work = torch.zeros(sum(L.partials for _, L, _, _ in tables), dtype=torch.float64, device="cuda")
    state = torch.zeros(64, dtype=torch.uint8, device="cuda")
    args = B.AdamwArgs(1e-3, 0.9, 0.999, 1e-8, 1.0, 1.0, 0, 0)
    near = lambda got, want: abs(float(got) - want) <= U * (1 + 1e-6) * want  # noqa: E731
    for turn in range(2):
        for order in (tables, tables[::-1]):
            for _, layout, plan, want in order:
                out = torch.full((2,), -7.0, device="cuda")
                B.grad_norm(layout, plan, 1.0, 1.0, out, work)
                assert near(out[0], want) and near(out[1], 1.0 / (want + 1e-6))
            for first in range(len(order)):                       # one table's sums behind another's, begun where any of them was
                some = order[first:first + 3]
                at = 0
                for _, layout, plan, _ in some:
                    B.grad_sumsq(layout, plan, work[at:])
                    at += layout.partials
                B.step_begin(args, state, work[:at])
                want = math.sqrt(sum(w * w for _, _, _, w in some))
                assert near(state.view(torch.float32)[4], want)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_sgd_clips_an_average_of_any_type_in_32_bits(co3, dtype):
    """The average times the factor goes to the weights as a float32 number, whatever the average is kept in: with a small factor
    a half-precision product would be among the subnormal numbers."""
    torch.manual_seed(33)
    model = torch.nn.Linear(48, 30).cuda()
    opt = co3.Co3SGD(model, 1, co3.Fmt(4, 3), lr=0.5, max_norm=1e-4)
    avg = torch.randn(opt.n, device="cuda").to(dtype)
    before = [p.detach().clone() for p in opt.params]
    opt.apply_average(avg)
    factor = opt.norm.compute()[1].clone()
    for p, b, a0, a1 in zip(opt.params, before, opt.seg_off[:-1], opt.seg_off[1:]):
        assert torch.equal(p.detach(), torch.add(b, (avg[a0:a1].float() * factor).view_as(p), alpha=-0.5))


def test_an_average_that_lies_elsewhere_now_is_the_one_that_is_stepped(co3):
    """The same tensor object with other memory, another object of the same memory, and the pipeline's own again."""
    def run(change):
        torch.manual_seed(34)
        model = torch.nn.Linear(48, 30).cuda()
        opt = co3.Co3AdamW(model, 1, co3.Fmt(4, 3), lr=0.1)
        avgs = [torch.randn(opt.n, device="cuda") for _ in range(4)]
        held = avgs[0].clone()
        opt.apply_average(held)
        change(opt, held, avgs)
        opt.pipe.avg[:opt.n] = avgs[3]
        opt.apply_average()
        assert opt.opt.t == 4
        return [p.detach().clone() for p in opt.params]

    def swapped(opt, held, avgs):
        held.data = avgs[1].clone()
        opt.apply_average(held)
        held.copy_(avgs[2])
        opt.apply_average(held[:])

    def separate(opt, held, avgs):
        opt.apply_average(avgs[1])
        opt.apply_average(avgs[2])
    assert all(torch.equal(a, b) for a, b in zip(run(swapped), run(separate)))
