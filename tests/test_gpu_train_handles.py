"""The training handles on the GPU: tensors that change their memory, and streams of their own."""
import pytest
import torch

from paper_2609_28053_amd import AdamW, BalanceLoss, ExpertRows, eqb
from test_gpu_adamw import HYPER, Model, bits_of, check
from test_gpu_balance import say

pytestmark = pytest.mark.gpu

D = dict(device="cuda")


def tensors(seed, *shapes):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return [torch.randn(s, generator=g, **D) for s in shapes]


SHAPES = ((64, 33), (5,), (300,))


@pytest.mark.parametrize("bits", [32, 8])
def test_a_parameter_that_moves_is_followed(bits):
    """p.data = ... between two steps: the new memory gets the step, bit for bit, and the old one keeps its values."""
    say(f"adamw {bits} bits, a parameter moves")
    still, moved = tensors(0, *SHAPES), tensors(0, *SHAPES)
    a, b = AdamW(still, lr=1e-2, state_bits=bits), AdamW(moved, lr=1e-2, state_bits=bits)
    first, second = tensors(1, *SHAPES), tensors(2, *SHAPES)
    a.step(first)
    b.step(first)
    old = moved[0].data
    was = old.clone()
    moved[0].data = old.clone()
    a.step(second)
    b.step(second)
    assert all(torch.equal(p, q) for p, q in zip(still, moved))
    assert torch.equal(old, was) and not torch.equal(moved[0], was)


T, E, K, H, P = 5000, 64, 4, 256, 3


def inputs():
    z, x, out, gy = tensors(3, (T, E), (T, H), (T * K, H), (T, H))
    idx = z.topk(K, dim=1).indices.to(torch.int32)
    bf = lambda t: t.to(torch.bfloat16)  # noqa: E731
    return dict(z=bf(z).view(torch.int16), idx=idx, x=bf(x), out=bf(out), gy=bf(gy), w=torch.sigmoid(z).gather(1, idx.long()),
                one=torch.ones(P, **D), valid=z[:, 0] < 1.0, grads=tensors(4, *SHAPES))


def pass_of(rows, loss, opt, i, stream):
    part = [0, 100, 3000, T]
    got = dict(rows=rows.plan(i["idx"], stream=stream).dispatch(i["x"], stream=stream)[:int(T * K)])
    got["y"] = rows.combine(i["out"], i["w"], stream=stream)
    got["grad_out"], got["grad_w"] = rows.combine_backward(i["gy"], i["out"], i["w"], stream=stream)
    got["loss"] = loss.forward(i["z"], i["idx"], i["valid"], part, stream=stream)
    got["grad_z"] = loss.backward(i["z"], i["one"], topk_idx=i["idx"], grad_score=got["grad_w"], valid=i["valid"],
                                  part_off=part, stream=stream)
    opt.step(i.pop("grads"), grad_scale=i["one"][:1], stream=stream)
    return got


def made(params, bits):
    return ExpertRows(T, E, K), BalanceLoss(T, E, K, P), AdamW(params, lr=1e-2, state_bits=bits)


def busy(stream, n=40):
    """Some milliseconds of products on the stream."""
    with torch.cuda.stream(stream):
        a = torch.ones((4096, 4096), dtype=torch.bfloat16, **D)
        for _ in range(n):
            a = (a @ a) * 2.0 ** -12
    return a


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("as_handle", [False, True])
def test_a_stream_of_their_own(bits, as_handle):
    """Calls with stream= behind a busy stream, their inputs dropped and overwritten-if-reused meanwhile: the same bits
    as on the current stream."""
    say(f"handles on a stream, {bits} bits")
    p, q = tensors(0, *SHAPES), tensors(0, *SHAPES)
    want = pass_of(*made(p, bits), inputs(), None)
    want = {k: v.clone() for k, v in want.items()}
    i, objects = inputs(), made(q, bits)
    sizes = [(t.shape, t.dtype) for t in i.values() if isinstance(t, torch.Tensor)] + [(g.shape, g.dtype) for g in i["grads"]]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    busy(s)
    got = pass_of(*objects, i, s.cuda_stream if as_handle else s)
    del i, objects                   # nothing else holds them while the stream still works
    for _ in range(3):
        junk = [torch.empty(shape, dtype=dtype, **D).view(torch.uint8).fill_(0xFF) for shape, dtype in sizes]
    s.synchronize()
    torch.cuda.synchronize()
    assert len(junk) == len(sizes)
    for k in want:
        assert torch.equal(want[k], got[k]), k
    assert all(torch.equal(a, b) for a, b in zip(p, q))


def test_buffers_filled_on_a_busy_stream():
    """A handle made on a busy stream and used on another at once: the call waits for the fills."""
    say("handles made on a busy stream")
    p, q = tensors(0, *SHAPES), tensors(0, *SHAPES)
    want = {k: v.clone() for k, v in pass_of(*made(p, 8), inputs(), None).items()}
    i = inputs()
    torch.cuda.synchronize()
    kept = busy(torch.cuda.current_stream())
    objects = made(q, 8)
    s = torch.cuda.Stream()
    got = pass_of(*objects, i, s)
    s.synchronize()
    assert kept.numel() and all(torch.equal(want[k], got[k]) for k in want)
    assert all(torch.equal(a, b) for a, b in zip(p, q))


@pytest.mark.parametrize("bits", [32, 8])
def test_a_counted_step_is_the_step_of_its_number(bits):
    """Bit for bit the step that a number given by the host makes, at the first steps and far on; a skipped one changes
    nothing, the counter included."""
    for taken in (0, 1, 6, 99999):
        say(f"adamw {bits} bits, counted step {taken + 1}")
        m = Model(taken, [1, 300, 2000, 255], bits, "bf16", True)
        counter = torch.zeros(8, dtype=torch.int64, **D)
        counter[0] = taken
        one = torch.ones(1, **D)
        before = [bits_of(t).copy() for t in m.tw + m.tc + m.tm + m.tv]
        eqb.eqb_adamw_step_counted(m.table(eqb), counter, seed=11, found_inf=one, **HYPER)
        assert all((a == bits_of(t)).all() for a, t in zip(before, m.tw + m.tc + m.tm + m.tv))
        assert int(counter[0]) == taken
        eqb.eqb_adamw_step_counted(m.table(eqb), counter, seed=11, found_inf=one * 0, **HYPER)
        check(m, taken + 1, 11)
        assert int(counter[0]) == taken + 1


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("on_device", [False, True])
def test_skipped_steps_do_not_count(bits, on_device):
    """Steps that found_inf skips, first ones and later ones, between steps that are taken: parameters and states end
    where those of an optimizer that made the taken steps alone end."""
    say(f"adamw {bits} bits, skipped steps")
    p, q = tensors(0, *SHAPES), tensors(0, *SHAPES)
    kw = dict(lr=1e-2, weight_decay=0.1, state_bits=bits, seed=3)
    alone, skipping = AdamW(p, **kw), AdamW(q, device_steps=on_device, **kw)
    zero, inf = torch.zeros(1, **D), torch.ones(1, **D)
    taken = 0
    for step, skip in enumerate((1, 1, 1, 0, 0, 1, 0)):
        grads = tensors(50 + step, *SHAPES)
        skipping.step(grads, found_inf=inf if skip else zero)
        if not skip:
            alone.step(grads)
            taken += 1
        assert skipping.steps == alone.steps == taken
    skipping.step(tensors(70, *SHAPES))               # without found_inf: counted as well
    alone.step(tensors(70, *SHAPES))
    assert skipping.steps == alone.steps == 4
    for a, b in zip(p + alone.exp_avg + alone.exp_avg_sq, q + skipping.exp_avg + skipping.exp_avg_sq):
        assert (bits_of(a) == bits_of(b)).all()
    third = AdamW([x.clone() for x in q], **kw)
    third.load_state_dict(skipping.state_dict())
    assert third.steps == 4
    third.step(tensors(71, *SHAPES))
    skipping.step(tensors(71, *SHAPES))
    assert all(torch.equal(a, b) for a, b in zip(third.params, q))


@pytest.mark.parametrize("bits", [32, 8])
def test_steps_in_a_graph(bits):
    """A captured step, replayed with eager work between the replays and one of them skipped: each replay is the next
    step.  Without device_steps the capture is refused."""
    say(f"adamw {bits} bits, steps in a graph")
    p, q = tensors(0, *SHAPES), tensors(0, *SHAPES)
    kw = dict(lr=1e-2, weight_decay=0.1, state_bits=bits, seed=3)
    eager, held = AdamW(p, **kw), AdamW(q, device_steps=True, **kw)
    grads, found = [torch.zeros(s, **D) for s in SHAPES], torch.zeros(1, **D)
    for g, x in zip(grads, tensors(50, *SHAPES)):
        g.copy_(x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        held.step(grads, found_inf=found)
    s.synchronize()
    eager.step(grads)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        held.step(grads, found_inf=found)
    for replay in range(5):
        for g, x in zip(grads, tensors(60 + replay, *SHAPES)):
            g.copy_(x)
        found.fill_(float(replay == 2))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        if replay != 2:
            eager.step(grads)
        assert all(torch.equal(a, b) for a, b in zip(p, q)), replay
        assert held.steps == eager.steps
    other = AdamW(p, **kw)
    other.step(grads)
    torch.cuda.synchronize()
    refused = torch.cuda.CUDAGraph()
    with pytest.raises(RuntimeError, match="device_steps"):
        with torch.cuda.graph(refused, stream=s):
            grads[0].add_(0.0)
            other.step(grads)
    torch.cuda.synchronize()


def test_batches_in_flight():
    """Two forward passes before the first backward pass, the routing's loads in one buffer that both write: the
    gradients are those of handles that serve one batch each."""
    say("two batches in flight")
    g = torch.Generator(device="cuda")
    g.manual_seed(9)
    batches = []
    for _ in range(2):
        z = torch.randn((T, E), generator=g, **D).to(torch.bfloat16)
        idx = (z.float() + torch.randn(E, generator=g, **D)).topk(K, dim=1).indices.to(torch.int32)
        batches.append((z.view(torch.int16), idx, torch.randn((T, H), generator=g, **D), torch.randn((T * K, H), generator=g, **D),
                        torch.rand((T, K), generator=g, **D)))
    one = torch.ones(1, **D)
    load_of = lambda idx: torch.bincount(idx.view(-1).long(), minlength=E).to(torch.int32).view(1, E)  # noqa: E731
    want = []
    for z, idx, gy, out, w in batches:
        rows, loss = ExpertRows(T, E, K), BalanceLoss(T, E, K)
        loss.forward(z, load=load_of(idx))
        want.append([*rows.plan(idx).combine_backward(gy, out, w), loss.backward(z, one)])
    rows, loss, load, kept = ExpertRows(T, E, K), BalanceLoss(T, E, K), torch.empty((1, E), dtype=torch.int32, **D), []
    for z, idx, gy, out, w in batches:
        load.copy_(load_of(idx))
        loss.forward(z, load=load)
        kept.append((rows.plan(idx).slot, loss.saved))
    load.fill_(0)
    for (z, idx, gy, out, w), (slot, saved), expected in zip(batches, kept, want):
        got = [*rows.combine_backward(gy, out, w, slot=slot), loss.backward(z, one, saved=saved)]
        assert all(torch.equal(a, b) for a, b in zip(got, expected))


@pytest.mark.parametrize("warm", [False, True])
def test_handles_in_a_graph(warm):
    """Plan, rows, loss and gradients through the handles in one graph, captured at their first call on the stream or
    after one, replayed on changing inputs with eager work between the replays."""
    say(f"handles in a graph, warm={warm}")
    z, idx = torch.zeros((T, E), dtype=torch.bfloat16, **D), torch.zeros((T, K), dtype=torch.int32, **D)
    x, out, gy = (torch.zeros(s, dtype=torch.bfloat16, **D) for s in ((T, H), (T * K, H), (T, H)))
    w, one, part = torch.zeros((T, K), **D), torch.ones(P, **D), eqb.PartOffsets([0, 100, 3000, T])

    def work(rows, loss):
        got = [rows.plan(idx).dispatch(x), rows.combine(out, w), *rows.combine_backward(gy, out, w)]
        got += [loss.forward(z.view(torch.int16), idx, part_off=part)]
        return got + [loss.backward(z.view(torch.int16), one, topk_idx=idx, grad_score=got[3], part_off=part)]

    held, eager = made([], 32)[:2], made([], 32)[:2]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    if warm:
        with torch.cuda.stream(s):
            work(*held)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        captured = work(*held)
    for replay in range(4):
        g = torch.Generator(device="cuda")
        g.manual_seed(replay)
        z.copy_(torch.randn((T, E), generator=g, **D))
        idx.copy_(z.float().topk(K, dim=1).indices)
        for t in (x, out, gy, w):
            t.copy_(torch.randn(t.shape, generator=g, **D))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, work(*eager))), replay
        torch.cuda.synchronize()
