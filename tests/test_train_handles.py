"""The training handles' host side without a GPU: the library's calls are replaced by
recorders, and tensors of the CPU pass for the GPU's."""
import pytest
import torch

from paper_2609_28053_amd import AdamW, eqb


@pytest.fixture
def calls(monkeypatch):
    """The arguments of every optimizer call, with the table's columns as they were."""
    def ptr(t, dtype=None, numel=None, name="tensor"):
        if t is None:
            return None
        if not t.is_contiguous() or (numel is not None and t.numel() != numel):
            raise ValueError(name)
        if dtype is not None and t.dtype is not dtype:
            raise TypeError(name)
        return t.data_ptr()

    seen = []

    def step(tensors, number, lr, beta1=0.9, beta2=0.95, eps=1e-8, seed=0, grad_scale=None, found_inf=None, stream=None):
        seen.append(dict({n: tensors.table[n].tolist() for n in tensors.table.dtype.names}, step=number, lr=lr))

    monkeypatch.setattr(eqb, "_ptr", ptr)
    def counted(tensors, counter, *a, **k):
        step(tensors, counter, *a, **k)

    monkeypatch.setattr(eqb, "eqb_adamw_step", step)
    monkeypatch.setattr(eqb, "eqb_adamw_step_counted", counted)
    return seen


def at(tensors):
    return [t.data_ptr() for t in tensors]


def model(bits=8):
    params = [torch.nn.Parameter(torch.randn(s)) for s in ((4, 5), (3,), (300,))]
    copies = [p.detach().to(torch.bfloat16) for p in params]
    return params, copies, AdamW(params, copies=copies, state_bits=bits, weight_decay=[0.1, 0.0, 0.2])


def grads_of(params):
    return [torch.randn_like(p) for p in params]


@pytest.mark.parametrize("bits", [8, 32])
def test_a_step_takes_the_memory_that_the_tensors_have_then(calls, bits):
    """Parameters, copies and states that were given other memory, or replaced in the optimizer's lists."""
    params, copies, opt = model(bits)
    opt.step(grads_of(params))
    params[0].data = params[0].data.clone()
    copies[1].data = copies[1].data.clone()
    opt.exp_avg[2] = opt.exp_avg[2].clone()
    opt.exp_avg_sq[0].data = opt.exp_avg_sq[0].data.clone()
    if bits == 8:
        opt.exp_avg_scale[1] = opt.exp_avg_scale[1].clone()
    for _ in range(2):
        grads = grads_of(params)
        opt.step(grads)
        got = calls[-1]
        assert got["param"] == at(params) and got["copy"] == at(copies) and got["grad"] == at(grads)
        assert got["exp_avg"] == at(opt.exp_avg) and got["exp_avg_sq"] == at(opt.exp_avg_sq)
        if bits == 8:
            assert got["exp_avg_scale"] == at(opt.exp_avg_scale) and got["exp_avg_sq_scale"] == at(opt.exp_avg_sq_scale)


def test_a_tables_memory_outlives_its_tensors(calls):
    """What a table names stays allocated while the table stands, whatever becomes of the tensors: it owns the storages
    that its addresses lie in."""
    params, copies, opt = model()
    grads = grads_of(params)
    table = eqb.AdamwTensors(params, grads, opt.exp_avg, opt.exp_avg_sq, copies, opt.exp_avg_scale, opt.exp_avg_sq_scale)
    kept = [t.untyped_storage()._cdata for t in params + copies + grads]
    before = table.table.copy()
    for t in params + copies + grads:
        t.data = torch.zeros_like(t.data)
    held = {s._cdata for _, storages in table._held.values() for s in storages}
    assert held.issuperset(kept) and (table.table == before).all()


def test_the_decay_of_a_step_is_the_one_it_has_then(calls):
    params, _, opt = model()
    opt.step(grads_of(params))
    opt.weight_decay[1] = 0.7
    opt.step(grads_of(params))
    opt.weight_decay = 0.25
    opt.step(grads_of(params))
    assert [c["weight_decay"] for c in calls] == [[0.1, 0.0, 0.2], [0.1, 0.7, 0.2], [0.25] * 3]


def test_memory_of_another_kind_is_refused(calls):
    params, copies, opt = model()
    opt.step(grads_of(params))
    params[2].data = torch.zeros(5)
    with pytest.raises(ValueError):
        opt.step([torch.zeros(4, 5), torch.zeros(3), torch.zeros(300)])
    params[2].data = torch.zeros(300, dtype=torch.float64)
    with pytest.raises(TypeError):
        opt.step([torch.zeros(4, 5), torch.zeros(3), torch.zeros(300)])
    params[2].data = torch.zeros(300)
    copies.append(torch.zeros(2, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        opt.step([torch.zeros(4, 5), torch.zeros(3), torch.zeros(300)])
    with pytest.raises(ValueError):
        opt.step([])


def test_a_refused_step_does_not_count(calls, monkeypatch):
    params, _, opt = model()
    opt.step(grads_of(params))
    taken = eqb.eqb_adamw_step

    def refuse(*a, **k):
        raise eqb.EqbError("eqb_adamw_step", eqb.EQB_ERR_INVALID_ARG)

    monkeypatch.setattr(eqb, "eqb_adamw_step", refuse)
    with pytest.raises(eqb.EqbError):
        opt.step(grads_of(params), lr=float("nan"))
    monkeypatch.setattr(eqb, "eqb_adamw_step", taken)
    opt.step(grads_of(params))
    assert [c["step"] for c in calls] == [1, 2] and opt.steps == 2


def test_steps_that_may_be_skipped_are_counted_on_the_device(calls):
    """From the first found_inf on the call gets the counter, which begins with the steps taken by then."""
    params, _, opt = model()
    opt._behind = set()
    opt.step(grads_of(params))
    opt.step(grads_of(params), found_inf=torch.zeros(1))
    opt.step(grads_of(params))
    assert calls[0]["step"] == 1
    assert all(c["step"] is opt._counter and c["step"].shape == (8,) for c in calls[1:])
    assert opt._counter.tolist() == [1] + [0] * 7 and opt.steps == 1          # the recorder does not count
    opt.load_state_dict(dict(opt.state_dict(), steps=40))
    assert opt.steps == 40 and opt._counter[0] == 40
    on = AdamW(params, device_steps=True)
    on.step(grads_of(params))
    assert calls[-1]["step"] is on._counter and on.steps == 0


def test_no_parameters(calls):
    """An optimizer of nothing takes its steps, whatever they are given."""
    for opt in (AdamW([]), AdamW([], state_bits=8, device_steps=True)):
        opt.step([])
        opt.step([], found_inf=torch.zeros(1))
        assert opt.steps == 2
    assert [c["step"] for c in calls] == [1, 2, 1, 2] and all(c["param"] == [] for c in calls)


@pytest.mark.parametrize("bits", [8, 32])
def test_a_state_that_does_not_fit_changes_nothing(bits):
    params, _, opt = model(bits)
    _, _, other = model(bits)
    for t in other.exp_avg + other.exp_avg_sq:
        t.view(torch.uint8).fill_(1)
    before = [t.clone() for t in opt.exp_avg + opt.exp_avg_sq]
    good = dict(other.state_dict(), steps=5)
    short = list(good["exp_avg_sq"])
    short[2] = short[2][:7]
    whole = [t.to(torch.float32).to(torch.int32) for t in good["exp_avg_sq"]]
    scale = dict(exp_avg_sq_scale=None if bits == 8 else good["exp_avg"])
    for bad in (dict(exp_avg_sq=short), dict(exp_avg_sq=whole), dict(exp_avg_sq=good["exp_avg_sq"][:2]), scale):
        with pytest.raises(ValueError):
            opt.load_state_dict(dict(good, **bad))
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(opt.exp_avg + opt.exp_avg_sq, before))
        assert opt.steps == 0
    with pytest.raises(KeyError):
        opt.load_state_dict({k: v for k, v in good.items() if k != "steps"})
    assert opt.steps == 0 and not opt.exp_avg[0].view(torch.uint8).any()
    opt.load_state_dict(good)
    assert opt.steps == 5 and all((t.view(torch.uint8) == 1).all() for t in opt.exp_avg + opt.exp_avg_sq)


def test_autograd_notices_a_step_between_forward_and_backward(calls):
    """A parameter or copy that autograd kept for a backward pass and that a step has overwritten is refused there, as
    with any change in place."""
    params, copies, opt = model()
    x = torch.randn(3, requires_grad=True)
    for weight in (params[1], copies[1]):
        y = (x * weight).sum()
        y.backward()
        y = (x * weight).sum()
        opt.step(grads_of(params))
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()


class Stream:
    """A stream that notes what waits on it."""

    def __init__(self, number):
        self.cuda_stream, self.waits = number, []

    def wait_event(self, event):
        self.waits.append(event)


@pytest.fixture
def streams(monkeypatch):
    """The stream that is current where memory is allocated and where the library is called: lists of numbers (0: the
    current stream outside)."""
    import contextlib
    now, where = [0], dict(alloc=[], call=[])

    @contextlib.contextmanager
    def on(s):
        now.append(s.cuda_stream)
        yield
        now.pop()

    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: Stream(now[-1]))
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: None)
    monkeypatch.setattr(eqb, "_stream", lambda s: now[-1] if s is None else s.cuda_stream)
    for name in ("empty", "empty_like"):
        real = getattr(torch, name)
        monkeypatch.setattr(torch, name, lambda *a, real=real, **k: (where["alloc"].append(now[-1]), real(*a, **k))[1])
    for name in ("eqb_dispatch_plan", "eqb_dispatch", "eqb_combine", "eqb_combine_backward", "eqb_balance_loss",
                 "eqb_balance_backward", "eqb_adamw_step"):
        def call(*a, **k):
            given = [x for x in list(a) + list(k.values()) if isinstance(x, Stream)]
            where["call"].append(given[0].cuda_stream if given else now[-1])
        monkeypatch.setattr(eqb, name, call)
    return where


def handles():
    from paper_2609_28053_amd import BalanceLoss, ExpertRows
    T, E, K, H = 6, 8, 2, 4
    rows, loss = ExpertRows(T, E, K, device="cpu"), BalanceLoss(T, E, K, device="cpu")
    rows.slot = torch.zeros((T, K), dtype=torch.int32)
    loss.load, loss.tokens = torch.zeros((1, E), dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    p = torch.zeros(3)
    opt = AdamW([p])
    x, r, w = torch.zeros(T, H), torch.zeros(T * K, H), torch.zeros(T, K)
    z, idx, one = torch.zeros(T, E), torch.zeros(T, K, dtype=torch.int32), torch.ones(1)
    return [(rows, lambda s: rows.plan(idx, stream=s)), (rows, lambda s: rows.dispatch(x, stream=s)),
            (rows, lambda s: rows.combine(r, w, stream=s)), (rows, lambda s: rows.combine_backward(x, r, w, stream=s)),
            (loss, lambda s: loss.forward(z, idx, stream=s)), (loss, lambda s: loss.backward(z, one, stream=s)),
            (opt, lambda s: opt.step([p.clone()], stream=s))]


def test_a_call_allocates_on_the_stream_that_it_works_on(calls, streams):
    for handle, call in handles():
        handle._fill, handle._behind = "filled", {0}
        for number in (7, 0):
            streams["alloc"].clear(), streams["call"].clear()
            call(Stream(number) if number else None)
            assert streams["call"] == [number] and set(streams["alloc"]) <= {number}


def test_the_first_call_on_a_stream_waits_for_the_fills(calls, streams):
    for handle, call in handles():
        handle._fill, handle._behind = "filled", {0}
        s = Stream(7)
        call(s)
        assert s.waits == ["filled"]
        call(s)
        assert s.waits == ["filled"]
        here = Stream(0)
        call(here)
        assert here.waits == []


@pytest.fixture
def numbers(monkeypatch, calls):
    """The library's calls as recorders that write their number into what they compute."""
    seen = []

    def fill(name, *outputs):
        seen.append(name)
        for t in outputs:
            t.fill_(len(seen))

    monkeypatch.setattr(eqb, "eqb_dispatch_plan", lambda idx, E, offsets, slot, ws=None, stream=None: fill("plan", offsets, slot))
    monkeypatch.setattr(eqb, "eqb_combine", lambda rows, slot, w, y, stream=None: fill(int(slot[0, 0]), y))
    monkeypatch.setattr(eqb, "eqb_dispatch", lambda x, slot, rows, stream=None: fill(int(slot[0, 0]), rows))
    monkeypatch.setattr(eqb, "eqb_combine_backward", lambda gy, r, slot, w, gr, gw, stream=None: fill(int(slot[0, 0]), gr, gw))
    monkeypatch.setattr(eqb, "eqb_balance_loss", lambda z, idx, K, a, load, tokens, prob, loss, *r, **k: fill(
        "loss", tokens, prob, loss, *([load] if idx is not None else [])))
    monkeypatch.setattr(eqb, "eqb_balance_backward", lambda z, load, tokens, *r, **k: seen.append(
        (int(load[0, 0]), int(tokens[0]))))
    return seen


def test_two_batches_in_flight_keep_their_plans(numbers):
    from paper_2609_28053_amd import ExpertRows
    rows = ExpertRows(6, 8, 2, device="cpu")
    idx, x, r, w = torch.zeros((6, 2), dtype=torch.int32), torch.zeros(6, 4), torch.zeros(12, 4), torch.zeros(6, 2)
    with pytest.raises(ValueError):
        rows.dispatch(x)
    first = rows.plan(idx).slot
    second = rows.plan(idx).slot
    rows.dispatch(x, slot=first), rows.combine(r, slot=first), rows.combine_backward(x, r, w, slot=first)
    rows.dispatch(x), rows.combine(r), rows.combine_backward(x, r, w)
    assert numbers == ["plan", "plan", 1, 1, 1, 2, 2, 2] and second is rows.slot


def test_two_batches_in_flight_keep_their_loads(numbers):
    """Counted loads and given ones, whose buffer the next routing fills again."""
    from paper_2609_28053_amd import BalanceLoss
    loss = BalanceLoss(6, 8, 2, device="cpu")
    z, idx, one = torch.zeros(6, 8), torch.zeros((6, 2), dtype=torch.int32), torch.ones(1)
    with pytest.raises(ValueError):
        loss.backward(z, one)
    a = loss.forward(z, idx)
    first = loss.saved
    routed = torch.full((1, 8), 50, dtype=torch.int32)
    b = loss.forward(z, load=routed)
    second = loss.saved
    routed.fill_(60)
    c = loss.forward(z, load=routed)
    routed.fill_(70)
    loss.backward(z, one, saved=first), loss.backward(z, one, saved=second), loss.backward(z, one)
    loss.load = loss.load * 2                     # loads that the program has changed (summed over ranks, say)
    loss.backward(z, one)
    assert numbers == ["loss"] * 3 + [(1, 1), (50, 2), (60, 3), (120, 3)]
    assert (float(a), float(b), float(c)) == (1.0, 2.0, 3.0)
