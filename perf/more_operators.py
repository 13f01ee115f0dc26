"""Performance cases of the routing by scores and of the experts' products in 8 bits.

Four kinds of call:
  route     the experts of every token by their scores (sigmoid or softmax, with a
            bias for balance, within the best groups), their weights, and the
            gradient with respect to the logits;
  quantize  rows, rows on their way to the experts, an expert's columns, or
            weights as E4M3 codes with a power of two for each block of 128;
  product   the experts' products of such codes: the rows with the weights, and
            the gradients with respect to both;
  gated     the gated activation between an expert's two products, as codes or
            with its gradient.
``run`` computes them from elementary torch operations, or, where ``own`` is set,
by the library's calls.
"""
import math

import torch

own = False

DEV = "cuda"
CHUNK = 1 << 16        # rows drawn or checked at a time
BLOCK = 128            # elements that share a scale
LARGEST = 448.0        # of the codes
EXPERTS = (8, 16, 32, 64, 128, 256)
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}


def listed():
    return [
        # a serving step of a few sequences: eight groups of experts, latency counts
        dict(name="route-decode", kind="route", T=8, E=256, K=8, groups=8, keep=4, pair=2, dtype="bf16", score="sigmoid",
             bias="normal", normalize=True, data="boost", grad=False),
        # one data-parallel rank's share of the paper's step, forward and backward
        dict(name="route-rank256", kind="route", T=147456, E=256, K=6, groups=8, keep=4, pair=2, dtype="bf16", score="sigmoid",
             bias="normal", normalize=True, data="boost", grad=True),
        # a softmax router on binary32 logits, experts masked out of rows, weights as they are
        dict(name="route-odd128", kind="route", T=99991, E=128, K=5, groups=1, keep=1, pair=1, dtype="f32", score="softmax",
             bias="none", normalize=False, data="masked", grad=True),
        # a rank's tokens on their way to the experts
        dict(name="quantize-dispatch", kind="quantize", form="dispatch", T=147456, E=256, K=6, H=1024, dtype="bf16", drop=0.0),
        # what a weight gradient contracts over: ragged experts, odd rows
        dict(name="quantize-columns", kind="quantize", form="columns", T=5003, E=32, K=4, H=1001, dtype="bf16", drop=0.05),
        # a layer's weights, for the products forward and backward
        dict(name="quantize-weights", kind="quantize", form="weights", E=64, N=2048, H=2048, dtype="bf16"),
        # a serving step: the weights of the chosen experts are the time
        dict(name="product-decode", kind="product", form="rows", T=8, E=256, K=8, N=2048, H=2048, dtype="bf16", drop=0.0),
        # a rank's rows through the first product
        dict(name="product-rank256", kind="product", form="rows", T=147456, E=256, K=6, N=1024, H=1024, dtype="bf16", drop=0.0),
        # a micro-batch of 64 experts: forward, and the gradients of rows and weights
        dict(name="product-train64", kind="product", form="train", T=16384, E=64, K=6, N=2048, H=2048, dtype="bf16", drop=0.1),
        # odd sizes, results in binary32
        dict(name="product-odd32", kind="product", form="train", T=5003, E=32, K=4, N=777, H=1001, dtype="f32", drop=0.05),
        # the rows of a serving step between the products
        dict(name="gated-decode", kind="gated", form="codes", T=8, E=256, K=8, H=2048, dtype="bf16", drop=0.0),
        # a micro-batch's, with the gradient
        dict(name="gated-train64", kind="gated", form="train", T=16384, E=64, K=6, H=2048, dtype="bf16", drop=0.1),
    ]


def _log(rng, low, high):
    return int(math.exp(rng.uniform(math.log(low), math.log(high + 0.99))))


def draw(rng):
    kind = rng.choice(["route", "quantize", "product", "product", "gated"])
    cost = lambda c: work(c)["bytes"] + work(c)["flops"] / 500  # noqa: E731
    most = max(cost(c) for c in listed() if c["kind"] == kind)
    while True:
        case = _draw(rng, kind)
        if cost(case) <= most and (kind != "product" or case["E"] * case["N"] * case["H"] <= 1 << 30):
            return case


def _draw(rng, kind):
    E = rng.choice(EXPERTS)
    odd = lambda n: n | 1 if rng.random() < 0.5 else n  # noqa: E731
    K, T = _log(rng, 1, min(E - 1, 16)), odd(_log(rng, 1, 147456))
    H = odd(_log(rng, 16, 4096)) if rng.random() < 0.5 else 128 * _log(rng, 1, 32)
    dtype, drop = rng.choice(["bf16", "bf16", "f16", "f32"]), rng.choice([0.0, 0.0, 0.1])
    if kind == "route":
        groups = rng.choice([g for g in (1, 1, 2, 4, 8, 16) if g <= E])
        keep = rng.randint(1, groups)
        K = min(K, keep * (E // groups))
        return dict(kind=kind, T=T, E=E, K=K, groups=groups, keep=keep,
                    pair=rng.choice([1, 2]) if E // groups > 1 else 1, dtype=dtype, score=rng.choice(["sigmoid", "softmax"]),
                    bias=rng.choice(["none", "normal", "steps"]),
                    # the weight of one expert alone, normalized, is a constant
                    normalize=K > 1 and rng.random() < 0.6,
                    data=rng.choice(["normal", "boost", "masked", "ties"]), grad=rng.random() < 0.7)
    if kind == "quantize":
        form = rng.choice(["rows", "dispatch", "columns", "weights"])
        if form == "weights":
            return dict(kind=kind, form=form, E=E, N=odd(_log(rng, 16, 4096)), H=H, dtype=dtype)
        return dict(kind=kind, form=form, T=T, E=E, K=K, H=H, dtype=dtype, drop=drop)
    if kind == "product":
        N = odd(_log(rng, 16, 4096)) if rng.random() < 0.5 else 128 * _log(rng, 1, 32)
        return dict(kind=kind, form=rng.choice(["rows", "rows", "train"]), T=T, E=E, K=K, N=N, H=H, dtype=dtype, drop=drop)
    return dict(kind=kind, form=rng.choice(["codes", "train"]), T=T, E=E, K=K, H=H, dtype=dtype, drop=drop)


# ------------------------------------------------------------------ inputs --
def _generator(seed, stream):
    g = torch.Generator(device=DEV)
    g.manual_seed((int(seed) * 1000003 + stream) % (1 << 62))
    return g


def _logits(T, E, data, dtype, seed):
    """A router's logits [T,E]: experts of unequal favour; "boost": one expert raised in a twentieth of the rows;
    "masked": a tenth of the experts masked out of each row, and all of them out of a few rows; "ties": steps of 1/4."""
    off = torch.randn(E, generator=_generator(seed, 0), device=DEV) * 0.7
    z = torch.empty((T, E), dtype=dtype, device=DEV)
    for c, t0 in enumerate(range(0, T, CHUNK)):
        g = _generator(seed, 1 + c)
        n = min(CHUNK, T - t0)
        x = torch.randn((n, E), generator=g, device=DEV) + off
        if data == "boost":
            e = torch.randint(0, E, (n, 1), generator=g, device=DEV)
            x.scatter_add_(1, e, (torch.rand((n, 1), generator=g, device=DEV) < 0.05).to(torch.float32) * 3)
        if data == "masked":
            x.masked_fill_(torch.rand((n, E), generator=g, device=DEV) < 0.1, -math.inf)
            x.masked_fill_(torch.rand((n, 1), generator=g, device=DEV) < 0.01, -math.inf)
        if data == "ties":
            x = torch.round(x * 4) / 4
        z[t0:t0 + n] = x
    return z


def _routed(case, seed):
    """The pairs of T tokens in the experts' order: how many each expert has (on the host, and as the offsets that the
    plan leaves on the device) and every pair's row."""
    T, E, K = case["T"], case["E"], case["K"]
    idx = torch.empty((T, K), dtype=torch.int64, device=DEV)
    for c, t0 in enumerate(range(0, T, CHUNK)):
        z = _logits(min(CHUNK, T - t0), E, "boost", torch.float32, seed * 64 + c)
        idx[t0:t0 + CHUNK] = z.topk(K, dim=1).indices
    flat = idx.view(-1)
    if case["drop"]:
        flat = torch.where(torch.rand(T * K, generator=_generator(seed, 0x20000), device=DEV) < case["drop"], E, flat)
    order = torch.sort(flat, stable=True).indices
    slot = torch.empty(T * K, dtype=torch.int32, device=DEV)
    slot[order] = torch.arange(T * K, device=DEV, dtype=torch.int32)
    slot = torch.where(flat < E, slot, -1).view(T, K)
    counts = torch.bincount(flat, minlength=E + 1)[:E]
    offsets = torch.zeros(E + 1, dtype=torch.int32, device=DEV)
    offsets[1:] = counts.cumsum(0)
    return dict(counts=counts.tolist(), offsets=offsets, slot=slot)


def _up(n, to=BLOCK):
    return -(-n // to) * to


def _starts(counts, R):
    """Where each expert's columns begin, on a whole block, and how many columns there are for R rows."""
    first, starts = 0, []
    for e, n in enumerate(counts):
        starts.append(BLOCK * (first // BLOCK + e))
        first += n
    return starts, BLOCK * (R // BLOCK + len(counts))


def _scale_width(H):
    return _up(-(-H // BLOCK), 4)


def _code_buffers(*shape):
    lead, H = shape[:-1], shape[-1]
    return (torch.zeros((*lead, _up(H)), dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn), _scale_buffer(*lead, H))


def _scale_buffer(*shape):
    return torch.zeros((*shape[:-1], _scale_width(shape[-1])), dtype=torch.uint8, device=DEV).view(torch.float8_e8m0fnu)


def _rows(case, seed, stream, width, dtype):
    """Rows of unequal size, as activations and gradients have them."""
    R = case["T"] * case["K"]
    g = _generator(seed, stream)
    size = torch.exp(torch.randn((R, 1), generator=g, device=DEV))
    x = torch.empty((R, width), dtype=dtype, device=DEV)
    for r0 in range(0, R, CHUNK):
        n = min(CHUNK, R - r0)
        x[r0:r0 + n] = torch.randn((n, width), generator=g, device=DEV) * size[r0:r0 + n]
    return x


def _weights(case, seed, dtype):
    E, N, H = case["E"], case["N"], case["H"]
    return torch.randn((E, N, H), generator=_generator(seed, 0x30000), device=DEV, dtype=dtype) * H ** -0.5


def prepare(case, seed):
    return {"route": _prepare_route, "quantize": _prepare_quantize, "product": _prepare_product,
            "gated": _prepare_gated}[case["kind"]](case, seed)


def _prepare_route(case, seed):
    T, E, K = case["T"], case["E"], case["K"]
    g = _generator(seed, 0x10000)
    bias = torch.randn(E, generator=g, device=DEV) * 0.1
    bias = {"none": None, "normal": bias, "steps": torch.round(bias * 1000) / 1000}[case["bias"]]
    state = dict(case=case, z=_logits(T, E, case["data"], TYPES[case["dtype"]], seed), bias=bias,
                 idx=torch.empty((T, K), dtype=torch.int32, device=DEV), weight=torch.empty((T, K), device=DEV))
    if case["grad"]:
        state.update(grad_weight=torch.randn((T, K), generator=g, device=DEV), grad_z=torch.empty((T, E), device=DEV))
    return state


def _prepare_quantize(case, seed):
    form, dt, H = case["form"], TYPES[case["dtype"]], case["H"]
    if form == "weights":
        codes, scales = _code_buffers(case["E"], case["N"], H)
        codes_t, scales_t = _code_buffers(case["E"], H, case["N"])
        scales, scales_t = _scale_buffer(case["E"], _up(case["N"]) // BLOCK, H), _scale_buffer(case["E"], _up(H) // BLOCK, case["N"])
        return dict(case=case, w=_weights(case, seed, dt), codes=codes, scales=scales, codes_t=codes_t, scales_t=scales_t)
    state = dict(case=case, **_routed(case, seed))
    R = case["T"] * case["K"]
    if form == "dispatch":
        state["x"] = _rows(dict(case, K=1), seed, 0x40000, H, dt)
    else:
        state["x"] = _rows(case, seed, 0x40000, H, dt)
    state["codes"], state["scales"] = _code_buffers(H, _starts(state["counts"], R)[1]) if form == "columns" else _code_buffers(R, H)
    return state


def _prepare_product(case, seed):
    N, H, dt = case["N"], case["H"], TYPES[case["dtype"]]
    R = case["T"] * case["K"]
    state = dict(case=case, **_routed(case, seed))
    w = _weights(case, seed, torch.bfloat16)
    x = _rows(case, seed, 0x40000, H, torch.bfloat16)
    state["x"], state["w"] = _plain_rows(x), _plain_weights(w)
    state["out"] = torch.zeros((R, N), dtype=dt, device=DEV)
    if case["form"] == "train":
        g = _rows(case, seed, 0x50000, N, torch.bfloat16)
        state["w_t"] = _plain_weights(w.transpose(1, 2).contiguous())
        state["g"], state["g_t"], state["x_t"] = _plain_rows(g), _plain_columns(g, state["counts"]), _plain_columns(x, state["counts"])
        state["grad_x"] = torch.zeros((R, H), dtype=dt, device=DEV)
        state["grad_w"] = torch.zeros((case["E"], N, H), device=DEV)
    return state


def _prepare_gated(case, seed):
    H, dt = case["H"], TYPES[case["dtype"]]
    R = case["T"] * case["K"]
    state = dict(case=case, **_routed(case, seed))
    state["x"] = _rows(case, seed, 0x40000, 2 * H, dt)
    if case["form"] == "codes":
        state["codes"], state["scales"] = _code_buffers(R, H)
    else:
        state.update(grad_h=_rows(case, seed, 0x50000, H, dt), h=torch.zeros((R, H), dtype=dt, device=DEV),
                     grad_x=torch.zeros((R, 2 * H), dtype=dt, device=DEV))
    return state


# --------------------------------------------------------------- the passes --
def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"route": _own_route, "quantize": _own_quantize, "product": _own_product, "gated": _own_gated}[kind](state)
    return {"route": _plain_route, "quantize": _plain_quantize, "product": _plain_product, "gated": _plain_gated}[kind](state)


SCALE = 2.5            # the factor of the chosen experts' weights


def _own_route(state):
    from paper_2609_28053_amd import eqb
    case, s = state["case"], state
    score = eqb.EQB_SCORE_SIGMOID if case["score"] == "sigmoid" else eqb.EQB_SCORE_SOFTMAX
    eqb.eqb_route_scored(s["z"], s["bias"], case["K"], s["idx"], s["weight"], score=score, groups=case["groups"],
                         top_groups=case["keep"], group_top=case["pair"], normalize=case["normalize"], scale=SCALE)
    if not case["grad"]:
        return dict(idx=s["idx"], weight=s["weight"])
    eqb.eqb_route_scored_backward(s["z"], s["idx"], s["grad_weight"], s["grad_z"], score=score,
                                  normalize=case["normalize"], scale=SCALE)
    return dict(idx=s["idx"], weight=s["weight"], grad_z=s["grad_z"])


def _plain_route(state):
    case, z = state["case"], state["z"]
    T, E, K, G = case["T"], case["E"], case["K"], case["groups"]
    some = z > -math.inf
    # the order of near scores is what it is in 64 bits
    zd = z.to(torch.float64)
    if case["score"] == "sigmoid":
        s = 1 / (1 + torch.exp(-zd))
    else:
        top = zd.amax(1, keepdim=True)
        s = torch.exp(zd - torch.where(top == -math.inf, 0.0, top))
        d = s.sum(1, keepdim=True)
        s = torch.where(d > 0, s / d, 0.0)
    q = s if state["bias"] is None else s + state["bias"].to(torch.float64)
    q = torch.where(some, q, -math.inf)
    if case["keep"] < G:
        best = q.view(T, G, E // G).topk(case["pair"], dim=2).values
        of_group = torch.where(best[..., 0] == -math.inf, -math.inf, torch.where(best == -math.inf, 0.0, best).sum(2))
        kept = torch.sort(of_group, dim=1, descending=True, stable=True).indices[:, :case["keep"]]
        inside = torch.zeros((T, G), dtype=torch.bool, device=DEV).scatter_(1, kept, True)
        q = torch.where(inside.repeat_interleave(E // G, 1), q, -math.inf)
    order = torch.sort(q, dim=1, descending=True, stable=True)
    chosen, at = order.values[:, :K] > -math.inf, order.indices[:, :K]
    sk = torch.where(chosen, s.gather(1, at), 0.0)
    S = sk.sum(1, keepdim=True)
    if case["normalize"]:
        weight = torch.where(S > 0, SCALE * sk / S, 0.0)
    else:
        weight = SCALE * sk
    got = dict(idx=torch.where(chosen, at, -1).to(torch.int32), weight=weight.to(torch.float32))
    if not case["grad"]:
        return got
    g = torch.where(chosen, state["grad_weight"].to(torch.float64), 0.0)
    if case["normalize"]:
        g = torch.where(S > 0, (g - (g * sk).sum(1, keepdim=True) / S) / S, 0.0)
    g = SCALE * g * sk
    if case["score"] == "sigmoid":
        grad = torch.zeros((T, E), dtype=torch.float64, device=DEV).scatter_add_(1, at, g / (1 + torch.exp(zd.gather(1, at))))
    else:
        grad = (-g.sum(1, keepdim=True) * s).scatter_add_(1, at, g)
    got["grad_z"] = grad.to(torch.float32)
    return got


def _exponents(top):
    """The least x >= -126 with top <= 448 2^x."""
    m, e = torch.frexp(top)
    return torch.where(top > 0, torch.where(m <= LARGEST / 512, e - 9, e - 8), -126).clamp(min=-126)


def _codes(y):
    return y.to(torch.float8_e4m3fn)


def _plain_rows(x):
    """Codes and scales of the blocks of 128 of each row."""
    R, H = x.shape
    v = torch.nn.functional.pad(x.to(torch.float32), (0, _up(H) - H)).view(R, -1, BLOCK)
    e = _exponents(v.abs().amax(2))
    codes = _codes(torch.ldexp(v, -e[..., None])).view(R, _up(H))
    return codes, _scales(e)


def _scales(e):
    wide = _up(e.shape[-1], 4) - e.shape[-1]
    return torch.nn.functional.pad((e + 127).to(torch.uint8), (0, wide)).view(torch.float8_e8m0fnu)


def _plain_columns(x, counts):
    """The same of each column in blocks of 128 rows of one expert; columns that belong to no block stay 0."""
    R, H = x.shape
    starts, wide = _starts(counts, R)
    kept = sum(counts)
    n = torch.tensor(counts, device=DEV)
    begin = torch.tensor(starts, device=DEV)
    at = torch.arange(kept, device=DEV) + (begin - (n.cumsum(0) - n)).repeat_interleave(n, output_size=kept)
    v = torch.zeros((H, wide), device=DEV)
    v[:, at] = x[:kept].to(torch.float32).t()
    v = v.view(H, -1, BLOCK)
    used = torch.zeros(wide // BLOCK, dtype=torch.bool, device=DEV)
    used[at // BLOCK] = True
    e = torch.where(used, _exponents(v.abs().amax(2)), -127)
    return _codes(torch.ldexp(v, torch.where(e > -127, -e, 0)[..., None])).view(H, wide), _scales(e)


def _plain_weights(w):
    """Codes of each expert's weights, a scale for each 128 x 128."""
    E, N, H = w.shape
    v = torch.nn.functional.pad(w.to(torch.float32), (0, _up(H) - H, 0, _up(N) - N)).view(E, -1, BLOCK, _up(H) // BLOCK, BLOCK)
    e = _exponents(v.abs().amax((2, 4)))
    codes = _codes(torch.ldexp(v, -e[:, :, None, :, None])).view(E, _up(N), _up(H))[:, :N].contiguous()
    return codes, _scales(e)


def _own_quantize(state):
    from paper_2609_28053_amd import eqb
    case, s = state["case"], state
    if case["form"] == "weights":
        eqb.eqb_quantize_weights(s["w"], s["codes"], s["scales"], s["codes_t"], s["scales_t"])
        return {k: s[k] for k in ("codes", "scales", "codes_t", "scales_t")}
    if case["form"] == "rows":
        eqb.eqb_quantize_rows(s["x"], s["codes"], s["scales"], s["offsets"][-1:])
    elif case["form"] == "dispatch":
        eqb.eqb_dispatch_quantized(s["x"], s["slot"], s["codes"], s["scales"])
    else:
        eqb.eqb_quantize_columns(s["x"], s["offsets"], s["codes"], s["scales"])
    return dict(codes=s["codes"], scales=s["scales"])


def _bytes(t):
    return t.view(torch.uint8)


def _plain_quantize(state):
    case, s = state["case"], state
    if case["form"] == "weights":
        codes, scales = _plain_weights(s["w"])
        codes_t, scales_t = _plain_weights(s["w"].transpose(1, 2).contiguous())
        return dict(codes=codes, scales=scales, codes_t=codes_t, scales_t=scales_t)
    if case["form"] == "columns":
        codes, scales = _plain_columns(s["x"], s["counts"])
        return dict(codes=codes, scales=scales)
    codes, scales = _plain_rows(s["x"])
    if case["form"] == "rows":
        kept = sum(s["counts"])
        _bytes(s["codes"])[:kept] = _bytes(codes)[:kept]
        _bytes(s["scales"])[:kept] = _bytes(scales)[:kept]
    else:
        # dropped pairs: the rows past the last expert's, which are 0
        T, K = s["slot"].shape
        flat = s["slot"].view(-1)
        pairs = (flat >= 0).nonzero()[:, 0]
        at, token = flat[pairs].long(), pairs // K
        _bytes(s["codes"])[at] = _bytes(codes)[token]
        _bytes(s["scales"])[at] = _bytes(scales)[token]
    return dict(codes=s["codes"], scales=s["scales"])


def _own_product(state):
    from paper_2609_28053_amd import eqb
    case, s = state["case"], state
    eqb.eqb_experts_product(*s["x"], *s["w"], s["offsets"], s["out"])
    if case["form"] == "rows":
        return dict(out=s["out"])
    eqb.eqb_experts_product(*s["g"], *s["w_t"], s["offsets"], s["grad_x"])
    eqb.eqb_experts_grad_weight(*s["g_t"], *s["x_t"], s["offsets"], s["grad_w"])
    return dict(out=s["out"], grad_x=s["grad_x"], grad_w=s["grad_w"])


def _values(codes, scales, width):
    """What codes [rows, .] with scales for blocks of a row stand for, `width` of each row."""
    e = (_bytes(scales).to(torch.int32) - 127)[:, :codes.shape[1] // BLOCK]
    return torch.ldexp(codes.to(torch.float32).view(codes.shape[0], -1, BLOCK), e[..., None]).view(codes.shape)[:, :width]


def _expert_values(codes, scales, width):
    return _values(codes, _bytes(scales).repeat_interleave(BLOCK, 0)[:codes.shape[0]], width)


def _plain_rows_product(x, w, counts, width, out):
    kept = sum(counts)
    a = _values(x[0][:kept], x[1][:kept], width)
    # an expert without rows has no product
    parts = [p @ _expert_values(w[0][e], w[1][e], width).t() for e, p in enumerate(a.split(counts)) if len(p)]
    if parts:
        out[:kept] = torch.cat(parts).to(out.dtype)
    return out


def _plain_product(state):
    case, s = state["case"], state
    N, H, counts = case["N"], case["H"], s["counts"]
    out = _plain_rows_product(s["x"], s["w"], counts, H, s["out"])
    if case["form"] == "rows":
        return dict(out=out)
    grad_x = _plain_rows_product(s["g"], s["w_t"], counts, N, s["grad_x"])
    g, x = _values(*s["g_t"], None), _values(*s["x_t"], None)
    starts = _starts(counts, case["T"] * case["K"])[0]
    grad_w = torch.stack([g[:, a:a + n] @ x[:, a:a + n].t() for a, n in zip(starts, counts)])
    return dict(out=out, grad_x=grad_x, grad_w=grad_w)


def _own_gated(state):
    from paper_2609_28053_amd import eqb
    case, s = state["case"], state
    count = s["offsets"][-1:]
    if case["form"] == "codes":
        eqb.eqb_gated_quantize(s["x"], s["codes"], s["scales"], count)
        return dict(codes=s["codes"], scales=s["scales"])
    eqb.eqb_gated(s["x"], s["h"], count)
    eqb.eqb_gated_backward(s["grad_h"], s["x"], s["grad_x"], count)
    return dict(h=s["h"], grad_x=s["grad_x"])


def _plain_gated(state):
    case, s = state["case"], state
    H, kept = case["H"], sum(s["counts"])
    x = s["x"][:kept].to(torch.float32)
    gate, up = x[:, :H], x[:, H:]
    sig = 1 / (1 + torch.exp(-gate))
    h = gate * sig * up
    if case["form"] == "codes":
        codes, scales = _plain_rows(h)
        _bytes(s["codes"])[:kept] = _bytes(codes)
        _bytes(s["scales"])[:kept] = _bytes(scales)
        return dict(codes=s["codes"], scales=s["scales"])
    s["h"][:kept] = h.to(s["h"].dtype)
    gh = s["grad_h"][:kept].to(torch.float32)
    s["grad_x"][:kept, :H] = (gh * up * sig * (1 + gate * (1 - sig))).to(s["h"].dtype)
    s["grad_x"][:kept, H:] = (gh * gate * sig).to(s["h"].dtype)
    return dict(h=s["h"], grad_x=s["grad_x"])


# --------------------------------------------------------------- the floors --
def work(case):
    kind, E = case["kind"], case["E"]
    if kind == "route":
        T, K, size = case["T"], case["K"], SIZE[case["dtype"]]
        some = 4 * E if case["bias"] != "none" else 0
        got = dict(bytes=T * (E * size + 8 * K) + some, flops=T * E * 6)
        if case["grad"]:
            # the chosen logits, or all of them where the softmax's other experts have gradients too
            dense = case["score"] == "softmax" and not case["normalize"]
            got["bytes"] += T * ((E if dense else K) * size + 8 * K + 4 * E)
            got["flops"] += T * (E * 6 if dense else K * 10)
        return got
    if kind == "quantize" and case["form"] == "weights":
        n = E * case["N"] * case["H"]
        return dict(bytes=n * (SIZE[case["dtype"]] + 2) + 2 * n // BLOCK ** 2, flops=3 * n)
    T, K, H = case["T"], case["K"], case["H"]
    pairs = int(T * K * (1 - case["drop"]))
    if kind == "quantize":
        read = (T if case["form"] == "dispatch" else pairs) * H * SIZE[case["dtype"]]
        some = 4 * T * K if case["form"] == "dispatch" else 4 * (E + 1)
        return dict(bytes=read + pairs * H + pairs * H // BLOCK + some, flops=3 * pairs * H)
    if kind == "gated":
        size = SIZE[case["dtype"]]
        if case["form"] == "codes":
            return dict(bytes=pairs * H * (2 * size + 1) + pairs * H // BLOCK, flops=10 * pairs * H)
        return dict(bytes=pairs * H * size * (3 + 5), flops=25 * pairs * H)
    N, size = case["N"], SIZE[case["dtype"]]
    # the weights of the experts that rows go to
    weights = min(E, pairs) * N * H
    got = dict(bytes=pairs * (H + H // BLOCK) + weights + pairs * N * size, flops=2 * pairs * N * H)
    if case["form"] == "train":
        got["bytes"] += pairs * (N + N // BLOCK) + weights + pairs * H * size
        got["bytes"] += pairs * (N + H) + pairs * (N + H) // BLOCK + 4 * E * N * H
        got["flops"] *= 3
    return got


# ------------------------------------------------------ the values in 64 bits --
def exact(case, seed):
    if case["kind"] == "product" and work(case)["flops"] > 1e13:
        return None
    return {"route": _exact_route, "quantize": _exact_quantize, "product": _exact_product, "gated": _exact_gated}[case["kind"]](case, seed)


def _exact_route(case, seed):
    s = _prepare_route(case, seed)
    T, E, K, G = case["T"], case["E"], case["K"], case["groups"]
    idx = torch.full((T, K), -1, dtype=torch.int32, device=DEV)
    weight = torch.zeros((T, K), dtype=torch.float64, device=DEV)
    grad = torch.zeros((T, E), dtype=torch.float64, device=DEV)
    for t0 in range(0, T, CHUNK):
        z = s["z"][t0:t0 + CHUNK].double()
        n = len(z)
        row = torch.arange(n, device=DEV)
        p = torch.sigmoid(z) if case["score"] == "sigmoid" else torch.softmax(z, 1).nan_to_num(0.0)
        q = p + (0.0 if s["bias"] is None else s["bias"].double())
        q[z == -math.inf] = -math.inf

        def largest(v):
            top = v.amax(1)
            return top, torch.where(v == top[:, None], torch.arange(v.shape[1], device=DEV), v.shape[1]).amin(1)

        groups = torch.zeros((n, G), dtype=torch.float64, device=DEV)
        for j in range(G):
            mine = q[:, j * (E // G):(j + 1) * (E // G)].clone()
            for k in range(case["pair"]):
                top, at = largest(mine)
                groups[:, j] += torch.where(top == -math.inf, -math.inf if k == 0 else 0.0, top)
                mine[row, at] = -math.inf
        allowed = torch.zeros((n, G), dtype=torch.bool, device=DEV)
        for _ in range(case["keep"]):
            at = largest(torch.where(allowed, -math.inf, groups))[1]
            # where the rest are all empty it does not matter which
            allowed[row, at] = True
        q[~allowed.repeat_interleave(E // G, 1)] = -math.inf
        pick = torch.zeros((n, E), dtype=torch.bool, device=DEV)
        for k in range(K):
            top, at = largest(q)
            ok = top > -math.inf
            idx[t0:t0 + n, k] = torch.where(ok, at, -1).to(torch.int32)
            weight[t0:t0 + n, k] = torch.where(ok, p[row, at], 0.0)
            pick[row, at] |= ok
            q[row, at] = -math.inf
        chosen = p * pick
        S = chosen.sum(1, keepdim=True)
        if case["normalize"]:
            weight[t0:t0 + n] = (weight[t0:t0 + n] / S).nan_to_num(0.0)
        if case["grad"]:
            g = torch.zeros((n, E), dtype=torch.float64, device=DEV)
            for k in range(K):
                i = idx[t0:t0 + n, k].long()
                on = (i >= 0).nonzero()[:, 0]
                g[on, i[on]] = s["grad_weight"][t0:t0 + n][on, k].double()
            if case["normalize"]:
                g = torch.where(pick, ((g - (g * chosen).sum(1, keepdim=True) / S) / S).nan_to_num(0.0), 0.0)
            if case["score"] == "sigmoid":
                grad[t0:t0 + n] = g * chosen * torch.sigmoid(-z)
            else:
                grad[t0:t0 + n] = p * (g - (g * chosen).sum(1, keepdim=True))
    out = dict(idx=idx, weight=SCALE * weight)
    return dict(out, grad_z=SCALE * grad) if case["grad"] else out


def _exact_codes(v):
    """Codes (as values) and scales of the blocks along the last axis."""
    top = v.abs().amax(-1)
    e = torch.ceil(torch.log2(top / LARGEST)).clamp(min=-126)
    y = v * torch.exp2(-e)[..., None]
    unit = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / unit) * unit, e


def _exact_scales(e):
    out = torch.full((*e.shape[:-1], _up(e.shape[-1], 4)), 2.0 ** -127, dtype=torch.float64, device=DEV)
    out[..., :e.shape[-1]] = torch.exp2(e)
    return out


def _exact_rows(x):
    R, H = x.shape
    v = torch.zeros((R, _up(H)), dtype=torch.float64, device=DEV)
    v[:, :H] = x
    y, e = _exact_codes(v.view(R, -1, BLOCK))
    return y.view(R, -1), _exact_scales(e)


def _exact_quantize(case, seed):
    s = _prepare_quantize(case, seed)
    H = case["H"]
    if case["form"] == "weights":
        got = {}
        E, N = case["E"], case["N"]
        for t, rows, wide in (("", N, H), ("_t", H, N)):
            codes = torch.zeros((E, rows, _up(wide)), dtype=torch.float64, device=DEV)
            scales = torch.zeros((E, _up(rows) // BLOCK, _scale_width(wide)), dtype=torch.float64, device=DEV)
            for e in range(E):
                v = torch.zeros((_up(rows), _up(wide)), dtype=torch.float64, device=DEV)
                v[:rows, :wide] = s["w"][e].t() if t else s["w"][e]
                tiles = v.view(-1, BLOCK, _up(wide) // BLOCK, BLOCK).transpose(1, 2)
                y, x = _exact_codes(tiles.reshape(*tiles.shape[:2], BLOCK * BLOCK))
                codes[e] = y.view(tiles.shape).transpose(1, 2).reshape(v.shape)[:rows]
                scales[e] = _exact_scales(x)
            got.update({"codes" + t: codes, "scales" + t: scales})
        return got
    if case["form"] == "columns":
        starts, wide = _starts(s["counts"], s["x"].shape[0])
        codes = torch.zeros((H, wide), dtype=torch.float64, device=DEV)
        scales = torch.full((H, _scale_width(wide)), 2.0 ** -127, dtype=torch.float64, device=DEV)
        first = 0
        for a, n in zip(starts, s["counts"]):
            if n:
                y, sc = _exact_rows(s["x"][first:first + n].double().t())
                codes[:, a:a + y.shape[1]] = y
                scales[:, a // BLOCK:a // BLOCK + y.shape[1] // BLOCK] = sc[:, :y.shape[1] // BLOCK]
            first += n
        return dict(codes=codes, scales=scales)
    R = s["codes"].shape[0]
    codes = torch.zeros(s["codes"].shape, dtype=torch.float64, device=DEV)
    scales = torch.full(s["scales"].shape, 2.0 ** -127, dtype=torch.float64, device=DEV)
    y, sc = _exact_rows(s["x"].double())
    if case["form"] == "rows":
        kept = sum(s["counts"])
        codes[:kept], scales[:kept] = y[:kept], sc[:kept]
    else:
        for k in range(case["K"]):
            to = s["slot"][:, k].long()
            on = to >= 0
            codes[to[on]], scales[to[on]] = y[on], sc[on]
    return dict(codes=codes, scales=scales)


def _exact_values(codes, scales):
    return codes.to(torch.float64) * _bytes(scales).double().sub(127).exp2().repeat_interleave(BLOCK, 1)[:, :codes.shape[1]]


def _exact_product(case, seed):
    s = _prepare_product(case, seed)
    train = case["form"] == "train"
    got = {k: torch.zeros(s[k].shape, dtype=torch.float64, device=DEV) for k in (("out", "grad_x", "grad_w") if train else ("out",))}
    starts = _starts(s["counts"], case["T"] * case["K"])[0]
    g_t, x_t = (_exact_values(*s["g_t"]), _exact_values(*s["x_t"])) if train else (None, None)
    first = 0
    for e, n in enumerate(s["counts"]):
        mine = slice(first, first + n)
        first += n
        if not n:
            continue
        for to, x, w in (("out", "x", "w"), ("grad_x", "g", "w_t"))[:2 if train else 1]:
            codes, scales = (t[e] for t in s[w])
            wide = _exact_values(codes, _bytes(scales).repeat_interleave(BLOCK, 0)[:len(codes)].contiguous())
            got[to][mine] = torch.mm(_exact_values(s[x][0][mine], s[x][1][mine]), wide.t())
        if train:
            cols = slice(starts[e], starts[e] + _up(n))
            got["grad_w"][e] = torch.mm(g_t[:, cols], x_t[:, cols].t())
    return got


def _exact_gated(case, seed):
    s = _prepare_gated(case, seed)
    H, kept = case["H"], sum(s["counts"])
    if case["form"] == "codes":
        codes = torch.zeros(s["codes"].shape, dtype=torch.float64, device=DEV)
        scales = torch.full(s["scales"].shape, 2.0 ** -127, dtype=torch.float64, device=DEV)
    else:
        h = torch.zeros(s["h"].shape, dtype=torch.float64, device=DEV)
        grad_x = torch.zeros(s["grad_x"].shape, dtype=torch.float64, device=DEV)
    for r0 in range(0, kept, CHUNK):
        at = slice(r0, min(kept, r0 + CHUNK))
        x = s["x"][at].double()
        gate, up = x.split(H, 1)
        act = torch.sigmoid(gate)
        if case["form"] == "codes":
            codes[at], scales[at] = _exact_rows(gate * act * up)
            continue
        h[at] = gate * act * up
        gh = s["grad_h"][at].double()
        grad_x[at, :H] = gh * up * (act + gate * act * torch.sigmoid(-gate))
        grad_x[at, H:] = gh * gate * act
    return dict(codes=codes, scales=scales) if case["form"] == "codes" else dict(h=h, grad_x=grad_x)
