"""What the library does around a layer's experts besides routing, as cases that can be prepared, run and compared.

The experts' rows lie in buffers [E, C, d] as `dispatch_tokens` fills them: expert j's are the first expert_offsets[j+1] - expert_offsets[j]
of its C, the rest is zero on the way in and out.  The operators:

  products   y = x . W of every expert's rows, their gradients with respect to x and W
  swiglu     the gated unit [g | u] = x . W, h = u * silu(g), and its gradient
  combine    the gradient of the gate-weighted sum of the experts' rows, with respect to the rows and to the gates
  mxfp4      rows in blocks of 32 four-bit numbers with a common power of two, and the products of such rows and weights
"""
import math

import torch

own = False

DEVICE = "cuda:0"


def _case(name, kind, T, d, E, k, factor, n, dtype="bf16", bias="zipf", transposed=False):
    """`factor`: the experts' capacity over T*k/E.  `n`: the experts' inner width.  `transposed`: weights of [E, out, in], not [E, in, out]."""
    case = dict(kind=kind, T=T, d=d, E=E, k=k, factor=factor, n=n, dtype=dtype, bias=bias, transposed=transposed)
    return dict(case, name=name) if name else case


def listed():
    return [
        # the smallest call anyone makes: a unit test, an interactive request
        _case("products 64 tokens, fp32", "products", 64, 64, 8, 2, 1.0, 128, dtype="fp32", bias="none"),
        # one training batch through a coarse top-2 layer's inner product, weights as linear layers keep them
        _case("products 4096 tokens, top 2 of 16", "products", 4096, 1024, 16, 2, 1.0, 1024, bias="normal", transposed=True),
        # the same products' backward pass at the size of a fine-grained training layer: dx and dW
        _case("products backward 16384 tokens", "products_backward", 16384, 2048, 64, 8, 1.0, 1024),
        # widths and counts that fit no tile, fp32 throughout
        _case("products 10007 tokens, fp32, ragged", "products", 10007, 1000, 96, 6, 1.1, 500, dtype="fp32", bias="normal"),
        # a serving step: a few hundred sequences decode one token each; the weights are all there is to read
        _case("swiglu 256 tokens, 64 experts", "swiglu", 256, 2048, 64, 8, 1.25, 1024),
        # prefill or training with capacity to spare, keeping what the backward pass needs; the most work of all
        _case("swiglu 32768 tokens, room to spare", "swiglu_train", 32768, 2048, 64, 8, 1.25, 1024, bias="none"),
        # the gated unit's backward pass
        _case("swiglu backward 16384 tokens", "swiglu_backward", 16384, 2048, 64, 8, 1.0, 1024),
        # from the layer's result back to the experts' rows: a small fine-tuning batch, and the largest layer
        _case("combine backward 256 tokens", "combine_backward", 256, 2048, 64, 8, 1.25, 1024),
        _case("combine backward 65536 tokens", "combine_backward", 65536, 2048, 128, 8, 1.0, 1024),
        # the inner weights of a fine-grained layer's experts, once per load of a model
        _case("mxfp4 weights of 64 experts", "quantise", 64 * 1024, 2048, 1, 1, 1.0, 1024, bias="none"),
        # the serving step with rows and weights in four bits; the rows are quantised on the way
        _case("mxfp4 swiglu 256 tokens, 64 experts", "mxfp4_swiglu", 256, 2048, 64, 8, 1.25, 1024),
        # the outer product of a prefill batch in four bits
        _case("mxfp4 products 16384 tokens", "mxfp4_products", 16384, 1024, 64, 8, 1.0, 2048),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi, step):
    """A width between lo and hi: mostly a multiple of 64, else of `step`."""
    step = 64 if rng.random() < 0.7 else step
    return max(step, step * round(_log_uniform(rng, lo, hi) / step))


def draw(rng):
    """A case of the same ranges: one token or tens of thousands, expert counts on and off the powers of two, widths on and off the tiles."""
    kind = rng.choice(("products", "products", "products_backward", "products_backward", "swiglu", "swiglu", "swiglu_train", "swiglu_backward",
                       "combine_backward", "combine_backward", "quantise", "mxfp4_swiglu", "mxfp4_products"))
    if kind == "quantise":
        rows = _log_uniform(rng, 1, 65536)
        return _case(None, kind, rows, 32 * rng.randint(1, 64), 1, 1, 1.0, 64, dtype=rng.choice(("bf16", "fp32")), bias="none")
    mx = kind.startswith("mxfp4")
    dtype = "bf16" if mx else rng.choices(("bf16", "fp32"), (4, 1))[0]
    E = rng.choice((1, 8, 16, 20, 32, 48, 64, 64, 96, 128))
    k = min(E, rng.choice((1, 2, 2, 4, 6, 8)))
    step = 32 if mx else rng.choice((8, 8, 8, 1))       # now and then rows that are no whole number of 16 bytes
    d = _width(rng, 64, 2048, step)
    n = _width(rng, 64, 1024, 32 if mx else step)
    factor = rng.choice((1.0, 1.0, 1.1, 1.25, 1.5))
    bias = rng.choice(("none", "normal", "zipf"))
    transposed = not mx and rng.random() < 0.5
    T = _log_uniform(rng, 1, 65536 if kind == "combine_backward" else 32768)
    case = _case(None, kind, T, d, E, k, factor, n, dtype=dtype, bias=bias, transposed=transposed)
    # no more work than the largest listed one; products in fp32 take twenty times as long
    most = {"flops": 1.8e12 if dtype == "bf16" else 9e10, "bytes": 2.6e9}
    while any(work(case)[w] > most[w] for w in most):
        case["T"] = max(1, case["T"] * 2 // 3)
    return case


def _capacity(case):
    return min(case["T"], max(1, math.ceil(case["factor"] * case["T"] * case["k"] / case["E"] - 1e-9)))


def _pairs(case):
    return min(case["T"] * case["k"], case["E"] * _capacity(case))


def _counts(case, gen):
    """Tokens per expert: shares by popularity, what does not fit an expert going to those with room, all pairs placed."""
    E, C, left = case["E"], _capacity(case), _pairs(case)
    if case["bias"] == "none":
        share = torch.ones(E, dtype=torch.float64)
    elif case["bias"] == "normal":
        share = torch.exp(torch.randn(E, generator=gen, dtype=torch.float64) * math.sqrt(0.5))
    else:
        share = (torch.arange(1, E + 1, dtype=torch.float64) ** -1.2)[torch.randperm(E, generator=gen)]
    share = share * torch.exp(0.05 * torch.randn(E, generator=gen, dtype=torch.float64))
    counts = [0] * E
    while left > 0:
        open_ = [j for j in range(E) if counts[j] < C]
        total = sum(float(share[j]) for j in open_)
        give = {j: min(C - counts[j], int(left * float(share[j]) / total)) for j in open_}
        if not any(give.values()):
            give = {j: 1 for j in sorted(open_, key=lambda j: -float(share[j]))[:left]}
        for j, g in give.items():
            counts[j] += g
        left -= sum(give.values())
    return torch.tensor(counts, dtype=torch.int32)


def _offsets(counts):
    return torch.cat([torch.zeros(1, dtype=torch.int32), counts.cumsum(0).to(torch.int32)]).to(DEVICE)


def _filled(offsets, C):
    """[E, C, 1]: whether a place of the buffers holds a row."""
    return (torch.arange(C, device=DEVICE)[None, :] < (offsets[1:] - offsets[:-1])[:, None])[..., None]


def _normal(shape, gen, dtype, scale=1.0):
    out = torch.empty(shape, device=DEVICE, dtype=dtype)
    for part in out.view(-1).split(1 << 28):            # normal numbers are made in 32 bits
        part.copy_(torch.randn(part.shape, generator=gen, device=DEVICE).mul_(scale))
    return out


def _pack_mxfp4(x):
    """Weights as they lie in memory: codes, two to a byte (the first one low), and the blocks' exponents + 127."""
    values, exponents = _mxfp4(x)
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=x.device)
    code = torch.bucketize(values.abs(), grid).to(torch.uint8) + 8 * (values < 0).to(torch.uint8)
    code = code.reshape(*x.shape[:-1], x.shape[-1] // 2, 2)
    return code[..., 0] + 16 * code[..., 1], (exponents + 127).to(torch.uint8)


def prepare(case, seed):
    gen, host = torch.Generator(device=DEVICE).manual_seed(seed), torch.Generator().manual_seed(seed)
    kind, T, d, E, k, n = (case[w] for w in ("kind", "T", "d", "E", "k", "n"))
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    if kind == "quantise":
        # rows of different sizes, as weights of different inputs have
        x = _normal((T, d), gen, dtype, 1 / math.sqrt(d))
        return dict(case=case, x=x.mul_(torch.exp(torch.randn(T, 1, generator=gen, device=DEVICE)).to(dtype)))
    C, counts = _capacity(case), _counts(case, host)
    offsets = _offsets(counts)
    state = dict(case=case, offsets=offsets)
    rows = lambda width: _normal((E, C, width), gen, dtype).mul_(_filled(offsets, C))  # noqa: E731
    if kind == "combine_backward":
        # a token's experts are distinct: pair p of those sorted by expert is token p modulo T's, and no expert has more than T
        p = torch.arange(_pairs(case), device=DEVICE)
        expert = torch.repeat_interleave(torch.arange(E, device=DEVICE), counts.to(DEVICE))
        token = torch.randperm(T, generator=gen, device=DEVICE)[p % T]
        order = torch.argsort(expert * T + token)
        pos = torch.empty_like(p)
        pos[order] = p - offsets.long()[expert[order]]
        assign = torch.full((T, k), -1, dtype=torch.int32, device=DEVICE)
        token_pos = torch.zeros((T, k), dtype=torch.int32, device=DEVICE)
        assign[token, p // T], token_pos[token, p // T] = expert.int(), pos.int()
        gates = torch.rand((T, k), generator=gen, device=DEVICE).mul_(2 / k) * (assign >= 0)
        return dict(state, assign=assign, token_pos=token_pos, gates=gates, expert_out=rows(d), dy=torch.randn((T, d), generator=gen, device=DEVICE))
    if kind == "swiglu_backward":
        return dict(state, gate_up=rows(2 * n), dh=rows(n))
    state["x"] = rows(d)
    out = 2 * n if "swiglu" in kind else n
    if kind.startswith("mxfp4"):
        state["wq"], state["ws"] = _pack_mxfp4(_normal((E, out, d), gen, dtype, 1 / math.sqrt(d)))
    else:
        state["w"] = _normal((E, out, d) if case["transposed"] else (E, d, out), gen, dtype, 1 / math.sqrt(d))
    if kind == "products_backward":
        state["dy"] = rows(n)
    return state


def run(state):
    return _own(state) if own else _plain(state)


def _own(state):
    import paper_2508_12801_amd as ms
    case = state["case"]
    kind, offsets, transposed = case["kind"], state.get("offsets"), case["transposed"]
    if kind == "products":
        return dict(y=ms.expert_matmul(state["x"], state["w"], offsets, transposed=transposed))
    if kind == "products_backward":
        x, dy = state["x"], state["dy"]
        dw = ms.expert_matmul_wgrad(dy, x, offsets) if transposed else ms.expert_matmul_wgrad(x, dy, offsets)
        return dict(dx=ms.expert_matmul(dy, state["w"], offsets, transposed=not transposed), dw=dw)
    if kind in ("swiglu", "swiglu_train"):
        r = ms.expert_swiglu(state["x"], state["w"], offsets, transposed=transposed, want_gate_up=kind == "swiglu_train")
        return dict(h=r["h"], gate_up=r["gate_up"]) if kind == "swiglu_train" else dict(h=r["h"])
    if kind == "swiglu_backward":
        r = ms.expert_swiglu_backward(state["gate_up"], state["dh"], offsets)
        return dict(dgate_up=r["dgate_up"], h=r["h"])
    if kind == "combine_backward":
        r = ms.combine_backward(state["dy"], state["expert_out"], state["assign"], state["token_pos"], state["gates"], offsets)
        return dict(dexpert_out=r["dexpert_out"], dgates=r["dgates"])
    xq, xs = ms.mxfp4_quantise(state["x"])
    if kind == "quantise":
        return dict(values=ms.mxfp4_dequantise(xq, xs, dtype=state["x"].dtype))
    product = ms.expert_swiglu_mxfp4 if kind == "mxfp4_swiglu" else ms.expert_matmul_mxfp4
    return dict(y=product(xq, xs, state["wq"], state["ws"], offsets))


def _mxfp4(x):
    """(the four-bit numbers, their blocks' exponents): the largest of a block lies in 4..8 of its power of two, beyond 6 counts as 6."""
    x = x.float().reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    exponents = (torch.frexp(x.abs().amax(-1))[1] - 3).clamp_(min=-127)
    exponents = torch.where(x.abs().amax(-1) == 0, -127, exponents)
    x = torch.ldexp(x, -exponents[..., None])
    a = x.abs()
    # half way between two numbers goes to the one whose last bit is zero
    v = 0.5 * ((a > 0.25).float() + (a >= 0.75) + (a > 1.25) + (a >= 1.75)) + 1.0 * ((a > 2.5).float() + (a >= 3.5)) + 2.0 * (a > 5.0)
    return torch.copysign(v, x).flatten(-2), exponents


def _unpacked(wq, ws):
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=wq.device)
    grid = torch.cat([grid, -grid])
    values = torch.stack([grid[(wq & 15).int()], grid[(wq >> 4).int()]], dim=-1).flatten(-2)
    return _scaled(values, ws.int() - 127)


def _scaled(values, exponents):
    return torch.ldexp(values.reshape(*exponents.shape, 32), exponents[..., None]).flatten(-2)


def _plain(state):
    case = state["case"]
    kind, transposed = case["kind"], case["transposed"]
    if kind == "quantise":
        return dict(values=_scaled(*_mxfp4(state["x"])).to(state["x"].dtype))
    filled = _filled(state["offsets"], _capacity(case))
    rows = lambda t: torch.where(filled, t.float(), 0.0)  # noqa: E731
    if kind == "combine_backward":
        E, C, d = state["expert_out"].shape
        dy, has = state["dy"], state["assign"] >= 0
        place = (state["assign"] * C + state["token_pos"]).long()[has]
        token = torch.nonzero(has)[:, 0]
        dexpert_out = torch.zeros((E * C, d), dtype=state["expert_out"].dtype, device=DEVICE)
        dexpert_out[place] = (state["gates"][has][:, None] * dy[token]).to(dexpert_out.dtype)
        dgates = torch.zeros_like(state["gates"])
        dgates[has] = (state["expert_out"].view(E * C, d)[place].float() * dy[token]).sum(1)
        return dict(dexpert_out=dexpert_out.view(E, C, d), dgates=dgates)
    if kind == "swiglu_backward":
        gate, up = rows(state["gate_up"]).chunk(2, dim=-1)
        dh, s = rows(state["dh"]), 1 / (1 + torch.exp(-gate))
        dgate = dh * up * s * (1 + gate * (1 - s))
        return dict(dgate_up=torch.cat([dgate, dh * gate * s], dim=-1).to(state["dh"].dtype), h=(up * gate * s).to(state["dh"].dtype))
    if kind.startswith("mxfp4"):
        x, w = rows(_scaled(*_mxfp4(state["x"]))), _unpacked(state["wq"], state["ws"]).transpose(1, 2)
    else:
        x, w = rows(state["x"]), state["w"].float()
        w = w.transpose(1, 2) if transposed else w
    dtype = state["x"].dtype
    if kind == "products_backward":
        dy = rows(state["dy"])
        dw = torch.matmul(x.transpose(1, 2), dy)
        return dict(dx=torch.matmul(dy, w.transpose(1, 2)).to(dtype), dw=dw.transpose(1, 2).contiguous() if transposed else dw)
    y = torch.matmul(x, w)
    if "swiglu" not in kind:
        return dict(y=y.to(dtype))
    gate, up = y.chunk(2, dim=-1)
    h = (up * gate / (1 + torch.exp(-gate))).to(dtype)
    return dict(h=h, gate_up=y.to(dtype)) if kind == "swiglu_train" else dict(y=h) if kind == "mxfp4_swiglu" else dict(h=h)


def _rounded_blocks(x):
    """Values of rows in four bits, from the format's definition: one bit behind the leading one, steps of 1/2 below 1, in units of the block's power of two."""
    x = x.double().reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    unit = torch.exp2(torch.floor(torch.log2(x.abs().amax(-1, keepdim=True))).clamp(min=-125.0) - 2)
    m = (x / unit).abs()
    step = torch.exp2(torch.floor(torch.log2(m)).clamp(min=0.0) - 1)
    return (torch.sign(x) * torch.clamp(torch.round(m / step) * step, max=6.0) * unit).flatten(-2)


def _unpacked_blocks(wq, ws):
    code = torch.stack([wq % 16, wq // 16], dim=-1).flatten(-2).long()
    sign, exponent, last = 1.0 - 2.0 * (code // 8), code // 2 % 4, (code % 2).double()
    value = torch.where(exponent == 0, 0.5 * last, torch.exp2(exponent.double() - 1) * (1 + 0.5 * last))
    return sign * value * torch.exp2(ws.double() - 127).repeat_interleave(32, dim=-1)


def exact(case, seed):
    state, kind = prepare(case, seed), case["kind"]
    if kind == "quantise":
        return dict(values=_rounded_blocks(state["x"]))
    offsets = state["offsets"].tolist()
    n_rows = [b - a for a, b in zip(offsets, offsets[1:])]
    if kind == "combine_backward":
        eo, assign, pos = state["expert_out"], state["assign"].long(), state["token_pos"].long()
        dexpert_out = torch.zeros(eo.shape, dtype=torch.float64, device=DEVICE)
        dgates = torch.zeros(assign.shape, dtype=torch.float64, device=DEVICE)
        for s in range(case["k"]):
            at = torch.nonzero(assign[:, s] >= 0)[:, 0]
            for i in at.split(8192):
                e, p, dy = assign[i, s], pos[i, s], state["dy"][i].double()
                dexpert_out[e, p] = state["gates"][i, s].double()[:, None] * dy
                dgates[i, s] = torch.linalg.vecdot(eo[e, p].double(), dy)
        return dict(dexpert_out=dexpert_out, dgates=dgates)
    C = _capacity(case)
    out = {}

    def put(name, j, value, buffer=True):
        if name not in out:
            out[name] = torch.zeros((case["E"], C if buffer else value.shape[0], value.shape[1]), dtype=torch.float64, device=DEVICE)
        out[name][j, :value.shape[0]] = value

    for j, r in enumerate(n_rows):
        if kind == "swiglu_backward":
            n = case["n"]
            g, u, dh = state["gate_up"][j, :r, :n].double(), state["gate_up"][j, :r, n:].double(), state["dh"][j, :r].double()
            s = torch.sigmoid(g)
            put("dgate_up", j, torch.cat([dh * u * (s + g * s * torch.sigmoid(-g)), dh * (g * s)], dim=1))
            put("h", j, g * s * u)
            continue
        if kind.startswith("mxfp4"):
            x, w = _rounded_blocks(state["x"][j, :r]), _unpacked_blocks(state["wq"][j], state["ws"][j]).T
        else:
            x, w = state["x"][j, :r].double(), state["w"][j].double()
            w = w.T if case["transposed"] else w
        if kind == "products_backward":
            dy = state["dy"][j, :r].double()
            put("dx", j, dy @ w.T)
            put("dw", j, dy.T @ x if case["transposed"] else x.T @ dy, buffer=False)
            continue
        y = x @ w
        if "swiglu" not in kind:
            put("y", j, y)
            continue
        g, u = y[:, :case["n"]], y[:, case["n"]:]
        put("y" if kind == "mxfp4_swiglu" else "h", j, torch.nn.functional.silu(g) * u)
        if kind == "swiglu_train":
            put("gate_up", j, y)
    return out


def work(case):
    """Every pair's rows in, every place's rows out, weights once; products count two operations to a multiplication."""
    kind, T, d, E, k, n = (case[w] for w in ("kind", "T", "d", "E", "k", "n"))
    C, P, size = _capacity(case), _pairs(case), 2 if case["dtype"] == "bf16" else 4
    four = 0.5 + 1 / 32
    if kind == "quantise":
        return {"bytes": T * d * (2 * size), "flops": 4 * T * d}
    if kind == "combine_backward":
        return {"bytes": 4 * T * d + P * d * size + E * C * d * size + 4 * 4 * T * k, "flops": 3 * P * d}
    if kind == "swiglu_backward":
        return {"bytes": (3 * P + 3 * E * C) * n * size, "flops": 12 * P * n}
    if kind == "products":
        return {"bytes": (P * d + E * d * n + E * C * n) * size, "flops": 2 * P * d * n}
    if kind == "products_backward":
        return {"bytes": (2 * P * n + P * d + E * d * n + E * C * d) * size + 4 * E * d * n, "flops": 4 * P * d * n}
    if kind == "mxfp4_products":
        return {"bytes": int(P * d * 2 + E * d * n * four + E * C * n * 2), "flops": 2 * P * d * n}
    if kind == "mxfp4_swiglu":
        return {"bytes": int(P * d * 2 + 2 * E * d * n * four + E * C * n * 2), "flops": 4 * P * d * n}
    kept = 3 if kind == "swiglu_train" else 1
    return {"bytes": (P * d + 2 * E * d * n + kept * E * C * n) * size, "flops": 4 * P * d * n}
