"""Cases of the operators on 8-bit floats with scales and on tokens dealt to experts, their plain forms, and their values in 64 bits.

The operators: quantising to 8-bit floats (e4m3) with a scale in 32 bits for each block of 128 numbers of a row, or of 128
rows, and reading them back; a root-mean-square norm with the residual's addition, whose result is such numbers; the
contraction of two such matrices, and of rows sorted by expert with their experts' weights; sorting tokens by expert, spreading
them out and joining them again with weights, and the gradients of that.

`run` computes the plain form with elementary torch operations, or with `own` set calls the framework.
"""

import math

import torch

own = False

# ------------------------------------------------------------------------------------------------
# cases
# ------------------------------------------------------------------------------------------------


def listed():
    return [
        # the hidden states of a few decoded tokens in front of a layer's products: a launch's latency
        {"name": "norm 4x4096 bf16", "op": "norm", "rows": 4, "cols": 4096, "dtype": "bfloat16", "residual": True},
        # those of a long prompt
        {"name": "norm 16384x8192 bf16", "op": "norm", "rows": 16384, "cols": 8192, "dtype": "bfloat16", "residual": True},
        # what attention gives for a short prompt, on its way into a projection; rows end inside a block
        {"name": "quantize 513x4104 bf16", "op": "quantize", "rows": 513, "cols": 4104, "dtype": "bfloat16", "block_rows": 1},
        # a weight matrix converted once; blocks at its edges are short
        {"name": "quantize 16380x8190 f32", "op": "quantize", "rows": 16380, "cols": 8190, "dtype": "float32", "block_rows": 128},
        # one decoded token through a projection: the weights are read once
        {"name": "dot 1x8192x8192", "op": "dot", "m": 1, "n": 8192, "k": 8192, "block_rows": 128},
        # a prompt of odd length through a projection whose sizes fill neither tiles nor blocks
        {"name": "dot 333x5000x4104", "op": "dot", "m": 333, "n": 5000, "k": 4104, "block_rows": 128},
        # the framework's largest dense product, in this format
        {"name": "dot 8192x8192x8192", "op": "dot", "m": 8192, "n": 8192, "k": 8192, "block_rows": 128},
        # a few decoded tokens through their experts: most of the experts that they meet have a row each
        {"name": "experts 8x2 of 64", "op": "experts", "tokens": 8, "choices": 2, "experts": 64, "n": 2048, "k": 4096, "gather": True},
        # a prompt through its experts, some of which have several times the rows that others have
        {"name": "experts 8192x2 of 16", "op": "experts", "tokens": 8192, "choices": 2, "experts": 16, "n": 4096, "k": 4096, "gather": True},
        # a batch of decoded tokens sorted, spread out and joined: latency
        {"name": "tokens 32x4 of 64", "op": "tokens", "tokens": 32, "choices": 4, "experts": 64, "cols": 4096, "dtype": "bfloat16",
         "dropped": False, "grad": False},
        # a prompt's, with places that overflowed
        {"name": "tokens 16384x4 of 128", "op": "tokens", "tokens": 16384, "choices": 4, "experts": 128, "cols": 4096, "dtype": "bfloat16",
         "dropped": True, "grad": False},
        # a training step's way back, odd sizes
        {"name": "tokens 8191x6 of 160, grad", "op": "tokens", "tokens": 8191, "choices": 6, "experts": 160, "cols": 2050, "dtype": "bfloat16",
         "dropped": True, "grad": True},
    ]


def _spread(rng, low, high):
    """A whole number whose logarithm is spread evenly, odd ones and multiples of 128 among them."""
    n = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    if rng.random() < 0.4 and n >= 256:
        n = n // 128 * 128
    return max(low, min(high, n))


def draw(rng):
    op = rng.choice(["norm", "quantize", "dot", "experts", "tokens"])
    while True:
        if op == "norm":
            case = {"op": op, "rows": _spread(rng, 1, 32768), "cols": _spread(rng, 1, 16384), "dtype": rng.choice(["bfloat16", "float32"]),
                    "residual": rng.random() < 0.7}
            if case["rows"] * case["cols"] > 1 << 26:
                continue
        elif op == "quantize":
            case = {"op": op, "rows": _spread(rng, 1, 32768), "cols": _spread(rng, 1, 16384), "dtype": rng.choice(["bfloat16", "float32"]),
                    "block_rows": rng.choice([1, 1, 128])}
            if case["rows"] * case["cols"] > 1 << 26:
                continue
        elif op == "dot":
            case = {"op": op, "m": _spread(rng, 1, 8192), "n": _spread(rng, 16, 16384), "k": _spread(rng, 16, 16384),
                    "block_rows": rng.choice([128, 128, 128, 1])}
            if case["m"] * case["n"] * case["k"] > 1 << 38:
                continue
        elif op == "experts":
            case = {"op": op, "tokens": _spread(rng, 1, 8192), "choices": rng.choice([1, 2, 4, 6, 8]), "experts": rng.choice([8, 16, 60, 64, 128]),
                    "n": _spread(rng, 64, 8192), "k": _spread(rng, 64, 8192), "gather": rng.random() < 0.5}
            if case["experts"] * case["n"] * case["k"] > 1 << 28:
                continue
            if case["tokens"] * case["choices"] * case["n"] * case["k"] > 1 << 38 or case["tokens"] * case["choices"] * max(case["n"], case["k"]) > 1 << 26:
                continue
        else:
            case = {"op": op, "tokens": _spread(rng, 1, 16384), "choices": rng.choice([1, 2, 4, 6, 8]), "experts": rng.choice([8, 16, 60, 64, 128, 256]),
                    "cols": _spread(rng, 8, 8192), "dtype": rng.choice(["bfloat16", "bfloat16", "float32"]), "dropped": rng.random() < 0.5,
                    "grad": rng.random() < 0.5}
            if case["tokens"] * case["choices"] * case["cols"] > 1 << 27:
                continue
        return case


def _size(case):
    return 2 if case["dtype"] == "bfloat16" else 4


def _f8_bytes(rows, cols, block_rows):
    return rows * cols + 4 * -(-rows // block_rows) * -(-cols // 128)


def _popular(case):
    """A quarter of the tokens choose among so many experts, the others among all."""
    return max(case["choices"], case["experts"] // 4)


def _loads(case):
    """Rows of each expert, before experts are renamed: in either group of tokens choices go round."""
    loads = [0] * case["experts"]
    few = -(-case["tokens"] // 4)
    for pool, tokens in ((_popular(case), few), (case["experts"], case["tokens"] - few)):
        each, more = divmod(tokens * case["choices"], pool)
        for e in range(pool):
            loads[e] += each + (e < more)
    return loads


def work(case):
    op = case["op"]
    if op == "norm":
        n = case["rows"] * case["cols"]
        return {"bytes": (1 + 2 * case["residual"]) * n * _size(case) + case["cols"] * _size(case) + _f8_bytes(case["rows"], case["cols"], 1), "flops": 6 * n}
    if op == "quantize":
        n = case["rows"] * case["cols"]
        return {"bytes": 2 * n * _size(case) + _f8_bytes(case["rows"], case["cols"], case["block_rows"]), "flops": 4 * n}
    if op == "dot":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": _f8_bytes(m, k, 1) + _f8_bytes(n, k, case["block_rows"]) + 2 * m * n, "flops": 2 * m * n * k}
    rows = case["tokens"] * case["choices"]
    if op == "experts":
        n, k, met = case["n"], case["k"], sum(load > 0 for load in _loads(case))
        return {"bytes": _f8_bytes(case["tokens"] if case["gather"] else rows, k, 1) + met * _f8_bytes(n, k, 128) + 2 * rows * n, "flops": 2 * rows * n * k}
    spread, flat = rows * case["cols"] * _size(case), case["tokens"] * case["cols"] * _size(case)
    if case["grad"]:            # the joined gradient, rows and weights in, the rows', weights' and tokens' gradients out
        return {"bytes": 2 * flat + 2 * spread + 12 * rows, "flops": 4 * rows * case["cols"]}
    return {"bytes": 2 * flat + spread + 16 * rows + 4 * case["experts"], "flops": 2 * rows * case["cols"]}


# ------------------------------------------------------------------------------------------------
# the format, in elementary operations
# ------------------------------------------------------------------------------------------------
# Rows of K numbers are ceil(K / 128) blocks of 128 codes, zeros behind K; scales (..., rows / block_rows, blocks), rows of
# them filled up with zeros to multiples of 4.

_LEAST = 2.0 ** -126
_UNIT = 1.0 / 448.0                      # of the largest code; rounded to 32 bits where it is used


def _encode(x, block_rows):
    """(..., rows, K) in 32 bits -> codes (..., rows, blocks, 128) as float8_e4m3fn, scales in 32 bits."""
    rows, k = x.shape[-2:]
    x = torch.nn.functional.pad(x.float(), (0, -k % 128)).unflatten(-1, (-1, 128))
    top = x.abs().amax(-1)                                                # (..., rows, blocks)
    if block_rows > 1:
        top = torch.nn.functional.pad(top, (0, 0, 0, -rows % block_rows)).unflatten(-2, (-1, block_rows)).amax(-2)
    scale = (top * torch.tensor(_UNIT, dtype=torch.float32, device=x.device)).clamp(min=_LEAST)
    factor = scale.double().reciprocal().float()
    code = (x * _per_row(factor, rows, block_rows).unsqueeze(-1)).to(torch.float8_e4m3fn)
    return code, torch.nn.functional.pad(scale, (0, -scale.shape[-1] % 4))


def _per_row(scale, rows, block_rows):
    """Scales (..., rows / block_rows, blocks) -> (..., rows, blocks)."""
    return scale if block_rows == 1 else scale.repeat_interleave(block_rows, -2)[..., :rows, :]


def _values(code, scale, cols, block_rows):
    """Codes (..., rows, blocks, 128) and scales -> values (..., rows, cols) in 32 bits."""
    scale = _per_row(scale[..., :code.shape[-2]], code.shape[-3], block_rows)
    return (code.float() * scale.unsqueeze(-1)).flatten(-2)[..., :cols]


# ------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------


def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda")


def _activations(gen, rows, cols):
    """Rows as a network has them: a few of the columns are much larger than the others."""
    x = _normal(gen, rows, cols)
    loud = torch.rand(cols, generator=gen, device="cuda") < 0.01
    return x * torch.where(loud, 20.0, 1.0)


def _chosen(gen, case):
    """Experts (tokens, choices) of every token, each another one, as _loads counts them."""
    tokens, choices = case["tokens"], case["choices"]
    few = -(-tokens // 4)
    at = torch.arange(tokens, device="cuda")
    first = torch.where(at < few, at, at - few) * choices
    pool = torch.where(at < few, _popular(case), case["experts"]).unsqueeze(1)
    chosen = (first.unsqueeze(1) + torch.arange(choices, device="cuda")) % pool
    name = torch.randperm(case["experts"], generator=gen, device="cuda")
    order = torch.randperm(tokens, generator=gen, device="cuda")
    return name[chosen][order].to(torch.int32)


def _sort(chosen, experts):
    """Offsets of every expert's rows, each row's token (-1 behind the last), each choice's row (-1: dropped)."""
    flat = chosen.flatten().long()
    key = torch.where((flat >= 0) & (flat < experts), flat, experts)
    order = torch.argsort(key, stable=True)
    row = torch.empty_like(order)
    row[order] = torch.arange(order.numel(), device="cuda")
    ends = (key.unsqueeze(0) < torch.arange(experts + 1, device="cuda").unsqueeze(1)).sum(1)
    tokens = torch.where(torch.arange(order.numel(), device="cuda") < ends[-1], order // chosen.shape[1], -1)
    places = torch.where(key < experts, row, -1).view(chosen.shape)
    return ends.to(torch.int32), tokens.to(torch.int32), places.to(torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op = case["op"]
    if op == "norm":
        dtype = getattr(torch, case["dtype"])
        x = _activations(gen, case["rows"], case["cols"]).to(dtype)
        residual = (_normal(gen, case["rows"], case["cols"]) * 3.0).to(dtype) if case["residual"] else None
        return {"case": case, "x": x, "residual": residual, "weight": (1.0 + 0.2 * _normal(gen, case["cols"])).to(dtype), "eps": 1e-6}
    if op == "quantize":
        return {"case": case, "x": _activations(gen, case["rows"], case["cols"]).to(getattr(torch, case["dtype"]))}
    if op == "dot":
        m, n, k = case["m"], case["n"], case["k"]
        return {"case": case, "x": _encode(_activations(gen, m, k), 1), "w": _encode(_normal(gen, n, k) / math.sqrt(k), case["block_rows"]),
                "out": torch.empty(m, n, dtype=torch.bfloat16, device="cuda")}
    tokens, choices, experts = case["tokens"], case["choices"], case["experts"]
    rows = tokens * choices
    chosen = _chosen(gen, case)
    if op == "experts":
        n, k = case["n"], case["k"]
        offsets, token_of, _ = _sort(chosen, experts)
        x = _encode(_activations(gen, tokens if case["gather"] else rows, k), 1)
        return {"case": case, "x": x, "w": _encode(_normal(gen, experts, n, k) / math.sqrt(k), 128), "offsets": offsets,
                "tokens": token_of if case["gather"] else None, "out": torch.empty(rows, n, dtype=torch.bfloat16, device="cuda")}
    if case["dropped"]:
        chosen.view(-1)[5::16] = -1
    dtype = getattr(torch, case["dtype"])
    weights = torch.softmax(_normal(gen, tokens, choices), -1)
    state = {"case": case, "weights": weights, "spread": torch.zeros(rows, case["cols"], dtype=dtype, device="cuda")}
    if case["grad"]:
        return {**state, "places": _sort(chosen, experts)[2], "rows": _normal(gen, rows, case["cols"]).to(dtype),
                "grad": _normal(gen, tokens, case["cols"]).to(dtype)}
    return {**state, "chosen": chosen, "x": _normal(gen, tokens, case["cols"]).to(dtype)}


# ------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------


def _run_own(state):
    from paper_2105_09377_amd import binding as gs
    case = state["case"]
    op = case["op"]
    if op == "norm":
        y, total = gs.f8_norm(state["x"], state["weight"], residual=state["residual"], eps=state["eps"])
        return (y.values, y.scales, total) if case["residual"] else (y.values, y.scales)
    if op == "quantize":
        return gs.f8_dequantize(gs.f8_quantize(state["x"], block_rows=case["block_rows"]), out_dtype=state["x"].dtype)
    if op == "dot":
        x = gs.F8(*state["x"], (case["m"], case["k"]), 1, 1)
        w = gs.F8(*state["w"], (case["n"], case["k"]), 1, case["block_rows"])
        return gs.f8_dot(x, w, out=state["out"])
    if op == "experts":
        x = gs.F8(*state["x"], (state["x"][0].shape[0], case["k"]), 1, 1)
        w = gs.F8(*state["w"], (case["experts"], case["n"], case["k"]), 2, 128)
        return gs.f8_expert_dot(x, w, state["offsets"], tokens=state["tokens"], out=state["out"])
    if case["grad"]:
        rows, weights = gs.expert_join_grad(state["grad"], state["rows"], state["places"], state["weights"], grad_rows=state["spread"])
        return rows, weights, gs.expert_join(rows, state["places"])
    s = gs.expert_sort(state["chosen"], case["experts"])
    rows = gs.expert_split(state["x"], s.places, out=state["spread"])
    return s.offsets, s.tokens, s.places, rows, gs.expert_join(rows, s.places, state["weights"])


def _join(rows, places, weights):
    """Sums of every token's rows, times their weights, in 32 bits."""
    kept = (places >= 0).unsqueeze(-1)
    part = torch.where(kept, rows[places.long().clamp(min=0)].float(), 0.0)
    return (part if weights is None else part * weights.unsqueeze(-1)).sum(1)


def _by_place(state, places, values):
    """Values (tokens, choices, cols) in the order of their rows; rows that nobody has keep what they hold."""
    at = places.flatten().long()
    rows = torch.cat((state["spread"], state["spread"][:1]))             # one more, for what has no place
    rows[torch.where(at >= 0, at, at.numel())] = values.flatten(0, 1).to(rows.dtype)
    return rows[:-1]


def run(state):
    if own:
        return _run_own(state)
    case = state["case"]
    op = case["op"]
    if op == "norm":
        x = state["x"]
        if case["residual"]:
            x = (x.float() + state["residual"].float()).to(x.dtype)
        # (64 bits: numbers next to a border between two codes)
        wide = x.double()
        y = wide * torch.rsqrt(wide.square().mean(-1, keepdim=True) + state["eps"]) * state["weight"].double()
        code, scale = _encode(y, 1)
        return (code, scale, x) if case["residual"] else (code, scale)
    if op == "quantize":
        return _values(*_encode(state["x"], case["block_rows"]), case["cols"], case["block_rows"]).to(state["x"].dtype)
    if op == "dot":
        w = _values(*state["w"], case["k"], case["block_rows"])
        return torch.matmul(_values(*state["x"], case["k"], 1), w.t()).to(torch.bfloat16)
    if op == "experts":
        # every expert's rows in a matrix of its own, filled up to as many as the largest has
        x = _values(*state["x"], case["k"], 1)
        if case["gather"]:
            x = x[state["tokens"].long()]
        most, first = max(_loads(case)), state["offsets"][:-1].long()
        row = torch.arange(x.shape[0], device="cuda")
        expert = (row.unsqueeze(1) >= state["offsets"][1:].long()).sum(1)
        at = row - first[expert]
        wide = torch.zeros(case["experts"], most, case["k"], device="cuda")
        wide[expert, at] = x
        w = _values(*state["w"], case["k"], 128).transpose(1, 2).contiguous()
        return torch.bmm(wide, w)[expert, at].to(torch.bfloat16)
    if case["grad"]:
        places, weights = state["places"], state["weights"]
        grad = state["grad"].float().unsqueeze(1)
        kept = (places >= 0).unsqueeze(-1)
        rows = _by_place(state, places, grad * weights.unsqueeze(-1))
        grad_weights = (torch.where(kept, state["rows"][places.long().clamp(min=0)].float(), 0.0) * grad).sum(-1)
        return rows, grad_weights, _join(rows, places, None).to(rows.dtype)
    offsets, token_of, places = _sort(state["chosen"], case["experts"])
    rows = _by_place(state, places, state["x"].unsqueeze(1).expand(-1, case["choices"], -1))
    return offsets, token_of, places, rows, _join(rows, places, state["weights"]).to(rows.dtype)


# ------------------------------------------------------------------------------------------------
# the definitions in 64 bits, apart from the plain form
# ------------------------------------------------------------------------------------------------


def _nearest64(x):
    """The nearest numbers with four bits from 2^-6 on, and multiples of 2^-9 below, ties to even ones; at most 448."""
    _, exponent = torch.frexp(x)
    step = torch.ldexp(torch.ones_like(x), (exponent - 1).clamp(min=-6) - 3)
    return (torch.round(x / step) * step).clamp(-448.0, 448.0)


def _round32(x):
    return x.to(torch.float32).to(torch.float64)


def _blocks64(x, block_rows):
    """(rows, K) -> codes (rows, blocks, 128) and scales (rows / block_rows, blocks), in 64 bits; scale and factor are numbers of 32."""
    rows, k = x.shape
    x = torch.cat((x, x.new_zeros(rows, -k % 128)), 1).reshape(rows, -1, 128)
    top = x.abs().max(2).values
    groups = -(-rows // block_rows)
    top = torch.stack([top[g * block_rows:(g + 1) * block_rows].max(0).values for g in range(groups)]) if block_rows > 1 else top
    unit = _round32(torch.tensor(1.0 / 448.0, dtype=torch.float64, device=x.device))
    scale = torch.maximum(_round32(top * unit), torch.full_like(top, _LEAST))
    of = torch.arange(rows, device=x.device) // block_rows
    return _nearest64(_round32(x * _round32(1.0 / scale)[of].unsqueeze(2))), scale


def _read64(code, scale, cols, block_rows):
    """(rows, blocks, 128) codes, scales -> (rows, cols)."""
    of = torch.arange(code.shape[0], device=code.device) // block_rows
    units = scale.double()[:, :code.shape[1]][of]
    return (code.double() * units.unsqueeze(2)).reshape(code.shape[0], -1)[:, :cols]


def _padded(scale):
    return torch.cat((scale, scale.new_zeros(scale.shape[0], -scale.shape[1] % 4)), 1)


def _places64(chosen, experts):
    """As _sort: a choice's row is what smaller experts have, and what its own had before."""
    flat = chosen.flatten().cpu().tolist()
    counts = [0] * experts
    rank = []
    for e in flat:
        rank.append(counts[e] if 0 <= e < experts else -1)
        if 0 <= e < experts:
            counts[e] += 1
    offsets = [0]
    for c in counts:
        offsets.append(offsets[-1] + c)
    places = [offsets[e] + r if r >= 0 else -1 for e, r in zip(flat, rank)]
    token_of = [-1] * len(flat)
    for i, p in enumerate(places):
        if p >= 0:
            token_of[p] = i // chosen.shape[1]
    return offsets, token_of, places


def exact(case, seed):
    state = prepare(case, seed)
    op = case["op"]
    if op == "norm":
        total = state["x"].double()
        if case["residual"]:
            total = (total + state["residual"].double()).to(state["x"].dtype).double()
        y = total / torch.sqrt((total * total).sum(1, keepdim=True) / case["cols"] + state["eps"]) * state["weight"].double()
        code, scale = _blocks64(_round32(y), 1)
        return (code, _padded(scale), total) if case["residual"] else (code, _padded(scale))
    if op == "quantize":
        return _read64(*_blocks64(state["x"].double(), case["block_rows"]), case["cols"], case["block_rows"])
    if op == "dot":
        return _read64(*state["x"], case["k"], 1) @ _read64(*state["w"], case["k"], case["block_rows"]).t().contiguous()
    if op == "experts":
        x = _read64(*state["x"], case["k"], 1)
        out = torch.zeros(case["tokens"] * case["choices"], case["n"], dtype=torch.float64, device="cuda")
        ends = state["offsets"].tolist()
        for e in range(case["experts"]):
            if ends[e + 1] > ends[e]:
                rows = x[state["tokens"][ends[e]:ends[e + 1]].long()] if case["gather"] else x[ends[e]:ends[e + 1]]
                out[ends[e]:ends[e + 1]] = rows @ _read64(state["w"][0][e], state["w"][1][e], case["k"], 128).t().contiguous()
        return out
    tokens, choices = case["tokens"], case["choices"]
    if case["grad"]:
        places = state["places"].tolist()
        rows = torch.zeros(tokens * choices, case["cols"], dtype=torch.float64, device="cuda")
        grad_weights = torch.zeros(tokens, choices, dtype=torch.float64, device="cuda")
        grad_x = torch.zeros(tokens, case["cols"], dtype=torch.float64, device="cuda")
        for j in range(choices):
            t = torch.tensor([i for i in range(tokens) if places[i][j] >= 0], dtype=torch.int64, device="cuda")
            p = torch.tensor([q[j] for q in places if q[j] >= 0], dtype=torch.int64, device="cuda")
            g = state["grad"][t].double()
            rows[p] = g * state["weights"][t, j].double().unsqueeze(1)
            grad_weights[t, j] = (g * state["rows"][p].double()).sum(1)
            grad_x[t] += rows[p].to(state["grad"].dtype).double()
        return rows, grad_weights, grad_x
    offsets, token_of, places = _places64(state["chosen"], case["experts"])
    place = torch.tensor(places, device="cuda").view(tokens, choices)
    rows = torch.zeros(tokens * choices, case["cols"], dtype=torch.float64, device="cuda")
    joined = torch.zeros(tokens, case["cols"], dtype=torch.float64, device="cuda")
    for j in range(choices):
        t = torch.nonzero(place[:, j] >= 0).squeeze(1)
        rows[place[t, j]] = state["x"][t].double()
        joined[t] += state["x"][t].double() * state["weights"][t, j].double().unsqueeze(1)
    return (torch.tensor(offsets, dtype=torch.int32), torch.tensor(token_of, dtype=torch.int32), torch.tensor(places, dtype=torch.int32).view(tokens, choices),
            rows, joined)
