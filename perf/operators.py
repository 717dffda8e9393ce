"""The work that training and sampling the search agent gives this library, as cases to be timed.

Three operators.  `sample`: a token per row of logits - an action per knob, a candidate out of a trajectory's scores, an
entry of a vocabulary - with temperature, top-k, top-p and min-p, from one given uniform number per row.  `linear_scan` and
its backward pass: the gated linear recurrence h_t = a_t h_{t-1} + b_t, as discounted returns over a trajectory, as a
sequence layer in training, and as its step for single tokens.  `AdamW`: one step over all tensors of a model, with the two
moments held in 32 bits or in 8.

Where `own` is false a pass is made of elementary torch operations in 32 bits; where it is true it is the library's call.
Two things are defined in whole numbers, so that every way of computing them gives the same answer: the weights that a draw
adds up are exp(d), rounded to multiples of 2^-38, and their sums are exact; the random bits of the 8-bit moments are
SplitMix64 of (seed, step, tensor, element).
"""
import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_GAMMA = 0x9E3779B97F4A7C15
_M64 = (1 << 64) - 1
BLOCK = 256                                              # elements that share a scale where moments are held in 8 bits
LR, BETA1, BETA2, EPS, DECAY = 1e-3, 0.9, 0.999, 1e-8, 0.01


def listed():
    return [
        # an action per knob of every configuration of an ordinary trajectory (65,536 configurations, 8 knobs, 3 directions)
        {"name": "sample_actions", "kind": "sample", "rows": 524288, "v": 3, "type": "f32", "temperature": 0, "top_k": 0, "top_p": 0, "min_p": 0},
        # a few draws out of a small trajectory's scores: latency
        {"name": "sample_small", "kind": "sample", "rows": 8, "v": 2000, "type": "f32", "temperature": 1, "top_k": 1, "top_p": 1, "min_p": 0},
        # a serving batch over a vocabulary, every request with its own settings
        {"name": "sample_vocab", "kind": "sample", "rows": 64, "v": 128003, "type": "bf16", "temperature": 1, "top_k": 1, "top_p": 1, "min_p": 1},
        # a candidate for every space of the `batched` workload, out of the nucleus of its scores
        {"name": "sample_nucleus", "kind": "sample", "rows": 64, "v": 262144, "type": "f32", "temperature": 1, "top_k": 0, "top_p": 1, "min_p": 0},
        # one draw out of all scores of the `large` workload: a single long row
        {"name": "sample_long_row", "kind": "sample", "rows": 1, "v": 8388608, "type": "f32", "temperature": 1, "top_k": 0, "top_p": 0, "min_p": 0},
        # one token of a recurrent layer, 64 sequences: latency
        {"name": "scan_step", "kind": "scan", "batch": 64, "t": 1, "c": 2048, "type": "bf16", "gate": "f32", "backward": 0, "returns": 0},
        # discounted returns backwards in time over the trajectories of the `batched` workload, cut into episodes
        {"name": "scan_returns", "kind": "scan", "batch": 64, "t": 262144, "c": 1, "type": "f32", "gate": "f32", "backward": 0, "returns": 1},
        # one long sequence: few channels, so that time has to be cut
        {"name": "scan_long", "kind": "scan", "batch": 1, "t": 65521, "c": 1024, "type": "bf16", "gate": "f32", "backward": 0, "returns": 0},
        # the backward pass of a layer in training
        {"name": "scan_train", "kind": "scan", "batch": 8, "t": 4093, "c": 2048, "type": "bf16", "gate": "bf16", "backward": 1, "returns": 0},
        # the search agent's own network (first layer shared, a head of 3 directions per knob, a value head): latency
        {"name": "adamw_agent", "kind": "adamw", "layers": 1, "width": 128, "type": "f32", "bits": 32, "master": 0},
        # an ordinary model in 32 bits throughout
        {"name": "adamw_f32", "kind": "adamw", "layers": 16, "width": 2048, "type": "f32", "bits": 32, "master": 0},
        # a larger one in bf16, with master weights in 32 bits and moments in 8
        {"name": "adamw_8bit", "kind": "adamw", "layers": 12, "width": 4096, "type": "bf16", "bits": 8, "master": 1},
    ]


def _between(rng, lo, hi):
    """A whole number in lo..hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    """Another case: any of the three, sizes between the smallest and the largest listed."""
    kind = rng.choice(["sample", "sample", "scan", "scan", "adamw"])
    if kind == "sample":
        case = {"kind": kind, "v": _between(rng, 3, 8388608), "type": rng.choice(["f32", "bf16", "f16"])}
        case["rows"] = _between(rng, 1, min(524288, max(1, 16777216 // case["v"])))
        for f in ("temperature", "top_k", "top_p", "min_p"):
            case[f] = rng.randint(0, 1)
        return case
    if kind == "scan":
        if rng.random() < 0.3:
            batch = _between(rng, 1, 64)
            return {"kind": kind, "batch": batch, "t": _between(rng, 100, min(262144, 16777216 // batch)), "c": 1, "type": "f32", "gate": "f32",
                    "backward": rng.randint(0, 1), "returns": 1}
        c = _between(rng, 16, 4096)
        t = _between(rng, 1, 65536)
        dtype = rng.choice(["f32", "bf16", "f16"])
        return {"kind": kind, "batch": _between(rng, 1, max(1, min(64, 67000000 // (c * t)))), "t": t, "c": c, "type": dtype,
                "gate": rng.choice(["f32", dtype]), "backward": rng.randint(0, 1), "returns": 0}
    dtype = rng.choice(["f32", "bf16"])
    return {"kind": kind, "layers": rng.randint(1, 16), "width": _between(rng, 32, 3000), "type": dtype, "bits": rng.choice([32, 8]),
            "master": rng.randint(0, 1) if dtype == "bf16" else 0}


def _shapes(case):
    """Tensors of the network: 8 knobs in, `layers` of width x width where there is more than the shared one, the two heads."""
    w = case["width"]
    shapes = [(w, 8), (w,)]
    for _ in range(case["layers"] - 1):
        shapes += [(w, w), (w,)]
    return shapes + [(24, w), (24,), (1, w), (1,)]


# ---- inputs ------------------------------------------------------------------------------------------------------

def _views(flat, sizes, starts):
    return [flat[a:a + n] for a, n in zip(starts, sizes)]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": case, "seed": seed, "kind": case["kind"]}
    rand = lambda *shape: torch.rand(*shape, generator=gen, device="cuda")        # noqa: E731
    randn = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")      # noqa: E731
    if case["kind"] == "sample":
        rows, v = case["rows"], case["v"]
        s["logits"] = (randn(rows, v) * 2.0).to(_TYPES[case["type"]])
        s["uniform"] = rand(rows)
        s["temperature"] = 0.5 + rand(rows) if case["temperature"] else None
        s["top_k"] = torch.randint(1, 256, (rows,), generator=gen, device="cuda", dtype=torch.int32) if case["top_k"] else None
        s["top_p"] = 0.5 + 0.49 * rand(rows) if case["top_p"] else None
        s["min_p"] = 0.1 * rand(rows) if case["min_p"] else None
        if own:                                          # scratch memory, as a serving loop keeps it
            from paper_1905_12799_amd import binding as rls
            s["workspace"] = torch.empty(rls.sample_workspace_bytes(rows, v) + 256, dtype=torch.uint8, device="cuda")
        return s
    if case["kind"] == "scan":
        b, t, c, dtype = case["batch"], case["t"], case["c"], _TYPES[case["type"]]
        if case["returns"]:
            s["a"] = torch.full((b, t, c), 0.9 * 0.99, device="cuda")
            s["reset"] = (rand(b, t) < 1.0 / 512).to(torch.uint8)
            s["state"] = None
        else:
            s["a"] = torch.sigmoid(randn(b, t, c) + 4.0).to(_TYPES[case["gate"]])
            s["reset"] = None
            s["state"] = randn(b, c)
        s["b"] = randn(b, t, c).to(dtype)
        if case["backward"]:
            s["h"] = _scan(s["a"].float(), s["b"].float(), s["state"], s["reset"], bool(case["returns"])).to(dtype)
            s["dh"] = randn(b, t, c).to(dtype)
            s["dlast"] = randn(b, c)
            del s["b"]
        if own:
            from paper_1905_12799_amd import binding as rls
            need = rls.linear_scan_workspace_bytes(b, t, c)
            s["workspace"] = torch.empty(need + 256, dtype=torch.uint8, device="cuda")
        return s
    shapes = _shapes(case)
    sizes = [int(torch.Size(x).numel()) for x in shapes]
    starts, end = [], 0
    for n in sizes:
        starts.append(end)
        end += -(-n // BLOCK) * BLOCK
    dtype = _TYPES[case["type"]]
    # a model's tensors lie in one buffer per array, each at a multiple of 256 elements; what lies between them stays as it is
    p = randn(end) * 0.02
    g = (randn(end) * 1e-3).to(dtype)
    m = randn(end) * 3e-4
    v = (randn(end) * 1e-3).square_().add_(1e-8)
    s["flat"] = {"param": p.to(dtype)}
    if case["master"]:
        s["flat"]["master"] = p
    if case["bits"] == 8:
        for name, x in (("m", m), ("v", v.sqrt())):
            blocks = x.view(-1, BLOCK)
            scale = _power_of_two(blocks.abs().amax(1))
            s["flat"][name] = (blocks / scale[:, None]).to(torch.float8_e4m3fn).view(torch.uint8).view(-1)
            s["flat"][name + "_scale"] = scale
    else:
        s["flat"]["m"], s["flat"]["v"] = m, v
    s["sizes"], s["step"] = sizes, 100
    s["grads"] = [x.view(k) for x, k in zip(_views(g, sizes, starts), shapes)]
    s["views"] = {}
    for name, x in s["flat"].items():
        if name.endswith("_scale"):
            s["views"][name] = _views(x, [-(-n // BLOCK) for n in sizes], [a // BLOCK for a in starts])
        else:
            s["views"][name] = [y.view(k) for y, k in zip(_views(x, sizes, starts), shapes)]
    if own:                                              # the optimizer that a training program keeps: the addresses of its tensors
        from paper_1905_12799_amd import binding as rls
        w = s["views"]
        s["optimizer"] = rls.AdamW(w["param"], exp_avg=w["m"], exp_avg_sq=w["v"], exp_avg_scale=w.get("m_scale"),
                                   exp_avg_sq_scale=w.get("v_scale"), master=w.get("master"), state_bits=case["bits"], step=s["step"], seed=seed)
    return s


# ---- one pass ------------------------------------------------------------------------------------------------------

def run(s):
    if s["kind"] == "sample":
        if own:
            from paper_1905_12799_amd import binding as rls
            token, logprob = rls.sample(s["logits"], s["uniform"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"],
                                        workspace=s["workspace"])
        else:
            token, logprob = _sample(s["logits"], s["uniform"], s["temperature"], s["top_k"], s["top_p"], s["min_p"])
        return {"token": token, "logprob": logprob}
    if s["kind"] == "scan":
        return _run_scan(s)
    return _run_adamw(s)


def _run_scan(s):
    reverse, dtype = bool(s["case"]["returns"]), _TYPES[s["case"]["type"]]
    if own:
        from paper_1905_12799_amd import binding as rls
        if s["case"]["backward"]:
            da, db, dstate = rls.linear_scan_backward(s["a"], s["h"], s["dh"], h0=s["state"], reset=s["reset"], dh_last=s["dlast"], reverse=reverse,
                                                      workspace=s["workspace"])
            return {"da": da, "db": db, "dstate": dstate}
        h, last = rls.linear_scan(s["a"], s["b"], h0=s["state"], reset=s["reset"], reverse=reverse, workspace=s["workspace"])
        return {"h": h, "last": last}
    a = s["a"].float()
    if not s["case"]["backward"]:
        h = _scan(a, s["b"].float(), s["state"], s["reset"], reverse)
        return {"h": h.to(dtype), "last": h[:, 0 if reverse else -1].clone()}
    h, dh = s["h"].float(), s["dh"].float()
    if s["reset"] is not None:
        a = a.masked_fill(s["reset"].bool()[:, :, None], 0.0)
    if reverse:
        a, h, dh = a.flip(1), h.flip(1), dh.flip(1)
    dh = torch.cat([dh[:, :-1], (dh[:, -1] + s["dlast"])[:, None]], 1)
    later = torch.cat([a[:, 1:], torch.zeros_like(a[:, :1])], 1)                  # what carries the next step's gradient back
    db = _scan(later, dh, None, None, True)
    first = torch.zeros_like(h[:, :1]) if s["state"] is None else s["state"][:, None]
    da = db * torch.cat([first, h[:, :-1]], 1)
    dstate = a[:, 0] * db[:, 0]
    if reverse:
        da, db = da.flip(1), db.flip(1)
    if s["reset"] is not None:
        da = da.masked_fill(s["reset"].bool()[:, :, None], 0.0)
    return {"da": da.to(s["a"].dtype), "db": db.to(dtype), "dstate": dstate}


def _scan(a, b, state, reset, reverse):
    """h_t = a_t h_{t-1} + b_t by doubling: after the pass of distance k every place has taken in the 2 k before it."""
    if reset is not None:
        a = a.masked_fill(reset.bool()[:, :, None], 0.0)
    if reverse:
        a, b = a.flip(1), b.flip(1)
    h = b.clone()
    if state is not None:
        h[:, 0] += a[:, 0] * state
    k, t = 1, a.shape[1]
    while k < t:
        h = torch.cat([h[:, :k], h[:, k:] + a[:, k:] * h[:, :-k]], 1)
        a = torch.cat([a[:, :k], a[:, k:] * a[:, :-k]], 1)
        k *= 2
    return h.flip(1) if reverse else h


def _sample(logits, uniform, temperature, top_k, top_p, min_p):
    """d = (logit - largest) / temperature and exp(d) in 32 bits, weights in multiples of 2^-38, their sums in whole numbers."""
    rows, v = logits.shape
    x = logits.float()
    x = torch.where(x.isnan(), -torch.inf, x)
    top = x.amax(1, keepdim=True)
    d = x - top
    if temperature is not None:
        d = d * (1.0 / temperature)[:, None]
    d = torch.where(x == top, 0.0, torch.where(x == -torch.inf, -torch.inf, d))
    e = torch.exp(d)
    w = torch.round(e.double() * 2.0 ** 38).long()
    w = torch.where(top == -torch.inf, 0, w)
    if top_k is not None or top_p is not None:
        order = torch.sort(d, dim=1, descending=True, stable=True).indices
        ws = w.gather(1, order)
        place = torch.arange(v, device=x.device)[None]
        if top_k is not None:
            ws = torch.where(place < top_k[:, None], ws, 0)
        if top_p is not None:
            before = ws.cumsum(1) - ws
            inside = before.double() < top_p.double()[:, None] * ws.sum(1, keepdim=True).double()
            ws = torch.where(inside | (place < 1), ws, 0)
        w = torch.zeros_like(w).scatter_(1, order, ws)
    if min_p is not None:
        w = torch.where((e >= min_p[:, None]) | (d == 0), w, 0)
    run_sum = w.cumsum(1)
    total = run_sum[:, -1:]
    mark = uniform.double()[:, None] * total.double()
    token = torch.minimum((run_sum.double() <= mark).sum(1), (run_sum < total).sum(1))
    logprob = d.gather(1, token[:, None].clamp(max=v - 1))[:, 0] - torch.log((total[:, 0].double() * 2.0 ** -38).float())
    empty = total[:, 0] == 0
    return torch.where(empty, -1, token).to(torch.int32), torch.where(empty, -torch.inf, logprob)


def _power_of_two(largest):
    """The scale of a block whose largest magnitude is given: the power of two that brings it to at most 448, and above 224."""
    mantissa, exponent = torch.frexp(largest)
    e = torch.where(mantissa <= 0.875, exponent - 9, exponent - 8)
    e = torch.where(largest == 0, -120, e).clamp(min=-120)
    return torch.ldexp(torch.ones_like(largest), e)


def _mix(z):
    """The output function of SplitMix64 (Steele, Lea, Flood 2014), on whole numbers."""
    z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & _M64
    z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & _M64
    return z ^ (z >> 31)


def _signed(c):
    return c - (1 << 64) if c >> 63 else c


def _random_bits(n, seed, step, tensor):
    """32 bits per element: the halves of SplitMix64 draw q for the elements 2 q and 2 q + 1."""
    base = _mix((_mix((seed + _GAMMA * step) & _M64) + _GAMMA * (tensor + 1)) & _M64)
    z = torch.arange(1, n // 2 + 1, device="cuda") * _signed(_GAMMA) + _signed(base)
    z = (z ^ ((z >> 30) & ((1 << 34) - 1))) * _signed(0xBF58476D1CE4E5B9)
    z = (z ^ ((z >> 27) & ((1 << 37) - 1))) * _signed(0x94D049BB133111EB)
    z = z ^ ((z >> 31) & ((1 << 33) - 1))
    return torch.stack([z & 0xFFFFFFFF, (z >> 32) & 0xFFFFFFFF], 1).view(-1)


def _encode(x, bits16, positive):
    """Blocks of values as 8-bit floats (1-4-3) times a power of two, rounded up or down at random in proportion: (codes, scales)."""
    largest = x.abs().amax(1)
    scale = _power_of_two(largest)
    y = x.abs() / scale[:, None]
    small = y < 2.0 ** -6
    y = torch.where(small, y + 2.0 ** -6, y)
    code = ((y.view(torch.int32) + ((bits16.int() << 4) + 8)) >> 20) - 968
    code = torch.where(small, code, code + 8)
    code = code.clamp(max=126)
    if positive:
        code = torch.where(x > 0, code.clamp(min=1), code)
    else:
        code = torch.where(x < 0, code + 128, code)
    return code.to(torch.uint8), scale


def _run_adamw(s):
    case, views = s["case"], s["views"]
    s["step"] += 1
    if own:
        s["optimizer"].step(s["grads"], lr=LR, betas=(BETA1, BETA2), eps=EPS, weight_decay=DECAY)
    else:
        step = s["step"]
        scale_m, scale_v = LR / (1.0 - BETA1 ** step), (1.0 - BETA2 ** step) ** -0.5
        for i, n in enumerate(s["sizes"]):
            param, g = views["param"][i].view(-1), s["grads"][i].view(-1).float()
            p = views["master"][i].view(-1) if case["master"] else param.float()
            m, v = views["m"][i].view(-1), views["v"][i].view(-1)
            if case["bits"] == 8:
                blocks = -(-n // BLOCK)
                pad = blocks * BLOCK - n
                fill = lambda x: torch.nn.functional.pad(x, (0, pad))              # noqa: E731
                codes_m, codes_v, g = fill(m), fill(v), fill(g)
                m = (codes_m.view(torch.float8_e4m3fn).float().view(blocks, BLOCK) * views["m_scale"][i][:, None]).view(-1)
                v = (codes_v.view(torch.float8_e4m3fn).float().view(blocks, BLOCK) * views["v_scale"][i][:, None]).square().view(-1)
            m = m * BETA1 + g * (1.0 - BETA1)
            v = v * BETA2 + (g * (1.0 - BETA2)) * g
            root = torch.sqrt(v)
            if case["bits"] == 8:
                bits = _random_bits(blocks * BLOCK, s["seed"], step, i).view(blocks, BLOCK)
                code, views["m_scale"][i][:] = _encode(m.view(blocks, BLOCK), bits & 0xFFFF, False)
                views["m"][i].view(-1)[:] = code.view(-1)[:n]
                code, views["v_scale"][i][:] = _encode(root.view(blocks, BLOCK), bits >> 16, True)
                views["v"][i].view(-1)[:] = code.view(-1)[:n]
                m, root = m[:n], root[:n]
            else:
                views["m"][i].view(-1)[:], views["v"][i].view(-1)[:] = m, v
            p = p * (1.0 - LR * DECAY) - (m / (root * scale_v + EPS)) * scale_m
            if case["master"]:
                views["master"][i].view(-1)[:] = p
            param[:] = p.to(param.dtype)
    out = dict(s["flat"])
    if case["bits"] == 8:
        out["m"], out["v"] = out["m"].view(torch.float8_e4m3fn), out["v"].view(torch.float8_e4m3fn)
    return out


# ---- what a pass cannot do without ---------------------------------------------------------------------------------

def work(case):
    """Inputs read once, outputs written once.  Per logit a subtraction, an exponential and a sum; per place of a recurrence a
    multiplication and an addition, three of each with gradients; per parameter some fifteen operations."""
    size = {"f32": 4.0, "bf16": 2.0, "f16": 2.0}
    if case["kind"] == "sample":
        n = float(case["rows"]) * case["v"]
        settings = sum(4.0 for f in ("temperature", "top_k", "top_p", "min_p") if case[f])
        return {"bytes": n * size[case["type"]] + case["rows"] * (4.0 + settings + 8.0), "flops": 3.0 * n}
    if case["kind"] == "scan":
        n = float(case["batch"]) * case["t"] * case["c"]
        wide, gate = size[case["type"]], size[case["gate"]]
        state = 8.0 * case["batch"] * case["c"]
        flags = float(case["batch"]) * case["t"] if case["returns"] else 0.0
        if case["backward"]:
            return {"bytes": n * (3 * wide + 2 * gate) + flags + 1.5 * state, "flops": 3.0 * n}
        return {"bytes": n * (2 * wide + gate) + flags + state, "flops": 2.0 * n}
    n = float(sum(int(torch.Size(x).numel()) for x in _shapes(case)))
    wide = size[case["type"]]
    moments = 16.0 if case["bits"] == 32 else 4.0 + 4 * 4.0 / BLOCK
    weights = wide + 8.0 if case["master"] else 2 * wide
    return {"bytes": n * (wide + moments + weights), "flops": 15.0 * n}


# ---- the same in 64 bits, from the definitions ---------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "sample":
        return _exact_sample(s)
    if case["kind"] == "scan":
        return _exact_scan(s)
    return _exact_adamw(s)


def _exact_sample(s):
    """Row by row: probabilities, the sets that the settings leave, the first place where the running sum passes the number drawn."""
    rows, v = s["logits"].shape
    if rows > 4096 and v > 8:
        return None
    x = s["logits"].double()
    one = torch.ones(rows, 1, dtype=torch.float64, device="cuda")
    t = one if s["temperature"] is None else s["temperature"].double()[:, None]
    p = torch.softmax(x / t, 1)
    keep = torch.ones_like(p, dtype=torch.bool)
    if s["top_k"] is not None or s["top_p"] is not None:
        ps, order = torch.sort(p, dim=1, descending=True, stable=True)
        rank = torch.arange(v, device="cuda").expand(rows, v)
        if s["top_k"] is not None:
            ps = ps * (rank < s["top_k"][:, None])
        ps = ps / ps.sum(1, keepdim=True)
        inside = ps > 0
        if s["top_p"] is not None:
            inside &= (ps.cumsum(1) - ps) < s["top_p"].double()[:, None]
        keep = torch.zeros_like(keep).scatter_(1, order, inside)
    if s["min_p"] is not None:
        keep &= p >= s["min_p"].double()[:, None] * p.amax(1, keepdim=True)
    p = p * keep
    p = p / p.sum(1, keepdim=True)
    passed = p.cumsum(1) > s["uniform"].double()[:, None]
    token = (~passed).sum(1).clamp(max=v - 1)
    return {"token": token.to(torch.int32), "logprob": torch.log(p.gather(1, token[:, None])[:, 0])}


def _exact_recurrence(a, b, state):
    """One step after the other within pieces of about sqrt(T) steps, all pieces at once; then from piece to piece."""
    n, t, c = a.shape
    size = max(1, int(t ** 0.5))
    pieces = -(-t // size)
    pad = pieces * size - t
    a = torch.cat([a, torch.ones(n, pad, c, dtype=a.dtype, device=a.device)], 1).view(n, pieces, size, c)
    b = torch.cat([b, torch.zeros(n, pad, c, dtype=a.dtype, device=a.device)], 1).view(n, pieces, size, c)
    h, f = torch.empty_like(b), torch.empty_like(a)
    h[:, :, 0], f[:, :, 0] = b[:, :, 0], a[:, :, 0]
    for i in range(1, size):
        h[:, :, i] = a[:, :, i] * h[:, :, i - 1] + b[:, :, i]
        f[:, :, i] = a[:, :, i] * f[:, :, i - 1]
    for j in range(pieces):
        h[:, j] += f[:, j] * state[:, None]
        state = h[:, j, -1]
    return h.view(n, pieces * size, c)[:, :t]


def _exact_scan(s):
    reverse = bool(s["case"]["returns"])
    turn = (lambda x: x.flip(1)) if reverse else (lambda x: x)
    a = turn(s["a"].double())
    n, t, c = a.shape
    state = torch.zeros(n, c, dtype=torch.float64, device="cuda") if s["state"] is None else s["state"].double()
    if s["reset"] is not None:
        a = a * (turn(s["reset"]) == 0)[:, :, None]
    if not s["case"]["backward"]:
        h = _exact_recurrence(a, turn(s["b"].double()), state)
        return {"h": turn(h), "last": h[:, -1]}
    dh = turn(s["dh"].double()).clone()
    dh[:, -1] += s["dlast"].double()
    back = torch.zeros_like(a)
    back[:, 1:] = a[:, 1:].flip(1)
    g = _exact_recurrence(back, dh.flip(1), torch.zeros_like(state)).flip(1)
    h = turn(s["h"].double())
    before = torch.cat([state[:, None], h[:, :-1]], 1)
    da = g * before
    if s["reset"] is not None:
        da = da * (turn(s["reset"]) == 0)[:, :, None]
    return {"da": turn(da), "db": turn(g), "dstate": a[:, 0] * g[:, 0]}


def _exact_adamw(s):
    case, t = s["case"], s["step"] + 1
    grad = torch.zeros(s["flat"]["param"].shape, dtype=torch.float64, device="cuda")
    inside = torch.zeros_like(grad, dtype=torch.bool)
    start = 0
    for n, g in zip(s["sizes"], s["grads"]):
        grad[start:start + n] = g.reshape(-1).double()
        inside[start:start + n] = True
        start += -(-n // BLOCK) * BLOCK
    m, v = s["flat"]["m"], s["flat"]["v"]
    if case["bits"] == 8:
        wide = lambda x, k: x.view(torch.float8_e4m3fn).float().double() * k.double().repeat_interleave(BLOCK)      # noqa: E731
        m, v = wide(m, s["flat"]["m_scale"]), wide(v, s["flat"]["v_scale"]) ** 2
    m, v = m.double(), v.double()
    old = (s["flat"]["master"] if case["master"] else s["flat"]["param"]).double()
    m1 = BETA1 * m + (1 - BETA1) * grad
    v1 = BETA2 * v + (1 - BETA2) * grad ** 2
    p = old - LR * DECAY * old - LR * (m1 / (1 - BETA1 ** t)) / ((v1 / (1 - BETA2 ** t)).sqrt() + EPS)
    out = {"param": torch.where(inside, p, s["flat"]["param"].double())}
    if case["master"]:
        out["master"] = torch.where(inside, p, old)
    if case["bits"] == 8:                                # (a code rounded at random has no such value)
        out.update(m=None, v=None, m_scale=None, v_scale=None)
    else:
        out["m"], out["v"] = torch.where(inside, m1, m), torch.where(inside, v1, v)
    return out
